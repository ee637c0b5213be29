// The library as one translation unit: the verification path, then the operators that stand beside it and use its
// device helpers and the context.
#include "tli.cu"
#include "tli_rows.cu"
#include "tli_embed.cu"
