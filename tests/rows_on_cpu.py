"""The kernels of csrc/tli_rows.cu, from their source, on the CPU: one fiber per thread (cuda_on_cpu.h), blocks one after the other, the
threads between two collectives in an order of choice.  For what a run on a GPU shows by luck only: two threads at one word of
shared memory without a barrier between them, threads that part before a barrier."""
import ctypes
import os
import re
import subprocess
import tempfile

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_05202_b200", "csrc")

SHIM = r"""
#include "cuda_on_cpu.h"
#include "tli.h"
static float ex2(float x) { return exp2f(x); }
static float max_nan(float a, float b) { return a != a || b != b ? NAN : a < b ? b : a; }
static void mask_bf16_vector(uint4 &r, uint32_t bits) {
    unsigned short h[8];
    memcpy(h, &r, 16);
    for (int i = 0; i < 8; ++i) if (!(bits >> i & 1)) h[i] = 0xff80u;
    memcpy(&r, h, 16);
}
"""

MAX_BF16 = r"""
static uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    return __float_as_uint(max_nan(bf16_lo(a), bf16_lo(b))) >> 16 | (__float_as_uint(max_nan(bf16_hi(a), bf16_hi(b))) & 0xffff0000u);
}
"""

LAUNCH = r"""
constexpr unsigned long long kCanary = 0x5ca1ab1ec0ffee11ull;
template <typename F> static bool grid(unsigned gx, unsigned gy, unsigned threads, size_t smem, int order, unsigned seed, F f) {
    gridDim = {gx, gy, 1}; blockDim = {threads, 1, 1};
    for (unsigned y = 0; y < gy; ++y)
        for (unsigned x = 0; x < gx; ++x) {
            blockIdx = {x, y, 0};
            memset(reinterpret_cast<void *>(&S), 0xa5, sizeof S);
            memset(pick_smem, 0xa5, sizeof pick_smem);
            memcpy(pick_smem + smem, &kCanary, 8);
            if (!emu::run_block(threads, order, seed + 7919u * (y * gx + x), f)) return false;
            if (memcmp(pick_smem + smem, &kCanary, 8)) { snprintf(emu::message, sizeof emu::message, "a block wrote behind its shared memory"); return false; }
        }
    return true;
}
template <int DT, int U> static bool launch(const RowsParams &P, int order, unsigned seed) {
    const unsigned rows = P.B * P.R, strips = (P.nstrip + kRowWarps - 1) / kRowWarps;
    if (!grid(strips, rows, kRowThreads, 0, order, seed, [&] { tli_rows_scan_kernel<DT, U>(P); })) return false;
    if (!grid(rows, 1, kPickThreads, pick_smem_bytes(P.nstrip, (P.nstrip + P.coarse - 1) / P.coarse * 32), order, seed, [&] { tli_rows_pick_kernel<DT>(P); })) return false;
    if (P.listcap > 0 && (P.top_k || P.top_p || P.min_p)) {
        if (!grid(2, 1, kPickThreads, settle_smem_bytes(P.nstrip), order, seed, [&] { tli_rows_spread_kernel<DT, U>(P); })) return false;
    }
    return P.sample || grid(strips, rows, kRowThreads, 0, order, seed, [&] { tli_rows_mask_kernel<DT, U>(P); });
}
}  // namespace

// 0: done; else emulator_message() says what happened.  left: rows that the pick kernel left to the spread kernel.
extern "C" int rows_on_cpu(int sample, int B, int R, int V, int dtype, const void *z, long long sb, long long sr, const unsigned *mask, const float *tau,
                           const int *top_k, const float *top_p, const float *min_p, const float *u, int *tokens, float *prob, int *status, void *out,
                           int order, unsigned seed, int *left) {
    RowsParams P;
    memset(&P, 0, sizeof P);
    P.B = B; P.R = R; P.V = V; P.sample = sample; P.z = z; P.sb = sb; P.sr = sr; P.mask = mask;
    P.tau = tau; P.top_k = top_k; P.top_p = top_p; P.min_p = min_p; P.u = u;
    P.tokens = tokens; P.prob = prob; P.status = status; P.out = out; P.osb = static_cast<long long>(R) * V; P.osr = V;
    const RowsLayout L = rows_layout(static_cast<long long>(B) * R, V, dtype);
    char *ws = static_cast<char *>(aligned_alloc(256, (L.total + 255) / 256 * 256));
    memset(ws, 0xa5, L.total);
    P.nstrip = L.nstrip; P.coarse = L.coarse; P.ulog = L.U == 2 ? 1 : L.U == 4 ? 2 : 3;
    P.gmax = ws + L.gmax;
    P.ssum = reinterpret_cast<StripSum *>(ws + L.ssum);
    P.border = reinterpret_cast<RowBorder *>(ws + L.border);
    P.plan = reinterpret_cast<RowPlan *>(ws + L.plan);
    P.todo = reinterpret_cast<int *>(ws + L.todo);
    P.lists = reinterpret_cast<unsigned long long *>(ws + L.lists);
    P.listcap = L.listcap;
    bool ok;
#define RUN(U) (dtype == TLI_F32 ? launch<TLI_F32, U>(P, order, seed) : launch<TLI_BF16, U>(P, order, seed))
    ok = L.U == 2 ? RUN(2) : L.U == 4 ? RUN(4) : RUN(8);
    *left = *P.todo;
    free(ws);
    return ok ? 0 : 1;
}
extern "C" void exp2_on_cpu(const double *x, double *out, int n) {            // (the weights' powers of two, without threads)
    double tab[16];
    for (int i = 0; i < 16; ++i) exp2_table_init(tab, i);
    for (int i = 0; i < n; ++i) out[i] = exp2_neg(x[i], tab);
}
extern "C" const char *emulator_message() { return emu::message; }
"""


def _definition(text, start):
    """From ``start`` to the brace that closes what it opens (and a semicolon behind it)."""
    at = text.index(start)
    i, depth = text.index("{", at), 0
    while True:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
        if depth == 0:
            return text[at:i] + (";" if text[i:i + 1] == ";" else "")


def source(edit=lambda text: text):
    """One C++ file; ``edit``: a change of csrc/tli_rows.cu's text."""
    tli = open(os.path.join(CSRC, "tli.cu")).read()
    rows = edit(open(os.path.join(CSRC, "tli_rows.cu")).read())
    helpers = [_definition(tli, s) for s in (
        "template <> struct Elt<TLI_F32>", "template <> struct Elt<TLI_BF16>", "__device__ __forceinline__ int float_order(",
        "__device__ __forceinline__ float order_float(", "__device__ __forceinline__ float warp_max(", "__device__ __forceinline__ double warp_sum(",
        "__device__ __forceinline__ float bf16_lo(", "__device__ __forceinline__ float bf16_hi(", "template <int DT> __device__ __forceinline__ float load_elt(",
        "template <int DT> __device__ __forceinline__ void unpack(", "template <int DT> struct RowView", "__device__ __forceinline__ uint32_t mask_bits(",
        "size_t align_up(", "int chunks_per_row(")]
    kernels, host = rows.split("// ---- host ----")
    kernels = re.sub(r'asm volatile\("griddepcontrol\.\w+;" ::: "memory"\);', "", kernels).replace("#include <cuda_bf16.h>", "")
    for start in ("__device__ __forceinline__ float max_nan(", "__device__ __forceinline__ uint32_t max_nan_bf16x2("):
        kernels = kernels.replace(_definition(kernels, start), "")
    kernels = kernels.replace("extern __shared__ __align__(16) unsigned char pick_smem[];", "static unsigned char pick_smem[256 * 1024] __align__(16);")
    layout = _definition(host, "struct RowsLayout") + "\n" + _definition(host, "RowsLayout rows_layout(")
    return "\n".join([SHIM, "namespace {\ntemplate <int DT> struct Elt;"] + helpers + [MAX_BF16, "}", kernels, layout, LAUNCH])


def build(edit=lambda text: text):
    """The compiled kernels as a ctypes library."""
    with tempfile.TemporaryDirectory(prefix="rows_on_cpu_") as folder:
        cpp, lib = os.path.join(folder, "rows.cpp"), os.path.join(folder, "rows.so")
        with open(cpp, "w") as f:
            f.write(source(edit))
        subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-ffp-contract=off", "-fno-strict-aliasing", "-fPIC", "-shared", "-I", os.path.join(ROOT, "tests"),
                        "-I", os.path.join(ROOT, "include"), "-o", lib, cpp], check=True)
        handle = ctypes.CDLL(lib)                                    # (stays loaded without its file)
    handle.emulator_message.restype = ctypes.c_char_p
    return handle


def run(lib, z, dtype, ask, u=None, part=None, order=0, seed=0):
    """Sample (``u`` given) or filter the rows ``z`` (fp32 values [B,R,V]; of bf16 precision for dtype 1)."""
    B, R, V = z.shape
    z = np.ascontiguousarray(z, np.float32)
    raw = z if dtype == 0 else (z.view(np.uint32) >> 16).astype(np.uint16)
    space = np.zeros(raw.nbytes + 64, np.uint8)                      # on 16 bytes, and readable to the last whole vector
    at = -space.ctypes.data % 16
    space[at:at + raw.nbytes] = raw.reshape(-1).view(np.uint8)
    mask = None
    if part is not None:
        bits = np.zeros((V + 31) // 32 * 32 + 64, bool)
        bits[:V] = part
        mask = np.packbits(bits.reshape(-1, 32), axis=1, bitorder="little").view(np.uint32).reshape(-1)
    tau, k, p, mp = (np.ascontiguousarray(x) for x in ask)
    tokens, prob, status = np.full((B, R), -9, np.int32), np.full((B, R), -9, np.float32), np.full((B, R), -9, np.int32)
    out = np.zeros(raw.nbytes + 64, np.uint8)
    at_out = -out.ctypes.data % 16
    left = ctypes.c_int()
    ptr = lambda a: None if a is None else ctypes.c_void_p(a.ctypes.data)
    uu = None if u is None else np.ascontiguousarray(u, np.float32)
    rc = lib.rows_on_cpu(int(u is not None), B, R, V, dtype, ctypes.c_void_p(space.ctypes.data + at), ctypes.c_longlong(R * V), ctypes.c_longlong(V), ptr(mask),
                         ptr(tau), ptr(k), ptr(p), ptr(mp), ptr(uu), ptr(tokens), ptr(prob), ptr(status), ctypes.c_void_p(out.ctypes.data + at_out),
                         order, ctypes.c_uint(seed), ctypes.byref(left))
    if rc:
        raise AssertionError("order %d, seed %d: %s" % (order, seed, lib.emulator_message().decode()))
    res = out[at_out:at_out + raw.nbytes].view(raw.dtype).reshape(z.shape)
    kept = ((res != 0xff80) if dtype else (res != -np.inf)) if u is None else None
    return {"tokens": tokens, "prob": prob, "status": status, "kept": kept, "left": left.value}
