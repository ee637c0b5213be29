// The losses of tli_loss.cu from hidden rows and the output head's weight, z = hidden * weight^T, and their gradients.  The logits
// are formed tile by tile in tensor memory and never written.  (Part of tli_lib.cu: uses the parts before it.)
//
// A call is a chain of launches:
//   tli_head_targets_kernel   which rows take part, one bit each; for the gradient what their slopes are made of.
//   tli_head_gather_kernel    those rows of `hidden` one after the other (work is in proportion to them, any stride and alignment will
//                             do, and a row that is left out may hold anything); for few rows tli_head_prepare_kernel does both.
//   tli_head_gemm_kernel      <STATS>  forward: (max, sum) of every row over every tile of the vocabulary.
//   tli_head_loss_kernel               forward: the tiles' pairs joined, the targets' logits, the loss.
//                             <SLOPE>  backward, for a run of the vocabulary: G = g dz in bf16, [rows, run], to the workspace;
//                             <GRADS>  d hidden += G * weight and d weight = G^T * hidden of that run, one list of tiles.
//   tli_head_rows_kernel      d hidden from its fp32 sums to bf16, at the rows' places.
// A run's G has 256 MB at most, whatever the vocabulary.  Side by side in one session, 8192 tokens x 128 256 x 2048: 9.9 ms; with 128 MB, about what L2
// holds, 11.2 (more launches and shorter sums of d hidden), with 64 MB 10.9, with 32 MB 14.1, with 512 MB 10.2.  (A card that has worked for seconds at its
// power limit, 1.38 GHz, takes 10.6 to 11.0; the first calls after a pause 9.5.)
// G is held in bf16, the type of the operands of both its products (as two bf16 parts it would double them).  Its rounding is off by half a step, 2^-8
// at most, and is most of what d hidden and d weight are off beside the rounding of their own: 0.0019 to 0.0023 of fp64 in the norm, 0.0017 without it.
// d hidden gets back what is left off a row's kHeadNear largest elements; d weight gets nothing back (its rows would need a list of their targets each).
//
// tli_head_gemm_kernel: persistent, one CTA per SM or one pair (CG = 2) per two SMs.  A tile of D is 128 CG rows x 256 columns of fp32 in
// tensor memory, two of them, so that the epilogue of one runs under the products of the next.  Warp 0 fills a ring of stages of
// 64 elements of the contracted axis by TMA, warp 1 issues tcgen05.mma (bf16, fp32 sums), warps 2 to 9 are the epilogue: two threads per
// row of D, 128 columns each (with one thread per row it took 6 us a tile, as long as the products at H = 1024).  What leaves, leaves by
// TMA from a slab of each warp's own, so that no warp waits for another.  (Four threads per row and slabs for them take the room of a
// stage: 17 % slower where the products count.)  With CG = 2 each CTA loads half of both operands and the pair's leader issues the products of both.
// What bounds it: the matrix unit and the shared memory that feeds it (32 KB in and 32 KB out per stage and CTA of 512 cycles).  Tensor pipe active
// 86 % of the cycles for STATS at H = 2048 (4096 rows, 64 000 ids), 64 % for SLOPE (179 us) and 79 % for GRADS (284 us) at H = 1024 (2000 rows, 49 152
// ids, one run, 1.6 GHz; there the epilogue and the first and last tiles weigh more); L2 at half its rate, DRAM at a quarter and less.  Long calls run at
// the power limit (1.4 GHz and below).
// With one row block the weight is read once for STATS and SLOPE each (DRAM: 131 MB in 17 us of a call of 32).
// Operands come as they lie in memory: rows along the contracted axis (K-major) or across it (MN-major), 128-byte swizzle either way.
// Waits on the barriers in shared memory are bounded: when one runs out the context's error word is set, every role stops, copies in flight
// are waited for, tensor memory is given back, and the rows' status says TLI_ROW_TIMEOUT.  (Not bounded are the barriers of the CTA and the
// pair, which every thread comes to, after a time-out too, and the allocation of tensor memory, which waits for kernels that hold it.)

#include <cuda.h>

namespace {

constexpr int kHeadEpilogue = 8;           // warps of the epilogue: two per quarter of the rows, 128 columns each
constexpr int kHeadThreads = 64 + 32 * kHeadEpilogue;
// The matrix unit cuts what a sum cannot hold (it does not round): a sum of 2048 products of a logit was 1e-5 off where one rounded at every step
// is 4e-6 off.  The logits that the statistics are made of are therefore summed in parts, which the epilogue adds up: 128 elements where the
// weight's way through the SM is what counts (one token: 32.3 us, 31.6 with 256, 33.5 with 64), else half of H but 512 to 1024 (8192 x
// 128 256 x 2048: one part 3.07 ms and 1e-5 off, two 3.16 and 5e-6, four 3.35 and 2e-6).  SLOPE forms its logits in one part whatever H is: what that
// leaves off grows with H, by the same count to 3e-4 at 65 536, a tenth of what rounding G to bf16 does.
constexpr int kHeadK = 64;                 // elements of the contracted axis in a stage: 128 bytes, one swizzle span
constexpr int kHeadN = 256;                // columns of a tile
constexpr int kHeadABytes = 128 * kHeadK * 2;
constexpr int kHeadSlab = 32 * 128;        // what a warp of the epilogue has on its way out: 32 rows of 128 bytes
enum : int { HEAD_STATS = 0, HEAD_SLOPE = 1, HEAD_GRADS = 2 };

template <int CG> struct HeadRing {
    static constexpr int kStages = CG == 1 ? 4 : 6;
    static constexpr int kBBytes = kHeadN / CG * kHeadK * 2;
    static constexpr int kStageBytes = kHeadABytes + kBBytes;
    static constexpr int kSmem = kStages * kStageBytes + kHeadEpilogue * kHeadSlab + 1024;
};

struct HeadGemm {
    // STATS, SLOPE: a = rows, b = weight, out = G.  GRADS: a = G (K-major), b = weight (MN-major), a2 = G (MN-major), b2 = rows (MN-major),
    // out = d weight, out2 = sums of d hidden
    CUtensorMap a, b, a2, b2, out, out2;
    const int *n_valid;
    unsigned *error;
    int H, V, c0, cols;                    // the run of the vocabulary: [c0, c0 + cols)
    int bn, k_part;                        // STATS, SLOPE: columns of a tile; STATS: stages of a part of a sum
    int early;                             // one row block: what a CTA does first does not depend on how many rows take part
    int a_rows;                            // rows of a box of a
    int splits, first, want_dh, want_dw;   // GRADS: runs the contraction of d hidden is cut into; whether its sums start here
    const uint32_t *mask;
    const float4 *rowp;                    // {s, m, f, -} of a row
    const int *tid; const float *tval; int k;     // SLOPE: the rows' targets, ids (-1) and elements of G
    float2 *part; long long part_pitch;    // STATS: [tile of the vocabulary][row]
    // GRADS, with a mask: the operands of d hidden once more, for weight rows outside it that are not finite
    const __nv_bfloat16 *G, *weight; long long pitch, weight_stride;
};

// ---- tensor memory, matrix instructions, tensor copies ----

__device__ __forceinline__ uint64_t umma_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    // start, leading and stride byte offsets in 16-byte units; version 1; 128-byte swizzle
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 | static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <int CG> __device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    const uint32_t p = accumulate;
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(p) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(p) : "memory");
}
// The barrier (of both CTAs of a pair) gets an arrival when all products issued so far by this thread are done.
template <int CG> __device__ __forceinline__ void umma_commit(uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 32 columns of this thread's row (one of the 32 that a warp may read)
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&x)[32]) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
                   "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&x)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
// A box of a tensor to shared memory.  CG = 2: counted on the barrier at `bar`, which may be the pair's other CTA's.
template <int CG> __device__ __forceinline__ void tensor_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tensor_store(const CUtensorMap *map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void tensor_store3(const CUtensorMap *map, int x, int y, int z, uint32_t src, bool add) {
    if (add) asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
    else asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4 &v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A tile: where its operands start and how long its contraction is.
struct HeadTile {
    int m, n;                              // first row (of the pair) and first column of D
    int k0, ks;                            // first element of the contracted axis, steps of kHeadK
    int split;                             // GRADS: of d hidden; -1: a tile of d weight
};
// The tiles of CTA (pair) `cta` of `ctas`, one after the other.  GRADS: d hidden's tiles are the long ones and come first, dealt out in turn;
// where they do not come out even, the CTAs with one less begin with as many more of d weight's tiles as one of them is worth.  Tiles side
// by side run at the same time: they share the operand that is not in L2.
template <int MODE, int CG> struct HeadTiles {
    int cta, ctas, mb, nb, hb, t2, t3, k2, k3, extra, ahead;
    __device__ __forceinline__ HeadTiles(const HeadGemm &P, int rows, int cta_, int ctas_) {
        cta = cta_; ctas = ctas_;
        mb = P.early ? 1 : (rows + 128 * CG - 1) / (128 * CG);
        if constexpr (MODE == HEAD_GRADS) {
            hb = (P.H + kHeadN - 1) / kHeadN;
            nb = (P.cols + 128 * CG - 1) / (128 * CG);
            t2 = P.want_dh ? mb * hb * P.splits : 0;
            t3 = P.want_dw ? nb * hb : 0;
            k2 = (P.cols + kHeadK - 1) / kHeadK;
            k3 = (rows + kHeadK - 1) / kHeadK;
            extra = t2 % ctas;                                     // CTAs with one more tile of d hidden
            ahead = (k2 / P.splits + kTileSteps) / (k3 + kTileSteps);
        } else {
            hb = t3 = k3 = extra = ahead = 0;
            nb = (P.cols + P.bn - 1) / P.bn;
            t2 = mb * nb;
            k2 = (P.H + kHeadK - 1) / kHeadK;
        }
    }
    static constexpr int kTileSteps = 3;                           // what a tile costs beside its steps, in steps
    // the CTA's i-th tile; false: it has no more
    __device__ __forceinline__ bool get(const HeadGemm &P, int i, HeadTile &w) const {
        const int t = cta + i * ctas;
        w.split = 0;
        if constexpr (MODE == HEAD_GRADS) {
            const int mine = t2 / ctas + (cta < extra);
            if (i < mine) {                                        // d hidden: a row block's columns next to one another
                const int r = t / hb;
                w.n = t % hb * kHeadN;
                w.m = r % mb * 128 * CG;
                w.split = r / mb;
                const int a = static_cast<int>(static_cast<long long>(k2) * w.split / P.splits), b = static_cast<int>(static_cast<long long>(k2) * (w.split + 1) / P.splits);
                w.k0 = a * kHeadK; w.ks = b - a;
                return true;
            }
            const int j = i - mine, before = ahead * (ctas - extra);      // tiles of the CTAs that are ahead
            const int u = cta < extra ? before + j * ctas + cta : j < ahead ? j * (ctas - extra) + cta - extra : before + (j - ahead) * ctas + cta;
            w.n = u % hb * kHeadN;
            w.m = u / hb * 128 * CG;
            w.split = -1;
            w.k0 = 0; w.ks = k3;
            return u < t3;
        } else {                                                   // the row blocks of a tile of the weight next to one another
            w.m = t % max(mb, 1) * 128 * CG;
            w.n = t / max(mb, 1) * P.bn;
            w.k0 = 0; w.ks = k2;
            return t < t2;
        }
    }
};

struct HeadShared {
    uint64_t full[6], empty[6], tfull[2], tempty[2], drain;
    uint32_t tmem;
    int error;
};

template <int MODE, int CG>
__global__ void __launch_bounds__(kHeadThreads, 1) tli_head_gemm_kernel(const __grid_constant__ HeadGemm P) {
    using R = HeadRing<CG>;
    extern __shared__ uint8_t head_smem[];
    __shared__ HeadShared sm;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = CG == 1 ? 0u : cluster_cta_rank();
    const uint32_t ring = (smem_addr(head_smem) + 1023u) & ~1023u, slab = ring + R::kStages * R::kStageBytes;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < R::kStages; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.tfull[i], 1); mbar_init(&sm.tempty[i], kHeadEpilogue * CG); }
        mbar_init(&sm.drain, 1);
        sm.error = 0;
        for (const CUtensorMap *map : {&P.a, &P.b, &P.a2, &P.b2, &P.out, &P.out2})
            if (MODE == HEAD_GRADS || (map != &P.a2 && map != &P.b2 && map != &P.out2 && (MODE == HEAD_SLOPE || map != &P.out)))
                asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sm.tmem)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tmem_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    tmem_fence_after();
    const uint32_t tmem = sm.tmem;
    const int cta = blockIdx.x / CG, ctas = gridDim.x / CG;
    // The weight's boxes of step k of a tile; stages are counted by it.
    auto load_weight = [&](const HeadTile &w, int k, unsigned st) {
        const uint32_t b = ring + st * R::kStageBytes + kHeadABytes, bar = CG == 1 ? smem_addr(&sm.full[st]) : cluster_addr(smem_addr(&sm.full[st]), 0u);
        const int x = w.k0 + k * kHeadK;
        if constexpr (MODE != HEAD_GRADS) {
            tensor_load<CG>(b, &P.b, x, P.c0 + w.n + static_cast<int>(rank) * (P.bn / CG), bar);
        } else {
            for (int i = 0; i < kHeadN / CG / 64; ++i) tensor_load<CG>(b + i * 8192, &P.b, w.n + static_cast<int>(rank) * (kHeadN / CG) + i * 64, P.c0 + x, bar);
        }
    };
    const unsigned bytes = CG * ((MODE == HEAD_GRADS ? static_cast<unsigned>(kHeadABytes) : P.a_rows * (kHeadK * 2u)) + static_cast<unsigned>((MODE == HEAD_GRADS ? kHeadN : P.bn) / CG) * (kHeadK * 2u));
    // The weight is an input of the call, and the call's first kernel lets its dependents start only when the kernels before the call are
    // done: it may be read before the kernels in between are.
    unsigned early = 0;
    if (P.early && threadIdx.x == 0) {
        HeadTile w;
        if (HeadTiles<MODE, CG>(P, 1, cta, ctas).get(P, 0, w) && w.split >= 0) {
            early = min(w.ks, R::kStages);
            for (unsigned k = 0; k < early; ++k) {
                if (rank == 0) mbar_arrive_expect_tx(&sm.full[k], bytes);
                load_weight(w, k, k);
            }
        }
    }
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int rows = *reinterpret_cast<const volatile int *>(P.n_valid);
    const HeadTiles<MODE, CG> tiles(P, rows, cta, ctas);
    HeadTile w;

    if (warp == 0) {
        if (lane == 0) {
            asm volatile("fence.proxy.async;" ::: "memory");       // what kernels before this one stored, to the copies' view
            unsigned it = 0;
            bool ok = true;
            for (int i = 0; ok && tiles.get(P, i, w); ++i) {
                const int m = w.m + static_cast<int>(rank) * 128;
                for (int k = 0; k < w.ks; ++k, ++it) {
                    const unsigned st = it % R::kStages, par = (it / R::kStages + 1) & 1u;
                    const uint32_t a = ring + st * R::kStageBytes, b = a + kHeadABytes;
                    const uint32_t bar = CG == 1 ? smem_addr(&sm.full[st]) : cluster_addr(smem_addr(&sm.full[st]), 0u);
                    const int x = w.k0 + k * kHeadK;
                    if (it >= early) {
                        ok = mbar_wait(&sm.empty[st], par, &sm.error, P.error);
                        if (!ok) break;
                        if (rank == 0) mbar_arrive_expect_tx(&sm.full[st], bytes);
                        if (MODE != HEAD_GRADS || w.split >= 0) load_weight(w, k, st);
                    }
                    if (MODE != HEAD_GRADS || w.split >= 0) {      // rows [rows, H], or G [rows, run], along the contracted axis
                        tensor_load<CG>(a, &P.a, x, m, bar);
                    } else {                                       // both across it
                        for (int i = 0; i < 2; ++i) tensor_load<CG>(a + i * 8192, &P.a2, m + i * 64, x, bar);
                        for (int i = 0; i < kHeadN / CG / 64; ++i) tensor_load<CG>(b + i * 8192, &P.b2, w.n + static_cast<int>(rank) * (kHeadN / CG) + i * 64, x, bar);
                    }
                }
            }
            // every stage handed back: no arrival is under way when the CTA leaves
            for (unsigned j = it > R::kStages ? it - R::kStages : 0; j < it && ok; ++j) ok = mbar_wait(&sm.empty[j % R::kStages], (j / R::kStages) & 1u, &sm.error, P.error);
            if (!ok && rank == 0) {                                // no CTA of the pair may leave while copies to it are in flight
                it = max(it, early);
                for (unsigned j = it > R::kStages ? it - R::kStages : 0; j < it; ++j)
                    for (unsigned i = 0; i < kWaitLimit && !mbar_test(&sm.full[j % R::kStages], (j / R::kStages) & 1u); ++i) __nanosleep(64);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t base = 1u << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(128 * CG >> 4) << 24;
            unsigned it = 0, acc = 0;
            bool ok = true;
            for (int i = 0; ok && tiles.get(P, i, w); ++i) {
                const bool dw = MODE == HEAD_GRADS && w.split < 0, dh = MODE == HEAD_GRADS && !dw;
                const int bn = MODE == HEAD_GRADS ? kHeadN : P.bn;
                const uint32_t idesc = base | static_cast<uint32_t>(bn >> 3) << 17 | (dw ? 1u << 15 | 1u << 16 : dh ? 1u << 16 : 0u);
                const uint32_t a_step = dw ? 128u : 2u, b_step = dw || dh ? 128u : 2u;        // 16 elements of the contracted axis, in 16 bytes
                const int part = MODE == HEAD_STATS ? P.k_part : max(w.ks, 1);
                for (int k0 = 0; ok && (k0 < w.ks || k0 == 0); k0 += part, ++acc) {
                    ok = mbar_wait(&sm.tempty[acc & 1], (acc >> 1 & 1u) ^ 1u, &sm.error, P.error);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t d = tmem + (acc & 1) * kHeadN;
                    for (int k = k0; k < min(w.ks, k0 + part); ++k, ++it) {
                        const unsigned st = it % R::kStages;
                        ok = mbar_wait(&sm.full[st], (it / R::kStages) & 1u, &sm.error, P.error);
                        if (!ok) break;
                        tmem_fence_after();
                        const uint32_t a = ring + st * R::kStageBytes, b = a + kHeadABytes;
                        // across: blocks of 64 are 8 KB apart, groups of 8 of the contracted axis 1 KB; along: groups of 8 rows 1 KB
                        uint64_t ad = dw ? umma_desc(a, 8192, 1024) : umma_desc(a, 16, 1024), bd = dw || dh ? umma_desc(b, 8192, 1024) : umma_desc(b, 16, 1024);
#pragma unroll
                        for (int i = 0; i < kHeadK / 16; ++i) umma<CG>(d, ad + i * a_step, bd + i * b_step, idesc, (k - k0 | i) != 0);
                        umma_commit<CG>(&sm.empty[st]);
                    }
                    if (ok) umma_commit<CG>(&sm.tfull[acc & 1]);
                }
            }
            if (!ok) {
                umma_commit<CG>(&sm.drain);
                for (unsigned i = 0; i < kWaitLimit && !mbar_test(&sm.drain, 0u); ++i) __nanosleep(64);
            }
        }
    } else {
        const int quarter = warp & 3, group = warp - 2 >> 2, row = quarter * 32 + lane, c0 = group * 128;
        const uint32_t mine = slab + (warp - 2) * kHeadSlab;       // this warp's slab
        const uint32_t tm = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + c0;
        unsigned acc = 0, turn = 0;
        bool ok = true;
        // 16 bytes of this thread's row of the slab; the slab is free again; the slab is full, and lane 0 may send it
        auto slab_put = [&](int i, const uint4 &v) { st_shared16(mine + lane * 128 + ((i ^ (lane & 7)) << 4), v); };
        auto slab_free = [&]() {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
        };
        auto slab_full = [&]() {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        };
        for (int i = 0; tiles.get(P, i, w); ++i) {
            const int m = w.m + static_cast<int>(rank) * 128, pos = m + row, m_warp = m + quarter * 32;
            // What depends on the row is a value here and no branch: a compiler that makes two paths of one (rows that count and rows that
            // do not) parts the warp in front of the instructions below that a whole warp has to take.  Where one lane alone has done
            // something (an arrival, a store), the warp meets again before it goes on to them.
            float s = 0.f, top = 0.f, f = 0.f;
            // (G is contracted over its rows in steps of kHeadK: the zeros of the last one are stored too)
            const int rows_stored = MODE == HEAD_SLOPE ? (rows + kHeadK - 1) / kHeadK * kHeadK : rows;
            uint32_t live = pos < rows ? 0xffffffffu : 0u, store = lane == 0 && (MODE == HEAD_GRADS && w.split < 0 ? P.c0 + m_warp < P.V : m_warp < rows_stored);
            asm volatile("" : "+r"(live), "+r"(store));
            if constexpr (MODE != HEAD_GRADS) {
                const float4 r = __ldg(P.rowp + max(0, min(pos, rows - 1)));
                s = r.x; top = r.y; f = r.z;
            }
            // A sum has been formed; (after a time-out the warps go on, tile by tile, with whatever tensor memory holds)
            auto sum_wait = [&]() {
                if (lane == 0) ok = ok && mbar_wait(&sm.tfull[acc & 1], acc >> 1 & 1u, &sm.error, P.error);
                __syncwarp();
                tmem_fence_after();
                return tm + (acc & 1) * kHeadN;
            };
            // ... and has been read
            auto sum_free = [&]() {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 1) mbar_arrive(&sm.tempty[acc & 1]);
                    else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr(smem_addr(&sm.tempty[acc & 1]), 0u)) : "memory");
                }
                __syncwarp();
                ++acc;
            };
            // which of 32 columns from column c of the tile on take part
            auto columns = [&](int c) {
                const int left = c < (MODE == HEAD_GRADS ? kHeadN : P.bn) ? P.cols - w.n - c : 0;
                uint32_t bits = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                if (P.mask && left > 0) bits &= __ldg(P.mask + ((P.c0 + w.n + c) >> 5));
                return bits;
            };
            // 32 columns of d hidden, this thread's row, over the ids inside the mask alone, without the matrix unit: for tiles that a weight
            // row outside the mask made NaN (a row that is NaN itself is none of them, and costs nothing).  2000 x 1024 x 49 152, half of the
            // ids inside: 25 ms a call, 0.46 without such a row; 1000 x 4096 x 128 256: 137 ms, no tile near the waits' limit of 17 s.
            auto inside_only = [&](float (&x)[32], int column) {
                const __nv_bfloat16 *g = P.G + max(0, min(pos, rows - 1)) * P.pitch, *wt = P.weight + P.c0 * P.weight_stride + column;
                const int end = min(w.k0 + w.ks * kHeadK, P.cols);
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = 0.f;
#pragma unroll 1
                for (int v = w.k0; v < end; v += 8) {              // (eight ids have their bits in one word: runs and splits begin at multiples of 64)
                    uint32_t in = __ldg(P.mask + ((P.c0 + v) >> 5)) >> ((P.c0 + v) & 31) & 0xffu;
                    if (end - v < 8) in &= (1u << (end - v)) - 1u;
                    if (!in) continue;
                    float gv[8];
                    unpack<TLI_BF16>(*reinterpret_cast<const uint4 *>(g + v), gv);
#pragma unroll
                    for (int u = 0; u < 8; ++u)
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            float y[8];
                            unpack<TLI_BF16>((in >> u & 1u) && column + i < P.H ? __ldg(reinterpret_cast<const uint4 *>(wt + (v + u) * P.weight_stride + i)) : make_uint4(0, 0, 0, 0), y);
#pragma unroll
                            for (int j = 0; j < 8; ++j) x[i + j] = fmaf(gv[u], y[j], x[i + j]);
                        }
                }
                __syncwarp();
            };
            if constexpr (MODE == HEAD_STATS) {
                const bool any = m_warp < rows && c0 < P.bn;       // the same for the warp
                float x[4][32];
                const uint32_t d0 = sum_wait();
#pragma unroll
                for (int q = 0; q < 4; ++q) tmem_load32(d0 + q * 32, x[q]);
                tmem_wait_load();
                sum_free();
#pragma unroll 1
                for (int k0 = P.k_part; k0 < w.ks; k0 += P.k_part) {
                    const uint32_t d = sum_wait();
                    if (any) {
#pragma unroll
                        for (int i0 = 0; i0 < 128; i0 += 16) {
                            float y[16];
                            tmem_load16(d + i0, y);
                            tmem_wait_load();
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i0 >> 5][(i0 & 31) + i] += y[i];
                        }
                    }
                    sum_free();
                }
                float best = kMaskBelow, sum = 0.f;
                if (any) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t bits = columns(c0 + q * 32);
                        if (bits != 0xffffffffu) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[q][i] = bits >> i & 1u ? x[q][i] : -INFINITY;
                        }
                    }
                    float high[4] = {best, best, best, best};
#pragma unroll
                    for (int i = 0; i < 128; ++i) high[i & 3] = fmaxf(high[i & 3], x[i >> 5][i & 31]);
                    best = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3]));
                    const uint64_t s2 = pack2(s, s), c2 = pack2(-best, -best);
                    uint64_t a2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < 128; i += 2) {
                        float y0, y1;
                        unpack2(mul2(add2(pack2(x[i >> 5][i & 31], x[i >> 5][i + 1 & 31]), c2), s2), y0, y1);
                        a2[i >> 1 & 3] = add2(a2[i >> 1 & 3], pack2(ex2(y0), ex2(y1)));
                    }
                    float w0, w1;
                    unpack2(add2(add2(a2[0], a2[1]), add2(a2[2], a2[3])), w0, w1);
                    sum = w0 + w1;
                }
                // the row's two pairs into one (the place is written again two tiles later at the earliest, behind the next tile's barrier)
                float2 *pairs = reinterpret_cast<float2 *>(head_smem + (slab - smem_addr(head_smem))) + (turn++ & 1) * 128;
                if (group) pairs[row] = make_float2(best, sum);
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (!group) {
                    const float2 o = pairs[row];
                    join_stats(s, best, sum, o.x, o.y);
                    if (live) P.part[static_cast<long long>(w.n / P.bn) * P.part_pitch + pos] = make_float2(best, sum);
                }
                __syncwarp();
            } else if constexpr (MODE == HEAD_SLOPE) {
                // The targets of the warp's 32 rows that lie among its columns: the warp reads all of them side by side and keeps a bit for
                // each (a thread through its own row's list: 0.19 ms a run instead of 0.08 for 32 targets per row).
                const int first = P.c0 + w.n + c0, entries = max(0, min(32, rows - m_warp)) * P.k;
                const long long base = static_cast<long long>(m_warp) * P.k;
                uint32_t hit[TLI_MAX_TARGETS / 32], hits = 0;
#pragma unroll
                for (int b = 0; b < TLI_MAX_TARGETS / 32; ++b) {
                    hit[b] = 0;
                    if (b * 32 >= P.k) continue;
#pragma unroll 8
                    for (int i = 0; i < 32; ++i) {
                        const int e = (b * 32 + i) * 32 + lane;
                        const int v = e < entries ? __ldg(P.tid + base + e) - first : -1;
                        hit[b] |= (static_cast<unsigned>(v) < 128u ? 1u : 0u) << i;
                    }
                    hits |= hit[b];
                }
                const bool some = __any_sync(0xffffffffu, hits != 0);
                const uint32_t d = sum_wait();
                const int columns_here = m_warp < rows_stored ? 128 : 0;      // (32 rows none of which is stored: nothing to do)
#pragma unroll 1
                for (int c = 0; c < columns_here; c += 64) {
                    float x[2][32];
                    tmem_load32(d + c, x[0]);
                    tmem_load32(d + c + 32, x[1]);
                    tmem_wait_load();
                    slab_free();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t bits = columns(c0 + c + h * 32) & live;
                        const bool whole = __all_sync(0xffffffffu, bits == 0xffffffffu);      // nothing to leave out, as in most tiles
                        const uint64_t s2 = pack2(s, s), t2 = pack2(-top, -top), f2 = pack2(f, f);
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            float y[8];
#pragma unroll
                            for (int j = 0; j < 8; j += 2) {
                                float a, b;
                                unpack2(mul2(add2(pack2(x[h][i + j], x[h][i + j + 1]), t2), s2), a, b);
                                unpack2(mul2(pack2(ex2(a), ex2(b)), f2), y[j], y[j + 1]);
                            }
                            if (!whole) {
#pragma unroll
                                for (int j = 0; j < 8; ++j) y[j] = bits >> (i + j) & 1u ? y[j] : 0.f;
                            }
                            slab_put(h * 4 + i / 8, pack_vector<TLI_BF16>(y));
                        }
                    }
                    if (some) {
                        __syncwarp();
#pragma unroll
                        for (int b = 0; b < TLI_MAX_TARGETS / 32; ++b)
                            for (uint32_t left = hit[b]; left; left &= left - 1) {
                                const int e = (b * 32 + __ffs(left) - 1) * 32 + lane, v = __ldg(P.tid + base + e) - first - c, r = e / P.k;
                                if (static_cast<unsigned>(v) < 64u)
                                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(mine + r * 128 + (((v >> 3) ^ (r & 7)) << 4) + (v & 7) * 2),
                                                 "h"(__bfloat16_as_ushort(__float2bfloat16_rn(__ldg(P.tval + base + e)))) : "memory");
                            }
                        __syncwarp();
                    }
                    slab_full();
                    if (store) tensor_store(&P.out, w.n + c0 + c, m_warp, mine);
                    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    __syncwarp();
                }
                sum_free();
            } else if (w.split >= 0) {                             // d hidden: fp32 sums, 32 columns a slab
                const uint32_t d = sum_wait();
#pragma unroll 1
                for (int h = 0; h < 128 && w.n + c0 + h < P.H && m_warp < rows; h += 32) {
                    float x[32];
                    tmem_load32(d + h, x);
                    tmem_wait_load();
                    slab_free();
                    if (w.ks == 0) {                               // (a split of a short run may have no step)
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = 0.f;
                    } else if (P.mask) {                           // G is 0 outside the mask, but 0 times a weight that is no number is none
                        float none = 0.f;
#pragma unroll
                        for (int i = 0; i < 32; ++i) none = fmaf(x[i], 0.f, none);
                        if (__any_sync(0xffffffffu, none != none && pos < rows && isfinite(__ldg(P.rowp + max(0, min(pos, rows - 1))).z)))
                            inside_only(x, w.n + c0 + h);
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        slab_put(i / 4, make_uint4(__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3])));
                    }
                    slab_full();
                    if (store) tensor_store3(&P.out2, w.n + c0 + h, m_warp, w.split, mine, !P.first);
                    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    __syncwarp();
                }
                sum_free();
            } else {                                               // d weight: bf16, 64 columns a slab
                const uint32_t d = sum_wait();
#pragma unroll 1
                for (int c = 0; c < 128 && w.n + c0 + c < P.H; c += 64) {
                    float x[2][32];
                    tmem_load32(d + c, x[0]);
                    tmem_load32(d + c + 32, x[1]);
                    tmem_wait_load();
                    slab_free();
                    if (w.ks == 0) {                               // (no row takes part)
#pragma unroll
                        for (int i = 0; i < 64; ++i) x[i >> 5][i & 31] = 0.f;
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            float y[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = x[h][i + j];
                            slab_put(h * 4 + i / 8, pack_vector<TLI_BF16>(y));
                        }
                    slab_full();
                    if (store) tensor_store(&P.out, w.n + c0 + c, P.c0 + m_warp, mine);
                    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    __syncwarp();
                }
                sum_free();
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    if (warp == 1) {
        tmem_fence_after();
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// ---- rows and targets ----

constexpr int kHeadNear = 4;

struct HeadRows {
    TargetParams T;
    int H, V;
    const __nv_bfloat16 *hidden; long long hidden_stride; int vec;     // vec: rows lie on 16-byte boundaries
    const __nv_bfloat16 *weight; long long weight_stride;
    const float *g;
    float *loss, *stats, *target_logits;
    int *status;
    const unsigned *error;
    // in the workspace
    uint32_t *taking;                      // a bit per row, a byte per CTA of the targets kernel
    int *n_valid, *pos;                    // rows that take part; place of a row among them, -1
    float4 *by_row, *rowp;                 // {s, m, f, -} of a row; of the rows that take part, in their order
    int *tid; float *tval;                 // gradient: the targets' ids (-1) and elements of G, of all rows
    int *tid_of; float *tval_of;           // ... of the rows that take part, in their order
    int *near_id; float *near_off;         // ... the kHeadNear largest of a row, and what bf16 leaves off them
    __nv_bfloat16 *rows;                   // [N, H]
    const float2 *part; long long part_pitch; int tiles;
    const float *sums; int splits, groups; // d hidden: [splits][N, H]; threads that share them
    __nv_bfloat16 *grad_hidden; long long grad_hidden_stride; int out_vec;
};

// Row `row` by one warp: whether it takes part, and in r what a tile of it needs.  GRAD: also its targets' elements, g/tau (q - mass).
// Q: targets per lane, 1, 2, 4 or TLI_MAX_TARGETS / 32 (the short forms have less code: read once, code is what these kernels wait for).
template <bool GRAD, int Q> __device__ __forceinline__ bool head_row(const HeadRows &P, long long row, float4 &r) {
    const int lane = threadIdx.x & 31, k = P.T.k;
    int id[Q];
    float t[Q];
    bool any = false;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        id[q] = -1; t[q] = 0.f;
        if (q * 32 + lane < k) id[q] = row_target(P.T, row, q * 32 + lane, t[q]);
        any |= id[q] >= 0;
    }
    any = __any_sync(0xffffffffu, any);
    float tau, s;
    const bool scale_ok = row_scale(P.T.tau, row, tau, s);
    bool takes = any && scale_ok;
    const int status = (any ? 0 : TLI_ROW_LEFT_OUT) | (scale_ok ? 0 : TLI_ROW_BAD_TEMPERATURE);
    r = make_float4(s, 0.f, 0.f, 0.f);
    if constexpr (GRAD) {
        const RowSlope slope(P.T.tau, P.stats, P.g, row);
        takes = takes && !slope.zero;
        r.y = slope.m; r.z = slope.f;
        if (takes) {
            float mass[Q], W = 1.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) mass[q] = 1.f;
            if (P.T.teacher) {
                float tm = -INFINITY, w[Q];
#pragma unroll
                for (int q = 0; q < Q; ++q) if (id[q] >= 0) tm = fmaxf(tm, t[q]);
                tm = warp_max(tm);
                W = 0.f;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    w[q] = id[q] >= 0 ? ex2((t[q] - tm) * s) : 0.f;
                    W += w[q];
                    mass[q] = 0.f;
                }
                W = warp_sum(W);
#pragma unroll
                for (int b = 0; b < Q; ++b) {
                    if (b * 32 >= k) break;
#pragma unroll 8
                    for (int l = 0; l < 32; ++l) {
                        const int other = __shfl_sync(0xffffffffu, id[b], l);
                        const float more = __shfl_sync(0xffffffffu, w[b], l);
#pragma unroll
                        for (int q = 0; q < Q; ++q) {
                            if (q * 32 >= k) break;
                            mass[q] += id[q] == other ? more : 0.f;
                        }
                    }
                }
            }
            float val[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const long long at = row * k + q * 32 + lane;
                if (q * 32 + lane >= k) break;
                P.tid[at] = id[q];
                if (id[q] >= 0) P.tval[at] = val[q] = fmaf(-slope.h, mass[q] / W, slope(__ldg(P.target_logits + at)));
            }
            // The row's few largest elements of G are most of it, and their rounding most of the error of d hidden: what it leaves off is kept.
            // (The same id twice is one element.)
#pragma unroll 1
            for (int n = 0; n < kHeadNear; ++n) {
                float most = -1.f, v = 0.f;
                int v_id = -1;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (q * 32 >= k) break;
                    if (id[q] >= 0 && fabsf(val[q]) > most) { most = fabsf(val[q]); v = val[q]; v_id = id[q]; }
                }
                const float all = warp_max(most);
                const unsigned who = __ballot_sync(0xffffffffu, v_id >= 0 && most == all);
                const int from = who ? __ffs(who) - 1 : 0;
                v = __shfl_sync(0xffffffffu, v, from);
                v_id = who ? __shfl_sync(0xffffffffu, v_id, from) : -1;
                if (lane == 0) {
                    P.near_id[row * kHeadNear + n] = v_id;
                    P.near_off[row * kHeadNear + n] = v - __bfloat162float(__float2bfloat16_rn(v));
                }
#pragma unroll
                for (int q = 0; q < Q; ++q) id[q] = id[q] == v_id ? -1 : id[q];
            }
        }
    }
    if (lane == 0 && P.status) P.status[row] = status | (!takes && !status ? TLI_ROW_FALLBACK : 0);
    return takes;
}
// The same question alone, by one thread.
template <bool GRAD> __device__ __forceinline__ bool head_takes(const HeadRows &P, long long row) {
    float tau, s, t;
    if (!row_scale(P.T.tau, row, tau, s) || (GRAD && __ldg(P.stats + 2 * row + 1) == 0.f)) return false;
    for (int j = 0; j < P.T.k; ++j)
        if (row_target(P.T, row, j, t) >= 0) return true;
    return false;
}
// A row of `hidden` (and its targets, for the gradient) to its place, by one warp: the first 256 vectors are read ahead of knowing it.
struct HeadCopy {
    static constexpr int kAhead = 8;
    uint4 v[kAhead];
    __device__ __forceinline__ void load(const HeadRows &P, long long row) {
        if (!P.vec) return;
        const uint4 *from = reinterpret_cast<const uint4 *>(P.hidden + row * P.hidden_stride);
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int i = (threadIdx.x & 31) + q * 32;
            if (i < P.H / 8) v[q] = __ldg(from + i);
        }
    }
    __device__ __forceinline__ void store(const HeadRows &P, long long row, long long pos) const {
        const int lane = threadIdx.x & 31;
        if (P.tid_of)
            for (int j = lane; j < P.T.k; j += 32) {               // (by the lanes that have written them, if this kernel has)
                P.tid_of[pos * P.T.k + j] = __ldcg(P.tid + row * P.T.k + j);
                P.tval_of[pos * P.T.k + j] = __ldcg(P.tval + row * P.T.k + j);
            }
        __nv_bfloat16 *to = P.rows + pos * P.H;
        const __nv_bfloat16 *from = P.hidden + row * P.hidden_stride;
        if (P.vec) {
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (lane + q * 32 < P.H / 8) reinterpret_cast<uint4 *>(to)[lane + q * 32] = v[q];
#pragma unroll 8
            for (int i = lane + kAhead * 32; i < P.H / 8; i += 32) reinterpret_cast<uint4 *>(to)[i] = __ldg(reinterpret_cast<const uint4 *>(from) + i);
        } else {
#pragma unroll 4
            for (int i = lane; i < P.H; i += 32) to[i] = from[i];
        }
    }
};
// The number of rows that take part, and zeros behind them up to the next multiple of kHeadK (the contraction of d weight goes that far).
__device__ __forceinline__ void head_end(const HeadRows &P, int total) {
    if (threadIdx.x == 0) *P.n_valid = total;
    const long long end = min(static_cast<long long>(P.T.N), (static_cast<long long>(total) + kHeadK - 1) / kHeadK * kHeadK);
    const long long nv = (end - total) * (P.H / 8);
    for (long long i = threadIdx.x; i < nv; i += blockDim.x) reinterpret_cast<uint4 *>(P.rows + static_cast<long long>(total) * P.H)[i] = make_uint4(0, 0, 0, 0);
}

constexpr int kGatherThreads = 256, kGatherRows = kGatherThreads / 32;
constexpr int kHeadOneLaunch = 1024;       // lookups up to which every CTA looks at all rows before its own, instead of a launch that does

// Few rows: both steps at once.  Eight warps have a row each, eight more count those before them meanwhile.
template <bool GRAD, int Q>
__global__ void __launch_bounds__(2 * kGatherThreads, 1) tli_head_prepare_kernel(const __grid_constant__ HeadRows P) {
    __shared__ int sums[kGatherRows], taking[kGatherRows];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row0 = blockIdx.x * kGatherRows, row = row0 + warp;
    bool takes = false;
    float4 r;
    HeadCopy copy;
    if (warp < kGatherRows) {
        if (row < P.T.N) {
            copy.load(P, row);                                     // (on its way while the targets are looked up)
            takes = head_row<GRAD, Q>(P, row, r);
        }
        if (lane == 0) taking[warp] = takes;
    } else {
        int before = 0;
        if (P.T.k == 1 && !P.T.teacher) {                          // labels: four rows' lookups at a time, step by step
#pragma unroll 1
            for (int i0 = threadIdx.x - kGatherThreads; i0 < row0; i0 += 4 * kGatherThreads) {
                int id[4];
                bool in[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = i0 + q * kGatherThreads;
                    in[q] = i < row0;
                    id[q] = in[q] ? __ldg(P.T.ids + i) : -1;
                    float tau, s;
                    if (in[q]) in[q] = (!P.T.tau || row_scale(P.T.tau, i, tau, s)) && !(GRAD && __ldg(P.stats + 2 * i + 1) == 0.f);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) id[q] = table_id(P.T.map, P.T.n_ids, id[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) before += in[q] && id[q] >= 0 && (!P.T.mask || (__ldg(P.T.mask + (id[q] >> 5)) >> (id[q] & 31) & 1u));
            }
        } else {
            for (int i = threadIdx.x - kGatherThreads; i < row0; i += kGatherThreads) before += head_takes<GRAD>(P, i);
        }
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) sums[warp - kGatherRows] = before;
    }
    __syncthreads();
    // (Not before the wait: see the early loads of the weight.  And not before the lookups: behind 28 MB of weight each of them took 4 us.)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int total = 0, pos = 0;
#pragma unroll
    for (int i = 0; i < kGatherRows; ++i) {
        total += sums[i] + taking[i];
        pos += sums[i] + (i < warp ? taking[i] : 0);
    }
    if (warp < kGatherRows && row < P.T.N) {
        if (lane == 0) {
            P.pos[row] = takes ? pos : -1;
            if (takes) P.rowp[pos] = r;
        }
        if (takes) copy.store(P, row, pos);
    }
    if (blockIdx.x == gridDim.x - 1) head_end(P, total);
}

// A bit per row, eight rows per CTA.
template <bool GRAD, int Q>
__global__ void __launch_bounds__(kGatherThreads) tli_head_targets_kernel(const __grid_constant__ HeadRows P) {
    __shared__ int taking[kGatherRows];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // (not before: see the early loads of the weight)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * kGatherRows + warp;
    bool takes = false;
    if (row < P.T.N) {
        float4 r;
        takes = head_row<GRAD, Q>(P, row, r);
        if (lane == 0) P.by_row[row] = r;
    }
    if (lane == 0) taking[warp] = takes;
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < kGatherRows; ++i) bits |= static_cast<unsigned>(taking[i]) << i;
        reinterpret_cast<unsigned char *>(P.taking)[blockIdx.x] = static_cast<unsigned char>(bits);
    }
}

// The rows that take part, in order, a warp each.
__global__ void __launch_bounds__(kGatherThreads) tli_head_gather_kernel(const __grid_constant__ HeadRows P) {
    __shared__ int sums[kGatherRows];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row = blockIdx.x * kGatherRows + warp, at = row / 32;
    HeadCopy copy;
    if (row < P.T.N) copy.load(P, row);                            // (an input of the call: before the targets are there)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int before = 0;
    for (int i = threadIdx.x; i < at; i += kGatherThreads) before += __popc(__ldcg(P.taking + i));
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) sums[warp] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int i = 0; i < kGatherRows; ++i) before += sums[i];
    uint32_t word = __ldcg(P.taking + at);
    if (P.T.N - at * 32 < 32) word &= (1u << (P.T.N - at * 32)) - 1u;     // (of the last word only the rows there are)
    if (row < P.T.N) {
        const int bit = row & 31;
        const bool takes = word >> bit & 1u;
        const int pos = before + __popc(word & ((1u << bit) - 1u));
        if (lane == 0) {
            P.pos[row] = takes ? pos : -1;
            if (takes) P.rowp[pos] = __ldcg(P.by_row + row);
        }
        if (takes) copy.store(P, row, pos);
    }
    if (blockIdx.x == gridDim.x - 1) head_end(P, before + __popc(word));
}

// ---- forward: the loss ----

__device__ __forceinline__ float dot_bf16(const uint4 &a, const uint4 &b, float acc) {
    float x[8], y[8];
    unpack<TLI_BF16>(a, x);
    unpack<TLI_BF16>(b, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = fmaf(x[i], y[i], acc);
    return acc;
}
// ROWS rows per CTA: eight, a warp each, for few targets; one, its targets dealt out to the warps four at a time, for more.  (Beyond 128 targets the 64
// registers of four CTAs per SM leave 124 bytes a thread in local memory.)
template <int Q, int ROWS>
__global__ void __launch_bounds__(256, 4) tli_head_loss_kernel(const __grid_constant__ HeadRows P) {
    __shared__ float sh_m[256 / ROWS][ROWS], sh_s[256 / ROWS][ROWS], sh_z[ROWS == 1 ? Q * 32 : 1];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, k = P.T.k;
    const long long row0 = static_cast<long long>(blockIdx.x) * ROWS, row = row0 + (ROWS == 1 ? 0 : warp), at = row * k;
    // The targets' logits are made of the call's inputs: a CTA on an SM without products (one token: 143 tiles on 148 SMs) begins with them.  Beside a CTA of
    // the products there is no room, their ring leaves 1792 bytes of shared memory.
    int id[Q];
    float t[Q], z[Q], tau = 1.f, s = 1.f;
    bool takes = false;
#pragma unroll
    for (int q = 0; q < Q; ++q) { id[q] = -1; t[q] = 0.f; z[q] = 0.f; }
    if (row < P.T.N) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (q * 32 + lane < k) id[q] = row_target(P.T, row, q * 32 + lane, t[q]);
            takes |= id[q] >= 0;
        }
        takes = __any_sync(0xffffffffu, takes);
        takes = row_scale(P.T.tau, row, tau, s) && takes;
    }
    if (takes) {
        const __nv_bfloat16 *h = P.hidden + row * P.hidden_stride;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (q * 32 >= k) break;
#pragma unroll 1
            for (int l = ROWS == 1 ? warp * 4 : 0; l < 32 && q * 32 + l < k; l += ROWS == 1 ? 32 : 4) {
                float dot[4] = {};
                const __nv_bfloat16 *w[4];
                bool on[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int v = __shfl_sync(0xffffffffu, id[q], l + u);
                    on[u] = v >= 0;
                    w[u] = P.weight + max(v, 0) * P.weight_stride;
                }
                if (P.vec) {
#pragma unroll 2
                    for (int i = lane; i < P.H / 8; i += 32) {
                        const uint4 x = __ldg(reinterpret_cast<const uint4 *>(h) + i);
                        uint4 y[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) y[u] = on[u] ? __ldg(reinterpret_cast<const uint4 *>(w[u]) + i) : make_uint4(0, 0, 0, 0);
#pragma unroll
                        for (int u = 0; u < 4; ++u) if (on[u]) dot[u] = dot_bf16(x, y[u], dot[u]);
                    }
                } else {
                    for (int i = lane; i < P.H; i += 32) {
                        const float x = __bfloat162float(h[i]);
#pragma unroll
                        for (int u = 0; u < 4; ++u) if (on[u]) dot[u] = fmaf(x, __bfloat162float(w[u][i]), dot[u]);
                    }
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    dot[u] = warp_sum(dot[u]);
                    if (ROWS == 1 && lane == u) sh_z[q * 32 + l + u] = on[u] ? dot[u] : 0.f;
                    if (ROWS > 1 && l + u == lane && on[u]) z[q] = dot[u];
                }
            }
        }
    }
    if (ROWS == 1) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < Q; ++q) if (id[q] >= 0 && takes) z[q] = sh_z[q * 32 + lane];
    }
    float tau_r = 1.f, s_r = 1.f;                                  // of the row whose tiles this thread joins
    if (row0 + threadIdx.x % ROWS < P.T.N) row_scale(P.T.tau, row0 + threadIdx.x % ROWS, tau_r, s_r);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (row < P.T.N && (ROWS > 1 || warp == 0)) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (q * 32 + lane < k) P.target_logits[at + q * 32 + lane] = z[q];
    }
    {
        const int r = threadIdx.x % ROWS, t0 = threadIdx.x / ROWS; // neighbouring threads: neighbouring rows of a tile
        const int pos = row0 + r < P.T.N ? __ldcg(P.pos + row0 + r) : -1;
        float m = kMaskBelow, sum = 0.f;
        if (pos >= 0) {
            const float2 *part = P.part + pos;
#pragma unroll 1
            for (int i = t0; i < P.tiles; i += 256 / ROWS * 4) {
                float2 p[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) p[q] = i + q * (256 / ROWS) < P.tiles ? __ldcg(part + (i + q * (256 / ROWS)) * P.part_pitch) : make_float2(kMaskBelow, 0.f);
#pragma unroll
                for (int q = 0; q < 4; ++q) join_stats(s_r, m, sum, p[q].x, p[q].y);
            }
        }
        sh_m[t0][r] = m; sh_s[t0][r] = sum;
    }
    __syncthreads();
    if (row >= P.T.N || (ROWS == 1 && warp > 0)) return;
    const int timeout = *reinterpret_cast<const volatile unsigned *>(P.error) ? TLI_ROW_TIMEOUT : 0;
    if (!takes) {
        if (lane == 0) {
            P.loss[row] = 0.f;
            reinterpret_cast<float2 *>(P.stats)[row] = make_float2(0.f, 0.f);
            if (P.status && timeout) P.status[row] |= timeout;
        }
        return;
    }
    float m = sh_m[lane][warp], sum = sh_s[lane][warp];
#pragma unroll
    for (int i = 32; i < 256 / ROWS; i += 32) join_stats(s, m, sum, sh_m[lane + i][warp], sh_s[lane + i][warp]);
    const float top = warp_max(m);
    sum = warp_sum(sum * ex2((m - top) * s));
    m = top;
    float W = 1.f, ent;
    if (P.T.teacher) {
        float tm = -INFINITY;
#pragma unroll
        for (int q = 0; q < Q; ++q) if (id[q] >= 0) tm = fmaxf(tm, t[q]);
        tm = warp_max(tm);
        W = 0.f; ent = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float w = id[q] >= 0 ? ex2((t[q] - tm) * s) : 0.f;
            W += w;
            if (w != 0.f) ent += w * (((m - z[q]) + (t[q] - tm)) / tau);
        }
        W = warp_sum(W);
        ent = warp_sum(ent);
    } else {
        ent = (m - z[0]) / tau;                                    // of lane 0
    }
    if (lane == 0) {
        const bool none = sum == 0.f, bad = sum != sum || W != W;
        P.loss[row] = none ? 0.f : bad ? NAN : logf(sum) + (P.T.teacher ? ent / W - logf(W) : ent);
        reinterpret_cast<float2 *>(P.stats)[row] = none ? make_float2(0.f, 0.f) : make_float2(m, bad ? NAN : sum);
        if (P.status) P.status[row] = timeout | (none ? TLI_ROW_FALLBACK : bad ? TLI_ROW_NONFINITE : 0);
    }
}

// ---- backward: d hidden at its rows' places ----

// Four columns of a row by P.groups threads, which share the splits (3 rows of 96 columns in 148 splits by one thread each: 35 us).
constexpr int kRowsThreads = 256;
template <bool SHARED>
__global__ void __launch_bounds__(kRowsThreads) tli_head_rows_kernel(const __grid_constant__ HeadRows P) {
    __shared__ float4 shared[SHARED ? kRowsThreads : 1];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int groups = SHARED ? P.groups : 1, units = P.H / 4, tx = kRowsThreads / groups, group = SHARED ? threadIdx.x / tx : 0;
    const long long i = static_cast<long long>(blockIdx.x) * tx + threadIdx.x % tx, row = i / units;
    const bool in = i < static_cast<long long>(P.T.N) * units;
    const int u = static_cast<int>(i % units), pos = in ? __ldcg(P.pos + row) : -1;
    if (in && group == 0 && u == 0 && P.status && *reinterpret_cast<const volatile unsigned *>(P.error)) P.status[row] |= TLI_ROW_TIMEOUT;
    if (!P.grad_hidden) return;
    float x[4] = {};
    if (pos >= 0) {
        const float *p = P.sums + static_cast<long long>(pos) * P.H + u * 4;
        const long long next = static_cast<long long>(P.T.N) * P.H;
#pragma unroll 1
        for (int sp = group; sp < P.splits; sp += 8 * groups) {
            float4 a[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) a[q] = sp + q * groups < P.splits ? __ldcg(reinterpret_cast<const float4 *>(p + (sp + q * groups) * next)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 8; ++q) { x[0] += a[q].x; x[1] += a[q].y; x[2] += a[q].z; x[3] += a[q].w; }
        }
    }
    if (SHARED) {
        shared[threadIdx.x] = make_float4(x[0], x[1], x[2], x[3]);
        __syncthreads();
        if (group == 0)
            for (int g = 1; g < groups; ++g) {
                const float4 a = shared[g * tx + threadIdx.x];
                x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
            }
    }
    if (group > 0 || !in) return;
    if (pos >= 0) {
#pragma unroll
        for (int n = 0; n < kHeadNear; ++n) {
            const int v = __ldcg(P.near_id + row * kHeadNear + n);
            if (v < 0) break;
            const float off = __ldcg(P.near_off + row * kHeadNear + n);
            const uint2 w = __ldg(reinterpret_cast<const uint2 *>(P.weight + v * P.weight_stride + u * 4));
            x[0] = fmaf(off, bf16_lo(w.x), x[0]); x[1] = fmaf(off, bf16_hi(w.x), x[1]);
            x[2] = fmaf(off, bf16_lo(w.y), x[2]); x[3] = fmaf(off, bf16_hi(w.y), x[3]);
        }
    }
    __nv_bfloat16 *to = P.grad_hidden + row * P.grad_hidden_stride + u * 4;
    if (P.out_vec) {
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[2 * j + 1]), "f"(x[2 * j]));
        *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = __float2bfloat16_rn(x[j]);
    }
}

// ---- host ----

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}
// [outer, inner] of bf16 or fp32 elements with `pitch` elements from row to row ([depth, outer, inner] if depth > 0, slices one after the
// other), boxes of 128 bytes x `box` rows.
bool tensor_map(CUtensorMap *map, bool f32, const void *base, long long inner, long long outer, long long pitch, int box, long long depth = 0) {
    const EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t elt = f32 ? 4 : 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(outer), static_cast<cuuint64_t>(depth)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(pitch) * elt, static_cast<cuuint64_t>(pitch) * outer * elt};
    const cuuint32_t boxes[3] = {static_cast<cuuint32_t>(128 / elt), static_cast<cuuint32_t>(box), 1}, ones[3] = {1, 1, 1};
    return fn(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, depth > 0 ? 3 : 2, const_cast<void *>(base), dims, strides, boxes, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr long long kHeadRunBytes = 256ll << 20;       // of G
constexpr int kHeadMinSteps = 8;                       // of the contraction in a split of d hidden

struct HeadPlan {
    int cg, bn, tiles;                     // CTAs per tile; columns of a forward tile, tiles of the vocabulary
    int run, runs, splits;                 // backward: columns of a run of G, runs, cuts of d hidden's contraction
    size_t taking, n_valid, pos, by_row, rowp, tid, tval, tid_of, tval_of, near_id, near_off, rows, part, G, sums, total;
};

HeadPlan head_plan(int N, int H, int k, int V, int num_sms, bool grad) {
    HeadPlan L;
    memset(&L, 0, sizeof L);
    // One CTA per tile where one row block holds all rows: the weight is then read once, whoever reads it.
    L.cg = N <= 128 ? 1 : 2;
    L.bn = kHeadN;
    if (!grad && L.cg == 1) {
        // The weight streams through the SMs: the width that leaves the last wave fullest (a CTA's time is waves * columns).
        long long best = -1;
        for (int bn = kHeadN; bn >= 64; bn -= 32) {
            const long long tiles = (V + bn - 1) / bn, time = (tiles + num_sms - 1) / num_sms * bn;
            if (best < 0 || time < best) { best = time; L.bn = bn; }
        }
    }
    L.tiles = (V + L.bn - 1) / L.bn;
    size_t off = 0;
    const size_t n = static_cast<size_t>(N), words = (n + 31) / 32;
    auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
    L.taking = take(4 * words);
    L.n_valid = take(4);
    L.pos = take(4 * n);
    L.by_row = take(16 * n);
    L.rowp = take(16 * n);
    L.rows = take(2 * n * H);
    if (!grad) {
        L.part = take(8 * n * L.tiles);
    } else {
        const long long most = std::max<long long>(kHeadN, kHeadRunBytes / (2ll * std::max(N, 1)) / kHeadN * kHeadN);
        L.runs = static_cast<int>((V + most - 1) / most);
        L.run = static_cast<int>(align_up((V + L.runs - 1) / L.runs, kHeadN));
        L.runs = (V + L.run - 1) / L.run;
        const int blocks = (N + 128 * L.cg - 1) / (128 * L.cg) * ((H + kHeadN - 1) / kHeadN), steps = (std::min(V, L.run) + kHeadK - 1) / kHeadK;
        L.splits = std::max(1, std::min(num_sms / L.cg / std::max(blocks, 1), steps / kHeadMinSteps));
        L.tid = take(4 * n * k);
        L.tval = take(4 * n * k);
        L.tid_of = take(4 * n * k);
        L.tval_of = take(4 * n * k);
        L.near_id = take(4 * n * kHeadNear);
        L.near_off = take(4 * n * kHeadNear);
        L.G = take(2 * n * L.run);
        L.sums = take(4 * n * H * L.splits);
    }
    L.total = off;
    return L;
}

template <int MODE, int CG> int launch_head_gemm(const HeadGemm &P, const tli_ctx *ctx, long long tiles, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    pdl_config(cfg, attr, stream);
    if (CG == 2) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    static SmemAllowed allowed;
    cudaError_t e = allowed.set(reinterpret_cast<const void *>(tli_head_gemm_kernel<MODE, CG>), HeadRing<CG>::kSmem, ctx->device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
    cfg.gridDim = dim3(static_cast<unsigned>(std::max<long long>(1, std::min<long long>(tiles, ctx->num_sms / CG)) * CG));
    cfg.blockDim = dim3(kHeadThreads);
    cfg.dynamicSmemBytes = HeadRing<CG>::kSmem;
    e = cudaLaunchKernelEx(&cfg, tli_head_gemm_kernel<MODE, CG>, P);
    return e == cudaSuccess ? TLI_OK : cuda_fail(e, "launch tli_head_gemm_kernel");
}
template <int MODE> int launch_head_gemm(const HeadGemm &P, int cg, const tli_ctx *ctx, long long tiles, cudaStream_t stream) {
    return cg == 1 ? launch_head_gemm<MODE, 1>(P, ctx, tiles, stream) : launch_head_gemm<MODE, 2>(P, ctx, tiles, stream);
}
template <typename K> int launch_plain(K kernel, const HeadRows &P, long long blocks, int threads, cudaStream_t stream, const char *what) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, stream);
    cfg.gridDim = dim3(static_cast<unsigned>(blocks)); cfg.blockDim = dim3(threads);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P);
    return e == cudaSuccess ? TLI_OK : cuda_fail(e, what);
}

// Which rows take part, and those one after the other.
template <bool GRAD, int Q> int launch_head_rows(const HeadRows &R, cudaStream_t stream) {
    const long long N = R.T.N, gathers = (N + kGatherRows - 1) / kGatherRows;
    if (Q == 1 && N * R.T.k <= kHeadOneLaunch) return launch_plain(tli_head_prepare_kernel<GRAD, 1>, R, gathers, 2 * kGatherThreads, stream, "launch tli_head_prepare_kernel");
    const int rc = launch_plain(tli_head_targets_kernel<GRAD, Q>, R, gathers, kGatherThreads, stream, "launch tli_head_targets_kernel");
    return rc == TLI_OK ? launch_plain(tli_head_gather_kernel, R, gathers, kGatherThreads, stream, "launch tli_head_gather_kernel") : rc;
}
template <bool GRAD> int launch_head_rows(const HeadRows &R, cudaStream_t stream) {
    if (R.T.k <= 32) return launch_head_rows<GRAD, 1>(R, stream);
    if (R.T.k <= 64) return launch_head_rows<GRAD, 2>(R, stream);
    return R.T.k <= 128 ? launch_head_rows<GRAD, 4>(R, stream) : launch_head_rows<GRAD, TLI_MAX_TARGETS / 32>(R, stream);
}

size_t head_workspace(const tli_ctx *ctx, int32_t N, int32_t H, int32_t k, int32_t side, bool grad) {
    if (!ctx || ctx->n_shards != 1 || N < 0 || N > TLI_MAX_HEAD_TOKENS || H < 8 || H > TLI_MAX_H || H % 8 || k < 1 || k > TLI_MAX_TARGETS) return 0;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return 0;
    return head_plan(N, H, k, side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d, ctx->num_sms, grad).total;
}

// The bytes from the first to the last element of a bf16 matrix.
struct Span {
    const char *begin, *end;
    Span(const void *p, int64_t rows, int64_t stride, int64_t width) : begin(static_cast<const char *>(p)), end(begin) {
        if (p && rows > 0) end += ((rows - 1) * stride + width) * 2;
    }
    bool meets(const Span &o) const { return begin < o.end && o.begin < end; }
};

// What both head calls check and set up alike.
int prepare_head(const tli_ctx *ctx, int32_t N, int32_t H, int32_t k, int32_t side, int32_t ids_side, int32_t support, const void *hidden, int64_t hidden_stride,
                 const void *weight, int64_t weight_stride, const int32_t *ids, const void *teacher, int32_t teacher_dtype, const float *temperature, void *workspace,
                 size_t workspace_bytes, bool grad, HeadRows &R, HeadPlan &L) {
    memset(&R, 0, sizeof R);
    int V;
    const int rc = check_targets(ctx, N, k, side, ids_side, support, ids, teacher, teacher_dtype, temperature, R.T, V);
    if (rc != TLI_OK) return rc;
    if (H < 8 || H % 8) return TLI_ERR_ARG;
    if (N > TLI_MAX_HEAD_TOKENS || H > TLI_MAX_H) return TLI_ERR_UNSUPPORTED;
    if ((N > 0 && !hidden) || reinterpret_cast<uintptr_t>(hidden) % 2 || hidden_stride < 0) return TLI_ERR_ARG;
    if (!weight || !on_vectors(weight, weight_stride, 2) || weight_stride < H) return TLI_ERR_ARG;
    L = head_plan(N, H, k, V, ctx->num_sms, grad);
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < L.total) return TLI_ERR_WORKSPACE;
    char *ws = reinterpret_cast<char *>(workspace);
    R.H = H; R.V = V;
    R.hidden = reinterpret_cast<const __nv_bfloat16 *>(hidden); R.hidden_stride = hidden_stride; R.vec = on_vectors(hidden, hidden_stride, 2);
    R.weight = reinterpret_cast<const __nv_bfloat16 *>(weight); R.weight_stride = weight_stride;
    R.error = ctx->d_counters + 3 * (TLI_MAX_B + 1);
    R.taking = reinterpret_cast<uint32_t *>(ws + L.taking);
    R.n_valid = reinterpret_cast<int *>(ws + L.n_valid);
    R.pos = reinterpret_cast<int *>(ws + L.pos);
    R.by_row = reinterpret_cast<float4 *>(ws + L.by_row);
    R.rowp = reinterpret_cast<float4 *>(ws + L.rowp);
    R.rows = reinterpret_cast<__nv_bfloat16 *>(ws + L.rows);
    return TLI_OK;
}
void head_gemm_common(const HeadRows &R, const tli_ctx *ctx, HeadGemm &G) {
    memset(&G, 0, sizeof G);
    G.n_valid = R.n_valid;
    G.error = ctx->d_counters + 3 * (TLI_MAX_B + 1);
    G.H = R.H; G.V = R.V;
    G.mask = R.T.mask;
    G.rowp = R.rowp;
}

}  // namespace

extern "C" {

size_t tli_head_loss_workspace_bytes(const tli_ctx *ctx, int32_t N, int32_t H, int32_t k, int32_t side) { return head_workspace(ctx, N, H, k, side, false); }
size_t tli_head_loss_grad_workspace_bytes(const tli_ctx *ctx, int32_t N, int32_t H, int32_t k, int32_t side) { return head_workspace(ctx, N, H, k, side, true); }

int tli_head_loss(tli_ctx *ctx, const tli_head_loss_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    HeadRows R;
    HeadPlan L;
    int rc = prepare_head(ctx, a->N, a->H, a->k, a->side, a->ids_side, a->support, a->hidden, a->hidden_stride, a->weight, a->weight_stride, a->ids, a->teacher,
                          a->teacher_dtype, a->temperature, a->workspace, a->workspace_bytes, false, R, L);
    if (rc != TLI_OK) return rc;
    if (a->N == 0) return TLI_OK;
    if (!a->loss || !a->stats || !a->target_logits || !aligned4({a->loss, a->target_logits, a->status}) || !aligned8(a->stats)) return TLI_ERR_ARG;
    R.loss = a->loss; R.stats = a->stats; R.target_logits = a->target_logits; R.status = a->status;
    R.part = reinterpret_cast<const float2 *>(reinterpret_cast<char *>(a->workspace) + L.part); R.part_pitch = a->N; R.tiles = L.tiles;
    HeadGemm G;
    head_gemm_common(R, ctx, G);
    G.cols = R.V; G.bn = L.bn; G.early = a->N <= 128 * L.cg;
    G.k_part = L.cg == 1 ? 2 : std::min(16, std::max(8, (R.H + 2 * kHeadK - 1) / (2 * kHeadK)));
    G.a_rows = std::min(128, (a->N + 7) / 8 * 8);
    G.part = const_cast<float2 *>(R.part); G.part_pitch = R.part_pitch;
    if (!tensor_map(&G.a, false, R.rows, R.H, a->N, R.H, G.a_rows) || !tensor_map(&G.b, false, R.weight, R.H, R.V, R.weight_stride, L.bn / L.cg)) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    rc = launch_head_rows<false>(R, stream);
    if (rc == TLI_OK) rc = launch_head_gemm<HEAD_STATS>(G, L.cg, ctx, static_cast<long long>(L.tiles) * ((a->N + 128 * L.cg - 1) / (128 * L.cg)), stream);
    if (rc != TLI_OK) return rc;
    // 1000 rows of 32 targets (V 4136, H 1960): 80 us a call with a warp per row and a target at a time, 72 with four at a time, 47 with a CTA per row
    if (a->k <= 4) rc = launch_plain(tli_head_loss_kernel<1, 8>, R, (a->N + 7) / 8, 256, stream, "launch tli_head_loss_kernel");
    else if (a->k <= 32) rc = launch_plain(tli_head_loss_kernel<1, 1>, R, a->N, 256, stream, "launch tli_head_loss_kernel");
    else if (a->k <= 128) rc = launch_plain(tli_head_loss_kernel<4, 1>, R, a->N, 256, stream, "launch tli_head_loss_kernel");
    else rc = launch_plain(tli_head_loss_kernel<TLI_MAX_TARGETS / 32, 1>, R, a->N, 256, stream, "launch tli_head_loss_kernel");
    return rc;
}

int tli_head_loss_grad(tli_ctx *ctx, const tli_head_loss_grad_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    HeadRows R;
    HeadPlan L;
    int rc = prepare_head(ctx, a->N, a->H, a->k, a->side, a->ids_side, a->support, a->hidden, a->hidden_stride, a->weight, a->weight_stride, a->ids, a->teacher,
                          a->teacher_dtype, a->temperature, a->workspace, a->workspace_bytes, true, R, L);
    if (rc != TLI_OK) return rc;
    if (a->N > 0 && (!a->stats || !a->target_logits)) return TLI_ERR_ARG;
    if (!aligned4({a->target_logits, a->grad_loss, a->status}) || !aligned8(a->stats)) return TLI_ERR_ARG;
    if (!a->grad_hidden && !a->grad_weight) return TLI_ERR_ARG;
    if (a->grad_hidden && (reinterpret_cast<uintptr_t>(a->grad_hidden) % 2 || (a->N > 1 && a->grad_hidden_stride < a->H))) return TLI_ERR_ARG;
    if (a->grad_weight && (!on_vectors(a->grad_weight, a->grad_weight_stride, 2) || a->grad_weight_stride < a->H)) return TLI_ERR_ARG;
    // (hidden has been copied when the gradients are written, the weight is read to the end)
    const Span dh(a->grad_hidden, a->N, a->grad_hidden_stride, a->H), dw(a->grad_weight, R.V, a->grad_weight_stride, a->H), w(a->weight, R.V, a->weight_stride, a->H);
    if (dh.meets(w) || dw.meets(w) || dh.meets(dw)) return TLI_ERR_ARG;
    char *ws = reinterpret_cast<char *>(a->workspace);
    R.stats = const_cast<float *>(a->stats); R.target_logits = const_cast<float *>(a->target_logits); R.g = a->grad_loss; R.status = a->status;
    R.tid = reinterpret_cast<int *>(ws + L.tid); R.tval = reinterpret_cast<float *>(ws + L.tval);
    R.tid_of = reinterpret_cast<int *>(ws + L.tid_of); R.tval_of = reinterpret_cast<float *>(ws + L.tval_of);
    R.near_id = reinterpret_cast<int *>(ws + L.near_id); R.near_off = reinterpret_cast<float *>(ws + L.near_off);
    __nv_bfloat16 *slopes = reinterpret_cast<__nv_bfloat16 *>(ws + L.G);
    R.sums = reinterpret_cast<const float *>(ws + L.sums); R.splits = L.splits;
    R.grad_hidden = reinterpret_cast<__nv_bfloat16 *>(a->grad_hidden); R.grad_hidden_stride = a->grad_hidden_stride;
    R.out_vec = on_vectors(a->grad_hidden, a->grad_hidden_stride, 2);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const int N = a->N;
    if (N == 0) {
        if (!a->grad_weight) return TLI_OK;
        const cudaError_t e = cudaMemset2DAsync(a->grad_weight, a->grad_weight_stride * 2, 0, a->H * 2ll, R.V, stream);
        return e == cudaSuccess ? TLI_OK : cuda_fail(e, "cudaMemset2DAsync");
    }
    HeadGemm S, G;
    head_gemm_common(R, ctx, S);
    head_gemm_common(R, ctx, G);
    S.tid = R.tid_of; S.tval = R.tval_of; S.k = a->k;
    S.bn = kHeadN; S.early = G.early = N <= 128 * L.cg;
    S.a_rows = std::min(128, (N + 7) / 8 * 8);
    bool maps = tensor_map(&S.a, false, R.rows, R.H, N, R.H, S.a_rows) && tensor_map(&S.b, false, R.weight, R.H, R.V, R.weight_stride, kHeadN / L.cg) &&
                tensor_map(&S.out, false, slopes, L.run, N, L.run, 32) && tensor_map(&G.a, false, slopes, L.run, N, L.run, 128);
    G.G = slopes; G.pitch = L.run; G.weight = R.weight; G.weight_stride = R.weight_stride;
    G.splits = L.splits; G.want_dh = a->grad_hidden != nullptr; G.want_dw = a->grad_weight != nullptr;
    maps = maps && tensor_map(&G.a2, false, slopes, L.run, N, L.run, kHeadK) && tensor_map(&G.b, false, R.weight, R.H, R.V, R.weight_stride, kHeadK) &&
           tensor_map(&G.b2, false, R.rows, R.H, N, R.H, kHeadK) && tensor_map(&G.out2, true, R.sums, R.H, N, R.H, 32, L.splits);
    if (maps && a->grad_weight) maps = tensor_map(&G.out, false, a->grad_weight, R.H, R.V, a->grad_weight_stride, 32);
    if (!maps) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    const long long mb = (N + 128 * L.cg - 1) / (128 * L.cg), hb = (R.H + kHeadN - 1) / kHeadN;
    rc = launch_head_rows<true>(R, stream);
    for (int i = 0; i < L.runs && rc == TLI_OK; ++i) {
        const int c0 = i * L.run, cols = std::min(L.run, R.V - c0);
        S.c0 = G.c0 = c0;
        S.cols = G.cols = cols;
        G.first = i == 0;
        rc = launch_head_gemm<HEAD_SLOPE>(S, L.cg, ctx, mb * ((cols + kHeadN - 1) / kHeadN), stream);
        if (rc == TLI_OK) rc = launch_head_gemm<HEAD_GRADS>(G, L.cg, ctx, mb * hb * L.splits + (cols + 128 * L.cg - 1) / (128 * L.cg) * hb, stream);
    }
    R.groups = 1;
    while (R.groups < 32 && R.groups * 8 < L.splits) R.groups *= 2;        // eight splits a thread, on their way together
    const long long per_cta = kRowsThreads / R.groups;
    if (rc == TLI_OK && (a->grad_hidden || a->status)) {
        const long long ctas = (static_cast<long long>(N) * (R.H / 4) + per_cta - 1) / per_cta;
        rc = R.groups > 1 ? launch_plain(tli_head_rows_kernel<true>, R, ctas, kRowsThreads, stream, "launch tli_head_rows_kernel")
                          : launch_plain(tli_head_rows_kernel<false>, R, ctas, kRowsThreads, stream, "launch tli_head_rows_kernel");
    }
    return rc;
}

}  // extern "C"
