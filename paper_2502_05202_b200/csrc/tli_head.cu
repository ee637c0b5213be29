// The losses of tli_loss.cu from hidden rows and the output head's weight, z = hidden * weight^T, and their gradients.  The logits
// are formed tile by tile in tensor memory and never written.  (Part of tli_lib.cu: uses the parts before it.)
//
// A call is a chain of launches:
//   tli_head_targets_kernel   which rows take part, one bit each; for the gradient what their slopes are made of.
//   tli_head_gather_kernel    those rows of `hidden` one after the other (work is in proportion to them, any stride and alignment will
//                             do, and a row that is left out may hold anything).
//   tli_head_gemm_kernel      <STATS>  forward: (max, sum) of every row over every tile of the vocabulary.
//   tli_head_loss_kernel               forward: the tiles' pairs joined, the targets' logits, the loss.
//                             <SLOPE>  backward, for a run of the vocabulary: G = g dz in bf16, [rows, run], to the workspace;
//   tli_head_patch_kernel              the targets' elements of G again;
//                             <GRADS>  d hidden += G * weight and d weight = G^T * hidden of that run, one list of tiles.
//   tli_head_rows_kernel      d hidden from its fp32 sums to bf16, at the rows' places.
// The run keeps G near the size of L2 (128 MB), whatever the vocabulary.
//
// tli_head_gemm_kernel: persistent, one CTA per SM or one pair (CG = 2) per two SMs.  A tile of D is 128 CG rows x 256 columns of fp32 in
// tensor memory, two of them, so that the epilogue of one runs under the products of the next.  Warp 0 fills a ring of stages of
// 64 elements of the contracted axis by TMA, warp 1 issues tcgen05.mma (bf16, fp32 sums), warps 2 to 5 are the epilogue, a thread per
// row of D.  With CG = 2 each CTA loads half of both operands and the pair's leader issues the products of both.
// Operands come as they lie in memory: rows along the contracted axis (K-major) or across it (MN-major), 128-byte swizzle either way.
// All waits are bounded: when one runs out the context's error word is set, every role stops, copies in flight are waited for, tensor
// memory is given back, and the rows' status says TLI_ROW_TIMEOUT.

#include <cuda.h>

namespace {

constexpr int kHeadThreads = 192;
constexpr int kHeadK = 64;                 // elements of the contracted axis in a stage: 128 bytes, one swizzle span
constexpr int kHeadN = 256;                // columns of a tile
constexpr int kHeadABytes = 128 * kHeadK * 2;
constexpr int kHeadStageBuf = 128 * 128;   // a slab of the epilogue's on its way out: 128 rows of 128 bytes
constexpr int kHeadRowBlock = 32;          // rows per CTA of the targets and gather kernels
enum : int { HEAD_STATS = 0, HEAD_SLOPE = 1, HEAD_GRADS = 2 };

template <int CG> struct HeadRing {
    static constexpr int kStages = CG == 1 ? 4 : 6;
    static constexpr int kBBytes = kHeadN / CG * kHeadK * 2;
    static constexpr int kStageBytes = kHeadABytes + kBBytes;
    static constexpr int kSmem = kStages * kStageBytes + 2 * kHeadStageBuf + 1024;
};

struct HeadGemm {
    // STATS, SLOPE: a = rows, b = weight, out = G.  GRADS: a = G (K-major), b = weight (MN-major), a2 = G (MN-major), b2 = rows (MN-major),
    // out = d weight, out2 = sums of d hidden
    CUtensorMap a, b, a2, b2, out, out2;
    const int *n_valid;
    unsigned *error;
    int H, V, c0, cols;                    // the run of the vocabulary: [c0, c0 + cols)
    int bn;                                // STATS, SLOPE: columns of a tile
    int a_rows;                            // rows of a box of a
    int splits, first, want_dh, want_dw;   // GRADS: runs the contraction of d hidden is cut into; whether its sums start here
    const uint32_t *mask;
    const float4 *rowp;                    // {s, m, f, -} of a row
    float2 *part; long long part_pitch;    // STATS: [tile of the vocabulary][row]
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
template <int MODE, int CG> struct HeadTiles {
    int mb, nb, hb, t2, total, k2, k3;
    __device__ __forceinline__ HeadTiles(const HeadGemm &P, int rows) {
        mb = (rows + 128 * CG - 1) / (128 * CG);
        if constexpr (MODE == HEAD_GRADS) {
            hb = (P.H + kHeadN - 1) / kHeadN;
            nb = (P.cols + 128 * CG - 1) / (128 * CG);
            t2 = P.want_dh ? mb * hb * P.splits : 0;
            total = t2 + (P.want_dw ? nb * hb : 0);
            k2 = (P.cols + kHeadK - 1) / kHeadK;
            k3 = (rows + kHeadK - 1) / kHeadK;
        } else {
            hb = t2 = k3 = 0;
            nb = (P.cols + P.bn - 1) / P.bn;
            total = mb * nb;
            k2 = (P.H + kHeadK - 1) / kHeadK;
        }
    }
    __device__ __forceinline__ HeadTile at(const HeadGemm &P, int t) const {
        HeadTile w;
        w.split = 0;
        if constexpr (MODE == HEAD_GRADS) {
            w.n = t % hb * kHeadN;
            if (t < t2) {                                          // d hidden: a row block's columns next to one another
                const int r = t / hb;
                w.m = r % mb * 128 * CG;
                w.split = r / mb;
                const int a = static_cast<int>(static_cast<long long>(k2) * w.split / P.splits), b = static_cast<int>(static_cast<long long>(k2) * (w.split + 1) / P.splits);
                w.k0 = a * kHeadK; w.ks = b - a;
            } else {
                w.n = (t - t2) % hb * kHeadN;
                w.m = (t - t2) / hb * 128 * CG;
                w.split = -1;
                w.k0 = 0; w.ks = k3;
            }
        } else {                                                   // the row blocks of a tile of the weight next to one another
            w.m = t % mb * 128 * CG;
            w.n = t / mb * P.bn;
            w.k0 = 0; w.ks = k2;
        }
        return w;
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
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.tfull[i], 1); mbar_init(&sm.tempty[i], 4 * CG); }
        mbar_init(&sm.drain, 1);
        sm.error = 0;
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
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int rows = *reinterpret_cast<const volatile int *>(P.n_valid);
    const HeadTiles<MODE, CG> tiles(P, rows);
    const int first_tile = blockIdx.x / CG, step = gridDim.x / CG;

    if (warp == 0) {
        if (lane == 0) {
            asm volatile("fence.proxy.async;" ::: "memory");       // what kernels before this one stored, to the copies' view
            unsigned it = 0;
            bool ok = true;
            for (int t = first_tile; t < tiles.total && ok; t += step) {
                const HeadTile w = tiles.at(P, t);
                const int m = w.m + static_cast<int>(rank) * 128;
                const bool dw = MODE == HEAD_GRADS && w.split < 0, dh = MODE == HEAD_GRADS && !dw;
                const int bn = MODE == HEAD_GRADS ? kHeadN : P.bn;
                const unsigned bytes = (MODE == HEAD_GRADS ? static_cast<unsigned>(kHeadABytes) : P.a_rows * (kHeadK * 2u)) + static_cast<unsigned>(bn / CG) * (kHeadK * 2u);
                for (int k = 0; k < w.ks; ++k, ++it) {
                    const unsigned st = it % R::kStages, par = (it / R::kStages + 1) & 1u;
                    ok = mbar_wait(&sm.empty[st], par, &sm.error, P.error);
                    if (!ok) break;
                    const uint32_t a = ring + st * R::kStageBytes, b = a + kHeadABytes;
                    const uint32_t bar = CG == 1 ? smem_addr(&sm.full[st]) : cluster_addr(smem_addr(&sm.full[st]), 0u);
                    if (CG == 1 || rank == 0) mbar_arrive_expect_tx(&sm.full[st], bytes * CG);
                    const int x = w.k0 + k * kHeadK;
                    if constexpr (MODE != HEAD_GRADS) {
                        tensor_load<CG>(a, &P.a, x, m, bar);
                        tensor_load<CG>(b, &P.b, x, P.c0 + w.n + static_cast<int>(rank) * (bn / CG), bar);
                    } else if (dh) {                               // G [rows, run], weight [run, H] across the contracted axis
                        tensor_load<CG>(a, &P.a, x, m, bar);
                        for (int i = 0; i < kHeadN / CG / 64; ++i) tensor_load<CG>(b + i * 8192, &P.b, w.n + static_cast<int>(rank) * (kHeadN / CG) + i * 64, P.c0 + x, bar);
                    } else {                                       // both across it
                        for (int i = 0; i < 2; ++i) tensor_load<CG>(a + i * 8192, &P.a2, m + i * 64, x, bar);
                        for (int i = 0; i < kHeadN / CG / 64; ++i) tensor_load<CG>(b + i * 8192, &P.b2, w.n + static_cast<int>(rank) * (kHeadN / CG) + i * 64, x, bar);
                    }
                }
            }
            // every stage handed back: no arrival is under way when the CTA leaves
            for (unsigned j = it > R::kStages ? it - R::kStages : 0; j < it && ok; ++j) ok = mbar_wait(&sm.empty[j % R::kStages], (j / R::kStages) & 1u, &sm.error, P.error);
            if (!ok && rank == 0) {                                // no CTA of the pair may leave while copies to it are in flight
                for (unsigned j = it > R::kStages ? it - R::kStages : 0; j < it; ++j)
                    for (unsigned i = 0; i < kWaitLimit && !mbar_test(&sm.full[j % R::kStages], (j / R::kStages) & 1u); ++i) __nanosleep(64);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t base = 1u << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(128 * CG >> 4) << 24;
            unsigned it = 0, acc = 0;
            bool ok = true;
            for (int t = first_tile; t < tiles.total && ok; t += step, ++acc) {
                const HeadTile w = tiles.at(P, t);
                const bool dw = MODE == HEAD_GRADS && w.split < 0, dh = MODE == HEAD_GRADS && !dw;
                const int bn = MODE == HEAD_GRADS ? kHeadN : P.bn;
                const uint32_t idesc = base | static_cast<uint32_t>(bn >> 3) << 17 | (dw ? 1u << 15 | 1u << 16 : dh ? 1u << 16 : 0u);
                const uint32_t a_step = dw ? 128u : 2u, b_step = dw || dh ? 128u : 2u;        // 16 elements of the contracted axis, in 16 bytes
                ok = mbar_wait(&sm.tempty[acc & 1], (acc >> 1 & 1u) ^ 1u, &sm.error, P.error);
                if (!ok) break;
                tmem_fence_after();
                const uint32_t d = tmem + (acc & 1) * kHeadN;
                for (int k = 0; k < w.ks; ++k, ++it) {
                    const unsigned st = it % R::kStages;
                    ok = mbar_wait(&sm.full[st], (it / R::kStages) & 1u, &sm.error, P.error);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t a = ring + st * R::kStageBytes, b = a + kHeadABytes;
                    // across: blocks of 64 are 8 KB apart, groups of 8 of the contracted axis 1 KB; along: groups of 8 rows 1 KB
                    uint64_t ad = dw ? umma_desc(a, 8192, 1024) : umma_desc(a, 16, 1024), bd = dw || dh ? umma_desc(b, 8192, 1024) : umma_desc(b, 16, 1024);
#pragma unroll
                    for (int i = 0; i < kHeadK / 16; ++i) umma<CG>(d, ad + i * a_step, bd + i * b_step, idesc, (k | i) != 0);
                    umma_commit<CG>(&sm.empty[st]);
                }
                if (ok) umma_commit<CG>(&sm.tfull[acc & 1]);
            }
            if (!ok) {
                umma_commit<CG>(&sm.drain);
                for (unsigned i = 0; i < kWaitLimit && !mbar_test(&sm.drain, 0u); ++i) __nanosleep(64);
            }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const bool issuer = warp == 2 && lane == 0;
        const uint32_t tm = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        unsigned acc = 0, slabs = 0;
        bool ok = true;
        // the row's 128 bytes of a slab, 16 at a time, and the slab on its way
        auto slab_free = [&]() {
            if (issuer) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();                                          // (a barrier counts warps: a parted one would count twice)
            asm volatile("bar.sync 1, 128;" ::: "memory");
            return slab + (slabs++ & 1) * kHeadStageBuf;
        };
        auto slab_full = [&]() {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            asm volatile("bar.sync 1, 128;" ::: "memory");
        };
        auto slab_at = [&](uint32_t s, int i) { return s + row * 128 + ((i ^ (row & 7)) << 4); };
        for (int t = first_tile; t < tiles.total; t += step, ++acc) {
            const HeadTile w = tiles.at(P, t);
            const int m = w.m + static_cast<int>(rank) * 128, pos = m + row;
            // What depends on the row is a value here and no branch: a compiler that makes two paths of one (rows that count and rows that
            // do not) parts the warp in front of the instructions below that a whole warp has to take.
            float s = 0.f, top = 0.f, f = 0.f;
            uint32_t live = pos < rows ? 0xffffffffu : 0u, store = issuer && (MODE == HEAD_GRADS && w.split < 0 ? P.c0 + m < P.V : m < rows);
            asm volatile("" : "+r"(live), "+r"(store));
            if constexpr (MODE != HEAD_GRADS) {
                const float4 r = __ldg(P.rowp + min(pos, rows - 1));
                s = r.x; top = r.y; f = r.z;
            }
            if (lane == 0) ok = ok && mbar_wait(&sm.tfull[acc & 1], acc >> 1 & 1u, &sm.error, P.error);
            __syncwarp();
            // (after a time-out the warps still meet at the slabs' barriers, tile by tile, with whatever tensor memory holds)
            tmem_fence_after();
            const uint32_t d = tm + (acc & 1) * kHeadN;
            if constexpr (MODE == HEAD_STATS) {
                float best = kMaskBelow, sum = 0.f;
                if (m < rows) {
#pragma unroll 1
                    for (int c = 0; c < P.bn; c += 32) {
                        float x[32];
                        tmem_load32(d + c, x);
                        tmem_wait_load();
                        const int col = w.n + c, left = P.cols - col;
                        uint32_t bits = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                        if (P.mask && left > 0) bits &= __ldg(P.mask + ((P.c0 + col) >> 5));
                        if (bits != 0xffffffffu) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = bits >> i & 1u ? x[i] : -INFINITY;
                        }
                        float high = x[0];
#pragma unroll
                        for (int i = 1; i < 32; ++i) high = fmaxf(high, x[i]);
                        if (high > best) {
                            sum *= ex2((best - high) * s);
                            best = high;
                        }
                        const uint64_t s2 = pack2(s, s), c2 = pack2(-best, -best);
                        uint64_t a2[2] = {pack2(sum, 0.f), 0ull};
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float y0, y1;
                            unpack2(mul2(add2(pack2(x[i], x[i + 1]), c2), s2), y0, y1);
                            a2[i >> 1 & 1] = add2(a2[i >> 1 & 1], pack2(ex2(y0), ex2(y1)));
                        }
                        float w0, w1, w2, w3;
                        unpack2(a2[0], w0, w1);
                        unpack2(a2[1], w2, w3);
                        sum = (w0 + w1) + (w2 + w3);
                    }
                    if (live) P.part[static_cast<long long>(w.n / P.bn) * P.part_pitch + pos] = make_float2(best, sum);
                }
            } else if constexpr (MODE == HEAD_SLOPE) {
#pragma unroll 1
                for (int c = 0; c < P.bn; c += 64) {
                    const uint32_t to = slab_free();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x[32];
                        tmem_load32(d + c + h * 32, x);
                        tmem_wait_load();
                        const int col = w.n + c + h * 32, left = P.cols - col;
                        uint32_t bits = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                        if (P.mask && left > 0) bits &= __ldg(P.mask + ((P.c0 + col) >> 5));
                        bits &= live;
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            float y[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                y[j] = ex2((x[i + j] - top) * s) * f;
                                y[j] = bits >> (i + j) & 1u ? y[j] : 0.f;
                            }
                            st_shared16(slab_at(to, h * 4 + i / 8), pack_vector<TLI_BF16>(y));
                        }
                    }
                    slab_full();
                    if (issuer) {
                        if (store) tensor_store(&P.out, w.n + c, m, to);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            } else if (w.split >= 0) {                             // d hidden: fp32 sums, 32 columns a slab
#pragma unroll 1
                for (int c = 0; c < kHeadN && w.n + c < P.H; c += 32) {
                    const uint32_t to = slab_free();
                    float x[32];
                    tmem_load32(d + c, x);
                    tmem_wait_load();
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[i + j] = w.ks ? x[i + j] : 0.f;     // (a split of a short run may have no step)
                        st_shared16(slab_at(to, i / 4), make_uint4(__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3])));
                    }
                    slab_full();
                    if (issuer) {
                        if (store) tensor_store3(&P.out2, w.n + c, m, w.split, to, !P.first);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            } else {                                               // d weight: bf16, 64 columns a slab
#pragma unroll 1
                for (int c = 0; c < kHeadN && w.n + c < P.H; c += 64) {
                    const uint32_t to = slab_free();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x[32];
                        tmem_load32(d + c + h * 32, x);
                        tmem_wait_load();
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            float y[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = w.ks ? x[i + j] : 0.f;
                            st_shared16(slab_at(to, h * 4 + i / 8), pack_vector<TLI_BF16>(y));
                        }
                    }
                    slab_full();
                    if (issuer) {
                        if (store) tensor_store(&P.out, w.n + c, P.c0 + m, to);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 1) mbar_arrive(&sm.tempty[acc & 1]);
                else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr(smem_addr(&sm.tempty[acc & 1]), 0u)) : "memory");
            }
        }
        if (issuer) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
    uint32_t *taking;                      // a bit per row, a word per CTA of the targets kernel
    int *n_valid, *pos;                    // rows that take part; place of a row among them, -1
    float4 *by_row, *rowp;                 // {s, m, f, -} of a row; of the rows that take part, in their order
    int *tid; float *tval;                 // gradient: the targets' ids (-1) and elements of G
    __nv_bfloat16 *rows;                   // [N, H]
    const float2 *part; long long part_pitch; int tiles;
    __nv_bfloat16 *G; long long pitch; int c0, cols;
    const float *sums; int splits;         // d hidden: [splits][N, H]
    __nv_bfloat16 *grad_hidden; long long grad_hidden_stride; int out_vec;
};

// A warp per row.  GRAD: also what the row's slope is made of and its targets' elements, g/tau (q - mass).
template <bool GRAD>
__global__ void __launch_bounds__(kHeadRowBlock * 32) tli_head_targets_kernel(const __grid_constant__ HeadRows P) {
    constexpr int Q = TLI_MAX_TARGETS / 32;
    __shared__ uint32_t word;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, k = P.T.k;
    const long long row = static_cast<long long>(blockIdx.x) * kHeadRowBlock + warp;
    if (threadIdx.x == 0) word = 0;
    __syncthreads();
    if (row < P.T.N) {
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
        int status = (any ? 0 : TLI_ROW_LEFT_OUT) | (scale_ok ? 0 : TLI_ROW_BAD_TEMPERATURE);
        float4 r = make_float4(s, 0.f, 0.f, 0.f);
        if constexpr (GRAD) {
            const RowSlope slope(P.T.tau, P.stats, P.g, row);
            takes = takes && !slope.zero;
            r = make_float4(slope.s, slope.m, slope.f, 0.f);
            if (takes) {
                float mass[Q], W = 1.f;
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
                        for (int l = 0; l < 32; ++l) {
                            const int other = __shfl_sync(0xffffffffu, id[b], l);
                            const float more = __shfl_sync(0xffffffffu, w[b], l);
#pragma unroll
                            for (int q = 0; q < Q; ++q) mass[q] += id[q] == other ? more : 0.f;
                        }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < Q; ++q) mass[q] = 1.f;
                }
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const long long at = row * k + q * 32 + lane;
                    if (q * 32 + lane >= k) break;
                    P.tid[at] = id[q];
                    if (id[q] >= 0) P.tval[at] = fmaf(-slope.h, mass[q] / W, slope(__ldg(P.target_logits + at)));
                }
            }
        }
        if (lane == 0) {
            P.by_row[row] = r;
            if (GRAD && P.status) P.status[row] = status | (!takes && !status ? TLI_ROW_FALLBACK : 0);
            if (!GRAD && P.status) P.status[row] = status;
            if (takes) atomicOr(&word, 1u << warp);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) P.taking[blockIdx.x] = word;
}

// The rows that take part, in order.  The last CTA leaves their number, and zeros up to the next multiple of kHeadK (the contraction of
// d weight goes that far).
constexpr int kGatherThreads = 256;
__global__ void __launch_bounds__(kGatherThreads) tli_head_gather_kernel(const __grid_constant__ HeadRows P) {
    constexpr int WARPS = kGatherThreads / 32;
    __shared__ int sums[WARPS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.x;
    int before = 0;
    for (int i = threadIdx.x; i < b; i += kGatherThreads) before += __popc(__ldcg(P.taking + i));
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) sums[warp] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) before += sums[i];
    const uint32_t word = __ldcg(P.taking + b);
    for (int r = warp; r < kHeadRowBlock; r += WARPS) {
        const long long row = static_cast<long long>(b) * kHeadRowBlock + r;
        if (row >= P.T.N) break;
        const bool takes = word >> r & 1u;
        const long long pos = before + __popc(word & ((1u << r) - 1u));
        if (lane == 0) {
            P.pos[row] = takes ? static_cast<int>(pos) : -1;
            if (takes) P.rowp[pos] = __ldcg(P.by_row + row);
        }
        if (!takes) continue;
        __nv_bfloat16 *to = P.rows + pos * P.H;
        const __nv_bfloat16 *from = P.hidden + row * P.hidden_stride;
        if (P.vec) {
            for (int i = lane; i < P.H / 8; i += 32) reinterpret_cast<uint4 *>(to)[i] = __ldg(reinterpret_cast<const uint4 *>(from) + i);
        } else {
            for (int i = lane; i < P.H; i += 32) to[i] = from[i];
        }
    }
    if (b == static_cast<int>(gridDim.x) - 1) {
        const int total = before + __popc(word);
        if (threadIdx.x == 0) *P.n_valid = total;
        const long long end = min(static_cast<long long>(P.T.N), (static_cast<long long>(total) + kHeadK - 1) / kHeadK * kHeadK);
        const long long nv = (end - total) * (P.H / 8);
        for (long long i = threadIdx.x; i < nv; i += kGatherThreads) reinterpret_cast<uint4 *>(P.rows + static_cast<long long>(total) * P.H)[i] = make_uint4(0, 0, 0, 0);
    }
}

// ---- forward: the loss of eight rows per CTA ----

constexpr int kHeadLossRows = 8;
__device__ __forceinline__ float dot_bf16(const uint4 &a, const uint4 &b, float acc) {
    float x[8], y[8];
    unpack<TLI_BF16>(a, x);
    unpack<TLI_BF16>(b, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = fmaf(x[i], y[i], acc);
    return acc;
}
__global__ void __launch_bounds__(256) tli_head_loss_kernel(const __grid_constant__ HeadRows P) {
    constexpr int Q = TLI_MAX_TARGETS / 32;
    __shared__ float sh_m[32][kHeadLossRows], sh_s[32][kHeadLossRows];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, k = P.T.k;
    const long long row0 = static_cast<long long>(blockIdx.x) * kHeadLossRows;
    {
        const int r = threadIdx.x & 7, t0 = threadIdx.x >> 3;      // neighbouring threads: neighbouring rows of a tile
        const long long row = row0 + r;
        const int pos = row < P.T.N ? __ldcg(P.pos + row) : -1;
        float m = kMaskBelow, sum = 0.f;
        if (pos >= 0) {
            const float s = __ldcg(&P.rowp[pos].x);
            for (int t = t0; t < P.tiles; t += 32) {
                const float2 p = __ldcg(P.part + t * P.part_pitch + pos);
                join_stats(s, m, sum, p.x, p.y);
            }
        }
        sh_m[t0][r] = m; sh_s[t0][r] = sum;
    }
    __syncthreads();
    const long long row = row0 + warp;
    if (row >= P.T.N) return;
    const int pos = __ldcg(P.pos + row);
    const long long at = row * k;
    if (pos < 0) {
        for (int j = lane; j < k; j += 32) P.target_logits[at + j] = 0.f;
        if (lane == 0) {
            P.loss[row] = 0.f;
            reinterpret_cast<float2 *>(P.stats)[row] = make_float2(0.f, 0.f);
            if (P.status && *reinterpret_cast<const volatile unsigned *>(P.error)) P.status[row] |= TLI_ROW_TIMEOUT;
        }
        return;
    }
    float tau, s;
    row_scale(P.T.tau, row, tau, s);
    float m = sh_m[lane][warp], sum = sh_s[lane][warp];
    const float top = warp_max(m);
    sum = warp_sum(sum * ex2((m - top) * s));
    m = top;
    // the targets' logits, a target at a time
    const uint4 *h = reinterpret_cast<const uint4 *>(P.rows + static_cast<long long>(pos) * P.H);
    int id[Q];
    float t[Q], z[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        id[q] = -1; t[q] = 0.f; z[q] = 0.f;
        if (q * 32 + lane < k) id[q] = row_target(P.T, row, q * 32 + lane, t[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (q * 32 >= k) break;
        for (int l = 0; l < 32 && q * 32 + l < k; ++l) {
            const int v = __shfl_sync(0xffffffffu, id[q], l);
            float dot = 0.f;
            if (v >= 0) {
                const uint4 *w = reinterpret_cast<const uint4 *>(P.weight + v * P.weight_stride);
                for (int i = lane; i < P.H / 8; i += 32) dot = dot_bf16(__ldg(h + i), __ldg(w + i), dot);
                dot = warp_sum(dot);
            }
            if (l == lane) z[q] = dot;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (q * 32 + lane < k) P.target_logits[at + q * 32 + lane] = z[q];
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
        if (P.status) {
            const int timeout = *reinterpret_cast<const volatile unsigned *>(P.error) ? TLI_ROW_TIMEOUT : 0;
            P.status[row] = timeout | (none ? TLI_ROW_FALLBACK : bad ? TLI_ROW_NONFINITE : 0);
        }
    }
}

// ---- backward: the targets' elements of a run of G, and d hidden at its rows' places ----

__global__ void __launch_bounds__(256) tli_head_patch_kernel(const __grid_constant__ HeadRows P) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<long long>(P.T.N) * P.T.k) return;
    const int pos = __ldcg(P.pos + i / P.T.k);
    if (pos < 0) return;
    const int v = __ldcg(P.tid + i) - P.c0;
    if (v < 0 || v >= P.cols) return;
    P.G[pos * P.pitch + v] = __float2bfloat16_rn(__ldcg(P.tval + i));
}

__global__ void __launch_bounds__(256) tli_head_rows_kernel(const __grid_constant__ HeadRows P) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int units = P.H / 8;
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<long long>(P.T.N) * units) return;
    const long long row = i / units;
    const int u = static_cast<int>(i % units), pos = __ldcg(P.pos + row);
    if (u == 0 && P.status && *reinterpret_cast<const volatile unsigned *>(P.error)) P.status[row] |= TLI_ROW_TIMEOUT;
    if (!P.grad_hidden) return;
    float x[8] = {};
    if (pos >= 0) {
        for (int sp = 0; sp < P.splits; ++sp) {
            const float4 *p = reinterpret_cast<const float4 *>(P.sums + (static_cast<long long>(sp) * P.T.N + pos) * P.H + u * 8);
            const float4 a = __ldcg(p), b = __ldcg(p + 1);
            x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
            x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
        }
    }
    __nv_bfloat16 *to = P.grad_hidden + row * P.grad_hidden_stride + u * 8;
    if (P.out_vec) {
        *reinterpret_cast<uint4 *>(to) = pack_vector<TLI_BF16>(x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) to[j] = __float2bfloat16_rn(x[j]);
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

constexpr long long kHeadRunBytes = 128ll << 20;       // of G
constexpr int kHeadMinSteps = 8;                       // of the contraction in a split of d hidden

struct HeadPlan {
    int cg, bn, tiles;                     // CTAs per tile; columns of a forward tile, tiles of the vocabulary
    int run, runs, splits;                 // backward: columns of a run of G, runs, cuts of d hidden's contraction
    size_t taking, n_valid, pos, by_row, rowp, tid, tval, rows, part, G, sums, total;
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
    const size_t n = static_cast<size_t>(N), words = (n + kHeadRowBlock - 1) / kHeadRowBlock;
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
        L.splits = std::max(1, std::min((num_sms / L.cg + blocks - 1) / std::max(blocks, 1), steps / kHeadMinSteps));
        L.tid = take(4 * n * k);
        L.tval = take(4 * n * k);
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

size_t head_workspace(const tli_ctx *ctx, int32_t N, int32_t H, int32_t k, int32_t side, bool grad) {
    if (!ctx || ctx->n_shards != 1 || N < 0 || N > TLI_MAX_HEAD_TOKENS || H < 8 || H > TLI_MAX_H || H % 8 || k < 1 || k > TLI_MAX_TARGETS) return 0;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return 0;
    return head_plan(N, H, k, side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d, ctx->num_sms, grad).total;
}

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
    G.cols = R.V; G.bn = L.bn;
    G.a_rows = std::min(128, (a->N + 7) / 8 * 8);
    G.part = const_cast<float2 *>(R.part); G.part_pitch = R.part_pitch;
    if (!tensor_map(&G.a, false, R.rows, R.H, a->N, R.H, G.a_rows) || !tensor_map(&G.b, false, R.weight, R.H, R.V, R.weight_stride, L.bn / L.cg)) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    const long long blocks = (a->N + kHeadRowBlock - 1) / kHeadRowBlock;
    rc = launch_plain(tli_head_targets_kernel<false>, R, blocks, kHeadRowBlock * 32, stream, "launch tli_head_targets_kernel");
    if (rc == TLI_OK) rc = launch_plain(tli_head_gather_kernel, R, blocks, kGatherThreads, stream, "launch tli_head_gather_kernel");
    if (rc == TLI_OK) rc = launch_head_gemm<HEAD_STATS>(G, L.cg, ctx, static_cast<long long>(L.tiles) * ((a->N + 128 * L.cg - 1) / (128 * L.cg)), stream);
    if (rc == TLI_OK) rc = launch_plain(tli_head_loss_kernel, R, (a->N + kHeadLossRows - 1) / kHeadLossRows, 256, stream, "launch tli_head_loss_kernel");
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
    char *ws = reinterpret_cast<char *>(a->workspace);
    R.stats = const_cast<float *>(a->stats); R.target_logits = const_cast<float *>(a->target_logits); R.g = a->grad_loss; R.status = a->status;
    R.tid = reinterpret_cast<int *>(ws + L.tid); R.tval = reinterpret_cast<float *>(ws + L.tval);
    R.G = reinterpret_cast<__nv_bfloat16 *>(ws + L.G); R.pitch = L.run;
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
    S.bn = kHeadN;
    S.a_rows = std::min(128, (N + 7) / 8 * 8);
    bool maps = tensor_map(&S.a, false, R.rows, R.H, N, R.H, S.a_rows) && tensor_map(&S.b, false, R.weight, R.H, R.V, R.weight_stride, kHeadN / L.cg) &&
                tensor_map(&S.out, false, R.G, L.run, N, L.run, 128);
    head_gemm_common(R, ctx, G);
    G.splits = L.splits; G.want_dh = a->grad_hidden != nullptr; G.want_dw = a->grad_weight != nullptr;
    G.a = S.out;
    maps = maps && tensor_map(&G.a2, false, R.G, L.run, N, L.run, kHeadK) && tensor_map(&G.b, false, R.weight, R.H, R.V, R.weight_stride, kHeadK) &&
           tensor_map(&G.b2, false, R.rows, R.H, N, R.H, kHeadK) && tensor_map(&G.out2, true, R.sums, R.H, N, R.H, 128, L.splits);
    if (maps && a->grad_weight) maps = tensor_map(&G.out, false, a->grad_weight, R.H, R.V, a->grad_weight_stride, 128);
    if (!maps) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    const long long blocks = (N + kHeadRowBlock - 1) / kHeadRowBlock, mb = (N + 128 * L.cg - 1) / (128 * L.cg), hb = (R.H + kHeadN - 1) / kHeadN;
    rc = launch_plain(tli_head_targets_kernel<true>, R, blocks, kHeadRowBlock * 32, stream, "launch tli_head_targets_kernel");
    if (rc == TLI_OK) rc = launch_plain(tli_head_gather_kernel, R, blocks, kGatherThreads, stream, "launch tli_head_gather_kernel");
    for (int i = 0; i < L.runs && rc == TLI_OK; ++i) {
        const int c0 = i * L.run, cols = std::min(L.run, R.V - c0);
        S.c0 = G.c0 = R.c0 = c0;
        S.cols = G.cols = R.cols = cols;
        G.first = i == 0;
        rc = launch_head_gemm<HEAD_SLOPE>(S, L.cg, ctx, mb * ((cols + kHeadN - 1) / kHeadN), stream);
        if (rc == TLI_OK) rc = launch_plain(tli_head_patch_kernel, R, (static_cast<long long>(N) * a->k + 255) / 256, 256, stream, "launch tli_head_patch_kernel");
        if (rc == TLI_OK) rc = launch_head_gemm<HEAD_GRADS>(G, L.cg, ctx, mb * hb * L.splits + (cols + 128 * L.cg - 1) / (128 * L.cg) * hb, stream);
    }
    if (rc == TLI_OK && (a->grad_hidden || a->status))
        rc = launch_plain(tli_head_rows_kernel, R, (static_cast<long long>(N) * (R.H / 8) + 255) / 256, 256, stream, "launch tli_head_rows_kernel");
    return rc;
}

}  // extern "C"
