// Embedding rows for ids of either vocabulary, and the gradient of that lookup.
// (Part of tli_lib.cu: uses tli_ctx and the error helpers of tli.cu.)
//
//   tli_embed_kernel       out[i] = scale * table[t(ids[i])], t the id map, its inverse or the identity; one warp per
//                          token and run of 128 vectors.  A copy: bound by DRAM, or for a decoding step by the
//                          chain id -> map -> row.
//   gradient               dW[v] = scale * sum over the tokens i with t(ids[i]) = v of g[i], every row written.
//       tli_grad_sort_kernel     tokens by (table id, position), least significant digit first, two digits of ten bits,
//                                stable, so that every sum below has one order whatever the timing; the other CTAs of
//                                the same grid fill dW with zeros meanwhile (the dense write is the floor); one cluster of eight.
//       tli_grad_count_kernel, tli_grad_scatter_kernel   the same sort over more CTAs for many tokens.
//       tli_grad_sum_kernel      a window of sorted tokens per group of threads: rows whose tokens all lie in the
//                                window are written, the pieces of a row that crosses a window go to the workspace.
//       tli_grad_join_kernel     adds the pieces of such a row in window order.
// Sums are fp32; the scaled sum, an fp32 product, is rounded to the type of dW.

namespace {

constexpr int kEmbThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 1024;
constexpr int kSortCluster = 8;
constexpr int kSumThreads = 128;
constexpr int kSumMinTx = 4;               // threads across a row at least (32 windows of 2 KB of keys and positions in a block)

// table id of a token, -1 if it has none
__device__ __forceinline__ int table_id(const int *map, int n_ids, int id) {
    if (id < 0 || id >= n_ids) return -1;
    return map ? __ldg(map + id) : id;
}

struct EmbedParams {
    int N, H, n_ids, chunks;
    const int *map, *ids;
    const void *table; long long ts;
    void *out; long long os;
    float scale;
    int *table_ids;
};

template <int DT> __device__ __forceinline__ uint4 scale_vector(const uint4 &r, float c) {
    float z[Elt<DT>::kPerVec];
    unpack<DT>(r, z);
    if constexpr (DT == TLI_F32) {
        return make_uint4(__float_as_uint(z[0] * c), __float_as_uint(z[1] * c), __float_as_uint(z[2] * c), __float_as_uint(z[3] * c));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)                                // to nearest even
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(z[2 * i + 1] * c), "f"(z[2 * i] * c));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <int DT> __device__ __forceinline__ float element(const void *p, long long i) {
    if constexpr (DT == TLI_F32) return __ldg(reinterpret_cast<const float *>(p) + i);
    else return __uint_as_float(static_cast<uint32_t>(__ldg(reinterpret_cast<const unsigned short *>(p) + i)) << 16);
}
template <int DT> __device__ __forceinline__ void set_element(void *p, long long i, float x) {
    if constexpr (DT == TLI_F32) {
        reinterpret_cast<float *>(p)[i] = x;
    } else {
        unsigned short h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
        reinterpret_cast<unsigned short *>(p)[i] = h;
    }
}

constexpr int kEmbUnroll = 4;

// VEC: rows of both sides lie on 16-byte boundaries and H is a whole number of vectors; otherwise element by element.
// 16 384 bf16 rows of 4096: 134 MB written and 58 MB of distinct rows read in 32 us (29.4 at the measured copy bandwidth).  48 rows of
// 2048: 2.1 us, the chain id -> map -> row.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kEmbThreads) tli_embed_kernel(const __grid_constant__ EmbedParams P) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long task = static_cast<long long>(blockIdx.x) * (kEmbThreads / 32) + (threadIdx.x >> 5);
    const int i = static_cast<int>(task / P.chunks), chunk = static_cast<int>(task % P.chunks), lane = threadIdx.x & 31;
    if (i >= P.N) return;
    const int t = table_id(P.map, P.n_ids, __ldg(P.ids + i));
    if (chunk == 0 && lane == 0 && P.table_ids) P.table_ids[i] = t;
    const int first = chunk * (32 * kEmbUnroll) + lane;
    if constexpr (VEC) {
        const int nv = P.H / Elt<DT>::kPerVec;
        const uint4 *src = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(P.table) + t * P.ts * Elt<DT>::kBytes);
        uint4 *dst = reinterpret_cast<uint4 *>(reinterpret_cast<char *>(P.out) + i * P.os * Elt<DT>::kBytes);
        uint4 r[kEmbUnroll];
#pragma unroll
        for (int q = 0; q < kEmbUnroll; ++q)
            r[q] = t >= 0 && first + q * 32 < nv ? __ldg(src + first + q * 32) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int q = 0; q < kEmbUnroll; ++q)
            if (first + q * 32 < nv) dst[first + q * 32] = t >= 0 ? scale_vector<DT>(r[q], P.scale) : r[q];
    } else {
        float x[kEmbUnroll];
#pragma unroll
        for (int q = 0; q < kEmbUnroll; ++q)
            x[q] = t >= 0 && first + q * 32 < P.H ? element<DT>(P.table, t * P.ts + first + q * 32) * P.scale : 0.f;
#pragma unroll
        for (int q = 0; q < kEmbUnroll; ++q)
            if (first + q * 32 < P.H) set_element<DT>(P.out, i * P.os + first + q * 32, x[q]);
    }
}

struct GradParams {
    int N, H, n_ids, V, groups, tile, clustered;      // groups: CTAs of the sort (one cluster or not); tile: tokens of one of them
    int window, nwin, tx;                  // sorted tokens per window; threads across a row
    const int *map, *ids;
    const void *g; long long gs;
    void *out; long long os;
    float scale;
    int *key[2], *pos[2];                  // [N]: sorted by the low digit, by both
    int *n_valid;                          // tokens that have a table id
    int *count;                            // [groups][kDigits]
    float *piece;                          // [nwin][2][H]: of the row that came in from the window before, of the one that goes on
};

// One digit of the sort for tokens [first, last) of the source, by one CTA.  pass 0 takes the ids, pass 1 what
// pass 0 left.
struct SortShared { int wsum[kSortWarps]; };

__device__ __forceinline__ int sort_key(const GradParams &P, int pass, int i, int &pos) {
    if (pass == 0) { pos = i; return table_id(P.map, P.n_ids, __ldg(P.ids + i)); }
    pos = __ldcg(P.pos[0] + i);
    return __ldcg(P.key[0] + i);
}
__device__ __forceinline__ int digit_of(int pass, int key) { return pass == 0 ? key & (kDigits - 1) : key >> 10; }

__device__ __forceinline__ int sort_scan(int x, SortShared &sh, int &total) {       // inclusive, over 1024 threads
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sh.wsum[warp] = x;
    __syncthreads();
    int s = sh.wsum[lane], incl = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    const int before = __shfl_sync(0xffffffffu, incl - s, warp);
    total = __shfl_sync(0xffffffffu, incl, 31);
    __syncthreads();
    return x + before;
}

// the lanes of the warp that hold the same digit (-1 for none), by a ballot per bit: __match_any_sync takes a step per distinct value
__device__ __forceinline__ unsigned same_digit(int d) {
    unsigned peers = __ballot_sync(0xffffffffu, d >= 0);
#pragma unroll
    for (int b = 0; b < 10; ++b) {
        const bool bit = d >> b & 1;
        const unsigned with = __ballot_sync(0xffffffffu, bit);
        peers &= bit ? with : ~with;
    }
    return peers;
}
// cnt: [warps][kDigits] counters and [kDigits] first places.  A warp has eight tokens per lane on their way at a time: one at a time,
// a digit of 16 384 tokens takes 16 trips to L2 and back in a row.
constexpr int kSortBatch = 8;
template <bool CLUSTER> __device__ __forceinline__ int sort_digit(const GradParams &P, int pass, int cta, int n, int *cnt, SortShared &sh) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = min(n, cta * P.tile), last = min(n, first + P.tile);
    const int chunk = ((last - first + kSortWarps - 1) / kSortWarps + 31) & ~31;     // a warp's tokens, in order
    const int w0 = min(last, first + warp * chunk), w1 = min(last, w0 + chunk);
    const int warps = chunk ? (last - first + chunk - 1) / chunk : 0;                // that have any
    int *base = cnt + kSortWarps * kDigits, *mine = cnt + warp * kDigits;
#pragma unroll 4
    for (int w = 0; w < warps; ++w) cnt[w * kDigits + tid] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i0 = w0 + lane; i0 < w1; i0 += 32 * kSortBatch) {
        int key[kSortBatch], pos;
#pragma unroll
        for (int j = 0; j < kSortBatch; ++j) key[j] = i0 + j * 32 < w1 ? sort_key(P, pass, i0 + j * 32, pos) : -1;
#pragma unroll
        for (int j = 0; j < kSortBatch; ++j)
            if (key[j] >= 0) atomicAdd(mine + digit_of(pass, key[j]), 1);
    }
    __syncthreads();
    // thread d: digit d
    int sum = 0, others = 0, all = 0;
#pragma unroll 8
    for (int w = 0; w < warps; ++w) {
        const int c = cnt[w * kDigits + tid];
        cnt[w * kDigits + tid] = sum;
        sum += c;
    }
    if (CLUSTER) {
        __stcg(P.count + cta * kDigits + tid, sum);
        cluster_barrier();
    }
#pragma unroll 8
    for (int c = 0; c < P.groups; ++c) {
        const int x = __ldcg(P.count + c * kDigits + tid);
        if (c < cta) others += x;
        all += x;
    }
    int total;
    base[tid] = sort_scan(all, sh, total) - all + others;
    if (pass == 0 && cta == 0 && tid == 0) *P.n_valid = total;
    __syncthreads();
#pragma unroll 1
    for (int i0 = w0 + lane; i0 - lane < w1; i0 += 32 * kSortBatch) {
        int key[kSortBatch], pos[kSortBatch];
#pragma unroll
        for (int j = 0; j < kSortBatch; ++j) {
            key[j] = -1; pos[j] = 0;
            if (i0 + j * 32 < w1) key[j] = sort_key(P, pass, i0 + j * 32, pos[j]);
        }
#pragma unroll
        for (int j = 0; j < kSortBatch; ++j) {
            const int d = key[j] >= 0 ? digit_of(pass, key[j]) : -1;
            const unsigned peers = same_digit(d);
            const int rank = __popc(peers & ((1u << lane) - 1u));
            int at = 0;
            if (d >= 0) at = mine[d] + rank;
            __syncwarp();
            if (d >= 0) {
                if (rank == 0) mine[d] = at + __popc(peers);
                at += base[d];
                __stcg(P.key[pass] + at, key[j]);
                __stcg(P.pos[pass] + at, pos[j]);
            }
            __syncwarp();
        }
    }
    if (CLUSTER) cluster_barrier(); else __syncthreads();
    return total;
}
constexpr size_t kSortSmem = sizeof(int) * (kSortWarps + 1) * kDigits;

// dW = 0, by CTAs [0, n) of a grid
template <int OT>
__device__ void fill_zero(const GradParams &P, unsigned cta, unsigned n) {
    const size_t step = static_cast<size_t>(n) * kSortThreads, me = static_cast<size_t>(cta) * kSortThreads + threadIdx.x;
    if (P.os == P.H) {
        char *p = reinterpret_cast<char *>(P.out);
        const size_t bytes = static_cast<size_t>(P.V) * P.H * Elt<OT>::kBytes;
        const size_t head = min(bytes, static_cast<size_t>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15));
        const size_t nv = (bytes - head) / 16;
        uint4 *v = reinterpret_cast<uint4 *>(p + head);
        for (size_t i = me; i < nv; i += step) v[i] = make_uint4(0, 0, 0, 0);
        const size_t edge = bytes - nv * 16;                       // the bytes in front of and behind the vectors
        for (size_t i = me; i < edge; i += step) p[i < head ? i : nv * 16 + i] = 0;
    } else {
        const size_t total = static_cast<size_t>(P.V) * P.H;
        for (size_t i = me; i < total; i += step) set_element<OT>(P.out, static_cast<long long>(i / P.H) * P.os + i % P.H, 0.f);
    }
}

// The first cluster sorts, the others fill dW with zeros.  (Two passes of one cluster of eight and two barriers each against
// eight more launches; the fill hides it up to some 10^5 tokens.)  49 152 fp32 rows of 2048 (403 MB) in 71 us, 5.7 TB/s: the fill has the SMs of
// the clusters that fit together, 112 of 148.
template <int OT>
__global__ void __launch_bounds__(kSortThreads) tli_grad_sort_kernel(const __grid_constant__ GradParams P) {
    extern __shared__ __align__(16) int sort_smem[];
    __shared__ SortShared sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned sorters = P.clustered ? kSortCluster : 0u;
    if (blockIdx.x < sorters) {
        const int cta = static_cast<int>(cluster_cta_rank());
        const int n = sort_digit<true>(P, 0, cta, P.N, sort_smem, sh);
        sort_digit<true>(P, 1, cta, n, sort_smem, sh);
        return;
    }
    fill_zero<OT>(P, blockIdx.x - sorters, gridDim.x - sorters);
}

__global__ void __launch_bounds__(kSortThreads) tli_grad_count_kernel(const __grid_constant__ GradParams P, int pass) {
    __shared__ int cnt[kDigits];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    cnt[threadIdx.x] = 0;
    __syncthreads();
    const int n = pass == 0 ? P.N : __ldcg(P.n_valid);
    const int first = min(n, static_cast<int>(blockIdx.x) * P.tile), last = min(n, first + P.tile);
    for (int i = first + threadIdx.x; i < last; i += kSortThreads) {
        int pos;
        const int key = sort_key(P, pass, i, pos);
        if (key >= 0) atomicAdd(cnt + digit_of(pass, key), 1);
    }
    __syncthreads();
    P.count[blockIdx.x * kDigits + threadIdx.x] = cnt[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) tli_grad_scatter_kernel(const __grid_constant__ GradParams P, int pass) {
    extern __shared__ __align__(16) int sort_smem[];
    __shared__ SortShared sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    sort_digit<false>(P, pass, blockIdx.x, pass == 0 ? P.N : __ldcg(P.n_valid), sort_smem, sh);
}

// ---- sums over the sorted tokens ----
//
// Columns of a thread.  VEC: one 16-byte vector of the gradient; otherwise four columns, kSumThreads-like strides apart
// so that a warp's loads stay together.
template <int GT, bool VEC> struct Columns {
    static constexpr int kN = VEC ? Elt<GT>::kPerVec : 4;
    int col[VEC ? 1 : 4];
    __device__ __forceinline__ Columns(const GradParams &P, int block) {
        const int x = threadIdx.x % P.tx;
        if constexpr (VEC) {
            col[0] = (block * P.tx + x) * kN;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) col[k] = (block * 4 + k) * P.tx + x;
        }
    }
    __device__ __forceinline__ bool any(const GradParams &P) const { return col[0] < P.H; }
    __device__ __forceinline__ void load(const GradParams &P, long long i, float (&x)[kN]) const {
        if constexpr (VEC) {
            const uint4 r = __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(P.g) + (i * P.gs + col[0]) * Elt<GT>::kBytes));
            unpack<GT>(r, x);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = col[k] < P.H ? element<GT>(P.g, i * P.gs + col[k]) : 0.f;
        }
    }
    template <int OT> __device__ __forceinline__ void store(const GradParams &P, int v, const float (&acc)[kN]) const {
        if constexpr (VEC) {
            char *p = reinterpret_cast<char *>(P.out) + (v * P.os + col[0]) * Elt<OT>::kBytes;
            float z[kN];
#pragma unroll
            for (int k = 0; k < kN; ++k) z[k] = acc[k] * P.scale;
            if constexpr (OT == TLI_F32) {
#pragma unroll
                for (int k = 0; k < kN; k += 4) reinterpret_cast<float4 *>(p)[k / 4] = make_float4(z[k], z[k + 1], z[k + 2], z[k + 3]);
            } else {
                uint32_t w[kN / 2];
#pragma unroll
                for (int k = 0; k < kN / 2; ++k) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(z[2 * k + 1]), "f"(z[2 * k]));
                if constexpr (kN == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
                else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col[k] < P.H) set_element<OT>(P.out, v * P.os + col[k], acc[k] * P.scale);
        }
    }
    // fp32 pieces in the workspace
    __device__ __forceinline__ void put(const GradParams &P, float *p, const float (&acc)[kN]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < kN; k += 4) __stcg(reinterpret_cast<float4 *>(p + col[0]) + k / 4, make_float4(acc[k], acc[k + 1], acc[k + 2], acc[k + 3]));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col[k] < P.H) __stcg(p + col[k], acc[k]);
        }
    }
    __device__ __forceinline__ void add(const GradParams &P, const float *p, float (&acc)[kN]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < kN; k += 4) {
                const float4 y = __ldcg(reinterpret_cast<const float4 *>(p + col[0]) + k / 4);
                acc[k] += y.x; acc[k + 1] += y.y; acc[k + 2] += y.z; acc[k + 3] += y.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col[k] < P.H) acc[k] += __ldcg(p + col[k]);
        }
    }
};

constexpr int kSumBatch = 8;               // rows of the gradient a thread has in flight
constexpr int kMaxWindow = 256;

// Bound by the latency of a window's gathered rows, eight of them on their way: 16 384 bf16 rows of 2048 (67 MB) in 10 us, 32 768 of 1024 in 24.
// The windows of a block: their tokens' keys, with the one in front and the one behind (-1 where there is none), and positions.
template <int GT, int OT, bool VEC>
__global__ void __launch_bounds__(kSumThreads) tli_grad_sum_kernel(const __grid_constant__ GradParams P) {
    extern __shared__ __align__(16) int window_smem[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int n = __ldcg(P.n_valid), ty = threadIdx.x / P.tx, tx = threadIdx.x % P.tx;
    const int win = blockIdx.x * (kSumThreads / P.tx) + ty;
    const int a = min(n, win * P.window), count = min(n, a + P.window) - a;
    int *key = window_smem + ty * (2 * P.window + 2), *pos = key + P.window + 2;
    for (int i = tx; i < P.window + 2; i += P.tx) {
        const int at = a - 1 + i;
        key[i] = at >= 0 && at < n ? __ldcg(P.key[1] + at) : -1;
        if (i < P.window) pos[i] = a + i < n ? __ldcg(P.pos[1] + a + i) : 0;
    }
    __syncthreads();
    const Columns<GT, VEC> c(P, blockIdx.y);
    if (win >= P.nwin || count <= 0 || !c.any(P)) return;
    constexpr int kN = Columns<GT, VEC>::kN;
    float acc[kN] = {};
    bool from_before = key[0] == key[1];
    int cur = key[1];
    auto flush = [&](bool goes_on) {
        if (from_before) c.put(P, P.piece + (static_cast<size_t>(win) * 2) * P.H, acc);          // (it may go on as well)
        else if (goes_on) c.put(P, P.piece + (static_cast<size_t>(win) * 2 + 1) * P.H, acc);
        else c.template store<OT>(P, cur, acc);
    };
#pragma unroll 1
    for (int i = 0; i < count; i += kSumBatch) {
        float x[kSumBatch][kN];
#pragma unroll
        for (int j = 0; j < kSumBatch; ++j) c.load(P, pos[min(i + j, count - 1)], x[j]);
#pragma unroll
        for (int j = 0; j < kSumBatch; ++j) {
            if (i + j >= count) break;
            const int k = key[1 + i + j];
            if (k != cur) {
                flush(false);
                from_before = false;
                cur = k;
#pragma unroll
                for (int q = 0; q < kN; ++q) acc[q] = x[j][q];
            } else {
#pragma unroll
                for (int q = 0; q < kN; ++q) acc[q] += x[j][q];
            }
        }
    }
    flush(key[1 + count] == cur);
}

// The row that begins in a window and goes on in the next ones: their pieces in order, eight on their way at a time (2 to 8 us after the
// sums, most of it the launch).
template <int GT, int OT, bool VEC>
__global__ void __launch_bounds__(kSumThreads) tli_grad_join_kernel(const __grid_constant__ GradParams P) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int n = __ldcg(P.n_valid);
    const int win = blockIdx.x * (kSumThreads / P.tx) + threadIdx.x / P.tx;
    const Columns<GT, VEC> c(P, blockIdx.y);
    const int a = win * P.window, e = a + P.window;
    if (win >= P.nwin || e >= n || !c.any(P)) return;
    const int *key = P.key[1];
    const int cur = __ldcg(key + e - 1), next = __ldcg(key + e), before = a > 0 ? __ldcg(key + a - 1) : -1;
    if (next != cur || before == cur) return;                      // ends in this window, or began before it
    constexpr int kN = Columns<GT, VEC>::kN, kBatch = 8;
    float acc[kN] = {};
    c.add(P, P.piece + (static_cast<size_t>(win) * 2 + 1) * P.H, acc);
    bool more = true;
#pragma unroll 1
    for (int w = win + 1; more; w += kBatch) {
        bool in[kBatch];
        float x[kBatch][kN];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int first = (w + j) * P.window;                  // a window that begins with the row has a piece of it
            in[j] = first < n && __ldcg(key + first) == cur;
#pragma unroll
            for (int q = 0; q < kN; ++q) x[j][q] = 0.f;
            // (pieces of windows behind the row's end are stale or foreign, but there: they are read and not used)
            if (w + j < P.nwin) c.add(P, P.piece + (static_cast<size_t>(w + j) * 2) * P.H, x[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            more = more && in[j];
            if (more) {
#pragma unroll
                for (int q = 0; q < kN; ++q) acc[q] += x[j][q];
            }
        }
    }
    c.template store<OT>(P, cur, acc);
}

// ---- host ----

constexpr int kSortOneCluster = 131072;    // tokens one cluster sorts (it runs beside the zero fill)
constexpr int kSortTile = 16384;           // tokens per CTA beyond that

struct GradLayout { int groups, tile, clustered, window, nwin; size_t key0, pos0, key1, pos1, n_valid, count, piece, total; };

GradLayout grad_layout(int N, int H) {
    GradLayout L;
    L.clustered = N > 0 && N <= kSortOneCluster;
    L.groups = L.clustered ? kSortCluster : (N + kSortTile - 1) / kSortTile;
    L.tile = L.clustered ? ((N + kSortCluster - 1) / kSortCluster + 31) & ~31 : kSortTile;
    // short windows spread few tokens over more threads, long ones keep the pieces of many tokens few
    L.window = 8;
    while (L.window < kMaxWindow && N / L.window > 512) L.window *= 2;
    L.nwin = (N + L.window - 1) / L.window;
    size_t off = 0;
    L.key0 = off; off = align_up(off + sizeof(int) * N, 256);
    L.pos0 = off; off = align_up(off + sizeof(int) * N, 256);
    L.key1 = off; off = align_up(off + sizeof(int) * N, 256);
    L.pos1 = off; off = align_up(off + sizeof(int) * N, 256);
    L.n_valid = off; off += 256;
    L.count = off; off = align_up(off + sizeof(int) * kDigits * L.groups, 256);
    L.piece = off; off = align_up(off + sizeof(float) * 2 * L.nwin * static_cast<size_t>(H), 256);
    L.total = off;
    return L;
}

int embed_side(const tli_ctx *ctx, int32_t ids_side, int32_t table_side, int &n_ids, int &V, const int *&map) {
    if (ids_side != TLI_SIDE_TARGET && ids_side != TLI_SIDE_DRAFTER) return TLI_ERR_ARG;
    if (table_side != TLI_SIDE_TARGET && table_side != TLI_SIDE_DRAFTER) return TLI_ERR_ARG;
    n_ids = ids_side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d;
    V = table_side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d;
    map = ids_side == table_side ? nullptr : (ids_side == TLI_SIDE_DRAFTER ? ctx->d_map : ctx->d_inv);
    return TLI_OK;
}
bool on_vectors(const void *p, int64_t stride, size_t elt) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * static_cast<int64_t>(elt) % 16 == 0;
}
// As many clusters of a kernel as are resident together (two at least), asked once per device.
struct ClustersResident {
    std::atomic<int> known[64] = {};
    cudaError_t get(const void *fn, const cudaLaunchConfig_t *cfg, int device, int &n) {
        n = device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
        if (n > 0) return cudaSuccess;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, fn, cfg);
        if (e != cudaSuccess) return e;
        n = std::max(2, n);
        if (device < 64) known[device].store(n, std::memory_order_relaxed);
        return cudaSuccess;
    }
};
void pdl_config(cudaLaunchConfig_t &cfg, cudaLaunchAttribute *attr, cudaStream_t stream) {
    memset(&cfg, 0, sizeof cfg);
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = stream;
}

template <int GT, int OT, bool VEC> int launch_grad_sums(const GradParams &P, int device, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, stream);
    constexpr int kN = Columns<GT, VEC>::kN;
    const int per_block = P.tx * kN;
    cfg.gridDim = dim3((P.nwin + kSumThreads / P.tx - 1) / (kSumThreads / P.tx), (P.H + per_block - 1) / per_block);
    cfg.blockDim = dim3(kSumThreads);
    cfg.dynamicSmemBytes = sizeof(int) * (2 * P.window + 2) * (kSumThreads / P.tx);
    static SmemAllowed allowed;
    cudaError_t e = allowed.set(reinterpret_cast<const void *>(tli_grad_sum_kernel<GT, OT, VEC>), sizeof(int) * (2 * kMaxWindow + 2) * kSumThreads / kSumMinTx, device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
    e = cudaLaunchKernelEx(&cfg, tli_grad_sum_kernel<GT, OT, VEC>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_grad_sum_kernel");
    cfg.dynamicSmemBytes = 0;
    e = cudaLaunchKernelEx(&cfg, tli_grad_join_kernel<GT, OT, VEC>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_grad_join_kernel");
    return TLI_OK;
}

template <int OT> int launch_grad(GradParams &P, int gdtype, int device, int num_sms, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, stream);
    const size_t smem = kSortSmem;
    static SmemAllowed allowed_sort, allowed_scatter;
    cudaError_t e = allowed_sort.set(reinterpret_cast<const void *>(tli_grad_sort_kernel<OT>), smem, device);
    if (e == cudaSuccess) e = allowed_scatter.set(reinterpret_cast<const void *>(tli_grad_scatter_kernel), smem, device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
    cfg.blockDim = dim3(kSortThreads);
    {
        cudaLaunchAttribute both[2];
        both[0] = attr[0];
        both[1].id = cudaLaunchAttributeClusterDimension;
        both[1].val.clusterDim.x = kSortCluster; both[1].val.clusterDim.y = 1; both[1].val.clusterDim.z = 1;
        cfg.attrs = both; cfg.numAttrs = P.clustered ? 2 : 1;
        cfg.gridDim = dim3(num_sms); cfg.dynamicSmemBytes = 0;
        if (P.clustered) {
            // as many clusters as are resident together: the fill's shares are fixed, so a second wave would double its time
            static ClustersResident resident;
            int clusters = 0;
            cfg.gridDim = dim3(2 * kSortCluster); cfg.dynamicSmemBytes = smem;
            cudaLaunchConfig_t ask = cfg;
            ask.attrs = both + 1; ask.numAttrs = 1;
            e = resident.get(reinterpret_cast<const void *>(tli_grad_sort_kernel<OT>), &ask, device, clusters);
            if (e != cudaSuccess) return cuda_fail(e, "cudaOccupancyMaxActiveClusters");
            cfg.gridDim = dim3(clusters * kSortCluster);
        }
        e = cudaLaunchKernelEx(&cfg, tli_grad_sort_kernel<OT>, P);
        cfg.attrs = attr; cfg.numAttrs = 1;
    }
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_grad_sort_kernel");
    if (P.N == 0) return TLI_OK;
    if (!P.clustered) {
        for (int pass = 0; pass < 2; ++pass) {
            cfg.gridDim = dim3(P.groups); cfg.dynamicSmemBytes = 0;
            e = cudaLaunchKernelEx(&cfg, tli_grad_count_kernel, P, pass);
            if (e != cudaSuccess) return cuda_fail(e, "launch tli_grad_count_kernel");
            cfg.dynamicSmemBytes = smem;
            e = cudaLaunchKernelEx(&cfg, tli_grad_scatter_kernel, P, pass);
            if (e != cudaSuccess) return cuda_fail(e, "launch tli_grad_scatter_kernel");
        }
    }
    const size_t ge = gdtype == TLI_F32 ? 4 : 2;
    const bool vec = on_vectors(P.g, P.gs, ge) && on_vectors(P.out, P.os, Elt<OT>::kBytes) && P.H % 8 == 0;
    const int across = vec ? P.H / (gdtype == TLI_F32 ? 4 : 8) : (P.H + 3) / 4;
    P.tx = kSumMinTx;
    while (P.tx < kSumThreads && P.tx < across) P.tx *= 2;
    if (gdtype == TLI_F32) return vec ? launch_grad_sums<TLI_F32, OT, true>(P, device, stream) : launch_grad_sums<TLI_F32, OT, false>(P, device, stream);
    return vec ? launch_grad_sums<TLI_BF16, OT, true>(P, device, stream) : launch_grad_sums<TLI_BF16, OT, false>(P, device, stream);
}

}  // namespace

extern "C" {

int tli_embed(tli_ctx *ctx, const tli_embed_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    if (a->N < 0 || a->H < 1) return TLI_ERR_ARG;
    if (a->N > TLI_MAX_TOKENS || a->H > TLI_MAX_H) return TLI_ERR_UNSUPPORTED;
    if (a->dtype != TLI_F32 && a->dtype != TLI_BF16) return TLI_ERR_ARG;
    EmbedParams P;
    int V;
    const int rc = embed_side(ctx, a->ids_side, a->table_side, P.n_ids, V, P.map);
    if (rc != TLI_OK) return rc;
    if (a->N == 0) return TLI_OK;
    if (!a->ids || !a->table || !a->out || !aligned4({a->ids, a->table_ids}) || !on_device(ctx)) return TLI_ERR_ARG;
    const size_t elt = a->dtype == TLI_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(a->table) % elt || reinterpret_cast<uintptr_t>(a->out) % elt) return TLI_ERR_ARG;
    if (a->table_stride < 0 || (a->N > 1 && a->out_stride < a->H)) return TLI_ERR_ARG;
    P.N = a->N; P.H = a->H; P.ids = a->ids;
    P.table = a->table; P.ts = a->table_stride;
    P.out = a->out; P.os = a->out_stride;
    P.scale = a->scale; P.table_ids = a->table_ids;
    const int epv = static_cast<int>(16 / elt);
    const bool vec = on_vectors(P.table, P.ts, elt) && on_vectors(P.out, P.os, elt) && P.H % epv == 0;
    const int units = vec ? P.H / epv : P.H;
    P.chunks = (units + 32 * kEmbUnroll - 1) / (32 * kEmbUnroll);
    const long long tasks = static_cast<long long>(P.N) * P.chunks, per = kEmbThreads / 32;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, reinterpret_cast<cudaStream_t>(cuda_stream));
    cfg.gridDim = dim3(static_cast<unsigned>((tasks + per - 1) / per)); cfg.blockDim = dim3(kEmbThreads);
    cudaError_t e;
    if (a->dtype == TLI_F32) e = vec ? cudaLaunchKernelEx(&cfg, tli_embed_kernel<TLI_F32, true>, P) : cudaLaunchKernelEx(&cfg, tli_embed_kernel<TLI_F32, false>, P);
    else e = vec ? cudaLaunchKernelEx(&cfg, tli_embed_kernel<TLI_BF16, true>, P) : cudaLaunchKernelEx(&cfg, tli_embed_kernel<TLI_BF16, false>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_embed_kernel");
    return TLI_OK;
}

size_t tli_embed_grad_workspace_bytes(const tli_ctx *ctx, int32_t N, int32_t H) {
    if (!ctx || ctx->n_shards != 1 || N < 0 || H < 1 || N > TLI_MAX_TOKENS || H > TLI_MAX_H) return 0;
    return grad_layout(N, H).total;
}

int tli_embed_grad(tli_ctx *ctx, const tli_embed_grad_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    if (a->N < 0 || a->H < 1) return TLI_ERR_ARG;
    if (a->N > TLI_MAX_TOKENS || a->H > TLI_MAX_H) return TLI_ERR_UNSUPPORTED;
    if ((a->grad_dtype != TLI_F32 && a->grad_dtype != TLI_BF16) || (a->out_dtype != TLI_F32 && a->out_dtype != TLI_BF16)) return TLI_ERR_ARG;
    GradParams P;
    memset(&P, 0, sizeof P);
    const int rc = embed_side(ctx, a->ids_side, a->table_side, P.n_ids, P.V, P.map);
    if (rc != TLI_OK) return rc;
    if (!a->out || (a->N > 0 && (!a->ids || !a->grad)) || !aligned4({a->ids}) || !on_device(ctx)) return TLI_ERR_ARG;
    const size_t ge = a->grad_dtype == TLI_F32 ? 4 : 2, oe = a->out_dtype == TLI_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(a->grad) % ge || reinterpret_cast<uintptr_t>(a->out) % oe) return TLI_ERR_ARG;
    if (a->grad_stride < 0 || (P.V > 1 && a->out_stride < a->H)) return TLI_ERR_ARG;
    const GradLayout L = grad_layout(a->N, a->H);
    if (!a->workspace || reinterpret_cast<uintptr_t>(a->workspace) % 256 || a->workspace_bytes < L.total) return TLI_ERR_WORKSPACE;
    P.N = a->N; P.H = a->H; P.groups = L.groups; P.tile = L.tile; P.clustered = L.clustered; P.window = L.window; P.nwin = L.nwin;
    P.ids = a->ids;
    P.g = a->grad; P.gs = a->grad_stride;
    P.out = a->out; P.os = a->out_stride;
    P.scale = a->scale;
    char *ws = reinterpret_cast<char *>(a->workspace);
    P.key[0] = reinterpret_cast<int *>(ws + L.key0); P.pos[0] = reinterpret_cast<int *>(ws + L.pos0);
    P.key[1] = reinterpret_cast<int *>(ws + L.key1); P.pos[1] = reinterpret_cast<int *>(ws + L.pos1);
    P.n_valid = reinterpret_cast<int *>(ws + L.n_valid);
    P.count = reinterpret_cast<int *>(ws + L.count);
    P.piece = reinterpret_cast<float *>(ws + L.piece);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
    return a->out_dtype == TLI_F32 ? launch_grad<TLI_F32>(P, a->grad_dtype, ctx->device, ctx->num_sms, stream)
                                   : launch_grad<TLI_BF16>(P, a->grad_dtype, ctx->device, ctx->num_sms, stream);
}

}  // extern "C"
