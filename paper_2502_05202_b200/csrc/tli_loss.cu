// Losses of rows of logits, against a label or a teacher's top logits, and their gradients.
// (Part of tli_lib.cu: uses RowView, row_vectors, table_id, tli_ctx and the error helpers of the parts before it.)
//
//   tli_loss_kernel        one thread-block cluster (1 to 8 CTAs) per row: running (max, sum) per thread in one pass over the
//                          row, joined through warps, the CTA and distributed shared memory; the row's targets beside it.
//   tli_loss_grad_kernel   a row, or a run of it where rows are few, per CTA: g/tau q everywhere, then the targets' elements again.
//
// Both are passes over the logits: bound by DRAM, and for bf16 rows near the special-function unit's rate (one ex2 per
// element; 16 a clock and SM are 4.4e12/s where 6.5 TB/s of bf16 are 3.3e12/s).
//
// A weight is 2^((z - m) s) with s = log2(e)/tau and m the largest logit seen.  The difference comes first: z*s - m*s in one fma would
// save an instruction of four per pair, but the rounding of m*s, which all weights of a row share, is 2^-24 |m s| of them (and beyond
// |m s| = 2^30 nothing is left of them).

namespace {

// Threads of a CTA: 64 for rows that are a batch or two of theirs (and have as few targets), 256 otherwise: what a short row costs beside its bytes
// then overlaps with more rows' (5372 bf16 rows of 1726, 7 targets, gradient: 13 us against 24).
constexpr int kLossThreads = 256, kLossShort = 64;
// 16-byte vectors a thread has on their way.  bf16 rows are half compute: they want warps (six CTAs per SM) more than loads in flight.  1500 of
// 50 257 over the intersection: 54 us with eight and three CTAs, 46 with four and four, 42 with four and six; 8192 of 128 256: 361 with four and
// six, 377 with two and six (for six, 40 registers, the compiler keeps 52 bytes a thread in local memory, which those times have in them).  fp32 rows the other way: 4096 of 256 000 in 613 us with eight, 648 with four.  (The next batch asked for before
// this one is worked on costs registers, hence warps: 48 us.)
template <int DT> constexpr int kLossBatch = DT == TLI_F32 ? 8 : 4;
constexpr int kLossMaxCluster = 8;
constexpr long long kLossFill = 8;         // CTAs per SM that rows are cut for
constexpr float kMaskBelow = -1e30f;       // a logit below it is a mask
constexpr float kLog2e = 1.4426950408889634f;
static_assert(TLI_MAX_TARGETS <= kLossThreads, "a thread per target");

// What the targets of a row are looked up with.
struct TargetParams {
    int N, k, n_ids;
    const int *map;                        // NULL: the ids are the rows'
    const uint32_t *mask;                  // ids that take part; NULL: all
    const int *ids;
    const void *teacher; int teacher_bf16;
    const float *tau;
};

struct LossParams {
    TargetParams T;
    int V, cluster;
    const void *z; long long stride;
    float *loss, *stats; int *status;
    const float *g;
    void *grad; long long grad_stride;
    int seg, nseg;                         // gradient: vectors of a CTA's run, runs per row
    int same_grid;                         // ... the gradient's rows lie on the logits' 16-byte grid
};

// The scale of a row, s = log2(e)/tau; false where the temperature is none.
__device__ __forceinline__ bool row_scale(const float *tau, long long row, float &t, float &s) {
    t = tau ? __ldg(tau + row) : 1.f;
    s = kLog2e / t;
    return t > 0.f && t < INFINITY && s > 0.f && s < INFINITY;
}
// Target j of a row: its id among the rows' and its teacher logit; -1 if it does not take part.
__device__ __forceinline__ int row_target(const TargetParams &T, long long row, int j, float &teacher) {
    const long long at = row * T.k + j;
    teacher = 0.f;
    int id = __ldg(T.ids + at);
    if (T.teacher) {
        teacher = T.teacher_bf16 ? __uint_as_float(static_cast<uint32_t>(__ldg(reinterpret_cast<const unsigned short *>(T.teacher) + at)) << 16)
                                 : __ldg(reinterpret_cast<const float *>(T.teacher) + at);
        if (teacher < kMaskBelow) return -1;
    }
    id = table_id(T.map, T.n_ids, id);
    if (id >= 0 && T.mask && !(__ldg(T.mask + (id >> 5)) >> (id & 31) & 1u)) id = -1;
    return id;
}

__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}
// Sum and maximum over the CTA, the same in every thread; `sh` has a word per warp and is free again when they return.
template <int WARPS> __device__ __forceinline__ float block_sum(float x, float *sh) {
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) t += sh[i];
    __syncthreads();
    return t;
}
template <int WARPS> __device__ __forceinline__ float block_max(float x, float *sh) {
    x = warp_max(x);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    float t = sh[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) t = fmaxf(t, sh[i]);
    __syncthreads();
    return t;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// One more batch of vectors into a thread's (m, sum of 2^((z - m) s)).  NaN and +inf end as a NaN sum.
template <int DT, int B> __device__ __forceinline__ void loss_batch(const uint4 (&raw)[B], float s, float &m, float &sum) {
    float top;
    if constexpr (DT == TLI_BF16) {
        uint32_t mm = bf16x2_max(bf16x2_max(raw[0].x, raw[0].y), bf16x2_max(raw[0].z, raw[0].w));
#pragma unroll
        for (int q = 1; q < B; ++q) mm = bf16x2_max(mm, bf16x2_max(bf16x2_max(raw[q].x, raw[q].y), bf16x2_max(raw[q].z, raw[q].w)));
        top = fmaxf(bf16_lo(mm), bf16_hi(mm));
    } else {
        top = -INFINITY;
#pragma unroll
        for (int q = 0; q < B; ++q)
            top = fmaxf(top, fmaxf(fmaxf(__uint_as_float(raw[q].x), __uint_as_float(raw[q].y)), fmaxf(__uint_as_float(raw[q].z), __uint_as_float(raw[q].w))));
    }
    if (top > m) {
        sum *= ex2((m - top) * s);
        m = top;
    }
    const uint64_t s2 = pack2(s, s), c2 = pack2(-m, -m);
    uint64_t a[2] = {pack2(sum, 0.f), 0ull};
#pragma unroll
    for (int q = 0; q < B; ++q) {
        float z[Elt<DT>::kPerVec];
        unpack<DT>(raw[q], z);
#pragma unroll
        for (int i = 0; i < Elt<DT>::kPerVec; i += 2) {
            float x, y;
            unpack2(mul2(add2(pack2(z[i], z[i + 1]), c2), s2), x, y);
            a[(i >> 1) & 1] = add2(a[(i >> 1) & 1], pack2(ex2(x), ex2(y)));
        }
    }
    float w0, w1, w2, w3;
    unpack2(a[0], w0, w1);
    unpack2(a[1], w2, w3);
    sum = (w0 + w1) + (w2 + w3);
}

// Two (m, sum) into one.
__device__ __forceinline__ void join_stats(float s, float &m, float &sum, float m2, float sum2) {
    const float top = fmaxf(m, m2);
    sum = sum * ex2((m - top) * s) + sum2 * ex2((m2 - top) * s);
    m = top;
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// Bound by DRAM on large batches: 4096 fp32 rows of 256 000 (4.2 GB) in 0.61 ms, 6.8 TB/s; 8192 bf16 rows of 128 256 (2.1 GB) in 0.34 to 0.38 ms, 5.6 to
// 6.2 TB/s, with the special-function unit active 79 % of the cycles and DRAM at 77 % of its nominal rate.  On smaller ones by what a row costs beside its bytes (lookups, joins) and by how its CTAs fill the SMs: 1500
// bf16 rows of 50 257 over the intersection, 20 targets each, 41 us for 151 MB, 34 without mask and with even rows.
template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, (DT == TLI_F32 ? 3 : 6) * (kLossThreads / THREADS)) tli_loss_kernel(const __grid_constant__ LossParams P) {
    constexpr int WARPS = THREADS / 32, kBatch = kLossBatch<DT>;
    __shared__ float sh[WARPS], sh_m[WARPS], sh_s[WARPS];
    __shared__ float part[kLossMaxCluster][2];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int C = P.cluster, rank = static_cast<int>(blockIdx.x % C), tid = threadIdx.x;
    const long long row = blockIdx.x / C;
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const RowView<DT> rv(P.z, row * P.stride, P.V);
    const int nvec = rv.nvec(), per = (nvec + C - 1) / C, v0 = rank * per, v1 = min(nvec, v0 + per);
    float tau, s, teacher = 0.f, z_t = 0.f;
    uint4 raw[kBatch];
    auto load = [&](int at) {
        int v[kBatch];
#pragma unroll
        for (int q = 0; q < kBatch; ++q) v[q] = at + q * THREADS;
        row_vectors<DT, kBatch>(rv.vec0, rv.row, rv.head, P.V, v1, P.T.mask, v, raw);
    };
    load(v0 + tid);                                                // (on their way while the targets are looked up)
    const bool scale_ok = row_scale(P.T.tau, row, tau, s);
    const int target = tid < P.T.k ? row_target(P.T, row, tid, teacher) : -1;
    float m = kMaskBelow, sum = 0.f;
    if (v0 + tid < v1) loss_batch<DT, kBatch>(raw, s, m, sum);
    const int any = __syncthreads_or(target >= 0);                 // the same in every CTA of the cluster, as is scale_ok
    if (!any || !scale_ok) {
        if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (rank == 0 && tid == 0) {
            P.loss[row] = 0.f;
            reinterpret_cast<float2 *>(P.stats)[row] = make_float2(0.f, 0.f);
            if (P.status) P.status[row] = (any ? 0 : TLI_ROW_LEFT_OUT) | (scale_ok ? 0 : TLI_ROW_BAD_TEMPERATURE);
        }
        return;
    }
    if (rank == 0 && target >= 0) z_t = load_elt<DT>(rv.row, target);
#pragma unroll 1
    for (int at = v0 + tid + THREADS * kBatch; at < v1; at += THREADS * kBatch) {
        load(at);
        loss_batch<DT, kBatch>(raw, s, m, sum);
    }
    const float wm = warp_max(m);
    sum = warp_sum(sum * ex2((m - wm) * s));
    if ((tid & 31) == 0) { sh_m[tid >> 5] = wm; sh_s[tid >> 5] = sum; }
    __syncthreads();
    m = sh_m[0]; sum = sh_s[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) join_stats(s, m, sum, sh_m[i], sh_s[i]);
    if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");        // every CTA of the cluster is running
        if (rank > 0 && tid == 0) {
            const uint32_t to = cluster_addr(smem_addr(&part[rank][0]), 0u);
            st_cluster_f32(to, m);
            st_cluster_f32(to + 4, sum);
        }
        __syncwarp();
        cluster_barrier();
        if (rank > 0) return;
        for (int i = 1; i < C; ++i) join_stats(s, m, sum, part[i][0], part[i][1]);
    }
    // the targets: ln p_j = (t_j - max t)/tau - ln W
    float ent, W = 1.f;
    if (P.T.teacher && P.T.k <= 32) {                              // one warp has all of them
        if (tid >= 32) return;
        const float tm = warp_max(target >= 0 ? teacher : -INFINITY);
        const float w = target >= 0 ? ex2((teacher - tm) * s) : 0.f;
        W = warp_sum(w);
        ent = warp_sum(w != 0.f ? w * (((m - z_t) + (teacher - tm)) / tau) : 0.f);
    } else if (P.T.teacher) {
        const float tm = block_max<WARPS>(target >= 0 ? teacher : -INFINITY, sh);
        const float w = target >= 0 ? ex2((teacher - tm) * s) : 0.f;
        W = block_sum<WARPS>(w, sh);
        ent = block_sum<WARPS>(w != 0.f ? w * (((m - z_t) + (teacher - tm)) / tau) : 0.f, sh);
    } else {
        ent = (m - z_t) / tau;                                     // of thread 0
    }
    if (tid == 0) {
        const bool none = sum == 0.f, bad = sum != sum || W != W;
        P.loss[row] = none ? 0.f : bad ? NAN : logf(sum) + (P.T.teacher ? ent / W - logf(W) : ent);
        reinterpret_cast<float2 *>(P.stats)[row] = none ? make_float2(0.f, 0.f) : make_float2(m, bad ? NAN : sum);
        if (P.status) P.status[row] = none ? TLI_ROW_FALLBACK : bad ? TLI_ROW_NONFINITE : 0;
    }
}

// What the gradient of row n is made of: dz = f 2^((z - m) s) - h p.
struct RowSlope {
    float s, m, f, h;                      // f = g/(tau sum), h = g/tau
    bool zero;
    __device__ __forceinline__ RowSlope(const float *taus, const float *stats, const float *g, long long row) {
        float tau;
        const bool ok = row_scale(taus, row, tau, s);
        const float2 st = __ldg(reinterpret_cast<const float2 *>(stats) + row);
        zero = !ok || st.y == 0.f;
        m = st.x;
        h = (g ? __ldg(g + row) : 1.f) / tau;
        f = h / st.y;
    }
    __device__ __forceinline__ float operator()(float z) const { return ex2((z - m) * s) * f; }
};

template <int DT> __device__ __forceinline__ uint4 pack_vector(const float (&x)[Elt<DT>::kPerVec]) {
    if constexpr (DT == TLI_F32) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// The probability mass of the teacher on a target's id, in every thread that has a target: all targets of the row with that id.
template <int THREADS> __device__ __forceinline__ float target_mass(const TargetParams &T, int target, float teacher, float s, float *sh, int *sh_id, float *sh_w) {
    constexpr int WARPS = THREADS / 32;
    const float tm = block_max<WARPS>(target >= 0 ? teacher : -INFINITY, sh);
    const float w = target >= 0 ? ex2((teacher - tm) * s) : 0.f;
    const float W = block_sum<WARPS>(w, sh);
    if (static_cast<int>(threadIdx.x) < T.k) { sh_id[threadIdx.x] = target; sh_w[threadIdx.x] = w; }
    __syncthreads();
    float mass = 0.f;
    if (target >= 0)
        for (int j = 0; j < T.k; ++j) mass += sh_id[j] == target ? sh_w[j] : 0.f;
    return mass / W;
}

// Bound by DRAM: 8192 bf16 rows of 128 256 (2.1 GB read, 2.1 written) in 0.65 ms, 6.4 TB/s; 4096 fp32 rows of as many in 0.67 ms, 6.3 TB/s; 2048 of 49 152 with 32 targets and a mask in 76 us, 5.3 TB/s
// (92 us with 32 KB of a row per CTA: the targets are then looked up three times a row).
template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS) tli_loss_grad_kernel(const __grid_constant__ LossParams P) {
    constexpr int EPV = Elt<DT>::kPerVec, kBatch = kLossBatch<DT>;
    __shared__ float sh[THREADS / 32], sh_w[THREADS];
    __shared__ int sh_id[THREADS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, seg = static_cast<int>(blockIdx.x % P.nseg);
    const long long row = blockIdx.x / P.nseg;
    const RowView<DT> rv(P.z, row * P.stride, P.V);
    const int nvec = rv.nvec(), v0 = seg * P.seg, v1 = min(nvec, v0 + P.seg);
    const RowSlope slope(P.T.tau, P.stats, P.g, row);
    char *out = reinterpret_cast<char *>(P.grad) + row * P.grad_stride * Elt<DT>::kBytes;
    const int e_lo = max(0, v0 * EPV - rv.head), e_hi = min(P.V, v1 * EPV - rv.head);
    uint4 raw[kBatch];
    auto load = [&](int at) {
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            const int v = at + q * THREADS, e0 = v * EPV - rv.head;
            raw[q] = make_uint4(Elt<DT>::kNegInfWord, Elt<DT>::kNegInfWord, Elt<DT>::kNegInfWord, Elt<DT>::kNegInfWord);
            if (v < v1) raw[q] = e0 >= 0 && e0 + EPV <= P.V ? __ldcg(rv.vec0 + v) : ragged_vector<DT>(rv.row, e0, P.V);
        }
    };
    load(v0 + tid);                                                // (on their way while the targets are looked up)
    // the targets of this run, their logits before anything is overwritten (the gradient may lie on the logits)
    int target = -1;
    float teacher = 0.f, z_t = 0.f;
    if (!slope.zero && tid < P.T.k) target = row_target(P.T, row, tid, teacher);
    const bool here = target >= e_lo && target < e_hi;
    if (here) z_t = load_elt<DT>(rv.row, target);
    const int any = __syncthreads_or(here);
    float mass = 1.f;
    if (any && P.T.teacher) mass = target_mass<THREADS>(P.T, target, teacher, slope.s, sh, sh_id, sh_w);
#pragma unroll 1
    for (int at = v0 + tid; at < v1; ) {
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            const int v = at + q * THREADS, e0 = v * EPV - rv.head;
            if (v >= v1) break;
            if (P.T.mask) raw[q] = mask_vector<DT>(raw[q], P.T.mask, e0);
            float x[EPV];
            unpack<DT>(raw[q], x);
#pragma unroll
            for (int i = 0; i < EPV; ++i) x[i] = slope.zero ? 0.f : slope(x[i]);
            if (P.same_grid && e0 >= 0 && e0 + EPV <= P.V) {
                *reinterpret_cast<uint4 *>(out + static_cast<long long>(e0) * Elt<DT>::kBytes) = pack_vector<DT>(x);
            } else {
#pragma unroll
                for (int i = 0; i < EPV; ++i)
                    if (e0 + i >= 0 && e0 + i < P.V) set_element<DT>(out, e0 + i, x[i]);
            }
        }
        at += THREADS * kBatch;
        if (at < v1 && !slope.zero) load(at);
    }
    if (any) {
        __syncthreads();
        if (here) set_element<DT>(out, target, fmaf(-slope.h, mass, slope(z_t)));
    }
}

// ---- host ----

// What the loss calls check alike.  Fills T; V: ids of the rows' vocabulary.
int check_targets(const tli_ctx *ctx, int32_t N, int32_t k, int32_t side, int32_t ids_side, int32_t support, const int32_t *ids,
                  const void *teacher, int32_t teacher_dtype, const float *temperature, TargetParams &T, int &V) {
    if (N < 0 || k < 1 || (!teacher && k != 1)) return TLI_ERR_ARG;
    if (k > TLI_MAX_TARGETS) return TLI_ERR_UNSUPPORTED;
    if (support != TLI_SUPPORT_ALL && support != TLI_SUPPORT_SHARED) return TLI_ERR_ARG;
    if (support == TLI_SUPPORT_SHARED && side != TLI_SIDE_DRAFTER) return TLI_ERR_ARG;
    if (teacher && teacher_dtype != TLI_F32 && teacher_dtype != TLI_BF16) return TLI_ERR_ARG;
    memset(&T, 0, sizeof T);
    const int rc = embed_side(ctx, ids_side, side, T.n_ids, V, T.map);
    if (rc != TLI_OK) return rc;
    if (N > 0 && !ids) return TLI_ERR_ARG;
    if (!aligned4({ids, temperature}) || reinterpret_cast<uintptr_t>(teacher) % (teacher_dtype == TLI_BF16 ? 2 : 4)) return TLI_ERR_ARG;
    if (!on_device(ctx)) return TLI_ERR_ARG;
    T.N = N; T.k = k; T.ids = ids; T.tau = temperature;
    T.mask = support == TLI_SUPPORT_SHARED ? ctx->d_mask : nullptr;
    T.teacher = teacher; T.teacher_bf16 = teacher && teacher_dtype == TLI_BF16;
    return TLI_OK;
}
// Rows of nvec vectors in `parts` CTAs each: whether the short CTA is the better one, up to `batches` of its batches.  5372 bf16 rows: 36 us against 41 at
// eight (16 000 ids), 69 against 66 at sixteen; 4000 fp32 rows, loss: 23 against 28 at four, the same at eight; gradient: 44 against 42 at four.
bool few_threads(long long nvec, int dtype, int k, int parts, int batches) {
    return parts == 1 && k <= kLossShort && nvec <= static_cast<long long>(batches) * kLossShort * (dtype == TLI_F32 ? kLossBatch<TLI_F32> : kLossBatch<TLI_BF16>);
}
bool aligned8(const void *p) { return reinterpret_cast<uintptr_t>(p) % 8 == 0; }

int check_loss(const tli_ctx *ctx, int32_t dtype, const void *logits, int64_t stride, const TargetParams &T, int V, LossParams &P) {
    if (T.N > TLI_MAX_TOKENS) return TLI_ERR_UNSUPPORTED;
    if (dtype != TLI_F32 && dtype != TLI_BF16) return TLI_ERR_ARG;
    const size_t elt = dtype == TLI_F32 ? 4 : 2;
    if ((T.N > 0 && !logits) || reinterpret_cast<uintptr_t>(logits) % elt || stride < 0) return TLI_ERR_ARG;
    memset(&P, 0, sizeof P);
    P.T = T; P.V = V; P.z = logits; P.stride = stride;
    return TLI_OK;
}

}  // namespace

extern "C" {

int tli_loss(tli_ctx *ctx, const tli_loss_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    TargetParams T;
    LossParams P;
    int V;
    int rc = check_targets(ctx, a->N, a->k, a->side, a->ids_side, a->support, a->ids, a->teacher, a->teacher_dtype, a->temperature, T, V);
    if (rc == TLI_OK) rc = check_loss(ctx, a->dtype, a->logits, a->stride, T, V, P);
    if (rc != TLI_OK) return rc;
    if (a->N == 0) return TLI_OK;
    if (!a->loss || !a->stats || !aligned4({a->loss, a->status}) || !aligned8(a->stats)) return TLI_ERR_ARG;
    P.loss = a->loss; P.stats = a->stats; P.status = a->status;
    // CTAs per row: as many as keep every SM busy, none with less than a batch per thread
    const long long nvec = (V + (a->dtype == TLI_F32 ? 3 : 7)) / (a->dtype == TLI_F32 ? 4 : 8) + 1;
    P.cluster = 1;
    while (P.cluster < kLossMaxCluster && static_cast<long long>(P.cluster) * a->N < kLossFill * ctx->num_sms && nvec > 2LL * P.cluster * kLossThreads) P.cluster *= 2;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    pdl_config(cfg, attr, reinterpret_cast<cudaStream_t>(cuda_stream));
    if (P.cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = P.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.gridDim = dim3(static_cast<unsigned>(a->N) * P.cluster); cfg.blockDim = dim3(kLossThreads);
    cudaError_t e;
    if (few_threads(nvec, a->dtype, a->k, P.cluster, a->dtype == TLI_F32 ? 4 : 8)) {
        cfg.blockDim = dim3(kLossShort);
        e = a->dtype == TLI_F32 ? cudaLaunchKernelEx(&cfg, tli_loss_kernel<TLI_F32, kLossShort>, P) : cudaLaunchKernelEx(&cfg, tli_loss_kernel<TLI_BF16, kLossShort>, P);
    } else {
        e = a->dtype == TLI_F32 ? cudaLaunchKernelEx(&cfg, tli_loss_kernel<TLI_F32, kLossThreads>, P) : cudaLaunchKernelEx(&cfg, tli_loss_kernel<TLI_BF16, kLossThreads>, P);
    }
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_loss_kernel");
    return TLI_OK;
}

int tli_loss_grad(tli_ctx *ctx, const tli_loss_grad_args *a, void *cuda_stream) {
    if (!ctx || !a || ctx->n_shards != 1) return TLI_ERR_ARG;
    TargetParams T;
    LossParams P;
    int V;
    int rc = check_targets(ctx, a->N, a->k, a->side, a->ids_side, a->support, a->ids, a->teacher, a->teacher_dtype, a->temperature, T, V);
    if (rc == TLI_OK) rc = check_loss(ctx, a->dtype, a->logits, a->stride, T, V, P);
    if (rc != TLI_OK) return rc;
    if (a->N == 0) return TLI_OK;
    const int64_t elt = a->dtype == TLI_F32 ? 4 : 2;
    if (!a->stats || !a->grad || !aligned4({a->grad_loss}) || !aligned8(a->stats) || reinterpret_cast<uintptr_t>(a->grad) % elt) return TLI_ERR_ARG;
    if (a->N > 1 && a->grad_stride < V) return TLI_ERR_ARG;
    if (rows_collide(reinterpret_cast<const char *>(a->logits), a->stride, 0, reinterpret_cast<const char *>(a->grad), a->grad_stride, 0, a->N, 1, V, elt)) return TLI_ERR_ARG;
    P.stats = const_cast<float *>(a->stats); P.g = a->grad_loss;
    P.grad = a->grad; P.grad_stride = a->grad_stride;
    P.same_grid = reinterpret_cast<uintptr_t>(a->grad) % 16 == reinterpret_cast<uintptr_t>(a->logits) % 16 &&
                  (a->N == 1 || (a->grad_stride - a->stride) * elt % 16 == 0);
    const long long nvec = (V + 16 / elt - 1) / (16 / elt) + 1;    // one more where a row begins inside a vector
    P.seg = static_cast<int>(nvec);
    while (P.seg > kLossThreads && (nvec + P.seg - 1) / P.seg * a->N < kLossFill * ctx->num_sms) P.seg = (P.seg + 1) / 2;
    P.seg = (P.seg + kLossThreads - 1) / kLossThreads * kLossThreads;
    P.nseg = static_cast<int>((nvec + P.seg - 1) / P.seg);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    pdl_config(cfg, attr, reinterpret_cast<cudaStream_t>(cuda_stream));
    cfg.gridDim = dim3(static_cast<unsigned>(a->N) * P.nseg); cfg.blockDim = dim3(kLossThreads);
    cudaError_t e;
    if (few_threads(nvec, a->dtype, a->k, P.nseg, a->dtype == TLI_F32 ? 2 : 8)) {
        cfg.blockDim = dim3(kLossShort);
        e = a->dtype == TLI_F32 ? cudaLaunchKernelEx(&cfg, tli_loss_grad_kernel<TLI_F32, kLossShort>, P) : cudaLaunchKernelEx(&cfg, tli_loss_grad_kernel<TLI_BF16, kLossShort>, P);
    } else {
        e = a->dtype == TLI_F32 ? cudaLaunchKernelEx(&cfg, tli_loss_grad_kernel<TLI_F32, kLossThreads>, P) : cudaLaunchKernelEx(&cfg, tli_loss_grad_kernel<TLI_BF16, kLossThreads>, P);
    }
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_loss_grad_kernel");
    return TLI_OK;
}

}  // extern "C"
