// Filtered sampling and filtered logits: temperature, top-k, top-p and min-p over rows of logits.
// (Part of tli_lib.cu: uses RowView, mask_bits, tli_ctx and the error helpers of tli.cu.)
//
// Mathematics.  Order the ids of a row by (logit descending, id ascending) and let w = exp((z - m)/tau),
// m the largest logit.  top-k keeps the first k, top-p the shortest prefix that holds p of their mass, min-p
// the ids with w >= min_p: three prefixes of one order, so what is kept is a prefix too, and one border
// (logit, id) says all of it.  The rest of the work is to find that border without sorting the row.
//
//   tli_rows_scan_kernel   reads every row once (HBM-bound): each lane leaves the largest of its U 16-byte vectors
//                          (a "group", 16*U bytes of the row) in the workspace, 1/(8U) or less of what it read;
//                          rows that need the whole mass (top-p without top-k, no filter at all) also leave a sum
//                          per strip of 32 groups.
//   tli_rows_pick_kernel   one CTA per row.  k groups have a largest element at or above the k-th largest group
//                          maximum, so at least k elements do: that maximum (taken from a histogram) is a
//                          floor under the border.  Only the groups that reach the floor are read again, their few
//                          elements sorted in shared memory, the border read off, the id drawn.  The same with
//                          mass instead of count for top-p.  Sets that do not fit the sort (flat rows, k in the
//                          thousands) go through a histogram over key digits instead: same border, more passes.
//   tli_rows_mask_kernel   (filter only) writes the row: -inf without reading it wherever the group maximum is
//                          below the border, the compared elements elsewhere.
//
// Weights and sums are fp64: the ids that come out are exact decisions (which id owns v * total, which one is
// the last inside top-p), and with 10^5 candidates an fp32 sum (2^-24 relative) would decide some of them by
// rounding.  An fp64 weight costs 13 fp64 operations; one pass over a row is then bound by the fp64 pipe only
// for 16-bit rows that need the whole mass.

namespace {

constexpr int kRowThreads = 256;                     // scan and mask kernels
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kPickThreads = 512;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kMaxGroups = 8192;                     // group maxima a pick CTA holds (coarser groups beyond)
constexpr int kListCap = 2048;                       // elements the sort takes
constexpr int kBins = 1024;

struct __align__(16) StripSum { double S; float m; int pad; };       // sum of 2^((z - m) s) over a strip, m its largest
struct __align__(16) RowBorder { float z; int id; int mode; int pad; };
enum : int { BORDER_APPLY = 0, BORDER_COPY = 1 };

struct RowsParams {
    int B, R, V, nstrip, coarse, sample;
    const void *z; long long sb, sr;
    const uint32_t *mask;                  // ids that can be kept; NULL: every id of the row
    const float *tau; const int *top_k; const float *top_p; const float *min_p; const float *u;
    int *tokens; float *prob; int *status;
    void *gmax;                            // [rows][nstrip * 32] in the rows' type
    StripSum *ssum;                        // [rows][nstrip]
    RowBorder *border;                     // [rows]
    void *out; long long osb, osr;
};

// ---- weights ----

// 2^(i/16); 16 doubles are one word line, so 32 lanes with any indices read it without a bank conflict
__device__ __forceinline__ void exp2_table_init(double *tab, int tid) {
    if (tid < 16) tab[tid] = exp2(tid / 16.0);
}
// 2^x for x in [-1021, 0]: x = n + i/16 + r, |r| <= 1/32, Taylor in r ln 2 to the sixth power
// (next term (ln2/32)^7/7! = 4e-16).
__device__ __forceinline__ double exp2_neg(double x, const double *tab) {
    constexpr double L = 0.693147180559945309417232;
    constexpr double c2 = L * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5, c6 = c5 * L / 6;
    constexpr double magic = 6755399441055744.0;                     // 1.5 * 2^52
    const double t = fma(x, 16.0, magic);
    const double r = fma(t - magic, -0.0625, x);
    const int n = __double2loint(t);
    double q = fma(r, c6, c5);
    q = fma(q, r, c4); q = fma(q, r, c3); q = fma(q, r, c2); q = fma(q, r, L); q = fma(q, r, 1.0);
    q *= tab[n & 15];
    return __hiloint2double(__double2hiint(q) + ((n >> 4) << 20), __double2loint(q));
}
// w(z) = exp((z - m)/tau), s = log2(e)/tau; 0 below cut (2^-1020 of the largest; -inf among them)
struct Weights {
    double m, s; float cut; const double *tab;
    __device__ __forceinline__ Weights(float m_, float tau, const double *tab_) {
        m = m_; s = 1.4426950408889634074 / tau; tab = tab_;
        cut = fmaxf(__double2float_ru(m - 1020.0 / s), -FLT_MAX);        // rounded up: z >= cut stays in exp2_neg's range
    }
    __device__ __forceinline__ double operator()(float z) const {
        const double w = exp2_neg((static_cast<double>(z) - m) * s, tab);
        return z >= cut ? w : 0.0;
    }
};

// ---- reading a row ----

template <int DT> __device__ __forceinline__ uint4 mask_vector(uint4 raw, const uint32_t *mask, int e0) {
    constexpr uint32_t NI = Elt<DT>::kNegInfWord;
    const uint32_t bits = mask_bits(mask, e0);
    if constexpr (DT == TLI_BF16) {
        mask_bf16_vector(raw, bits);
    } else {
        raw.x = (bits & 1u) ? raw.x : NI; raw.y = (bits & 2u) ? raw.y : NI;
        raw.z = (bits & 4u) ? raw.z : NI; raw.w = (bits & 8u) ? raw.w : NI;
    }
    return raw;
}
// Vector v of a row; ids outside the row or outside the mask read as -inf.
template <int DT>
__device__ __forceinline__ uint4 row_vector(const RowView<DT> &rv, const uint32_t *mask, int v, int nvec) {
    constexpr uint32_t NI = Elt<DT>::kNegInfWord;
    if (v >= nvec) return make_uint4(NI, NI, NI, NI);
    const uint4 raw = rv.load(v);
    return mask ? mask_vector<DT>(raw, mask, rv.first_elem(v)) : raw;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// largest element of U vectors, NaN if any is NaN
template <int DT, int U> __device__ __forceinline__ float vectors_max(const uint4 (&raw)[U]) {
    if constexpr (DT == TLI_BF16) {
        uint32_t mm = max_nan_bf16x2(max_nan_bf16x2(raw[0].x, raw[0].y), max_nan_bf16x2(raw[0].z, raw[0].w));
#pragma unroll
        for (int q = 1; q < U; ++q)
            mm = max_nan_bf16x2(mm, max_nan_bf16x2(max_nan_bf16x2(raw[q].x, raw[q].y), max_nan_bf16x2(raw[q].z, raw[q].w)));
        return max_nan(bf16_lo(mm), bf16_hi(mm));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int q = 0; q < U; ++q)
            m = max_nan(m, max_nan(max_nan(__uint_as_float(raw[q].x), __uint_as_float(raw[q].y)),
                                   max_nan(__uint_as_float(raw[q].z), __uint_as_float(raw[q].w))));
        return m;
    }
}
template <int DT> __device__ __forceinline__ void store_group(void *gmax, size_t i, float m) {
    if constexpr (DT == TLI_F32) __stcg(reinterpret_cast<float *>(gmax) + i, m);
    else __stcg(reinterpret_cast<unsigned short *>(gmax) + i, static_cast<unsigned short>(__float_as_uint(m) >> 16));
}
template <int DT> __device__ __forceinline__ float load_group(const void *gmax, size_t i) {
    if constexpr (DT == TLI_F32) return __ldcg(reinterpret_cast<const float *>(gmax) + i);
    else return __uint_as_float(static_cast<uint32_t>(__ldcg(reinterpret_cast<const unsigned short *>(gmax) + i)) << 16);
}

// What a row asks for, from its sequence's parameters.
struct RowAsk {
    float tau, p, least;
    int k;
    bool bad_tau, bad_filter, one, k_on, p_on, min_on;
    __device__ __forceinline__ RowAsk(const RowsParams &P, int b) {
        tau = __ldg(P.tau + b);
        k = P.top_k ? __ldg(P.top_k + b) : 0;
        p = P.top_p ? __ldg(P.top_p + b) : 1.f;
        least = P.min_p ? __ldg(P.min_p + b) : 0.f;
        bad_tau = !(tau >= 0.f && tau < INFINITY);
        bad_filter = p != p || least != least;
        one = tau == 0.f || k == 1 || p <= 0.f || least > 1.f;     // only the first id is kept
        k_on = k > 0 && k < P.V;
        p_on = p < 1.f;
        min_on = least > 0.f;
    }
    __device__ __forceinline__ bool plain() const { return !k_on && !p_on && !min_on; }
    // the mass of the whole row is asked for
    __device__ __forceinline__ bool whole_mass(int sample) const {
        return !bad_tau && !bad_filter && !one && !k_on && (p_on || (sample && !min_on));
    }
};

template <int DT, int U>
__global__ void __launch_bounds__(kRowThreads) tli_rows_scan_kernel(const RowsParams P) {
    __shared__ double tab[16];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.y, b = row / P.R;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int strip = blockIdx.x * kRowWarps + warp;
    const RowView<DT> rv(P.z, b * P.sb + (row - b * P.R) * P.sr, P.V);
    const int nvec = rv.nvec(), v0 = strip * (32 * U) + lane;
    uint4 raw[U];
    const bool live = strip < P.nstrip;
    if (live) {
#pragma unroll
        for (int q = 0; q < U; ++q) raw[q] = row_vector<DT>(rv, P.mask, v0 + q * 32, nvec);
    }
    const RowAsk ask(P, b);
    const bool sums = ask.whole_mass(P.sample);                    // the same for the whole CTA
    if (sums) {
        exp2_table_init(tab, threadIdx.x);
        __syncthreads();
    }
    if (!live) return;
    const float m = vectors_max<DT, U>(raw);
    store_group<DT>(P.gmax, static_cast<size_t>(row) * P.nstrip * 32 + strip * 32 + lane, m);
    if (!sums) return;
    const float ms = warp_max(m);
    double acc = 0.0;
    if (ms > -INFINITY && ms < INFINITY) {                         // NaN: not compared, the row is flagged later
        const Weights w(ms, ask.tau, tab);
#pragma unroll
        for (int q = 0; q < U; ++q) {
            float z[Elt<DT>::kPerVec];
            unpack<DT>(raw[q], z);
#pragma unroll
            for (int i = 0; i < Elt<DT>::kPerVec; ++i) acc += w(z[i]);
        }
    }
    acc = warp_sum(acc);
    if (lane == 0) {
        StripSum ss; ss.S = acc; ss.m = ms; ss.pad = 0;
        P.ssum[static_cast<size_t>(row) * P.nstrip + strip] = ss;
    }
}

// ---- block-wide steps of the pick kernel (all threads call them; each begins and ends with a barrier) ----

struct PickShared {
    double tab[16];
    double wsum[kPickWarps];
    unsigned long long wsum_u[kPickWarps];
    int wsum_i[kPickWarps];
    double bd[2];
    unsigned long long bu[2];
    int bi[4];
};

// inclusive prefix over the block's threads; total in `total`
template <typename T> __device__ __forceinline__ T block_scan(T x, T *slots, T &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) slots[warp] = x;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kPickWarps; ++i) {
        const T t = slots[i];
        if (i < warp) before += t;
        all += t;
    }
    total = all;
    __syncthreads();
    return x + before;
}
__device__ __forceinline__ int block_max_int(int x, int *slots) {
    x = __reduce_max_sync(0xffffffffu, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = x;
    __syncthreads();
    int r = slots[0];
#pragma unroll
    for (int i = 1; i < kPickWarps; ++i) r = max(r, slots[i]);
    __syncthreads();
    return r;
}
__device__ __forceinline__ int block_min_int(int x, int *slots) { return -block_max_int(-x, slots); }

// bitonic sort of a[0 .. n), n a power of two, descending.  Pairs at most 32 apart stay inside one warp's 64
// elements, so only the wider steps need a block barrier.
__device__ __forceinline__ void sort_descending(unsigned long long *a, int n) {
    __syncthreads();
    for (int size = 2; size <= n; size <<= 1) {
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
            if (stride > 32) __syncthreads(); else __syncwarp();
            for (int i = threadIdx.x; i < (n >> 1); i += kPickThreads) {
                const int x = 2 * i - (i & (stride - 1)), y = x + stride;
                const unsigned long long ax = a[x], ay = a[y];
                const bool down = (x & size) == 0;
                if ((ax < ay) == down) { a[x] = ay; a[y] = ax; }
            }
            if (stride > 32) __syncthreads();
        }
    }
    __syncthreads();
}

__device__ __forceinline__ uint32_t logit_key(float z) {           // monotone; -0 and +0 alike
    const uint32_t u = __float_as_uint(z + 0.f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// bin of a logit by its distance below the largest: 32 bins per factor of two, 2^-16 .. 2^16
__device__ __forceinline__ int distance_bin(float m, float z) {
    const int e = static_cast<int>(__float_as_uint(m - z) >> 18) - ((127 - 16) << 5);
    return min(max(e, 0), kBins - 1);
}

// The pick kernel's shared memory: the elements to sort (or the strip sums), histograms (count, two words of mass),
// the row's group maxima and the numbers of the groups to read again.
size_t pick_smem_bytes(int ngroups) { return kListCap * 8 + kBins * 12 + static_cast<size_t>(ngroups) * 6; }
constexpr size_t kPickSmemMax = kListCap * 8 + kBins * 12 + kMaxGroups * 6;

template <int DT, int U> struct Pick {
    const RowsParams &P;
    PickShared &sh;
    float *sg;                           // [ngroups]
    unsigned short *glist;               // [ng]
    unsigned *cnt, *mlo, *mhi;           // [kBins]
    unsigned long long *list;            // [kListCap]
    double *strips;                      // the same memory
    const RowView<DT> rv;
    const int row, nvec, ngroups;
    int ng;
    float m;

    __device__ __forceinline__ Pick(const RowsParams &P_, PickShared &sh_, unsigned char *smem, int row_, int b)
        : P(P_), sh(sh_), rv(P_.z, b * P_.sb + (row_ - b * P_.R) * P_.sr, P_.V), row(row_), nvec(rv.nvec()),
          ngroups((P_.nstrip + P_.coarse - 1) / P_.coarse * 32), ng(0) {
        list = reinterpret_cast<unsigned long long *>(smem);
        strips = reinterpret_cast<double *>(list);
        cnt = reinterpret_cast<unsigned *>(list + kListCap);
        mlo = cnt + kBins; mhi = mlo + kBins;
        sg = reinterpret_cast<float *>(mhi + kBins);
        glist = reinterpret_cast<unsigned short *>(sg + ngroups);
        m = 0.f;
    }

    // group maxima into shared memory, their maximum into m; false if a NaN or +inf is among them
    __device__ __forceinline__ bool load_groups() {
        const size_t base = static_cast<size_t>(row) * P.nstrip * 32;
        int best = INT_MIN;
        bool bad = false;
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads) {
            float x;
            if (P.coarse == 1) {
                x = load_group<DT>(P.gmax, base + g);
            } else {
                x = -INFINITY;
                const int s0 = (g >> 5) * P.coarse;
                for (int c = 0; c < P.coarse && s0 + c < P.nstrip; ++c)
                    x = max_nan(x, load_group<DT>(P.gmax, base + static_cast<size_t>(s0 + c) * 32 + (g & 31)));
            }
            sg[g] = x;
            bad |= !(x < INFINITY);
            best = max(best, float_order(x));
        }
        if (__syncthreads_or(bad)) return false;
        m = order_float(block_max_int(best, sh.wsum_i));
        return true;
    }

    // numbers of the groups whose maximum is at least `floor`, in an order that depends on the row only
    __device__ __forceinline__ void list_groups(float floor) {
        int mine = 0, total;
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads) mine += sg[g] >= floor;
        int at = block_scan(mine, sh.wsum_i, total) - mine;
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads)
            if (sg[g] >= floor) glist[at++] = static_cast<unsigned short>(g);
        ng = total;
        __syncthreads();
    }

    // f(z, id) for every element of the listed groups (elements outside the row or the mask come as -inf)
    template <typename F> __device__ __forceinline__ void each(F f) const {
        const int per = P.coarse * U;
        const int total = ng * per;
        for (int t = threadIdx.x; t < total; t += kPickThreads) {
            const int g = glist[t / per], j = t % per;
            const int v = ((g >> 5) * P.coarse + j / U) * (32 * U) + (j % U) * 32 + (g & 31);
            if (v >= nvec) continue;
            float z[Elt<DT>::kPerVec];
            unpack<DT>(row_vector<DT>(rv, P.mask, v, nvec), z);
            const int e0 = rv.first_elem(v);
#pragma unroll
            for (int i = 0; i < Elt<DT>::kPerVec; ++i) f(z[i], e0 + i);
        }
    }

    __device__ __forceinline__ void clear_bins(bool mass) {
        for (int i = threadIdx.x; i < kBins; i += kPickThreads) {
            cnt[i] = 0;
            if (mass) { mlo[i] = 0; mhi[i] = 0; }
        }
        __syncthreads();
    }
    // first bin at which the running count (from `before`) reaches `want`; -1 if none does.  `before` becomes the
    // count in front of that bin (or of everything).
    __device__ __forceinline__ int find_count(unsigned long long want, unsigned long long &before) {
        constexpr int per = kBins / kPickThreads;
        unsigned long long x[per], mine = 0, total;
#pragma unroll
        for (int i = 0; i < per; ++i) { x[i] = cnt[threadIdx.x * per + i]; mine += x[i]; }
        return find_bin<per>(x, mine, want, before, total);
    }
    __device__ __forceinline__ int find_mass(unsigned long long want, unsigned long long &before) {
        constexpr int per = kBins / kPickThreads;
        unsigned long long x[per], mine = 0, total;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int k = threadIdx.x * per + i;
            x[i] = (static_cast<unsigned long long>(mhi[k]) << 32) + mlo[k];
            mine += x[i];
        }
        return find_bin<per>(x, mine, want, before, total);
    }
    template <int per>
    __device__ __forceinline__ int find_bin(const unsigned long long (&x)[per], unsigned long long mine, unsigned long long want,
                                            unsigned long long &before, unsigned long long &total) {
        if (threadIdx.x == 0) sh.bi[0] = -1;
        unsigned long long run = before + block_scan(mine, sh.wsum_u, total) - mine;
        if (run < want && run + mine >= want) {                    // at most one thread
#pragma unroll
            for (int i = 0; i < per; ++i) {
                if (run < want && run + x[i] >= want) { sh.bi[0] = threadIdx.x * per + i; sh.bu[0] = run; }
                run += x[i];
            }
        }
        __syncthreads();
        const int bin = sh.bi[0];
        before = bin < 0 ? before + total : sh.bu[0];
        __syncthreads();
        return bin;
    }

    // A floor under the border from the group maxima: the smallest group maximum among the first bins that hold
    // `want` of them (by count, or by fixed-point mass: 2^18 per unit of weight, rounded down, so never too much).
    // Returns -FLT_MAX with ok = false if they do not hold that much.
    __device__ __forceinline__ float floor_from_groups(bool by_mass, unsigned long long want, double s, bool &ok) {
        clear_bins(false);
        const float sf = static_cast<float>(s);
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads) {
            const float x = sg[g];
            if (x > -INFINITY) {
                unsigned add = 1;
                if (by_mass) add = static_cast<unsigned>(ex2((x - m) * sf) * (262144.f * 0.9999f));
                if (add) atomicAdd(cnt + distance_bin(m, x), add);
            }
        }
        __syncthreads();
        unsigned long long before = 0;
        const int bin = find_count(want, before);
        ok = bin >= 0;
        if (!ok) return -FLT_MAX;
        int low = INT_MAX;
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads) {
            const float x = sg[g];
            if (x > -INFINITY && distance_bin(m, x) <= bin) low = min(low, float_order(x));
        }
        return order_float(block_min_int(low, sh.wsum_i));
    }

    // The id of the n-th lowest id (n >= 1) among the elements equal to z: two levels of a histogram over ids.
    __device__ __forceinline__ int nth_id_of(float z, unsigned long long n) {
        int base = 0, shift = 0;
        while ((P.V - 1) >> shift >= kBins) ++shift;
        unsigned long long before = 0;
        for (;;) {
            clear_bins(false);
            each([&](float x, int id) {
                const int k = (id - base) >> shift;
                if (x == z && id >= base && k < kBins) atomicAdd(cnt + k, 1u);
            });
            __syncthreads();
            const int bin = find_count(n, before);
            if (bin < 0) return INT_MAX;
            base += bin << shift;
            if (shift == 0) return base;
            shift = max(0, shift - 10);
        }
    }

    // The border by digits of the key: every level splits the interval of logits that holds it into at most 1024
    // bins.  Masses are 64-bit fixed-point numbers (two 32-bit shared atomics), so their sums do not depend on the
    // order of the atomics.  `zlow`: no element below it can be kept.  `Z`: mass of the row where there is no top-k.
    __device__ void border_by_digits(const RowAsk &ask, const Weights &w, float zlow, float zmin, double Z, float &bz, int &bid) {
        list_groups(zlow);
        const uint32_t top = logit_key(m), bottom = logit_key(zlow);
        bz = -INFINITY; bid = -1;                                  // everything finite
        bool cut = false;                                          // top-k leaves something out
        unsigned long long ties = 0, take = 0;                     // elements at the border's logit, and how many are kept
        uint32_t border = 0;
        if (ask.k_on) {
            uint32_t hi = top, lo = bottom;
            unsigned long long before = 0;
            for (;;) {
                const uint32_t range = hi - lo;
                const int shift = range < kBins ? 0 : 22 - __clz(range);
                clear_bins(false);
                each([&](float z, int) {
                    const uint32_t key = logit_key(z);
                    if (z >= zlow && key >= lo && key <= hi) atomicAdd(cnt + ((hi - key) >> shift), 1u);
                });
                __syncthreads();
                const int bin = find_count(static_cast<unsigned long long>(ask.k), before);
                if (bin < 0) break;                                // fewer than k finite logits
                if (shift == 0) {
                    cut = true;
                    border = hi - bin; ties = cnt[bin]; take = ask.k - before;
                    break;
                }
                hi -= static_cast<uint32_t>(bin) << shift;
                const uint32_t width = (1u << shift) - 1u;
                if (hi - lo > width) lo = hi - width;
            }
            __syncthreads();
        }
        if (ask.p_on) {
            double above = 0.0;
            if (ask.k_on) {                                        // the mass that top-k leaves
                double mine = 0.0;
                each([&](float z, int) { if (!cut || logit_key(z) > border) mine += w(z); });
                block_scan(mine, sh.wsum, above);
                Z = above + (cut ? static_cast<double>(take) * w(key_logit(border)) : 0.0);
            }
            const int e = ilogb(Z) + 1;                            // Z < 2^e, in units of 2^(e-62) it fits
            const double unit = scalbn(1.0, 62 - e);
            const unsigned long long want = max(1ull, static_cast<unsigned long long>(ceil(static_cast<double>(ask.p) * Z * unit)));
            uint32_t hi = top, lo = cut ? border + 1 : bottom;     // ties at the top-k border are counted apart
            unsigned long long before = 0;
            bool found = false;
            if (lo <= hi) {
                for (;;) {
                    const uint32_t range = hi - lo;
                    const int shift = range < kBins ? 0 : 22 - __clz(range);
                    clear_bins(true);
                    each([&](float z, int) {
                        const uint32_t key = logit_key(z);
                        if (z >= zlow && key >= lo && key <= hi) {
                            const unsigned long long f = __double2ull_rn(w(z) * unit);
                            const uint32_t k = (hi - key) >> shift, low = static_cast<uint32_t>(f);
                            const uint32_t old = atomicAdd(mlo + k, low);
                            const uint32_t high = static_cast<uint32_t>(f >> 32) + (old + low < old ? 1u : 0u);
                            if (high) atomicAdd(mhi + k, high);
                            if (shift == 0) atomicAdd(cnt + k, 1u);
                        }
                    });
                    __syncthreads();
                    const int bin = find_mass(want, before);
                    if (bin < 0) break;
                    if (shift == 0) {
                        found = true;
                        border = hi - bin; ties = cnt[bin];
                        break;
                    }
                    hi -= static_cast<uint32_t>(bin) << shift;
                    const uint32_t width = (1u << shift) - 1u;
                    if (hi - lo > width) lo = hi - width;
                }
                __syncthreads();
            }
            if (found || cut) {
                const unsigned long long f = __double2ull_rn(w(key_logit(border)) * unit);
                unsigned long long need = want > before && f ? (want - before + f - 1) / f : 1ull;
                if (want > before && !f) need = ~0ull;
                take = min(max(need, 1ull), found ? ties : take);
                cut = true;
            }
        }
        if (cut) { bz = key_logit(border); bid = take >= ties ? INT_MAX : nth_id_of(bz, take); }
        if (ask.min_on && zmin > bz) { bz = zmin; bid = INT_MAX; }
    }

    // The id that owns u * total over the kept elements, from a sum per strip.
    __device__ void draw_by_strips(const RowAsk &ask, const Weights &w, float bz, int bid, float u, int &token, double &prob) {
        auto kept = [&](float z, int id) { return z > bz || (z == bz && id <= bid); };
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (ask.whole_mass(P.sample) && bz == -INFINITY) {
            for (int i = threadIdx.x; i < P.nstrip; i += kPickThreads) {
                const StripSum ss = P.ssum[static_cast<size_t>(row) * P.nstrip + i];
                strips[i] = ss.S > 0.0 && ss.m >= w.cut ? ss.S * exp2_neg((static_cast<double>(ss.m) - w.m) * w.s, w.tab) : 0.0;
            }
        } else {
            for (int i = warp; i < P.nstrip; i += kPickWarps) {
                double acc = 0.0;
                if (sg[i / P.coarse * 32 + lane] >= bz) {
                    for (int q = 0; q < U; ++q) {
                        const int v = i * (32 * U) + q * 32 + lane;
                        float z[Elt<DT>::kPerVec];
                        unpack<DT>(row_vector<DT>(rv, P.mask, v, nvec), z);
                        const int e0 = rv.first_elem(v);
#pragma unroll
                        for (int j = 0; j < Elt<DT>::kPerVec; ++j)
                            if (kept(z[j], e0 + j)) acc += w(z[j]);
                    }
                }
                acc = warp_sum(acc);
                if (lane == 0) strips[i] = acc;
            }
        }
        __syncthreads();
        const int per = (P.nstrip + kPickThreads - 1) / kPickThreads, first = threadIdx.x * per;
        double mine = 0.0, total;
        int last = -1;
        for (int i = first; i < min(first + per, P.nstrip); ++i) {
            mine += strips[i];
            if (strips[i] > 0.0) last = i;
        }
        double run = block_scan(mine, sh.wsum, total) - mine;
        const double target = static_cast<double>(u) * total;
        last = block_max_int(last, sh.wsum_i);
        int hit = INT_MAX;
        for (int i = first; i < min(first + per, P.nstrip); ++i) {
            if (strips[i] > 0.0 && run + strips[i] > target) { hit = i; break; }
            run += strips[i];
        }
        const int strip = min(block_min_int(hit, sh.wsum_i), last);       // rounding can leave none above the target
        if (strip == hit || (hit == INT_MAX && strip == last && first <= last && last < first + per)) {
            double before = 0.0;                                   // the owner of the strip says what lies in front of it
            if (strip == hit) before = run; else before = run - strips[last];
            sh.bd[0] = before;
        }
        __syncthreads();
        if (warp == 0) {
            double base = sh.bd[0], w_last = 0.0, w_hit = 0.0;
            int id_last = -1, id_hit = -1;
            for (int q = 0; q < U && id_hit < 0; ++q) {
                const int v = strip * (32 * U) + q * 32 + lane;
                float z[Elt<DT>::kPerVec];
                double x[Elt<DT>::kPerVec], sum = 0.0;
                unpack<DT>(row_vector<DT>(rv, P.mask, v, nvec), z);
                const int e0 = rv.first_elem(v);
                int id_mine = -1;
                double w_mine = 0.0;
#pragma unroll
                for (int j = 0; j < Elt<DT>::kPerVec; ++j) {
                    x[j] = kept(z[j], e0 + j) ? w(z[j]) : 0.0;
                    sum += x[j];
                    if (x[j] > 0.0) { id_mine = e0 + j; w_mine = x[j]; }
                }
                double incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double y = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += y;
                }
                const unsigned over = __ballot_sync(0xffffffffu, sum > 0.0 && base + incl > target);
                const unsigned some = __ballot_sync(0xffffffffu, sum > 0.0);
                if (some) {
                    const int src = 31 - __clz(some);
                    id_last = __shfl_sync(0xffffffffu, id_mine, src);
                    w_last = __shfl_sync(0xffffffffu, w_mine, src);
                }
                if (over) {
                    const int src = __ffs(over) - 1;
                    double c = base + (incl - sum);
                    int id = id_mine;
                    double wt = w_mine;
#pragma unroll
                    for (int j = Elt<DT>::kPerVec - 1; j >= 0; --j) {      // smallest j whose running sum exceeds the target
                        double cj = c;
#pragma unroll
                        for (int i = 0; i <= j; ++i) cj += x[i];
                        if (x[j] > 0.0 && cj > target) { id = e0 + j; wt = x[j]; }
                    }
                    id_hit = __shfl_sync(0xffffffffu, id, src);
                    w_hit = __shfl_sync(0xffffffffu, wt, src);
                }
                base += __shfl_sync(0xffffffffu, incl, 31);
            }
            if (lane == 0) {
                sh.bi[1] = id_hit >= 0 ? id_hit : id_last;
                sh.bd[1] = (id_hit >= 0 ? w_hit : w_last) / total;
            }
        }
        __syncthreads();
        token = sh.bi[1];
        prob = sh.bd[1];
    }
};

template <int DT, int U>
__global__ void __launch_bounds__(kPickThreads) tli_rows_pick_kernel(const RowsParams P) {
    extern __shared__ __align__(16) unsigned char pick_smem[];
    __shared__ PickShared sh;
    const int tid = threadIdx.x, row = blockIdx.x, b = row / P.R;
    exp2_table_init(sh.tab, tid);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const RowAsk ask(P, b);
    Pick<DT, U> pk(P, sh, pick_smem, row, b);

    int status = 0, token = -1, mode = BORDER_APPLY, bid = -1;
    float bz = -INFINITY;
    double prob = 0.0;
    auto finish = [&]() {
        if (tid != 0) return;
        if (P.status) P.status[row] = status;
        if (P.sample) {
            P.tokens[row] = token;
            if (P.prob) P.prob[row] = static_cast<float>(prob);
        } else {
            RowBorder rb; rb.z = bz; rb.id = bid; rb.mode = mode; rb.pad = 0;
            P.border[row] = rb;
        }
    };

    if (ask.bad_tau) status |= TLI_ROW_BAD_TEMPERATURE;
    if (ask.bad_filter) status |= TLI_ROW_BAD_FILTER;
    if (status) { mode = BORDER_COPY; finish(); return; }
    if (!pk.load_groups()) { status = TLI_ROW_NONFINITE; mode = BORDER_COPY; finish(); return; }
    const float m = pk.m;
    if (!(m > -INFINITY)) { status = TLI_ROW_FALLBACK; finish(); return; }     // no id to keep

    if (ask.one) {                                                 // the lowest id at the largest logit
        pk.list_groups(m);
        int best = INT_MAX;
        pk.each([&](float z, int id) { if (z == m) best = min(best, id); });
        bz = m; bid = token = block_min_int(best, sh.wsum_i);
        prob = 1.0;
        finish();
        return;
    }
    const Weights w(m, ask.tau, sh.tab);
    // min-p as a logit: z >= m + tau ln(min_p), in fp64, to the next float above
    const float zmin = ask.min_on ? __double2float_ru(static_cast<double>(m) + static_cast<double>(ask.tau) * log(static_cast<double>(ask.least))) : -FLT_MAX;
    if (ask.plain()) {
        if (P.sample) { const float u = __ldg(P.u + row); pk.draw_by_strips(ask, w, bz, bid, u, token, prob); }
        finish();
        return;
    }
    double Z = 0.0;
    if (ask.p_on && !ask.k_on) {
        double mine = 0.0;
        for (int i = tid; i < P.nstrip; i += kPickThreads) {
            const StripSum ss = P.ssum[static_cast<size_t>(row) * P.nstrip + i];
            if (ss.S > 0.0 && ss.m >= w.cut) mine += ss.S * exp2_neg((static_cast<double>(ss.m) - w.m) * w.s, w.tab);
        }
        block_scan(mine, sh.wsum, Z);
    }

    // a floor under everything that can be kept
    float floor = -FLT_MAX;
    bool ok = true;
    if (ask.k_on) floor = pk.floor_from_groups(false, ask.k, w.s, ok);
    else if (ask.p_on) floor = pk.floor_from_groups(true, static_cast<unsigned long long>(ceil(static_cast<double>(ask.p) * Z * 262144.0)), w.s, ok);
    if (!ok && ask.p_on && !ask.k_on) {
        // ids of weight below (1-p) Z / V weigh less than (1-p) Z together: the border is at or above that weight
        const double t = log((1.0 - static_cast<double>(ask.p)) * Z / P.V) * ask.tau * (1.0 + 1e-9);
        floor = fmaxf(-FLT_MAX, __double2float_rd(static_cast<double>(m) + fmin(t, 0.0) - 1e-6 * fabs(static_cast<double>(m))));
    }
    const float zlow = ask.p_on ? floor : fmaxf(floor, zmin);
    bool drawn = false, found = false;
    if (ok) {
        pk.list_groups(zlow);
        if (tid == 0) sh.bi[2] = 0;
        __syncthreads();
        pk.each([&](float z, int id) {
            if (z >= zlow) {
                const int at = atomicAdd(&sh.bi[2], 1);
                if (at < kListCap)
                    pk.list[at] = (static_cast<unsigned long long>(logit_key(z)) << 32) | static_cast<uint32_t>(~id);
            }
        });
        __syncthreads();
        const int N = sh.bi[2];
        if (N <= kListCap) {
            int n2 = 32;
            while (n2 < N) n2 <<= 1;
            for (int i = N + tid; i < n2; i += kPickThreads) pk.list[i] = 0;
            sort_descending(pk.list, n2);                          // by (logit descending, id ascending)
            const int per = max(1, n2 / kPickThreads), first = tid * per;
            const int limit = ask.k_on ? min(N, ask.k) : N;
            double x[kListCap / kPickThreads], mine = 0.0, all;
#pragma unroll
            for (int i = 0; i < kListCap / kPickThreads; ++i) {
                x[i] = (i < per && first + i < limit) ? w(key_logit(static_cast<uint32_t>(pk.list[first + i] >> 32))) : 0.0;
                mine += x[i];
            }
            double run = block_scan(mine, sh.wsum, all) - mine;
            const double mass = static_cast<double>(ask.p) * (ask.k_on ? all : Z);
            found = !(ask.p_on && !ask.k_on && all < mass);        // (the floor is conservative; this holds but for rounding)
            if (found) {
                int count = 0, n;
#pragma unroll
                for (int i = 0; i < kListCap / kPickThreads; ++i) {
                    if (i < per && first + i < limit) {
                        const float z = key_logit(static_cast<uint32_t>(pk.list[first + i] >> 32));
                        const bool in = first + i == 0 || ((!ask.p_on || run < mass) && z >= zmin);
                        count += in;
                    }
                    run += x[i];
                }
                block_scan(count, sh.wsum_i, n);
                const unsigned long long edge = pk.list[n - 1];
                bz = key_logit(static_cast<uint32_t>(edge >> 32));
                bid = static_cast<int>(~static_cast<uint32_t>(edge));
                __syncthreads();
                if (P.sample) {                                    // the same elements by id
                    for (int i = tid; i < n2; i += kPickThreads) {
                        const unsigned long long e = pk.list[i];
                        pk.list[i] = i < n ? (e << 32) | (e >> 32) : 0ull;
                    }
                    int n3 = 32;
                    while (n3 < n) n3 <<= 1;
                    sort_descending(pk.list, n3);                  // ~id descending: id ascending
                    const int per3 = max(1, n3 / kPickThreads), first3 = tid * per3;
                    mine = 0.0;
#pragma unroll
                    for (int i = 0; i < kListCap / kPickThreads; ++i) {
                        x[i] = (i < per3 && first3 + i < n) ? w(key_logit(static_cast<uint32_t>(pk.list[first3 + i]))) : 0.0;
                        mine += x[i];
                    }
                    run = block_scan(mine, sh.wsum, all) - mine;
                    const double target = static_cast<double>(__ldg(P.u + row)) * all;
                    int hit = INT_MAX, last = -1;
#pragma unroll
                    for (int i = 0; i < kListCap / kPickThreads; ++i) {
                        run += x[i];
                        if (x[i] > 0.0) {
                            last = first3 + i;
                            if (hit == INT_MAX && run > target) hit = first3 + i;
                        }
                    }
                    last = block_max_int(last, sh.wsum_i);
                    hit = min(block_min_int(hit, sh.wsum_i), last);
                    const unsigned long long e = pk.list[hit];
                    token = static_cast<int>(~static_cast<uint32_t>(e >> 32));
                    prob = w(key_logit(static_cast<uint32_t>(e))) / all;
                    drawn = true;
                }
            }
        }
        __syncthreads();
    }
    if (!found) {
        if (ask.k_on || ask.p_on) pk.border_by_digits(ask, w, zlow, zmin, Z, bz, bid);
        else { bz = zmin; bid = INT_MAX; }
    }
    if (P.sample && !drawn) {
        const float u = __ldg(P.u + row);
        pk.draw_by_strips(ask, w, bz, bid, u, token, prob);
    }
    finish();
}

template <int DT, int U>
__global__ void __launch_bounds__(kRowThreads) tli_rows_mask_kernel(const RowsParams P) {
    constexpr uint32_t NI = Elt<DT>::kNegInfWord;
    constexpr int EPV = Elt<DT>::kPerVec;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.y, b = row / P.R, r = row - b * P.R;
    const int strip = blockIdx.x * kRowWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (strip >= P.nstrip) return;
    const RowView<DT> rv(P.z, b * P.sb + r * P.sr, P.V), ov(P.out, b * P.osb + r * P.osr, P.V);
    const int nvec = rv.nvec();
    const RowBorder rb = P.border[row];
    const bool copy = rb.mode == BORDER_COPY;
    const float gm = load_group<DT>(P.gmax, static_cast<size_t>(row) * P.nstrip * 32 + strip * 32 + lane);
    const bool read = copy || gm >= rb.z;                          // gm is never NaN where the border applies
    uint4 raw[U];
#pragma unroll
    for (int q = 0; q < U; ++q) {
        raw[q] = make_uint4(NI, NI, NI, NI);
        const int v = strip * (32 * U) + q * 32 + lane;
        // (the row may be the output too: coherent loads)
        if (read && v < nvec) {
            const int e0 = rv.first_elem(v);
            if (e0 >= 0 && e0 + EPV <= P.V) {
                raw[q] = __ldcg(rv.vec0 + v);
            } else {
                uint32_t x[EPV];
#pragma unroll
                for (int i = 0; i < EPV; ++i) {
                    const int e = e0 + i;
                    if constexpr (DT == TLI_F32) x[i] = e >= 0 && e < P.V ? __ldcg(reinterpret_cast<const unsigned *>(rv.row) + e) : 0xff800000u;
                    else x[i] = e >= 0 && e < P.V ? __ldcg(reinterpret_cast<const unsigned short *>(rv.row) + e) : 0xff80u;
                }
                if constexpr (DT == TLI_F32) raw[q] = make_uint4(x[0], x[1], x[2], x[3]);
                else raw[q] = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
            }
        }
    }
    const bool same_grid = rv.head == ov.head;
#pragma unroll
    for (int q = 0; q < U; ++q) {
        const int v = strip * (32 * U) + q * 32 + lane;
        if (v >= nvec) continue;
        const int e0 = rv.first_elem(v);
        if (read && !copy) {
            if (P.mask) raw[q] = mask_vector<DT>(raw[q], P.mask, e0);
            float z[EPV];
            unpack<DT>(raw[q], z);
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < EPV; ++i)
                if (z[i] > rb.z || (z[i] == rb.z && e0 + i <= rb.id)) bits |= 1u << i;
            if constexpr (DT == TLI_BF16) {
                mask_bf16_vector(raw[q], bits);
            } else {
                raw[q].x = (bits & 1u) ? raw[q].x : NI; raw[q].y = (bits & 2u) ? raw[q].y : NI;
                raw[q].z = (bits & 4u) ? raw[q].z : NI; raw[q].w = (bits & 8u) ? raw[q].w : NI;
            }
        }
        if (same_grid && e0 >= 0 && e0 + EPV <= P.V) {
            const_cast<uint4 *>(ov.vec0)[v] = raw[q];
        } else {
            const uint32_t x[4] = {raw[q].x, raw[q].y, raw[q].z, raw[q].w};
#pragma unroll
            for (int i = 0; i < EPV; ++i) {
                const int e = e0 + i;
                if (e < 0 || e >= P.V) continue;
                if constexpr (DT == TLI_F32) const_cast<uint32_t *>(reinterpret_cast<const uint32_t *>(ov.row))[e] = x[i];
                else const_cast<unsigned short *>(reinterpret_cast<const unsigned short *>(ov.row))[e] =
                         static_cast<unsigned short>(i & 1 ? x[i >> 1] >> 16 : x[i >> 1]);
            }
        }
    }
}

// ---- host ----

struct RowsLayout { int U, nstrip, coarse; size_t gmax, ssum, border, total; };

// Groups of 8 vectors; of 4 where a row has at most 8192 vectors, so that a short row still has enough groups for
// a top-k of a few hundred.
RowsLayout rows_layout(long long rows, int V, int dtype) {
    RowsLayout L;
    const int nvec = chunks_per_row(V, dtype, 1);
    L.U = nvec <= 8192 ? 4 : 8;
    L.nstrip = (nvec + 32 * L.U - 1) / (32 * L.U);
    L.coarse = (L.nstrip * 32 + kMaxGroups - 1) / kMaxGroups;
    const size_t elt = dtype == TLI_F32 ? 4 : 2;
    size_t off = 0;
    L.gmax = off; off = align_up(off + elt * rows * L.nstrip * 32, 256);
    L.ssum = off; off = align_up(off + sizeof(StripSum) * rows * L.nstrip, 256);
    L.border = off; off = align_up(off + sizeof(RowBorder) * rows, 256);
    L.total = off;
    return L;
}

size_t rows_workspace(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side) {
    if (!ctx || ctx->n_shards != 1 || B < 1 || R < 1 || static_cast<long long>(B) * R > TLI_MAX_B) return 0;
    if (dtype != TLI_F32 && dtype != TLI_BF16) return 0;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return 0;
    return rows_layout(static_cast<long long>(B) * R, side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d, dtype).total;
}

template <int DT, int U> int launch_rows(const RowsParams &P, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = stream;
    const unsigned rows = static_cast<unsigned>(P.B) * P.R;
    cfg.gridDim = dim3((P.nstrip + kRowWarps - 1) / kRowWarps, rows); cfg.blockDim = dim3(kRowThreads);
    cudaError_t e = cudaLaunchKernelEx(&cfg, tli_rows_scan_kernel<DT, U>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_rows_scan_kernel");
    e = cudaFuncSetAttribute(tli_rows_pick_kernel<DT, U>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPickSmemMax));
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
    cfg.gridDim = dim3(rows); cfg.blockDim = dim3(kPickThreads); cfg.dynamicSmemBytes = pick_smem_bytes((P.nstrip + P.coarse - 1) / P.coarse * 32);
    e = cudaLaunchKernelEx(&cfg, tli_rows_pick_kernel<DT, U>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_rows_pick_kernel");
    if (!P.sample) {
        cfg.gridDim = dim3((P.nstrip + kRowWarps - 1) / kRowWarps, rows); cfg.blockDim = dim3(kRowThreads); cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, tli_rows_mask_kernel<DT, U>, P);
        if (e != cudaSuccess) return cuda_fail(e, "launch tli_rows_mask_kernel");
    }
    return TLI_OK;
}

int run_rows(RowsParams &P, const tli_ctx *ctx, int32_t dtype, int32_t side, void *workspace, cudaStream_t stream) {
    P.V = side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d;
    P.mask = side == TLI_SIDE_TARGET ? nullptr : ctx->d_mask;
    const RowsLayout L = rows_layout(static_cast<long long>(P.B) * P.R, P.V, dtype);
    char *ws = reinterpret_cast<char *>(workspace);
    P.nstrip = L.nstrip; P.coarse = L.coarse;
    P.gmax = ws + L.gmax;
    P.ssum = reinterpret_cast<StripSum *>(ws + L.ssum);
    P.border = reinterpret_cast<RowBorder *>(ws + L.border);
    if (dtype == TLI_F32) return L.U == 4 ? launch_rows<TLI_F32, 4>(P, stream) : launch_rows<TLI_F32, 8>(P, stream);
    return L.U == 4 ? launch_rows<TLI_BF16, 4>(P, stream) : launch_rows<TLI_BF16, 8>(P, stream);
}

// What tli_sample() and tli_filter() check alike.
int check_rows(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side, const void *logits, int64_t sb, int64_t sr,
               const float *tau, const void *workspace, size_t workspace_bytes) {
    if (!ctx || ctx->n_shards != 1 || B < 1 || R < 1) return TLI_ERR_ARG;
    if (static_cast<long long>(B) * R > TLI_MAX_B) return TLI_ERR_UNSUPPORTED;
    if (dtype != TLI_F32 && dtype != TLI_BF16) return TLI_ERR_ARG;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return TLI_ERR_ARG;
    if (!logits || !tau) return TLI_ERR_ARG;
    const size_t elt = dtype == TLI_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % elt || sb < 0 || sr < 0) return TLI_ERR_ARG;
    const size_t need = rows_workspace(ctx, B, R, dtype, side);
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < need) return TLI_ERR_WORKSPACE;
    return TLI_OK;
}

}  // namespace

extern "C" {

size_t tli_sample_workspace_bytes(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side) {
    return rows_workspace(ctx, B, R, dtype, side);
}
size_t tli_filter_workspace_bytes(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side) {
    return rows_workspace(ctx, B, R, dtype, side);
}

int tli_sample(tli_ctx *ctx, const tli_sample_args *a, void *cuda_stream) {
    if (!a) return TLI_ERR_ARG;
    const int rc = check_rows(ctx, a->B, a->R, a->dtype, a->side, a->logits, a->stride_b, a->stride_r, a->temperature,
                              a->workspace, a->workspace_bytes);
    if (rc != TLI_OK) return rc;
    if (!a->uniforms || !a->tokens) return TLI_ERR_ARG;
    RowsParams P;
    memset(&P, 0, sizeof P);
    P.B = a->B; P.R = a->R; P.sample = 1;
    P.z = a->logits; P.sb = a->stride_b; P.sr = a->stride_r;
    P.tau = a->temperature; P.top_k = a->top_k; P.top_p = a->top_p; P.min_p = a->min_p; P.u = a->uniforms;
    P.tokens = a->tokens; P.prob = a->prob; P.status = a->status;
    return run_rows(P, ctx, a->dtype, a->side, a->workspace, reinterpret_cast<cudaStream_t>(cuda_stream));
}

int tli_filter(tli_ctx *ctx, const tli_filter_args *a, void *cuda_stream) {
    if (!a) return TLI_ERR_ARG;
    const int rc = check_rows(ctx, a->B, a->R, a->dtype, a->side, a->logits, a->stride_b, a->stride_r, a->temperature,
                              a->workspace, a->workspace_bytes);
    if (rc != TLI_OK) return rc;
    const size_t elt = a->dtype == TLI_F32 ? 4 : 2;
    if (!a->out || reinterpret_cast<uintptr_t>(a->out) % elt) return TLI_ERR_ARG;
    // rows of the output must not overlap one another
    const int64_t V = a->side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d;
    const int64_t ob = a->out_stride_b, orr = a->out_stride_r;
    if (ob < 0 || orr < 0) return TLI_ERR_ARG;
    if (a->R > 1 && orr < V) return TLI_ERR_ARG;
    if (a->B > 1 && ob < V) return TLI_ERR_ARG;
    if (a->B > 1 && a->R > 1 && !(ob >= (a->R - 1) * orr + V || orr >= (a->B - 1) * ob + V)) return TLI_ERR_ARG;
    RowsParams P;
    memset(&P, 0, sizeof P);
    P.B = a->B; P.R = a->R; P.sample = 0;
    P.z = a->logits; P.sb = a->stride_b; P.sr = a->stride_r;
    P.tau = a->temperature; P.top_k = a->top_k; P.top_p = a->top_p; P.min_p = a->min_p;
    P.status = a->status;
    P.out = a->out; P.osb = ob; P.osr = orr;
    return run_rows(P, ctx, a->dtype, a->side, a->workspace, reinterpret_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
