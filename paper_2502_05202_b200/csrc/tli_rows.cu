// Filtered sampling and filtered logits: temperature, top-k, top-p and min-p over rows of logits.
// (Part of tli_lib.cu: uses RowView, mask_bits, tli_ctx and the error helpers of tli.cu.)
//
// Mathematics.  Order the ids of a row by (logit descending, id ascending) and let w = exp((z - m)/tau),
// m the largest logit.  top-k keeps the first k, top-p the shortest prefix that holds p of their mass, min-p
// the ids with w >= min_p: three prefixes of one order, so what is kept is a prefix too, and one border
// (logit, id) says all of it.  The rest of the work is to find that border without sorting the row.
//
//   tli_rows_scan_kernel   reads every row once: each lane leaves the largest of its U 16-byte vectors (a "group") in the
//                          workspace, 1/(8U) or less of what it read; rows that need the whole mass (top-p without
//                          top-k, no filter at all) also leave a sum per strip of 32 groups.
//   tli_rows_pick_kernel   one CTA per row.  k groups have a largest element at or above the k-th largest group maximum, so at
//                          least k elements do: a histogram of the maxima gives a floor under the border (the same with mass
//                          instead of count for top-p).  Only the groups that reach the floor are read again; their elements
//                          are a list in shared memory in which the border and the draw are found by counting (up to 256) or
//                          by histograms over what is left of the interval (up to 4096).
//   tli_rows_spread_kernel the rows whose list would not fit, by all CTAs: a sample of 8192 elements brackets the border between two
//                          logits, one more pass over the row counts and weighs what lies above the bracket and lists what
//                          lies in it; the CTA that ends a row's last strips finds border and draw as above.  If the bracket
//                          was wrong (or a run of equal logits is longer than the list, or top-k of many thousands meets
//                          top-p, or min-p cuts above the bracket of a top-p without top-k: the bracket knows nothing of min-p)
//                          the border is found by key digits over the whole row by one CTA: the same border, more passes.  For the
//                          last of these that is the rule, not bad luck: 48 bf16 rows of 128 256 at top-p .95 with min-p .05
//                          take 366 us (filter 181) against 63 at top-p .95 alone and 25 at min-p .05 alone; 320 fp32 rows of 256 000
//                          1.9 ms (filter 1.0) against 311 and 79 us.
//   tli_rows_mask_kernel   (filter only) writes the row: -inf without reading it wherever the group maximum is
//                          below the border, the compared elements elsewhere.
//
// Bytes: a row once (sample), once and written once (filter).  At the measured copy bandwidth that is 50 us for 320 fp32 rows of
// 256 000; the call takes 84 us at top-k 50, 135 at top-p .5, 288 to 311 at top-p .9 to .95 (two thirds of that is the fp64 work of
// the scan and of the spread pass).  One fp32 row of 32 000: 18 us, three launches and 13 us of dependent steps.
//
// Weights and sums are fp64: the ids that come out are exact decisions (which id owns v * total, which one is
// the last inside top-p), and with 10^5 candidates an fp32 sum (2^-24 relative) would decide some of them by
// rounding.  A weight is off by 1.5e-13 of itself at most (3e-13 where it is a product of two, a strip's sum at its own largest logit and
// that logit's weight), a list's fixed-point mass by 4e-12, a sum of a whole row by less than 1e-12: an id is decided by these only where
// its border lies within 5e-12 of the mass.  An fp64 weight costs 12 fp64 operations; one pass over a row is then bound by the fp64 pipe only
// for 16-bit rows that need the whole mass.

#include <cuda_bf16.h>
#include <algorithm>
#include <atomic>
#include <initializer_list>

namespace {

constexpr int kRowThreads = 128;                     // scan and mask kernels
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kPickThreads = 256;                    // pick and spread kernels
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kMaxGroups = 8192;                     // group maxima a pick CTA holds (coarser groups beyond)
constexpr int kListCap = 4096;                       // elements the pick kernel searches in shared memory
constexpr int kSpreadCap = 8192;                     // ... the spread kernel
constexpr int kSample = 8192;                        // elements of a row that stand for it where the border is guessed
constexpr int kBins = 1024;

struct __align__(16) StripSum { double S; float m; int pad; };       // sum of 2^((z - m) s) over a strip, m its largest
struct __align__(16) RowBorder { float z; int id; int mode; int pad; };
enum : int { BORDER_APPLY = 0, BORDER_COPY = 1 };
// What the pick kernel leaves to the spread kernel: ids above (zhi, bid) are kept, below zlo none is.
struct __align__(16) RowPlan { double Z; float zlo, zhi; int bid, kind; float m, zmin; int listed, done; };
enum : int { PLAN_BRACKET = 0, PLAN_DRAW = 1 };                      // the border is in between; it is (zhi, bid)

struct RowsParams {
    int B, R, V, nstrip, ulog, coarse, sample;
    const void *z; long long sb, sr;
    const uint32_t *mask;                  // ids that can be kept; NULL: every id of the row
    const float *tau; const int *top_k; const float *top_p; const float *min_p; const float *u;
    int *tokens; float *prob; int *status;
    void *gmax;                            // [rows][nstrip * 32] in the rows' type
    StripSum *ssum;                        // [rows][nstrip]
    RowBorder *border;                     // [rows]
    RowPlan *plan;                         // [rows]
    int *todo;                             // [2 + rows]: how many rows the spread kernel has, and which; behind them its next task
    unsigned long long *lists; int listcap;    // [rows][listcap]
    void *out; long long osb, osr;
};

// ---- weights ----

// 2^(i/16), less i/16 in the exponent field (see exp2_parts); 16 doubles are one line of banks, so 32 lanes with any indices
// read it without a conflict
__device__ __forceinline__ void exp2_table_init(double *tab, int tid) {
    if (tid < 16) {
        const double t = exp2(tid / 16.0);
        tab[tid] = __hiloint2double(__double2hiint(t) - (tid << 16), __double2loint(t));
    }
}
// 2^x for x in [-1021, 0] as a product q * t: x = n/16 + r, |r| <= 1/32; q = 2^r by its Taylor series in r ln 2 to the fifth power
// (next term (ln2/32)^6/6! = 1.4e-13, the whole error 1.46e-13), t = 2^(n/16) = tab[n mod 16] with n/16 added to the exponent field (the table's entry lacks
// what the low four bits of n would add).  On this part an fp64 instruction holds the issue port for two cycles: the 12 of a
// weight and five others are what bounds a pass that weighs a whole row.
__device__ __forceinline__ void exp2_parts(double x, const double *tab, double &q, double &t) {
    constexpr double L = 0.693147180559945309417232;
    constexpr double c2 = L * L / 2, c3 = c2 * L / 3, c4 = c3 * L / 4, c5 = c4 * L / 5;
    constexpr double magic = 6755399441055744.0;                     // 1.5 * 2^52
    const double k = fma(x, 16.0, magic);
    const double r = fma(k - magic, -0.0625, x);
    const int n = __double2loint(k);
    t = tab[n & 15];
    t = __hiloint2double(__double2hiint(t) + (n << 16), __double2loint(t));
    q = fma(r, c5, c4);
    q = fma(q, r, c3); q = fma(q, r, c2); q = fma(q, r, L); q = fma(q, r, 1.0);
}
__device__ __forceinline__ double exp2_neg(double x, const double *tab) {
    double q, t;
    exp2_parts(x, tab, q, t);
    return q * t;
}
__device__ __forceinline__ int exponent(double x) { return ((__double2hiint(x) >> 20) & 0x7ff) - 1023; }     // of a normal number
__device__ __forceinline__ double two_to(int n) { return __hiloint2double((n + 1023) << 20, 0); }
// w(z) = exp((z - m)/tau), s = log2(e)/tau; 0 below cut (exp(-707) of the largest; -inf among them)
struct Weights {
    double m, s; float cut; const double *tab;
    Weights() = default;
    __device__ __forceinline__ Weights(float m_, float tau, const double *tab_) {
        m = m_; s = kLog2e / tau; tab = tab_; cut = cut_of(m_, tau);
    }
    static constexpr double kLog2e = 1.4426950408889634074;
    __device__ __forceinline__ static float cut_of(float m, float tau) {       // rounded up: z >= cut stays in exp2_neg's range
        return fmaxf(__double2float_ru(static_cast<double>(m) - 707.0 * static_cast<double>(tau)), -FLT_MAX);
    }
    __device__ __forceinline__ double operator()(float z) const {
        const double w = exp2_neg((static_cast<double>(z) - m) * s, tab);
        return z >= cut ? w : 0.0;
    }
    // acc + w(z), where w(z) is 0 + w(cut): for sums that hold a weight of 1, if w(cut) is nothing beside it
    __device__ __forceinline__ bool cut_is_nothing() const { return (m - static_cast<double>(cut)) * s > 200.0; }
    __device__ __forceinline__ double add(double acc, float z) const {
        double q, t;
        exp2_parts((static_cast<double>(fmaxf(z, cut)) - m) * s, tab, q, t);
        return fma(q, t, acc);
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
// A vector at an end of a row: what lies outside the row reads as -inf.  Out of line: two vectors of a row come here.
template <int DT> __device__ __noinline__ uint4 ragged_vector(const void *row, int e0, int V) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DT == TLI_F32) {
            const int e = e0 + k;
            w[k] = e >= 0 && e < V ? __ldcg(reinterpret_cast<const unsigned *>(row) + e) : 0xff800000u;
        } else {
            const int e = e0 + 2 * k;
            const unsigned short *h = reinterpret_cast<const unsigned short *>(row);
            const uint32_t lo = e >= 0 && e < V ? __ldcg(h + e) : 0xff80u, hi = e + 1 >= 0 && e + 1 < V ? __ldcg(h + e + 1) : 0xff80u;
            w[k] = lo | hi << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// B vectors of a row, v[] >= nvec for none; ids outside the row or outside the mask read as -inf.  The loads first, then what is rare and what
// needs their results: a vector finished before the next one is asked for costs a trip to memory each.
template <int DT, int B> __device__ __forceinline__ void row_vectors(const uint4 *vec0, const void *row, int head, int V, int nvec, const uint32_t *mask,
                                                                     const int (&v)[B], uint4 (&raw)[B]) {
    constexpr uint32_t NI = Elt<DT>::kNegInfWord;
    constexpr int EPV = Elt<DT>::kPerVec;
    bool ragged = false;
#pragma unroll
    for (int k = 0; k < B; ++k) {
        raw[k] = make_uint4(NI, NI, NI, NI);
        const int e0 = v[k] * EPV - head;
        const bool whole = v[k] < nvec && e0 >= 0 && e0 + EPV <= V;
        if (whole) raw[k] = __ldg(vec0 + v[k]);
        ragged |= v[k] < nvec && !whole;
    }
    if (ragged) {
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const int e0 = v[k] * EPV - head;
            if (v[k] < nvec && !(e0 >= 0 && e0 + EPV <= V)) raw[k] = ragged_vector<DT>(row, e0, V);
        }
    }
    if (mask) {
#pragma unroll
        for (int k = 0; k < B; ++k)
            if (v[k] < nvec) raw[k] = mask_vector<DT>(raw[k], mask, v[k] * EPV - head);
    }
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
    // min-p as a logit: z >= m + tau ln(min_p), in fp64, to the next value of the row's type above
    template <int DT> __device__ __forceinline__ float zmin(float m) const {
        if (!min_on) return -FLT_MAX;
        const float f = __double2float_ru(static_cast<double>(m) + static_cast<double>(tau) * log(static_cast<double>(least)));
        return DT == TLI_BF16 ? __bfloat162float(__float2bfloat16_ru(f)) : f;
    }
    __device__ __forceinline__ bool plain() const { return !k_on && !p_on && !min_on; }
    // the mass of the whole row is asked for
    __device__ __forceinline__ bool whole_mass(int sample) const {
        return !bad_tau && !bad_filter && !one && !k_on && (p_on || (sample && !min_on));
    }
};

// Bound by DRAM where no mass is asked for: 320 fp32 rows of 256 000 (328 MB) in 48 us, 6.8 TB/s; by the issue slots of the fp64
// weights where every row wants its mass: 95 us.  Small blocks (128 threads) because a row of 32 000 has only 16 to 32 strips.
template <int DT, int U>
__global__ void __launch_bounds__(kRowThreads) tli_rows_scan_kernel(const __grid_constant__ RowsParams P) {
    __shared__ double tab[16];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.y, b = row / P.R;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int strip = blockIdx.x * kRowWarps + warp;
    if (blockIdx.x == 0 && row == 0 && threadIdx.x == 0) { *P.todo = 0; P.todo[1 + P.B * P.R] = 0; }
    const RowView<DT> rv(P.z, b * P.sb + (row - b * P.R) * P.sr, P.V);
    const int nvec = rv.nvec(), v0 = strip * (32 * U) + lane;
    uint4 raw[U];
    const bool live = strip < P.nstrip;
    if (live) {
        int v[U];
#pragma unroll
        for (int q = 0; q < U; ++q) v[q] = v0 + q * 32;
        row_vectors<DT, U>(rv.vec0, rv.row, rv.head, P.V, nvec, P.mask, v, raw);
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
        if (w.cut_is_nothing()) {
#pragma unroll
            for (int q = 0; q < U; ++q) {
                float z[Elt<DT>::kPerVec];
                unpack<DT>(raw[q], z);
#pragma unroll
                for (int i = 0; i < Elt<DT>::kPerVec; ++i) acc = w.add(acc, z[i]);
            }
        } else {                                                   // tau below a step of the largest logit, or logits near the lowest value
#pragma unroll 1
            for (int q = 0; q < U; ++q) {
                float z[Elt<DT>::kPerVec];
                unpack<DT>(raw[0], z);
#pragma unroll
                for (int k = 0; k + 1 < U; ++k) raw[k] = raw[k + 1];
#pragma unroll
                for (int i = 0; i < Elt<DT>::kPerVec; ++i) acc += w(z[i]);
            }
        }
    }
    acc = warp_sum(acc);
    if (lane == 0) {
        StripSum ss; ss.S = acc; ss.m = ms; ss.pad = 0;
        P.ssum[static_cast<size_t>(row) * P.nstrip + strip] = ss;
    }
}

// ---- logits as integers ----

// monotone; -0 and +0 alike; 16 bits for bf16
template <int DT> __device__ __forceinline__ uint32_t logit_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    const uint32_t k = u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
    return DT == TLI_BF16 ? k >> 16 : k;
}
template <int DT> __device__ __forceinline__ float key_logit(uint32_t k) {
    if (DT == TLI_BF16) return __uint_as_float(((k & 0x8000u) ? k ^ 0x8000u : ~k & 0xffffu) << 16);
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// an element as one integer that falls along the order (logit descending, id ascending); never 0
using u64 = unsigned long long;
constexpr uint32_t kIdMask = (1u << 20) - 1u;
static_assert(TLI_MAX_V <= (1 << 20), "an id has 20 bits in a list element");
template <int DT> __device__ __forceinline__ u64 element_of(float z, int id) {
    return (static_cast<u64>(logit_key<DT>(z)) << 20) | (kIdMask - static_cast<uint32_t>(id));
}
template <int DT> __device__ __forceinline__ float element_logit(u64 e) { return key_logit<DT>(static_cast<uint32_t>(e >> 20)); }
__device__ __forceinline__ int element_id(u64 e) { return static_cast<int>(kIdMask - (static_cast<uint32_t>(e) & kIdMask)); }

// ---- the state of a pick or settle block ----
//
// These two kernels run each of their steps once or a few times per row, so what they cost is the fetching of their code:
// with every step inlined and unrolled they were 300 to 540 KB and took two to ten times as long.  The steps are
// functions that are called, their loops are not unrolled, and the block's state is in shared memory instead of registers.

struct __align__(16) PickState {
    double tab[16];
    alignas(16) u64 slot[kPickWarps];                  // (read as int4)
    u64 few[kPickThreads], few_mass[kPickThreads];     // a short list and its masses
    u64 found, before;
    int bin, listed;
    // the row
    Weights w;
    const uint4 *vec0; const void *row; const uint32_t *mask;
    int head, V, nvec, nstrip, ulog, coarse, ngroups;
    int ng;                  // groups listed; -1: the whole row is
    int room;                // elements the list has room for
    float m;
};
__shared__ PickState S;
// Dynamic shared memory: three words per bin of a histogram (zero between uses), the strip sums, the elements that may lie at
// the border; in the pick kernel also the row's group maxima and the numbers of the groups to read again.
extern __shared__ __align__(16) unsigned char pick_smem[];
constexpr size_t settle_smem_bytes(int nstrip) { return kBins * 12 + kSpreadCap * 8 + static_cast<size_t>(nstrip) * 8; }
constexpr size_t pick_smem_bytes(int nstrip, int ngroups) { return kBins * 12 + kListCap * 8 + static_cast<size_t>(nstrip) * 8 + static_cast<size_t>(ngroups) * 6; }
constexpr int kMaxRowStrips = (TLI_MAX_V + 6) / (4 * 32 * 8) + 1;
constexpr size_t kPickSmemMax = pick_smem_bytes(kMaxRowStrips, kMaxGroups), kSettleSmemMax = settle_smem_bytes(kMaxRowStrips);
__device__ __forceinline__ unsigned *bins() { return reinterpret_cast<unsigned *>(pick_smem); }
__device__ __forceinline__ u64 *list() { return reinterpret_cast<u64 *>(pick_smem + kBins * 12); }
__device__ __forceinline__ double *strips() { return reinterpret_cast<double *>(pick_smem + kBins * 12) + S.room; }
__device__ __forceinline__ float *group_max() { return reinterpret_cast<float *>(strips() + S.nstrip); }
__device__ __forceinline__ unsigned short *group_list() { return reinterpret_cast<unsigned short *>(group_max() + S.ngroups); }

template <int DT> __device__ __forceinline__ void enter_row(const RowsParams &P, int row, int b, int room) {      // (visible after the next barrier)
    for (int i = threadIdx.x; i < 3 * kBins / 4; i += kPickThreads) reinterpret_cast<uint4 *>(bins())[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) {
        const RowView<DT> rv(P.z, b * P.sb + (row - b * P.R) * P.sr, P.V);
        S.vec0 = rv.vec0; S.row = rv.row; S.head = rv.head; S.V = P.V; S.nvec = rv.nvec(); S.mask = P.mask;
        S.nstrip = P.nstrip; S.ulog = P.ulog; S.coarse = P.coarse; S.ng = -1; S.room = room;
        S.ngroups = (P.nstrip + P.coarse - 1) / P.coarse * 32;
    }
}
template <int DT, int B> __device__ __forceinline__ void state_vectors(const int (&v)[B], uint4 (&raw)[B]) {      // of the block's row
    row_vectors<DT, B>(S.vec0, S.row, S.head, S.V, S.nvec, S.mask, v, raw);
}
template <int DT> __device__ __forceinline__ float vector_element(const uint4 &r, int i) {               // i not known in advance
    if (DT == TLI_F32) return __uint_as_float(i < 2 ? (i == 0 ? r.x : r.y) : (i == 2 ? r.z : r.w));
    const uint32_t x = i < 4 ? (i < 2 ? r.x : r.y) : (i < 6 ? r.z : r.w);
    return i & 1 ? bf16_hi(x) : bf16_lo(x);
}

// ---- block-wide steps (every thread of the block calls them) ----

__device__ __noinline__ int block_max(int x) {
    x = __reduce_max_sync(0xffffffffu, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) reinterpret_cast<int *>(S.slot)[threadIdx.x >> 5] = x;
    __syncthreads();
    const int4 a = reinterpret_cast<const int4 *>(S.slot)[0], b = reinterpret_cast<const int4 *>(S.slot)[1];
    return max(max(max(a.x, a.y), max(a.z, a.w)), max(max(b.x, b.y), max(b.z, b.w)));
}
__device__ __forceinline__ int block_min(int x) { return ~block_max(~x); }
__device__ __noinline__ int block_sum(int x) {
    x = __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) reinterpret_cast<int *>(S.slot)[threadIdx.x >> 5] = x;
    __syncthreads();
    const int4 a = reinterpret_cast<const int4 *>(S.slot)[0], b = reinterpret_cast<const int4 *>(S.slot)[1];
    return a.x + a.y + a.z + a.w + b.x + b.y + b.z + b.w;
}
template <typename T> struct Prefix { T before, total; };
template <typename T> __device__ __noinline__ Prefix<T> block_prefix(T x) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    T *slot = reinterpret_cast<T *>(S.slot);
    __syncthreads();
    if (lane == 31) slot[warp] = incl;
    __syncthreads();
    Prefix<T> p;
    p.before = 0; p.total = 0;
#pragma unroll
    for (int i = 0; i < kPickWarps; ++i) {
        const T t = slot[i];
        if (i < warp) p.before += t;
        p.total += t;
    }
    p.before += incl - x;
    return p;
}

// First bin at which the running measure, from `before`, reaches `want` (-1 if none does), the measure in front of it (or of everything)
// and its own.
// A bin's measure is w0 + (w1 << shift) + (w2 << 38).  The bins come back zero unless they are to be kept.
struct BinAt { int bin; u64 before, measure; };
static_assert(kBins == 4 * kPickThreads, "four bins per thread");
__device__ __noinline__ BinAt find_bin(u64 want, u64 before, int shift, bool keep) {
    __syncthreads();
    uint4 *w = reinterpret_cast<uint4 *>(bins()) + threadIdx.x;
    const uint4 a = w[0], b = w[kBins / 4], c = w[kBins / 2];
    if (!keep) { w[0] = make_uint4(0, 0, 0, 0); w[kBins / 4] = w[0]; w[kBins / 2] = w[0]; }
    auto value = [shift](unsigned lo, unsigned mid, unsigned hi) { return lo + (static_cast<u64>(mid) << shift) + (static_cast<u64>(hi) << 38); };
    const u64 x0 = value(a.x, b.x, c.x), x1 = value(a.y, b.y, c.y), x2 = value(a.z, b.z, c.z), x3 = value(a.w, b.w, c.w);
    const u64 mine = x0 + x1 + x2 + x3;
    const Prefix<u64> p = block_prefix(mine);
    u64 run = before + p.before;
    if (run < want && run + mine >= want) {                        // at most one thread
        int k = 0;
        u64 x = x0;
        if (run + x < want) { run += x; x = x1; k = 1; if (run + x < want) { run += x; x = x2; k = 2; if (run + x < want) { run += x; x = x3; k = 3; } } }
        S.bin = threadIdx.x * 4 + k;
        S.before = run;
        S.found = x;
    }
    __syncthreads();
    BinAt r;
    const bool any = before < want && before + p.total >= want;
    r.bin = any ? S.bin : -1;
    r.before = any ? S.before : before + p.total;
    r.measure = any ? S.found : 0;
    __syncthreads();
    return r;
}
__device__ __forceinline__ int bin_shift(u64 range) { return range < kBins ? 0 : 54 - __clzll(range); }      // (range >> shift) < 1024
// an element's weight in units of 1/unit; sums of it do not depend on their order
template <int DT> __device__ __forceinline__ u64 mass_of(u64 e, double unit) { return __double2ull_rn(S.w(element_logit<DT>(e)) * unit); }
__device__ __forceinline__ void add_mass(int k, u64 f) {          // f < 2^57, in three words of 19 bits: kSpreadCap of them cannot overflow 32
    unsigned *w = bins() + k;
    atomicAdd(w, static_cast<uint32_t>(f) & 0x7ffffu);
    atomicAdd(w + kBins, static_cast<uint32_t>(f >> 19) & 0x7ffffu);
    const uint32_t c = static_cast<uint32_t>(f >> 38);
    if (c) atomicAdd(w + 2 * kBins, c);
}

// Among the n listed elements that are >= edge, in their order (BY_ID: in increasing id): the one at which the running
// measure (their number; BY_MASS: their fixed-point mass) reaches `want`, coming from `before`; 0 if none does.  A histogram
// of 1024 bins over the interval that is left, from the element `first` on, until few are left (a level costs some 4000 cycles, a
// few in front of another 10 each); then every thread adds up what is in front of its own.
enum : int { BY_MASS = 1, BY_ID = 2 };
constexpr int kFew = 64;
template <int DT> __device__ __noinline__ u64 find_element(int n, u64 edge, u64 want, u64 before, u64 first, u64 range, int how, double unit) {
    u64 low = 0;
    auto pos = [&](u64 e) { return (how & BY_ID) ? static_cast<u64>(element_id(e)) : first - e; };
    int few;
    do {
        const int shift = bin_shift(range);
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += kPickThreads) {
            const u64 e = list()[i], p = pos(e) - low;
            if (e >= edge && p <= range) {
                if (how & BY_MASS) add_mass(static_cast<int>(p >> shift), mass_of<DT>(e, unit));
                else atomicAdd(bins() + static_cast<int>(p >> shift), 1u);
            }
        }
        if (threadIdx.x == 0) S.listed = 0;
        const BinAt at = find_bin(want, before, 19, false);
        if (at.bin < 0) return 0;
        before = at.before;
        low += static_cast<u64>(at.bin) << shift;
        range = min(range - (static_cast<u64>(at.bin) << shift), (1ull << shift) - 1);
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += kPickThreads) {
            const u64 e = list()[i];
            if (e >= edge && pos(e) - low <= range) {
                const int k = atomicAdd(&S.listed, 1);
                if (k < kFew) S.few[k] = e;
            }
        }
        __syncthreads();
        few = S.listed;
        __syncthreads();
    } while (few > kFew);
    const u64 e = threadIdx.x < few ? S.few[threadIdx.x] : 0ull;
    const u64 f = !e ? 0ull : (how & BY_MASS) ? mass_of<DT>(e, unit) : 1ull;
    S.few_mass[threadIdx.x] = f;
    __syncthreads();
    if (e) {
#pragma unroll 4
        for (int j = 0; j < few; ++j) before += pos(S.few[j]) < pos(e) ? S.few_mass[j] : 0ull;
        if (before < want && before + f >= want) S.found = e;      // one thread: the bin's running measure passes `want` once
    }
    __syncthreads();
    return S.found;
}

// ---- steps of the pick kernel ----

// group maxima into shared memory; this thread's largest comes back (NaN if a NaN is among them)
template <int DT> __device__ __noinline__ float load_groups(const void *gmax, size_t base) {
    float best = -INFINITY;
    const int ngroups = S.ngroups, coarse = S.coarse;
    float *sg = group_max();
    if (coarse == 1) {
#pragma unroll 1
        for (int g0 = threadIdx.x; g0 < ngroups; g0 += 8 * kPickThreads) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = g0 + i * kPickThreads < ngroups ? load_group<DT>(gmax, base + g0 + i * kPickThreads) : -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (g0 + i * kPickThreads < ngroups) sg[g0 + i * kPickThreads] = x[i];
                best = max_nan(best, x[i]);
            }
        }
    } else {
#pragma unroll 1
        for (int g = threadIdx.x; g < ngroups; g += kPickThreads) {
            float x = -INFINITY;
            const int s0 = (g >> 5) * coarse;
#pragma unroll 1
            for (int c = 0; c < coarse && s0 + c < S.nstrip; ++c) x = max_nan(x, load_group<DT>(gmax, base + static_cast<size_t>(s0 + c) * 32 + (g & 31)));
            sg[g] = x;
            best = max_nan(best, x);
        }
    }
    return best;
}

// numbers of the groups whose maximum is at least `floor`, in any order; tmax: the largest of this thread's
__device__ __noinline__ void list_groups(float floor, float tmax) {
    const float *sg = group_max();
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) S.ng = 0;
    __syncthreads();
    int mine = 0;
    if (tmax >= floor) {
#pragma unroll 4
        for (int g = threadIdx.x; g < S.ngroups; g += kPickThreads) mine += sg[g] >= floor;
    }
    if (__any_sync(0xffffffffu, mine != 0)) {
        int at = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += y;
        }
        int base = 0;
        if (lane == 31) base = atomicAdd(&S.ng, at);
        at += __shfl_sync(0xffffffffu, base, 31) - mine;
        if (mine) {
            unsigned short *out = group_list();
#pragma unroll 1
            for (int g = threadIdx.x; g < S.ngroups; g += kPickThreads)
                if (sg[g] >= floor) out[at++] = static_cast<unsigned short>(g);
        }
    }
    __syncthreads();
}
// vectors of the listed groups (S.coarse << S.ulog of them each), and the t-th of them
__device__ __forceinline__ int listed_vectors() { return S.ng < 0 ? S.nvec : S.ng * (S.coarse << S.ulog); }
__device__ __forceinline__ int listed_vector(int t) {
    if (S.ng < 0) return t;
    const int per = S.coarse << S.ulog;
    const int k = S.coarse == 1 ? t >> S.ulog : t / per, j = t - k * per, g = group_list()[k];
    return ((((g >> 5) * S.coarse + (j >> S.ulog)) << S.ulog) + (j & ((1 << S.ulog) - 1))) * 32 + (g & 31);
}

// elements of the listed groups at or above zlow to the list, as far as they fit; returns how many there are.  One shared atomic
// per warp and batch of vectors: as many on one address as there are elements cost more than the loads.
template <int DT> __device__ __noinline__ int gather(float zlow) {
    constexpr int B = 4, EPV = Elt<DT>::kPerVec;
    const int lane = threadIdx.x & 31, total = listed_vectors();
    if (threadIdx.x == 0) S.listed = 0;
    __syncthreads();
#pragma unroll 1
    for (int t0 = threadIdx.x; t0 - lane < total; t0 += B * kPickThreads) {
        uint4 raw[B];
        int v[B];
#pragma unroll
        for (int k = 0; k < B; ++k) v[k] = t0 + k * kPickThreads < total ? listed_vector(t0 + k * kPickThreads) : S.nvec;
        state_vectors<DT, B>(v, raw);
        unsigned in = 0;
#pragma unroll
        for (int k = 0; k < B; ++k) {
            float z[EPV];
            unpack<DT>(raw[k], z);
#pragma unroll
            for (int i = 0; i < EPV; ++i) in |= static_cast<unsigned>(z[i] >= zlow) << (k * EPV + i);
        }
        if (!__any_sync(0xffffffffu, in != 0)) continue;
        int at = __popc(in);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, at, o);
            if (lane >= o) at += y;
        }
        int base = 0;
        if (lane == 31) base = atomicAdd(&S.listed, at);
        at += __shfl_sync(0xffffffffu, base, 31) - __popc(in);
#pragma unroll 1
        for (; in; in &= in - 1, ++at) {
            const int bit = __ffs(in) - 1, k = bit / EPV, i = bit % EPV;
            const uint4 r = k < 2 ? (k == 0 ? raw[0] : raw[1]) : (k == 2 ? raw[2] : raw[3]);
            const int vk = k < 2 ? (k == 0 ? v[0] : v[1]) : (k == 2 ? v[2] : v[3]);
            if (at < kListCap) list()[at] = element_of<DT>(vector_element<DT>(r, i), vk * EPV - S.head + i);
        }
    }
    __syncthreads();
    const int n = S.listed;
    __syncthreads();                                               // (the next step may count in the same word)
    return n;
}

// A floor under the border for a top-k of at most half as many as there are threads, from the threads' maxima (nearly as tight
// as the groups' own): k of them are at or above it, so at least k elements are.  Steps down from m that double, then halve.
__device__ __noinline__ float floor_from_threads(int k, float tmax) {
    const float m = S.m;
    float step = 1.f, low = m;
    int n = 0;
#pragma unroll 1
    for (int i = 0; i < 40; ++i, step *= 2.f) {
        low = m - step;
        if (!(low >= -FLT_MAX)) return -INFINITY;
        n = __syncthreads_count(tmax >= low);
        if (n >= k) break;
    }
    if (n < k) return -INFINITY;
    float high = m;                                                // (if fewer than k reach it; else the loop ends at once)
#pragma unroll 1
    for (int i = 0; i < 24 && n > k + k / 8 + 4; ++i) {
        const float mid = low + 0.5f * (high - low);
        if (mid <= low || mid >= high) break;
        const int c = __syncthreads_count(tmax >= mid);
        if (c >= k) { low = mid; n = c; } else high = mid;
    }
    return low;
}

// A floor under the border from the maxima of the groups: the smallest one among the first of 1024 equal parts of [q, m] that
// hold `want` of them, by count or by mass (2^18 per unit of weight, rounded down, so never too much).  q: as far again below m as
// the least of the threads' maxima.  -inf if they do not hold that much.
__device__ __noinline__ float floor_from_groups(bool by_mass, unsigned want, float tmax) {
    const float m = S.m, *sg = group_max();
    const float least = order_float(block_min(float_order(tmax > -1e30f ? tmax : m)));
    const float q = fmaxf(least - (m - least), -FLT_MAX), step = (m - q) * (1.f / kBins);
    if (!(step > 0.f) || !(step < INFINITY)) return -INFINITY;
    const float per = 1.f / step, sf = static_cast<float>(S.w.s);
#pragma unroll 2
    for (int g = threadIdx.x; g < S.ngroups; g += kPickThreads) {
        const float x = sg[g];
        if (x >= q) {
            const unsigned add = by_mass ? static_cast<unsigned>(ex2((x - m) * sf) * (262144.f * 0.9999f)) : 1u;
            if (add) atomicAdd(bins() + min(static_cast<int>((m - x) * per), kBins - 1), add);
        }
    }
    const int bin = find_bin(want, 0, 19, false).bin;
    if (bin < 0) return -INFINITY;
    int low = INT_MAX;                                             // the smallest of these bins, by the same rounding that put it there
#pragma unroll 2
    for (int g = threadIdx.x; g < S.ngroups; g += kPickThreads) {
        const float x = sg[g];
        if (x >= q && min(static_cast<int>((m - x) * per), kBins - 1) <= bin) low = min(low, float_order(x));
    }
    return order_float(block_min(low));
}

// ---- the border by digits of the key over the whole row ----
//
// For what the other ways leave: runs of equal logits longer than the list, a top-k of many thousands with top-p.  Every level
// splits the interval of logits that holds the border into at most 1024 bins and reads the row again.  Masses are 64-bit
// fixed-point numbers (two 32-bit shared atomics with a carry).

enum : int { PASS_COUNT_KEYS, PASS_WEIGH_KEYS, PASS_WEIGH, PASS_COUNT, PASS_COUNT_IDS, PASS_LOWEST_ID };
// One pass over the row (or its listed groups) for the elements whose logit is in [low, high]: their number, mass (the bits of a double: small
// weights count, however many there are) or lowest id, or a histogram of their keys down from `high`, or of their ids up from `base`.
template <int DT> __device__ __noinline__ u64 row_pass(int what, float low, float high, int shift, int base, double unit) {
    constexpr int EPV = Elt<DT>::kPerVec;
    const int total = listed_vectors();
    const uint32_t top = logit_key<DT>(high);
    u64 mine = what == PASS_LOWEST_ID ? INT_MAX : 0;
    double mass = 0.0;
#pragma unroll 1
    for (int t0 = threadIdx.x; t0 < total; t0 += 4 * kPickThreads) {
        uint4 raw[4];
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = t0 + k * kPickThreads < total ? listed_vector(t0 + k * kPickThreads) : S.nvec;
        state_vectors<DT, 4>(v, raw);
        unsigned in = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float z[EPV];
            unpack<DT>(raw[k], z);
#pragma unroll
            for (int i = 0; i < EPV; ++i) in |= static_cast<unsigned>(z[i] >= low && z[i] <= high) << (k * EPV + i);
        }
        if (what == PASS_COUNT) { mine += __popc(in); continue; }
#pragma unroll 1
        for (; in; in &= in - 1) {
            const int bit = __ffs(in) - 1, k = bit / EPV, i = bit % EPV;
            const float x = vector_element<DT>(k < 2 ? (k == 0 ? raw[0] : raw[1]) : (k == 2 ? raw[2] : raw[3]), i);
            const int id = (k < 2 ? (k == 0 ? v[0] : v[1]) : (k == 2 ? v[2] : v[3])) * EPV - S.head + i;
            if (what == PASS_LOWEST_ID) { mine = min(mine, static_cast<u64>(id)); continue; }
            if (what == PASS_COUNT_IDS) {
                if (id >= base && (id - base) >> shift < kBins) atomicAdd(bins() + ((id - base) >> shift), 1u);
                continue;
            }
            if (what == PASS_WEIGH) { mass += S.w(x); continue; }
            const u64 f = what == PASS_COUNT_KEYS ? 1ull : __double2ull_rn(S.w(x) * unit);
            const uint32_t j = (top - logit_key<DT>(x)) >> shift, lo = static_cast<uint32_t>(f);
            const uint32_t old = atomicAdd(bins() + j, lo);
            const uint32_t hi = static_cast<uint32_t>(f >> 32) + (old + lo < old ? 1u : 0u);
            if (hi) atomicAdd(bins() + kBins + j, hi);
        }
    }
    if (what == PASS_WEIGH) return static_cast<u64>(__double_as_longlong(block_prefix(mass).total));
    if (what == PASS_COUNT) return block_prefix(mine).total;
    if (what == PASS_LOWEST_ID) return static_cast<u64>(block_min(static_cast<int>(mine)));
    return 0;
}
struct Border { float z; int id; };
// The key at which the running measure, coming from `before`, reaches `want` within [lo, hi], and the measure in front of it; false if none does.
template <int DT> __device__ __noinline__ bool key_by_digits(int what, uint32_t lo, uint32_t hi, double unit, u64 want, uint32_t &key, u64 &before) {
    for (;;) {
        const int shift = bin_shift(hi - lo);
        row_pass<DT>(what, key_logit<DT>(lo), key_logit<DT>(hi), shift, 0, unit);
        const BinAt at = find_bin(want, before, 32, false);
        before = at.before;
        if (at.bin < 0) return false;
        hi -= static_cast<uint32_t>(at.bin) << shift;
        if (shift == 0) { key = hi; return true; }
        const uint32_t width = (1u << shift) - 1u;
        if (hi - lo > width) lo = hi - width;
    }
}
// What is known of the border (of top-k where there is one, else of top-p): it is within [low, high], with `above` elements of `mass`
// in front of them; low > high: nothing.  `Z`: mass of the row where there is no top-k.
struct Hint { float low, high; u64 above; double mass; };
template <int DT> __device__ __noinline__ Border border_by_digits(const RowAsk &ask, float zmin, double Z, const Hint &hint) {
    const uint32_t top = logit_key<DT>(S.m), bottom = logit_key<DT>(-FLT_MAX);
    const uint32_t near_lo = logit_key<DT>(hint.low), near_hi = logit_key<DT>(hint.high);
    Border r;
    r.z = -INFINITY; r.id = -1;                                    // everything finite
    bool cut = false;                                              // something is left out
    u64 take = 0, before = 0;                                      // how many of the elements at the border's logit are kept
    uint32_t key = 0;
    if (ask.k_on) {
        if (hint.low <= hint.high && hint.above < static_cast<u64>(ask.k)) {
            before = hint.above;
            cut = key_by_digits<DT>(PASS_COUNT_KEYS, near_lo, near_hi, 1.0, ask.k, key, before);
        }
        if (!cut) {
            before = 0;
            cut = key_by_digits<DT>(PASS_COUNT_KEYS, bottom, top, 1.0, ask.k, key, before);
        }
        take = ask.k - before;
    }
    if (ask.p_on) {
        if (ask.k_on) {                                            // the mass that top-k leaves
            const uint32_t lo = cut ? key + 1 : bottom;
            Z = cut ? static_cast<double>(take) * S.w(key_logit<DT>(key)) : 0.0;
            if (lo <= top) Z += __longlong_as_double(static_cast<long long>(row_pass<DT>(PASS_WEIGH, key_logit<DT>(lo), S.m, 0, 0, 0.0)));
        }
        const double unit = two_to(61 - exponent(Z));              // Z unit < 2^62
        const u64 want = max(1ull, static_cast<u64>(ceil(static_cast<double>(ask.p) * Z * unit)));
        const uint32_t lo = cut ? key + 1 : bottom;                // ties at the top-k border are counted apart
        uint32_t k = 0;
        bool by_p = false;
        if (!ask.k_on && hint.low <= hint.high) {
            before = __double2ull_rn(hint.mass * unit);
            if (before < want) by_p = key_by_digits<DT>(PASS_WEIGH_KEYS, near_lo, near_hi, unit, want, k, before);
        }
        if (!by_p) {
            before = 0;
            by_p = lo <= top && key_by_digits<DT>(PASS_WEIGH_KEYS, lo, top, unit, want, k, before);
        }
        if (by_p) key = k;
        if (by_p || cut) {
            const u64 f = __double2ull_rn(S.w(key_logit<DT>(key)) * unit);
            u64 need = 1;
            if (want > before) need = f ? (want - before + f - 1) / f : ~0ull;
            take = by_p ? max(need, 1ull) : min(max(need, 1ull), take);
            cut = true;
        }
    }
    if (cut) {
        r.z = key_logit<DT>(key);
        r.id = INT_MAX;
        if (take < row_pass<DT>(PASS_COUNT, r.z, r.z, 0, 0, 0.0)) {
            // the id of the last one that is kept, by digits of the id
            int base = 0, shift = bin_shift(S.V - 1);
            before = 0;
            for (;;) {
                row_pass<DT>(PASS_COUNT_IDS, r.z, r.z, shift, base, 0.0);
                const BinAt at = find_bin(take, before, 32, false);
                before = at.before;
                base += at.bin << shift;
                if (shift == 0) break;
                shift = max(0, shift - 10);
            }
            r.id = base;
        }
    }
    if (ask.min_on && zmin > r.z) { r.z = zmin; r.id = INT_MAX; }
    return r;
}

// ---- the border among thousands: a bracket from a sample ----

// Two logits that the k-th largest (or the last one inside top-p) lies between but for bad luck, from up to 8192 elements
// spread over the row: where the sample itself has that place, and four standard errors to both sides (up to eight, if few elements
// lie between; fewer, if as many would not fit `capacity`), not below `floor`.  The sample is counted and weighed in 1024 equal parts of [q, m], what is below q with the first;
// q: three times as far below m as the least of the threads' maxima.  (A logit of the type's lowest value is a mask to both.)
struct Bracket { float low, high; bool wide; };            // wide: with four standard errors it would not have fit
template <int DT> __device__ __noinline__ Bracket bracket(const RowAsk &ask, double Z, int capacity, float floor, float tmax) {
    constexpr int EPV = Elt<DT>::kPerVec, total = kSample / EPV, B = 4;
    static_assert(total % (B * kPickThreads) == 0 && kSample <= 8192, "whole batches; 8192 parts of 498 000 fit 32 bits");
    const bool whole = S.nvec <= total, by_mass = !ask.k_on;
    const float m = S.m, sf = static_cast<float>(S.w.s);
    Bracket r;
    r.low = -FLT_MAX; r.high = m; r.wide = false;
    float q = order_float(block_min(float_order(tmax > -1e30f ? tmax : m)));
    q = m - 3.f * (m - q);
    if (by_mass) q = fmaxf(q, m - 70.f * ask.tau);                 // (no weight worth a part is below that)
    const float width = (m - q) * (1.f / kBins), per_bin = 1.f / width;
    if (!(width > 0.f) || !(width < INFINITY) || !(per_bin < INFINITY)) return r;
    const double share = whole ? 1.0 : static_cast<double>(total) / S.nvec, spare = whole ? 0.0 : 4.0 * sqrt(1.0 - share);
    // by mass: (1-p) Z lies below the border, and the many small weights there are what a sample knows well; in units of
    // 1/2^18 of it, each clipped at 1.9, from the smallest logit up.  By count: from the largest down.
    const float unit = by_mass ? static_cast<float>(262144.0 / ((1.0 - static_cast<double>(ask.p)) * Z * share)) : 0.f;
    unsigned *w = bins();
#pragma unroll 1
    for (int j0 = threadIdx.x; j0 < total; j0 += B * kPickThreads) {
        uint4 raw[B];
        int v[B];
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const int j = j0 + k * kPickThreads;
            v[k] = whole ? j : static_cast<int>(static_cast<long long>(j) * S.nvec / total);
        }
        state_vectors<DT, B>(v, raw);
#pragma unroll
        for (int k = 0; k < B; ++k) {
            float z[EPV];
            unpack<DT>(raw[k], z);
#pragma unroll
            for (int i = 0; i < EPV; ++i) {
                if (!(z[i] > -INFINITY)) continue;
                const int up = max(min(static_cast<int>((z[i] - q) * per_bin), kBins - 1), 0);
                if (by_mass) {
                    const unsigned add = __float2uint_rn(fminf(ex2((z[i] - m) * sf) * unit, 498000.f));
                    if (add) { atomicAdd(w + up, add); atomicAdd(w + kBins + up, 1u); }
                } else {
                    atomicAdd(w + (kBins - 1 - up), 1u);
                }
            }
        }
    }
    __syncthreads();
    uint4 *own = reinterpret_cast<uint4 *>(w) + threadIdx.x;       // four bins of each thread, out of shared memory for good
    const uint4 a = own[0], c = by_mass ? own[kBins / 4] : a;
    own[0] = make_uint4(0, 0, 0, 0);
    own[kBins / 4] = own[0];
    const unsigned x[4] = {a.x, a.y, a.z, a.w}, n[4] = {c.x, c.y, c.z, c.w};
    const unsigned mine = a.x + a.y + a.z + a.w;
    const unsigned run0 = block_prefix(mine).before;
    // where the running measure reaches `at`, in bins, by proportion inside one; every thread looks at its own four
    auto place = [&](double at, float *out) {
        unsigned run = run0;
        if (static_cast<double>(run0) < at && static_cast<double>(run0) + mine >= at) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (run < at && static_cast<double>(run) + x[i] >= at) *out = threadIdx.x * 4 + i + static_cast<float>((at - run) / x[i]);
                run += x[i];
            }
        }
    };
    float *at = reinterpret_cast<float *>(S.few);
    if (threadIdx.x < 3) at[threadIdx.x] = -1.f;
    double want = 262144.0, off;
    if (by_mass) {
        __syncthreads();
        place(want, at + 2);
        __syncthreads();
        const float here = at[2] < 0.f ? static_cast<float>(kBins) : at[2];
        float square = 0.f;                                        // sum of the squared weights below the place, bin by bin from their mean
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (static_cast<float>(threadIdx.x * 4 + i) <= here && n[i]) square += static_cast<float>(x[i]) * static_cast<float>(x[i]) / static_cast<float>(n[i]);
        off = spare * sqrt(block_prefix(static_cast<double>(square)).total) + 1200.0;
    } else {
        want = ask.k * share;
        off = spare * (sqrt(want) + 1.0);
    }
#pragma unroll 1
    for (int round = 0; round < 4; ++round) {
        __syncthreads();
        if (threadIdx.x < 2) at[threadIdx.x] = -1.f;
        __syncthreads();
        place(fmax(1.0, want - off), at);
        place(want + off, at + 1);
        __syncthreads();
        const float near = by_mass ? fmaxf(at[0], (floor - q) * per_bin) : at[0], far = at[1];
        r.low = -FLT_MAX; r.high = m;
        if (by_mass) {
            if (near > 1.f) r.low = q + near * width;
            if (far >= 0.f) r.high = q + far * width;
        } else {
            if (far >= 0.f && far < kBins - 1) r.low = m - far * width;
            if (want - off >= 1.0 && near > 0.f) r.high = m - near * width;
        }
        if (round == 3) break;
        int inside = 0;
        const float last = far < 0.f ? static_cast<float>(kBins) : far;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float bin = static_cast<float>(threadIdx.x * 4 + i);
            if (bin + 1.f > near && bin < last)
                inside += static_cast<int>(static_cast<float>(n[i]) * (fminf(bin + 1.f, last) - fmaxf(bin, near)) + 0.5f);
        }
        const double expected = block_sum(inside) / share;
        if (round == 0 && expected < 0.0625 * capacity) {          // up to twice as wide: nearly free, and a miss is not
            off *= fmin(2.0, 0.0625 * capacity / fmax(expected, 1.0));
            continue;
        }
        if (expected <= 0.9 * capacity) break;
        r.wide = true;
        off *= fmax(0.4, 0.8 * capacity / expected);
    }
    __syncthreads();
    r.low = fmaxf(r.low, floor);
    r.high = fmaxf(fminf(r.high, m), r.low);
    if (DT == TLI_BF16) {                                          // values of the row's type, so that keys and logits say the same
        r.low = fmaxf(__bfloat162float(__float2bfloat16_rd(r.low)), -FLT_MAX);
        r.high = __bfloat162float(__float2bfloat16_ru(r.high));
    }
    return r;
}

// ---- border and draw from the list ----

// The border among the n listed elements (logits from ztop down to zlow), with `above` elements of mass `above_mass` in front of
// them, all kept as far as the list reaches; if they number fewer than k, nothing below zlow could be kept either.  Elements >= edge
// are kept, in the list and out of it (edge 0: the border is not here).  unit: for masses, so that no sum of them reaches 2^57.
struct Edge { u64 edge; double unit; };
template <int DT> __device__ __noinline__ Edge border_in_list(const RowAsk &ask, bool draw, float zmin, double Z, int n, float ztop, float zlow, u64 above, double above_mass) {
    const u64 first = element_of<DT>(ztop, 0), range = first - (static_cast<u64>(logit_key<DT>(zlow)) << 20);
    Edge r;
    r.edge = 1; r.unit = 1.0;
    if (ask.k_on && above + n >= static_cast<u64>(ask.k)) {
        r.edge = 0;
        if (above >= static_cast<u64>(ask.k)) return r;
        r.edge = find_element<DT>(n, 1, ask.k, above, first, range, 0, 0.0);
    }
    if (ask.p_on || draw) {
        // The unit by the mass itself: by the number of elements (a weight is at most 1) thousands of small weights beside a large one would round
        // to nothing.  The mass that top-k leaves is summed in units of 2^-50 (8192 weights fit 64 bits, and are off by 2^-38 at most) and not in
        // fp64, which would depend on the list's order.
        double mass = Z;
        if (!ask.p_on || ask.k_on) {
            constexpr double fine = 1125899906842624.0;            // 2^50
            static_assert(kSpreadCap <= 1 << 13 && kListCap <= kSpreadCap, "sums below 2^64");
            u64 all = 0;
#pragma unroll 4
            for (int i = threadIdx.x; i < n; i += kPickThreads) if (list()[i] >= r.edge) all += mass_of<DT>(list()[i], fine);
            mass = above_mass + static_cast<double>(block_prefix(all).total) / fine;
        }
        r.unit = two_to(56 - exponent(mass + 1e-11));
        if (ask.p_on) {
            const u64 before = __double2ull_rn(above_mass * r.unit);
            const u64 want = max(1ull, static_cast<u64>(ceil(static_cast<double>(ask.p) * mass * r.unit)));
            const u64 edge = above > 0 && before >= want ? 0ull : find_element<DT>(n, r.edge, want, before, first, range, BY_MASS, r.unit);
            r.edge = edge;
            if (edge == 0) return r;
        }
    }
    if (ask.min_on) r.edge = max(r.edge, static_cast<u64>(logit_key<DT>(zmin)) << 20);
    return r;
}
template <int DT> __device__ __forceinline__ Border border_of(u64 edge) {
    Border r;
    r.z = edge > 1 ? element_logit<DT>(edge) : -INFINITY;
    r.id = edge > 1 ? element_id(edge) : -1;
    return r;
}

struct Draw { int token; double prob; };
// (a number outside [0, 1) is the caller's mistake, but still draws a kept id)
__device__ __forceinline__ float uniform_of(const RowsParams &P, int row) { return fminf(fmaxf(__ldg(P.u + row), 0.f), 1.f); }
// Border and draw from a list of at most one element per thread: every thread counts, and weighs, what is in front of its own
// element, in the order of the logits and then in that of the ids.  Two trips through the list against ten block-wide steps.
template <int DT> __device__ __noinline__ Draw pick_from_short_list(const RowAsk &ask, bool draw, float u, float zmin, double Z, int n, Border &border) {
    const int tid = threadIdx.x;
    const u64 e = tid < n ? list()[tid] : 0ull;
    // the masses' unit: every sum formed here stays below 2^57
    const double unit = two_to(56 - exponent(ask.p_on && !ask.k_on ? Z : static_cast<double>(n)));
    const bool weigh = ask.p_on || draw;
    const double w = e && weigh ? S.w(element_logit<DT>(e)) : 0.0;
    const u64 f = __double2ull_rn(w * unit);
    S.few_mass[tid] = f;
    __syncthreads();
    int rank = 0;
    u64 ahead = 0;
    if (e) {
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const bool before = list()[j] > e;
            rank += before;
            ahead += before ? S.few_mass[j] : 0ull;
        }
    }
    const int k = ask.k_on ? min(ask.k, n) : n;
    u64 want = ~0ull;
    if (ask.p_on) {
        if (e && rank == k - 1) S.before = ahead + f;              // the mass that top-k leaves
        __syncthreads();
        want = max(1ull, static_cast<u64>(ceil(static_cast<double>(ask.p) * (ask.k_on ? static_cast<double>(S.before) : Z * unit))));
    }
    const bool kept = e && rank < k && (ask.p_on ? ahead < want : true) && (ask.min_on ? rank == 0 || element_logit<DT>(e) >= zmin : true);
    const int count = __syncthreads_count(kept);
    if (e && rank == count - 1) { S.found = e; S.before = ahead + f; }
    __syncthreads();
    const u64 edge = S.found, total = S.before;
    __syncthreads();                                               // (the draw leaves its element where the border was)
    border.z = element_logit<DT>(edge);
    border.id = element_id(edge);
    // fewer kept than asked for: only min-p or the end of the row can be the reason, and both hold below the list too
    Draw d = {-1, 0.0};
    if (!draw) return d;
    const u64 target = static_cast<u64>(static_cast<double>(u) * static_cast<double>(total));
    u64 own = f;
    if (target == 0) {                                             // the lowest id that has any weight
        own = w > 0.0;
        S.few_mass[tid] = own;
        __syncthreads();
    }
    if (kept) {
        u64 before = 0;
        const uint32_t id = static_cast<uint32_t>(e) & kIdMask;    // (falls as the id grows)
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const u64 x = list()[j];
            before += x >= edge && (static_cast<uint32_t>(x) & kIdMask) > id ? S.few_mass[j] : 0ull;
        }
        if (before <= target && target < before + own) S.found = e;
    }
    __syncthreads();
    const u64 hit = S.found;
    d.token = element_id(hit);
    d.prob = S.w(element_logit<DT>(hit)) * unit / static_cast<double>(total);
    return d;
}

// The id that owns u * total among the listed elements >= edge.
template <int DT> __device__ __noinline__ Draw draw_from_list(float u, int n, u64 edge, double unit) {
    u64 mine = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kPickThreads) if (list()[i] >= edge) mine += mass_of<DT>(list()[i], unit);
    const u64 total = block_prefix(mine).total, target = static_cast<u64>(static_cast<double>(u) * static_cast<double>(total));
    u64 hit;
    if (target > 0) {
        hit = find_element<DT>(n, edge, min(target + 1, total), 0, 0, S.V - 1, BY_MASS | BY_ID, unit);
    } else {                                                       // the lowest id that has any weight
        int low = INT_MAX;
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += kPickThreads)
            if (list()[i] >= edge && element_logit<DT>(list()[i]) >= S.w.cut) low = min(low, element_id(list()[i]));
        low = block_min(low);
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += kPickThreads)
            if (list()[i] >= edge && element_id(list()[i]) == low) S.found = list()[i];
        __syncthreads();
        hit = S.found;
    }
    Draw d;
    d.token = element_id(hit);
    d.prob = S.w(element_logit<DT>(hit)) * unit / static_cast<double>(total);
    return d;
}

// The id that owns u * total over what (bz, bid) keeps of the row, from strips(), a sum per strip.
template <int DT> __device__ __noinline__ Draw draw_by_strips(Border border, float u) {
    constexpr int EPV = Elt<DT>::kPerVec;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    const int per = (S.nstrip + kPickThreads - 1) / kPickThreads, first = threadIdx.x * per, end = min(first + per, S.nstrip);
    double mine = 0.0;
    int last = -1;
#pragma unroll 1
    for (int i = first; i < end; ++i) {
        mine += strips()[i];
        if (strips()[i] > 0.0) last = i;
    }
    const Prefix<double> p = block_prefix(mine);
    const double target = static_cast<double>(u) * p.total;
    last = block_max(last);
    double run = p.before;
    int hit = INT_MAX;
#pragma unroll 1
    for (int i = first; i < end; ++i) {
        if (strips()[i] > 0.0 && run + strips()[i] > target) { hit = i; break; }
        run += strips()[i];
    }
    const int lowest = block_min(hit), strip = min(lowest, last);  // rounding can leave none above the target
    double *before = reinterpret_cast<double *>(&S.before);        // what lies in front of the strip: its owner says
    if (strip == hit) *before = run;
    else if (lowest == INT_MAX && first <= last && last < end) *before = run - strips()[last];
    __syncthreads();
    // the strip's vectors of every lane, one per warp (there are at most as many)
    static_assert(kPickWarps >= 8, "a warp per vector of a strip");
    const int e0 = ((strip << (5 + S.ulog)) + warp * 32 + lane) * EPV - S.head;
    double x[EPV], sum = 0.0, w_mine = 0.0;
    int id_mine = -1;
#pragma unroll
    for (int j = 0; j < EPV; ++j) x[j] = 0.0;
    if (warp < (1 << S.ulog)) {
        const int v[1] = {(strip << (5 + S.ulog)) + warp * 32 + lane};
        uint4 r[1];
        state_vectors<DT, 1>(v, r);
        float z[EPV];
        unpack<DT>(r[0], z);
#pragma unroll
        for (int j = 0; j < EPV; ++j) {
            x[j] = z[j] > border.z || (z[j] == border.z && e0 + j <= border.id) ? S.w(z[j]) : 0.0;
            sum += x[j];
            if (x[j] > 0.0) { id_mine = e0 + j; w_mine = x[j]; }
        }
    }
    const double front = *before + block_prefix(sum).before;       // (block_prefix begins with a barrier)
    // the first lane whose running sum exceeds the target, else the last one that has any weight
    const int hit_at = block_min(sum > 0.0 && front + sum > target ? static_cast<int>(threadIdx.x) : INT_MAX);
    const int last_at = block_max(sum > 0.0 ? static_cast<int>(threadIdx.x) : -1);
    if (static_cast<int>(threadIdx.x) == (hit_at < INT_MAX ? hit_at : last_at)) {
        if (hit_at < INT_MAX) {
            double c = front;
            bool found = false;
#pragma unroll
            for (int j = 0; j < EPV; ++j) {                        // the first element whose running sum does (rounding: or the last)
                c += x[j];
                if (!found && x[j] > 0.0 && c > target) { found = true; id_mine = e0 + j; w_mine = x[j]; }
            }
        }
        S.found = static_cast<u64>(id_mine);
        *before = w_mine / p.total;
    }
    __syncthreads();
    Draw d;
    d.token = static_cast<int>(S.found);
    d.prob = *before;
    return d;
}

__device__ __noinline__ void finish_row(const RowsParams &P, int row, int status, int mode, Border border, int token, double prob) {
    if (threadIdx.x != 0) return;
    if (P.status) P.status[row] = status;
    if (P.sample) {
        P.tokens[row] = token;
        if (P.prob) P.prob[row] = static_cast<float>(prob);
    } else {
        RowBorder rb; rb.z = border.z; rb.id = border.id; rb.mode = mode; rb.pad = 0;
        P.border[row] = rb;
    }
}
// leaves the row to the spread kernel
__device__ __noinline__ void plan_row(const RowsParams &P, int row, int kind, float zlo, float zhi, int bid, float zmin, double Z) {
    if (threadIdx.x != 0) return;
    RowPlan pl;
    pl.Z = Z; pl.zlo = zlo; pl.zhi = zhi; pl.bid = bid; pl.kind = kind; pl.m = S.m; pl.zmin = zmin; pl.listed = 0; pl.done = 0;
    P.plan[row] = pl;
    P.todo[1 + atomicAdd(P.todo, 1)] = row;
}

// Bound by latency: some ten block-wide steps and three or four trips to L2 in a row, 10 to 12 us at top-k 50 for one row or 64, 17 us
// for rows of 256 000 (their 8000 group maxima); 20 to 45 us where a list of thousands or a bracket is needed.  Two or three CTAs
// share an SM (group maxima and list: 50 to 94 KB), so some 300 to 440 rows are one wave.
template <int DT>
__global__ void __launch_bounds__(kPickThreads, 3) tli_rows_pick_kernel(const __grid_constant__ RowsParams P) {
    const int tid = threadIdx.x, row = blockIdx.x, b = row / P.R;
    exp2_table_init(S.tab, tid);
    enter_row<DT>(P, row, b, kListCap);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const RowAsk ask(P, b);
    const float u = P.sample ? uniform_of(P, row) : 0.f;
    const Border all = {-INFINITY, -1};

    __syncthreads();
    const float tmax = load_groups<DT>(P.gmax, static_cast<size_t>(row) * P.nstrip * 32);
    const double scale = Weights::kLog2e / ask.tau;                // (beside the loads)
    const int bad = (ask.bad_tau ? TLI_ROW_BAD_TEMPERATURE : 0) | (ask.bad_filter ? TLI_ROW_BAD_FILTER : 0);
    if (bad) { finish_row(P, row, bad, BORDER_COPY, all, -1, 0.0); return; }
    // NaN lies above +inf, and that above every finite number, in this order
    const float m = order_float(block_max(tmax != tmax ? INT_MAX : float_order(tmax)));
    if (!(m < INFINITY)) { finish_row(P, row, TLI_ROW_NONFINITE, BORDER_COPY, all, -1, 0.0); return; }
    if (!(m > -INFINITY)) { finish_row(P, row, TLI_ROW_FALLBACK, BORDER_APPLY, all, -1, 0.0); return; }      // no id to keep
    if (tid == 0) {
        S.m = m;
        S.w.m = m; S.w.s = scale; S.w.tab = S.tab; S.w.cut = Weights::cut_of(m, ask.tau);
    }

    if (ask.one) {                                                 // the lowest id at the largest logit
        list_groups(m, tmax);
        Border first;
        first.z = m;
        first.id = static_cast<int>(row_pass<DT>(PASS_LOWEST_ID, m, m, 0, 0, 0.0));
        finish_row(P, row, 0, BORDER_APPLY, first, first.id, 1.0);
        return;
    }
    __syncthreads();
    double Z = 0.0;
    if (ask.whole_mass(P.sample)) {                                // the strips' sums at the row's own largest logit
        double mine = 0.0;
#pragma unroll 1
        for (int i = tid; i < P.nstrip; i += kPickThreads) {
            const StripSum ss = P.ssum[static_cast<size_t>(row) * P.nstrip + i];
            const double x = ss.S > 0.0 && ss.m >= S.w.cut ? ss.S * exp2_neg((static_cast<double>(ss.m) - S.w.m) * S.w.s, S.tab) : 0.0;
            strips()[i] = x;
            mine += x;
        }
        Z = block_prefix(mine).total;
    }
    Draw d = {-1, 0.0};
    if (ask.plain()) {
        if (P.sample) d = draw_by_strips<DT>(all, u);
        finish_row(P, row, 0, BORDER_APPLY, all, d.token, d.prob);
        return;
    }
    const float zmin = ask.zmin<DT>(m);

    // a floor under everything that can be kept
    float floor = -INFINITY;
    if (ask.k_on) {
        floor = ask.k <= kPickThreads / 2 ? floor_from_threads(ask.k, tmax) : floor_from_groups(false, ask.k, tmax);
        if (floor == -INFINITY && ask.p_on && P.V > kListCap && ask.k <= P.listcap * 3 / 4) {      // too few groups for that many: from a sample
            floor = bracket<DT>(ask, Z, P.listcap - ask.k, -FLT_MAX, tmax).low;
            if (floor == -FLT_MAX) floor = -INFINITY;
        }
    } else if (ask.p_on && Z < 8192.0) {
        floor = floor_from_groups(true, static_cast<unsigned>(ceil(static_cast<double>(ask.p) * Z * 262144.0)), tmax);
    }
    const bool ok = floor > -INFINITY || (!ask.k_on && !ask.p_on);
    const float zlow = ask.p_on ? fmaxf(floor, -FLT_MAX) : fmaxf(floor, zmin);
    list_groups(zlow, tmax);
    // Every listed group has an element.  Without a floor only short and mostly masked rows are worth a try; and beyond some 4096
    // vectors to read again (4 ns each for this one block) all blocks together are faster: with a limit of 8192 a call for 80 fp32 rows
    // of 256 000 at top-p .9 takes 137 us against 113 (48 bf16 rows of 128 256 at .95: 38 against 51), with one of 1024 the latter
    // at .9 takes 41 us against 29 (64 bf16 rows of 32 000, mixed filters: 55 against 63).
    const int vectors = S.ng * (P.coarse << P.ulog);
    const bool worth = P.V <= kListCap || (ok ? vectors <= 4096 : S.ng <= 256);
    const int n = worth ? gather<DT>(zlow) : INT_MAX;
    // (fewer than k above a sampled floor: there may be more below it)
    const bool whole = !(ask.k_on && n < ask.k && zlow == floor);
    Border border;
    if (n <= kPickThreads && whole) {
        d = pick_from_short_list<DT>(ask, P.sample, u, zmin, Z, n, border);
        finish_row(P, row, 0, BORDER_APPLY, border, d.token, d.prob);
        return;
    }
    if (n <= kListCap && whole) {
        const Edge at = border_in_list<DT>(ask, P.sample, zmin, Z, n, m, zlow, 0, 0.0);
        if (at.edge) {
            if (P.sample) d = draw_from_list<DT>(u, n, at.edge, at.unit);
            finish_row(P, row, 0, BORDER_APPLY, border_of<DT>(at.edge), d.token, d.prob);
            return;
        }
    }
    if (ask.k_on && ok && ask.k <= P.listcap * 3 / 4) {            // all that top-k can keep goes to the list
        plan_row(P, row, PLAN_BRACKET, floor, m, -1, zmin, Z);
        return;
    }
    if (ask.k_on || ask.p_on) {
        const Bracket br = bracket<DT>(ask, Z, P.listcap, ask.k_on ? -FLT_MAX : fmaxf(floor, -FLT_MAX), tmax);
        // A bracket too wide for the list is that of a row whose mass lies in a few large elements, with many small ones below them.  It comes here
        // when two of them share a group (the maxima do not hold the mass, or only far down): the list above the largest groups'
        // maxima is complete as far as it goes, and as a rule far enough.  (One such row of 48 bf16 rows of 128 256 ended in the digits: 359 us a
        // call against 35.)
        const int per = P.coarse << P.ulog;
        const float top = br.wide && !ask.k_on ? floor_from_groups(false, 2048 / per, tmax) : -INFINITY;
        if (top > -INFINITY) {
            list_groups(top, tmax);
            const int few = S.ng * per <= 8192 ? gather<DT>(top) : INT_MAX;
            if (few <= kListCap) {
                const Edge at = border_in_list<DT>(ask, P.sample, zmin, Z, few, m, top, 0, 0.0);
                if (at.edge) {
                    if (P.sample) d = draw_from_list<DT>(u, few, at.edge, at.unit);
                    finish_row(P, row, 0, BORDER_APPLY, border_of<DT>(at.edge), d.token, d.prob);
                    return;
                }
            }
        }
        plan_row(P, row, PLAN_BRACKET, br.low, br.high, -1, zmin, Z);
        return;
    }
    border.z = zmin; border.id = INT_MAX;                          // min-p alone: the border is known
    if (P.sample) plan_row(P, row, PLAN_DRAW, INFINITY, border.z, border.id, zmin, 0.0);
    else finish_row(P, row, 0, BORDER_APPLY, border, -1, 0.0);
}

// ---- rows whose kept set has thousands of elements ----

// Which of a vector's elements are at least `least`, a bit each, and their order: fp32 element i is bit i; bf16 element 2k + h (half
// h of word k) is bit 16h + k, so that one packed comparison and one and-or find two.
template <int DT> struct Least {
    float f;
    __nv_bfloat162 b;
    __device__ __forceinline__ explicit Least(float least) : f(least), b(__bfloat162bfloat162(__float2bfloat16_ru(least))) {}
    __device__ __forceinline__ unsigned bits(const uint4 &r) const {
        if constexpr (DT == TLI_F32) {
            return static_cast<unsigned>(__uint_as_float(r.x) >= f) | static_cast<unsigned>(__uint_as_float(r.y) >= f) << 1 |
                   static_cast<unsigned>(__uint_as_float(r.z) >= f) << 2 | static_cast<unsigned>(__uint_as_float(r.w) >= f) << 3;
        } else {
            auto two = [this](uint32_t x) { return __hge2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&x), b); };
            return (two(r.x) & 0x10001u) | (two(r.y) & 0x20002u) | (two(r.z) & 0x40004u) | (two(r.w) & 0x80008u);
        }
    }
    // the same order for a bit per element in increasing order
    __device__ __forceinline__ static unsigned arranged(unsigned x) {
        if (DT == TLI_F32) return x & 0xfu;
        x = (x & 0x55u) | (x & 0xaau) << 15;
        x = (x | x >> 1) & 0x330033u;
        return (x | x >> 2) & 0xf000fu;
    }
    static constexpr int kVectors = DT == TLI_F32 ? 8 : 4;         // of one word of bits, four places apart
    __device__ __forceinline__ static int vector(int bit) { return (DT == TLI_F32 ? bit : bit & 15) >> 2; }
    __device__ __forceinline__ static int element(int bit) { return DT == TLI_F32 ? bit & 3 : (bit & 3) * 2 + (bit >> 4); }
};

// Strips [strip, end) of such a row by one warp: what (zhi, bid) keeps is counted and, if asked for, weighed, strip by strip; what
// lies from there down to zlo goes to the row's list.  Every lane finds its candidates as bits first, then takes them one by one
// from a copy of its vectors in shared memory (they cannot be indexed in registers): what an element costs that is neither kept nor
// near the border is one comparison.  The next strip is on its way while one is worked on.  (Ballots per element instead of bits per
// lane: 304 fp32 rows of 256 000 at top-p .95 in 215 us against 149.  Weighing the kept ones of a warp 32 at a time from a queue costs as much as it saves.)
constexpr int kStash = 96;                               // 64 and one element of each lane
constexpr int kStage = 8 * 32;                           // vectors of a strip at most
static_assert(kPickWarps * (kStage * 16 + kStash * 8) <= kSpreadCap * 8, "strips and stashes take the place of the list");
template <int DT, int U> __device__ __forceinline__ void spread_strips(const RowsParams &P, RowPlan *plan, int row, int strip, int end, float zlo, float zhi, int bid, bool weigh) {
    using L = Least<DT>;
    constexpr int EPV = Elt<DT>::kPerVec, NW = (U + L::kVectors - 1) / L::kVectors;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nvec = S.nvec, head = S.head;
    const uint4 *vec0 = S.vec0;
    const uint32_t *mask = S.mask;
    const Weights w = S.w;
    uint4 *stage = reinterpret_cast<uint4 *>(list()) + warp * kStage + lane;
    u64 *stash = list() + kPickWarps * kStage * 2 + warp * kStash;
    const size_t groups = static_cast<size_t>(row) * P.nstrip * 32 + lane;
    const L least(fminf(zhi, zlo));
    const bool ties = bid >= 0;                                    // (then all of them: min-p's border)
    int stashed = 0;
    auto flush = [&]() {                                           // the stash to the row's list
        __syncwarp();
        int at = 0;
        if (lane == 0) at = atomicAdd(&plan->listed, stashed);
        at = __shfl_sync(0xffffffffu, at, 0);
        for (int i = lane; i < stashed; i += 32)
            if (at + i < P.listcap) __stcg(P.lists + static_cast<size_t>(row) * P.listcap + at + i, stash[i]);
        stashed = 0;
        __syncwarp();
    };
    uint4 next[U];
    unsigned in[U];                                                // the mask's bits of the vectors
#pragma unroll
    for (int q = 0; q < U; ++q) in[q] = ~0u;
    auto fetch = [&](int st, float gm) {
        int v[U];
#pragma unroll
        for (int q = 0; q < U; ++q) v[q] = gm >= least.f ? st * (32 * U) + q * 32 + lane : nvec;
        row_vectors<DT, U>(vec0, S.row, head, P.V, nvec, nullptr, v, next);
        if (mask) {
#pragma unroll
            for (int q = 0; q < U; ++q)
                if (v[q] < nvec) in[q] = mask_bits(mask, v[q] * EPV - head);
        }
    };
    float gm_after = strip + 1 < end ? load_group<DT>(P.gmax, groups + (strip + 1) * 32) : -INFINITY;
    fetch(strip, load_group<DT>(P.gmax, groups + strip * 32));
#pragma unroll 1
    for (; strip < end; ++strip) {
        unsigned bits[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) bits[i] = 0;
#pragma unroll
        for (int q = 0; q < U; ++q) {
            stage[q * 32] = next[q];                               // (read by this lane only)
            unsigned x = least.bits(next[q]);
            if (mask) x &= L::arranged(in[q]);
            bits[q / L::kVectors] |= x << q % L::kVectors * 4;
        }
        if (strip + 1 < end) fetch(strip + 1, gm_after);
        if (strip + 2 < end) gm_after = load_group<DT>(P.gmax, groups + (strip + 2) * 32);
        const int id0 = (strip * (32 * U) + lane) * EPV - head;
        double acc = 0.0;
        int count = 0, base = 0;
        unsigned now = bits[0];
        if (NW > 1 && now == 0) { now = bits[NW - 1]; base = L::kVectors; bits[NW - 1] = 0; }
        while (__any_sync(0xffffffffu, now != 0)) {                // two of each lane at a time
            float z[2];
            int id[2];
            bool kept[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                z[r] = -INFINITY; id[r] = 0;
                if (now) {
                    const int bit = __ffs(now) - 1, v = (base + L::vector(bit)) * 32, i = L::element(bit);
                    now &= now - 1;
                    if constexpr (DT == TLI_F32) z[r] = reinterpret_cast<const float *>(stage + v)[i];
                    else z[r] = __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const unsigned short *>(stage + v)[i]) << 16);
                    id[r] = id0 + v * EPV + i;
                    if (NW > 1 && now == 0) { now = bits[NW - 1]; base = L::kVectors; bits[NW - 1] = 0; }
                }
                kept[r] = z[r] > zhi || (ties && z[r] == zhi);
                count += kept[r];
            }
            if (weigh && __any_sync(0xffffffffu, kept[0] || kept[1])) {
                const double w0 = w(z[0]), w1 = w(z[1]);
                acc += kept[0] ? w0 : 0.0;
                acc += kept[1] ? w1 : 0.0;
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const bool near = !kept[r] && z[r] >= zlo;
                const unsigned who = __ballot_sync(0xffffffffu, near);
                if (who == 0) continue;
                if (stashed > kStash - 32) flush();
                if (near) stash[stashed + __popc(who & ((1u << lane) - 1u))] = element_of<DT>(z[r], id[r]);
                stashed += __popc(who);
            }
        }
        count = __reduce_add_sync(0xffffffffu, count);
        if (weigh) acc = warp_sum(acc);
        if (lane == 0) {
            StripSum ss; ss.S = acc; ss.m = 0.f; ss.pad = count;
            __stcg(reinterpret_cast<double2 *>(P.ssum + static_cast<size_t>(row) * P.nstrip + strip), *reinterpret_cast<const double2 *>(&ss));
        }
    }
    if (stashed) flush();
}

// Such a row's border in its list, and the draw.
template <int DT> __device__ __noinline__ void settle_row(const RowsParams &P, RowPlan *plan, int row, int b) {
    constexpr int EPV = Elt<DT>::kPerVec;
    const int tid = threadIdx.x;
    const RowAsk ask(P, b);
    const float zmin = __ldcg(&plan->zmin), zlo = __ldcg(&plan->zlo), zhi = __ldcg(&plan->zhi);
    const double Z = __ldcg(&plan->Z);
    const bool bracketed = __ldcg(&plan->kind) == PLAN_BRACKET;
    const int n = static_cast<int>(__ldcg(&plan->listed));
    if (bracketed && n <= P.listcap) {
#pragma unroll 8
        for (int i = tid; i < n; i += kPickThreads) list()[i] = __ldcg(P.lists + static_cast<size_t>(row) * P.listcap + i);
    }
    u64 above = 0;
    double mass = 0.0;
#pragma unroll 2
    for (int i = tid; i < P.nstrip; i += kPickThreads) {
        const double2 raw = __ldcg(reinterpret_cast<const double2 *>(P.ssum + static_cast<size_t>(row) * P.nstrip + i));
        const StripSum ss = *reinterpret_cast<const StripSum *>(&raw);
        strips()[i] = ss.S;
        mass += ss.S;
        above += ss.pad;
    }
    above = block_prefix(above).total;
    mass = block_prefix(mass).total;
    Border border = {zhi, __ldcg(&plan->bid)};
    if (bracketed) {
        Edge at = {0, 1.0};
        if (n <= P.listcap) {
            // (fewer than k in all is not something the bracket can say)
            if (!ask.k_on || above + n >= static_cast<u64>(ask.k)) at = border_in_list<DT>(ask, P.sample, zmin, Z, n, zhi, zlo, above, mass);
        }
        border = border_of<DT>(at.edge);
        if (at.edge && border.z <= zhi) {
            if (P.sample) {
                // the kept elements of the list join their strips, in fixed point so that their order does not matter
                // (the bins hold a strip each; a row of the largest vocabulary can have one more)
                static_assert(kMaxRowStrips <= kBins + 1, "one strip beyond the bins");
                if (tid == 0) S.before = 0;
                __syncthreads();
#pragma unroll 4
                for (int i = tid; i < n; i += kPickThreads) {
                    const u64 e = list()[i];
                    if (e < at.edge) continue;
                    const int strip = (element_id(e) + S.head) / EPV >> (5 + S.ulog);
                    if (strip < kBins) add_mass(strip, mass_of<DT>(e, at.unit));
                    else atomicAdd(&S.before, mass_of<DT>(e, at.unit));
                }
                __syncthreads();
                const double part = 1.0 / at.unit;                 // (a power of two)
#pragma unroll 1
                for (int i = tid; i < P.nstrip; i += kPickThreads) {
                    const unsigned *w = bins() + i;
                    const u64 more = i < kBins ? w[0] + (static_cast<u64>(w[kBins]) << 19) + (static_cast<u64>(w[2 * kBins]) << 38) : S.before;
                    strips()[i] += static_cast<double>(more) * part;
                }
            }
        } else {                                                   // bad luck, or min-p above the bracket: the long way
            const Hint hint = {zlo, zhi, above, mass};
            border = border_by_digits<DT>(ask, zmin, Z, hint);
            if (P.sample) {
                __syncthreads();
#pragma unroll 1
                for (int s = tid >> 5; s < P.nstrip; s += kPickWarps) {
                    double acc = 0.0;
#pragma unroll 1
                    for (int t = tid & 31; t < (32 << S.ulog) * EPV; t += 32) {
                        const int id = (s << (5 + S.ulog)) * EPV - S.head + t;
                        if (id < 0 || id >= P.V || (P.mask && !(__ldg(P.mask + (id >> 5)) >> (id & 31) & 1u))) continue;
                        const float z = load_elt<DT>(S.row, id);
                        if (z > border.z || (z == border.z && id <= border.id)) acc += S.w(z);
                    }
                    acc = warp_sum(acc);
                    if ((tid & 31) == 0) strips()[s] = acc;
                }
            }
        }
    }
    Draw d = {-1, 0.0};
    if (P.sample) d = draw_by_strips<DT>(border, uniform_of(P, row));
    finish_row(P, row, 0, BORDER_APPLY, border, d.token, d.prob);
}

// The rows that the pick kernel left, by all blocks: each takes some strips at a time (the next ones when it is done: the block
// that ends last with a row settles it, which takes 13 to 25 us, as long as several strips).  Two blocks of 128 registers per SM hold
// 16 warps with a strip of 4 KB on its way each.  304 fp32 rows of 256 000 at top-p .95 in 149 us (2.1 TB/s read again; the issue slots are
// 43% busy, the rest waits for the loads, for fp64 results and for the slowest warp of a task); ends 20 us after its last strip.
template <int DT, int U>
__global__ void __launch_bounds__(kPickThreads, 2) tli_rows_spread_kernel(const __grid_constant__ RowsParams P) {
    const int tid = threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int rows = __ldcg(P.todo);
    if (rows == 0) return;
    // strips of a warp at a time: some three turns for every block
    const long long all = static_cast<long long>(rows) * P.nstrip;
    const int each = static_cast<int>(min(8ll, max(1ll, all / (3ll * gridDim.x * kPickWarps))));
    const int nchunk = (P.nstrip + kPickWarps * each - 1) / (kPickWarps * each);
    exp2_table_init(S.tab, tid);
    int *next = P.todo + 1 + P.B * P.R;
    for (;;) {
        __syncthreads();                                           // the shared memory is free again
        if (tid == 0) S.listed = atomicAdd(next, 1);
        __syncthreads();
        const int task = S.listed;
        if (task >= rows * nchunk) return;
        const int row = __ldcg(P.todo + 1 + task / nchunk), b = row / P.R;
        RowPlan *plan = P.plan + row;
        const float zlo = __ldcg(&plan->zlo), zhi = __ldcg(&plan->zhi);
        const int bid = __ldcg(&plan->bid);
        if (tid == 0) {
            S.m = __ldcg(&plan->m);
            S.w = Weights(S.m, __ldg(P.tau + b), S.tab);
        }
        enter_row<DT>(P, row, b, kSpreadCap);
        __syncthreads();
        const int strip = (task % nchunk * kPickWarps + (tid >> 5)) * each;
        if (strip < P.nstrip)
            spread_strips<DT, U>(P, plan, row, strip, min(strip + each, P.nstrip), zlo, zhi, bid, P.sample || (P.top_p && __ldg(P.top_p + b) < 1.f));
        __threadfence();
        __syncthreads();
        if (tid == 0) S.listed = atomicAdd(&plan->done, 1);
        __syncthreads();
        if (S.listed != nchunk - 1) continue;
        __threadfence();
        settle_row<DT>(P, plan, row, b);
    }
}

// Bound by DRAM: 576 bf16 rows of 152 064 (175 MB written, up to as much read) in 42 us.
template <int DT, int U>
__global__ void __launch_bounds__(kRowThreads) tli_rows_mask_kernel(const __grid_constant__ RowsParams P) {
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

struct RowsLayout { int U, nstrip, coarse, listcap; size_t gmax, ssum, border, plan, todo, lists, total; };

// Groups of 8 vectors; of 4 and 2 where a row has at most 8192 and 4096 vectors, so that a short row still has enough groups for a
// top-k of a few hundred (or thousand: 64 bf16 rows of 32 000, top-k 1000 with top-p .99: 45 us against 59 with groups of 8 and, before
// lists were as long, 319 of 4) and the scan enough strips for the SMs (4.8 us against 6.1 with groups of 8).
RowsLayout rows_layout(long long rows, int V, int dtype) {
    RowsLayout L;
    const int nvec = chunks_per_row(V, dtype, 1);
    L.U = nvec <= 4096 ? 2 : nvec <= 8192 ? 4 : 8;
    L.nstrip = (nvec + 32 * L.U - 1) / (32 * L.U);
    L.coarse = (L.nstrip * 32 + kMaxGroups - 1) / kMaxGroups;
    const size_t elt = dtype == TLI_F32 ? 4 : 2;
    size_t off = 0;
    L.gmax = off; off = align_up(off + elt * rows * L.nstrip * 32, 256);
    L.ssum = off; off = align_up(off + sizeof(StripSum) * rows * L.nstrip, 256);
    L.border = off; off = align_up(off + sizeof(RowBorder) * rows, 256);
    L.plan = off; off = align_up(off + sizeof(RowPlan) * rows, 256);
    L.todo = off; off = align_up(off + sizeof(int) * (rows + 2), 256);
    // Bracketed elements of a row: a sample of 8192 puts the border within about V/50 of them, in 16 bits the ties at the bracket's
    // ends come along, and a top-k of thousands with top-p wants them all.  (V/20: 64 bf16 rows of 32 000, top-k 2500 to 5000 with
    // top-p, went through digits in 257 to 290 us against 79 to 119; where the list was long enough both are alike.)
    L.listcap = V <= kListCap ? 0 : std::min(kSpreadCap, std::max(2048, V / 4));
    L.lists = off; off = align_up(off + sizeof(unsigned long long) * rows * L.listcap, 256);
    L.total = off;
    return L;
}

size_t rows_workspace(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side) {
    if (!ctx || ctx->n_shards != 1 || B < 1 || R < 1 || static_cast<long long>(B) * R > TLI_MAX_B) return 0;
    if (dtype != TLI_F32 && dtype != TLI_BF16) return 0;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return 0;
    return rows_layout(static_cast<long long>(B) * R, side == TLI_SIDE_TARGET ? ctx->V_t : ctx->V_d, dtype).total;
}

// Raises a kernel's limit of dynamic shared memory once per device.
struct SmemAllowed {
    std::atomic<unsigned long long> devices{0};
    cudaError_t set(const void *fn, size_t bytes, int device) {
        const unsigned long long bit = device < 64 ? 1ull << device : 0ull;        // (beyond: every time)
        if (devices.load(std::memory_order_acquire) & bit) return cudaSuccess;
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
        if (e == cudaSuccess) devices.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

template <int DT, int U> int launch_rows(const RowsParams &P, int device, int num_sms, cudaStream_t stream) {
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
    const size_t smem = pick_smem_bytes(P.nstrip, (P.nstrip + P.coarse - 1) / P.coarse * 32);
    static SmemAllowed allowed, allowed_spread;
    e = allowed.set(reinterpret_cast<const void *>(tli_rows_pick_kernel<DT>), kPickSmemMax, device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
    cfg.gridDim = dim3(rows); cfg.blockDim = dim3(kPickThreads); cfg.dynamicSmemBytes = smem;
    e = cudaLaunchKernelEx(&cfg, tli_rows_pick_kernel<DT>, P);
    if (e != cudaSuccess) return cuda_fail(e, "launch tli_rows_pick_kernel");
    if (P.listcap > 0 && (P.top_k || P.top_p || P.min_p)) {        // (short rows and unfiltered ones are done)
        e = allowed_spread.set(reinterpret_cast<const void *>(tli_rows_spread_kernel<DT, U>), kSettleSmemMax, device);
        if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute");
        const long long blocks = static_cast<long long>(rows) * ((P.nstrip + kPickWarps - 1) / kPickWarps);
        cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>(blocks, 2LL * num_sms))); cfg.blockDim = dim3(kPickThreads);
        cfg.dynamicSmemBytes = settle_smem_bytes(P.nstrip);
        e = cudaLaunchKernelEx(&cfg, tli_rows_spread_kernel<DT, U>, P);
        if (e != cudaSuccess) return cuda_fail(e, "launch tli_rows_spread_kernel");
    }
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
    P.nstrip = L.nstrip; P.coarse = L.coarse; P.ulog = L.U == 2 ? 1 : L.U == 4 ? 2 : 3;
    P.gmax = ws + L.gmax;
    P.ssum = reinterpret_cast<StripSum *>(ws + L.ssum);
    P.border = reinterpret_cast<RowBorder *>(ws + L.border);
    P.plan = reinterpret_cast<RowPlan *>(ws + L.plan);
    P.todo = reinterpret_cast<int *>(ws + L.todo);
    P.lists = reinterpret_cast<unsigned long long *>(ws + L.lists);
    P.listcap = L.listcap;
#define TLI_ROWS(U) (dtype == TLI_F32 ? launch_rows<TLI_F32, U>(P, ctx->device, ctx->num_sms, stream) \
                                     : launch_rows<TLI_BF16, U>(P, ctx->device, ctx->num_sms, stream))
    return L.U == 2 ? TLI_ROWS(2) : L.U == 4 ? TLI_ROWS(4) : TLI_ROWS(8);
#undef TLI_ROWS
}

// The context's device is the current one (a launch elsewhere would read this device's pointers there).
bool on_device(const tli_ctx *ctx) {
    int current = -1;
    return cudaGetDevice(&current) == cudaSuccess && current == ctx->device;
}
bool aligned4(std::initializer_list<const void *> pointers) {
    uintptr_t bits = 0;
    for (const void *p : pointers) bits |= reinterpret_cast<uintptr_t>(p);
    return bits % 4 == 0;
}
// Whether rows of V elements written at `out` meet any read at `in` other than themselves.
bool rows_collide(const char *in, int64_t sb, int64_t sr, const char *out, int64_t ob, int64_t orr, int64_t B, int64_t R, int64_t V, int64_t elt) {
    if (B == 1) sb = ob = 0;
    if (R == 1) sr = orr = 0;
    if (in == out && sb == ob && sr == orr) return false;          // in place
    const int64_t in_span = ((B - 1) * sb + (R - 1) * sr + V) * elt, out_span = ((B - 1) * ob + (R - 1) * orr + V) * elt;
    if (out + out_span <= in || in + in_span <= out) return false;
    // rows of one pitch can lie in one another's gaps
    if (sb != ob || sr != orr) return true;
    const int64_t pitch = sr == 0 ? sb : sb == 0 ? sr : std::min(sb, sr), apart = (out > in ? out - in : in - out);
    if (pitch == 0 || sb % pitch || sr % pitch || apart % elt) return true;
    const int64_t gap = apart / elt % pitch;
    return gap < V || gap > pitch - V;
}

// What tli_sample() and tli_filter() check alike.
int check_rows(const tli_ctx *ctx, int32_t B, int32_t R, int32_t dtype, int32_t side, const void *logits, int64_t sb, int64_t sr,
               const float *tau, const void *workspace, size_t workspace_bytes) {
    if (!ctx || ctx->n_shards != 1 || B < 1 || R < 1) return TLI_ERR_ARG;
    if (static_cast<long long>(B) * R > TLI_MAX_B) return TLI_ERR_UNSUPPORTED;
    if (dtype != TLI_F32 && dtype != TLI_BF16) return TLI_ERR_ARG;
    if (side != TLI_SIDE_TARGET && side != TLI_SIDE_DRAFTER) return TLI_ERR_ARG;
    if (!logits || !tau || !on_device(ctx)) return TLI_ERR_ARG;
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
    if (!aligned4({a->temperature, a->top_k, a->top_p, a->min_p, a->uniforms, a->tokens, a->prob, a->status})) return TLI_ERR_ARG;
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
    if (!aligned4({a->temperature, a->top_k, a->top_p, a->min_p, a->status})) return TLI_ERR_ARG;
    if (rows_collide(reinterpret_cast<const char *>(a->logits), a->stride_b, a->stride_r, reinterpret_cast<const char *>(a->out), ob, orr, a->B, a->R, V,
                     static_cast<int64_t>(elt))) return TLI_ERR_ARG;
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
