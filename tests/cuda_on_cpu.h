// The CUDA constructs that the row kernels use, on one CPU thread: a block is a set of fibers, one per thread, that run from one
// collective (barrier, shuffle, ballot, reduction) to the next.  Between two of them the threads run one after the other in an order
// that the caller picks, so that whatever two threads do to one word without a collective in between happens in either order.  A block
// whose threads wait at different collectives, or for a thread that has left, ends with a message instead of hanging.
#pragma once
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <vector>
#include <ucontext.h>

// ---- fibers ----

struct Dim3 { unsigned x, y, z; };
static Dim3 threadIdx, blockIdx, gridDim, blockDim;

namespace emu {
enum { READY, AT_BARRIER, AT_WARP, DONE };
struct Fiber { ucontext_t ctx; char *stack; int state, line; unsigned long long put; };
static std::vector<Fiber> fibers;
static ucontext_t scheduler;
static std::function<void()> body;
static int current, order, block_count;
static unsigned long long warp_put[64][32];
static char message[256];
static unsigned long long random_state;
constexpr size_t kStack = 96 * 1024;

static unsigned next_random() {
    random_state = random_state * 6364136223846793005ull + 1442695040888963407ull;
    return static_cast<unsigned>(random_state >> 33);
}
static void yield(int state, int line, unsigned long long put) {
    Fiber &f = fibers[current];
    f.state = state; f.line = line; f.put = put;
    swapcontext(&f.ctx, &scheduler);
}
static void enter() {
    body();
    fibers[current].state = DONE;
    swapcontext(&fibers[current].ctx, &scheduler);
}
// orders: 0 ascending, 1 descending, 2 any thread at any time, 3 a warp that runs last, 4 one that runs first, 5 one thread that runs last
static int pick(const std::vector<int> &ready, int favourite) {
    const int n = static_cast<int>(ready.size());
    if (order == 0) return ready[0];
    if (order == 1) return ready[n - 1];
    if (order == 2) return ready[next_random() % n];
    int other = -1;
    for (int t : ready) {
        const bool chosen = order == 5 ? t == favourite : t / 32 == favourite;
        if (order == 4 && chosen) return t;
        if (!chosen) { other = t; break; }
    }
    return other >= 0 ? other : ready[0];
}
// One block of n threads; false (and a message) if it cannot end.
static bool run_block(int n, int order_, unsigned seed, const std::function<void()> &f) {
    order = order_; random_state = seed * 2654435761u + 12345u; body = f;
    next_random();
    while (static_cast<int>(fibers.size()) < n) {
        Fiber x{};
        x.stack = static_cast<char *>(malloc(kStack));
        fibers.push_back(x);
    }
    for (int t = 0; t < n; ++t) {
        Fiber &x = fibers[t];
        getcontext(&x.ctx);
        x.ctx.uc_stack.ss_sp = x.stack; x.ctx.uc_stack.ss_size = kStack; x.ctx.uc_link = nullptr;
        makecontext(&x.ctx, enter, 0);
        x.state = READY;
    }
    const int favourite = static_cast<int>(next_random() % (order_ == 5 ? n : n / 32));
    std::vector<int> ready;
    for (;;) {
        // whole warps that wait at one collective go on
        for (int w = 0; w < n / 32; ++w) {
            bool all = true;
            for (int l = 0; l < 32; ++l) all = all && fibers[w * 32 + l].state == AT_WARP;
            if (!all) continue;
            for (int l = 0; l < 32; ++l) {
                Fiber &x = fibers[w * 32 + l];
                if (x.line != fibers[w * 32].line) {
                    snprintf(message, sizeof message, "lanes of warp %d meet at lines %d and %d", w, fibers[w * 32].line, x.line);
                    return false;
                }
                warp_put[w][l] = x.put;
                x.state = READY;
            }
        }
        ready.clear();
        int barrier = 0, done = 0, line = -1, line2 = -1;
        for (int t = 0; t < n; ++t) {
            const Fiber &x = fibers[t];
            if (x.state == READY) ready.push_back(t);
            else if (x.state == DONE) ++done;
            else if (x.state == AT_BARRIER) { ++barrier; if (line < 0) line = x.line; else if (line != x.line) line2 = x.line; }
        }
        if (ready.empty()) {
            if (done == n) return true;
            if (barrier < n || line2 >= 0) {
                snprintf(message, sizeof message, "%d threads at barriers (lines %d, %d), %d left, %d inside a warp's collective", barrier, line, line2, done,
                         n - barrier - done);
                return false;
            }
            block_count = 0;
            for (int t = 0; t < n; ++t) { block_count += fibers[t].put != 0; fibers[t].state = READY; }
            continue;
        }
        // the chosen ones of this round, until no more of them can run
        while (!ready.empty()) {
            const int t = pick(ready, favourite);
            current = t;
            threadIdx = {static_cast<unsigned>(t), 0, 0};
            swapcontext(&scheduler, &fibers[t].ctx);
            for (size_t i = 0; i < ready.size(); ++i)
                if (ready[i] == t) { ready.erase(ready.begin() + i); break; }
            if (fibers[t].state != AT_WARP) continue;
            bool all = true;                                       // the last lane of a warp's collective: the warp may go on at once
            for (int l = 0; l < 32; ++l) all = all && fibers[t / 32 * 32 + l].state == AT_WARP;
            if (all) break;
        }
    }
}
template <typename T> static unsigned long long as_bits(T x) {
    unsigned long long b = 0;
    static_assert(sizeof(T) <= 8, "a word");
    memcpy(&b, &x, sizeof x);
    return b;
}
template <typename T> static T from_bits(unsigned long long b) {
    T x;
    memcpy(&x, &b, sizeof x);
    return x;
}
template <typename T> static unsigned long long *exchange(T x, int line) {
    yield(AT_WARP, line, as_bits(x));
    return warp_put[threadIdx.x / 32];
}
static int barrier(int line, int put) {
    yield(AT_BARRIER, line, put != 0);
    return block_count;
}
template <typename T> static T shuffle_up(T x, int o, int line) {
    const unsigned long long *w = exchange(x, line);
    const int lane = threadIdx.x % 32;
    return from_bits<T>(w[lane >= o ? lane - o : lane]);
}
template <typename T> static T shuffle_xor(T x, int o, int line) { const unsigned long long *w = exchange(x, line); return from_bits<T>(w[(threadIdx.x % 32) ^ o]); }
template <typename T> static T shuffle(T x, int from, int line) { return from_bits<T>(exchange(x, line)[from]); }
static unsigned ballot(bool p, int line) {
    const unsigned long long *w = exchange(static_cast<int>(p), line);
    unsigned r = 0;
    for (int l = 0; l < 32; ++l) r |= w[l] ? 1u << l : 0u;
    return r;
}
static int reduce_max(int x, int line) {
    const unsigned long long *w = exchange(x, line);
    int r = INT_MIN;
    for (int l = 0; l < 32; ++l) { const int y = from_bits<int>(w[l]); r = y > r ? y : r; }
    return r;
}
static int reduce_add(int x, int line) {
    const unsigned long long *w = exchange(x, line);
    unsigned r = 0;
    for (int l = 0; l < 32; ++l) r += from_bits<unsigned>(w[l]);
    return static_cast<int>(r);
}
}  // namespace emu

#define __syncthreads() emu::barrier(__LINE__, 0)
#define __syncthreads_count(p) emu::barrier(__LINE__, p)
#define __syncwarp() emu::exchange(0, __LINE__)
#define __shfl_up_sync(m, x, o) emu::shuffle_up(x, o, __LINE__)
#define __shfl_xor_sync(m, x, o) emu::shuffle_xor(x, o, __LINE__)
#define __shfl_sync(m, x, from) emu::shuffle(x, from, __LINE__)
#define __ballot_sync(m, p) emu::ballot(p, __LINE__)
#define __any_sync(m, p) (emu::ballot(p, __LINE__) != 0)
#define __reduce_max_sync(m, x) emu::reduce_max(x, __LINE__)
#define __reduce_add_sync(m, x) emu::reduce_add(x, __LINE__)

// ---- types, memory, arithmetic ----

#define __device__
#define __global__ static
#define __shared__ static
#define __forceinline__ inline
#define __noinline__ __attribute__((noinline))
#define __launch_bounds__(...)
#define __grid_constant__
#define __align__(n) __attribute__((aligned(n)))

struct __align__(16) uint4 { unsigned x, y, z, w; };
struct __align__(16) int4 { int x, y, z, w; };
struct __align__(16) double2 { double x, y; };
static inline uint4 make_uint4(unsigned x, unsigned y, unsigned z, unsigned w) { uint4 r = {x, y, z, w}; return r; }
template <typename T> static inline T __ldg(const T *p) { return *p; }
template <typename T> static inline T __ldcg(const T *p) { return *p; }
template <typename T> static inline void __stcg(T *p, T x) { *p = x; }
template <typename T, typename U> static inline T atomicAdd(T *p, U x) { const T old = *p; *p = old + static_cast<T>(x); return old; }
static inline void __threadfence() {}

template <typename T> static inline T min(T a, T b) { return b < a ? b : a; }
template <typename T> static inline T max(T a, T b) { return a < b ? b : a; }
static inline unsigned __float_as_uint(float x) { return emu::from_bits<unsigned>(emu::as_bits(x)); }
static inline float __uint_as_float(unsigned x) { return emu::from_bits<float>(x); }
static inline int __float_as_int(float x) { return static_cast<int>(__float_as_uint(x)); }
static inline float __int_as_float(int x) { return __uint_as_float(static_cast<unsigned>(x)); }
static inline int __double2hiint(double x) { return static_cast<int>(emu::as_bits(x) >> 32); }
static inline int __double2loint(double x) { return static_cast<int>(emu::as_bits(x)); }
static inline double __hiloint2double(int hi, int lo) { return emu::from_bits<double>(static_cast<unsigned long long>(static_cast<unsigned>(hi)) << 32 | static_cast<unsigned>(lo)); }
static inline long long __double_as_longlong(double x) { return static_cast<long long>(emu::as_bits(x)); }
static inline double __longlong_as_double(long long x) { return emu::from_bits<double>(static_cast<unsigned long long>(x)); }
static inline unsigned long long __double2ull_rn(double x) { return x > 0 ? static_cast<unsigned long long>(nearbyint(x)) : 0ull; }
static inline unsigned __float2uint_rn(float x) { return x > 0 ? static_cast<unsigned>(nearbyintf(x)) : 0u; }
static inline float __double2float_ru(double x) {
    const float f = static_cast<float>(x);
    return static_cast<double>(f) < x ? nextafterf(f, INFINITY) : f;
}
static inline int __popc(unsigned x) { return __builtin_popcount(x); }
static inline int __ffs(unsigned x) { return __builtin_ffs(static_cast<int>(x)); }
static inline int __clzll(unsigned long long x) { return x ? __builtin_clzll(x) : 64; }
static inline uint32_t __funnelshift_r(uint32_t lo, uint32_t hi, unsigned s) { return static_cast<uint32_t>((static_cast<uint64_t>(hi) << 32 | lo) >> (s & 31)); }

struct __nv_bfloat16 { unsigned short x; };
struct __nv_bfloat162 { __nv_bfloat16 x, y; };
static inline float __bfloat162float(__nv_bfloat16 h) { return __uint_as_float(static_cast<unsigned>(h.x) << 16); }
static inline __nv_bfloat16 bf16_towards(float f, bool up) {
    unsigned u = __float_as_uint(f);
    const bool cut = (u & 0xffffu) && f == f, away = up ? f > 0 : f < 0;
    u &= 0xffff0000u;
    if (cut && away) u += 0x10000u;
    return {static_cast<unsigned short>(u >> 16)};
}
static inline __nv_bfloat16 __float2bfloat16_ru(float f) { return bf16_towards(f, true); }
static inline __nv_bfloat16 __float2bfloat16_rd(float f) { return bf16_towards(f, false); }
static inline __nv_bfloat162 __bfloat162bfloat162(__nv_bfloat16 h) { return {h, h}; }
static inline unsigned __hge2_mask(__nv_bfloat162 a, __nv_bfloat162 b) {
    return (__bfloat162float(a.x) >= __bfloat162float(b.x) ? 0xffffu : 0u) | (__bfloat162float(a.y) >= __bfloat162float(b.y) ? 0xffff0000u : 0u);
}
