// cci_logprobs.cu -- log probabilities of given tokens, entropy and top alternatives of rows
// of logits, and the gradient of the first two.
//
// Row of V logits x, m = max x, e_v = exp(x_v - m), s = sum e_v:
//   logp    = x_t - m - log s                         (t: the row's token)
//   entropy = log s - sum e_v (x_v - m) / s           (a masked logit, -inf, adds nothing)
//   top     = the k largest logits with their log probabilities, ties to the lower index
//   dx_v    = dlogp (1[v = t] - p_v) - dentropy p_v (log p_v + entropy),  p_v = e_v / s
//
// Memory bound: one read of the logits forward, one read and one write backward.  The forward
// pass keeps the running maximum m, s and t = sum e_v (x_v - m) per thread and rescales them when the
// maximum moves, in base 2: y = (x - m) log2(e).  The difference comes first: it is exact or
// nearly so near the maximum whatever the logits' offset, and x log2(e) would overflow for logits
// at the type's lowest value.  What is subtracted is never below a logit, so no exponential is above 1 and every term
// of t is at most 0: nothing cancels, s of a row is at least 1, its logarithm and the entropy at least 0.
//
// Top alternatives: the pass notes the maximum of every run of 512 consecutive logits (32 to 128 in rows of
// up to 16384), which costs it one warp reduction.  Of the runs, ordered by maximum and then position,
// only the first k can hold one of the k largest logits: every other run has k maxima ahead of all it
// holds, and runs in order keep ties to the lower index.  Those k runs are read again (from L2)
// for the logits that reach the k-th run's maximum, about k of them; they are put in order by
// counting, for each, the ones above it.  Of the run of rank r no more than k - r logits count, so of those
// equal to that maximum the first k - r are taken; where logits rise and too many are above it, a
// warp draws a run's best k - r one by one.  So the cost has a bound whatever the logits.  Parts of a row of more than
// 262144 logits (64 runs a warp) rank every run against every other, in time that grows with the square of the part:
// 305 x 300001 bf16 55 us without alternatives and 102 with 5, 305 x 2^20 166 and 638, 1 x 2^24 129 and 783.
//
// Rows of up to 1024 logits take a warp each and stay in its registers.  Longer ones take one warp, four or eight,
// or, where the rows alone would not fill the SMs, a cluster of 2, 4 or 8 blocks that each read a
// part of the row and join in the first block's shared memory.
#include <cooperative_groups.h>

#include <type_traits>

#include "cci_kernels.h"
#include "cci_rowops.cuh"

namespace cci {
namespace lp {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxTop = 32;  // a warp's lanes
// shared memory for the runs' maxima: 2^24 logits in one block have 32768 runs
constexpr int kMaxMaxima = 160 * 1024;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// order of a logit among all (a larger key ranks first): its fp32 bits made monotonic, then the
// inverted index.  -0 is +0; NaN is never asked
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (static_cast<uint64_t>(o) << 32) | ~index;
}

__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t o = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ uint32_t index_of(uint64_t key) { return ~static_cast<uint32_t>(key); }

// running sums of a part of a row: maximum (or reference) m, s = sum 2^y, t = sum 2^y y with y = (x - m) log2(e).
// Nothing seen yet, or only -inf: m = -inf, s = t = 0
struct Sums {
    float m, s, t;
};

// what is subtracted: -inf - -inf would be NaN
__device__ __forceinline__ float ref_of(float m) { return m == neg_inf() ? 0.f : m; }

// the sums under a larger (or the same) maximum
__device__ __forceinline__ Sums moved(Sums a, float m)
{
    if (m == a.m || a.s == 0.f) return Sums{m, a.s, a.t};
    const float d = (ref_of(a.m) - ref_of(m)) * kLog2e;
    if (!(d > -150.f)) return Sums{m, isnan(a.s) ? a.s : 0.f, 0.f};  // below every fp32; NaN stays
    const float f = ex2(d);
    return Sums{m, a.s * f, (a.t + d * a.s) * f};
}

__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    a = moved(a, m);
    b = moved(b, m);
    return Sums{m, a.s + b.s, a.t + b.t};
}

__device__ __forceinline__ Sums warp_joined(Sums a)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
        b.t = __shfl_xor_sync(0xffffffffu, a.t, o);
        a = joined(a, b);
    }
    return a;
}

using row::add2;
using row::mul2;

// the larger; NaN if either is
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// a thread's running sums in four independent parts, two of each pair, against a reference m that is at least its
// maximum: that of all that its warp has seen (rows in one warp's registers: its own), so that the lanes move
// their sums together, and seldom (a row of 131072 logits over four warps: about five times).  Moved at every maximum
// of its own, a lane would hold up its warp in nearly every iteration
struct Running {
    float m;
    unsigned long long s[2], t[2];
};

__device__ __forceinline__ Sums sums_of(const Running &a)
{
    const unsigned long long s = add2(a.s[0], a.s[1]), t = add2(a.t[0], a.t[1]);
    return Sums{a.m, lo_of(s) + hi_of(s), lo_of(t) + hi_of(t)};
}

// the sums ready for elements of up to `top`
__device__ __forceinline__ void raise_to(Running &a, float top)
{
    if (top > a.m) {
        const Sums s = moved(sums_of(a), top);
        a = Running{top, {pack2(s.s, 0.f), 0ull}, {pack2(s.t, 0.f), 0ull}};
    }
}

// a logit below which nothing is left of exp(x - m) in fp32, but whose difference from m is finite.  None does
// for maxima next to the type's lowest value: -inf there
__device__ __forceinline__ float floor_of(float m)
{
    return ref_of(m) - fmaxf(140.f, fabsf(ref_of(m)) * 0.03f);
}

// adds n elements of at most a.m to the sums.  CLAMPED: none is below floor_of(a.m), which is finite
template <bool CLAMPED, int n>
__device__ __forceinline__ void add(Running &a, const float (&x)[n])
{
    const float m = ref_of(a.m);
    const unsigned long long neg = pack2(-m, -m), c = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
        unsigned long long y = mul2(add2(pack2(x[2 * i], x[2 * i + 1]), neg), c);
        // 2^-200 is 0, and 0 times it is no NaN, as 0 times -inf would be
        if constexpr (!CLAMPED) y = pack2(max_nan(lo_of(y), -200.f), max_nan(hi_of(y), -200.f));
        const unsigned long long e = pack2(ex2(lo_of(y)), ex2(hi_of(y)));
        a.s[i & 1] = add2(a.s[i & 1], e);
        ffma2(a.t[i & 1], e, y);
    }
}

// one element more
__device__ __forceinline__ void add1(Running &a, float x)
{
    const float f[2] = {x, neg_inf()};
    raise_to(a, fmaxf(x, neg_inf()));
    add<false>(a, f);
}

using row::warp_max;

// the lanes' largest (no NaN among them), in one instruction
__device__ __forceinline__ float lanes_max(float v)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

struct Row {
    const int64_t *tokens;
    int64_t ignore;
    float *logp, *entropy, *stats;
    float *top_logp;
    int32_t *top_idx;
    int k;
    uint32_t *status;
};

// what a row's sums say, once it has them all (one thread)
struct Result {
    float m, log_s;  // log of the sum of exp(x - m)
    bool empty;      // nothing but -inf
};

__device__ __forceinline__ Result finish(const Sums &a)
{
    Result r;
    r.empty = a.m == neg_inf() && a.s == 0.f;
    r.m = ref_of(a.m);
    r.log_s = r.empty ? 0.f : logf(a.s);
    return r;
}

__device__ __forceinline__ float logp_of(const Result &r, float x) { return r.empty ? neg_inf() : x - r.m - r.log_s; }

template <typename T>
__device__ __forceinline__ void write_row(const Row &o, int64_t n, const T *x, int64_t V, const Sums &a, const Result &r)
{
    const int64_t token = o.tokens[n];
    float lp = 0.f;
    if (token != o.ignore) {
        if (token >= 0 && token < V) {
            lp = logp_of(r, row::to_f32(x[token]));
        } else {
            report(o.status, CCI_ERR_INDEX);
            lp = __int_as_float(0x7fc00000);
        }
    }
    o.logp[n] = lp;
    o.entropy[n] = r.empty ? 0.f : r.log_s - a.t / a.s * kLn2;
    o.stats[2 * n] = a.m;
    o.stats[2 * n + 1] = r.log_s;
}

// place `rank` of the row's list: the entry of that key (0: none, where the row has fewer numbers)
__device__ __forceinline__ void write_top(const Row &o, int64_t n, int rank, uint64_t key, const Result &r)
{
    o.top_idx[n * o.k + rank] = key ? static_cast<int32_t>(index_of(key)) : -1;
    o.top_logp[n * o.k + rank] = key ? logp_of(r, logit_of(key)) : __int_as_float(0x7fc00000);
}

// the lanes' largest key
__device__ __forceinline__ uint64_t warp_best(uint64_t key)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, key, o);
        key = other > key ? other : key;
    }
    return key;
}

// how many of the first c keys of a list in shared memory (16-byte aligned, a zero past an odd end) are above
// `mine`: two a load, eight loads on their way
__device__ __forceinline__ int count_above(const uint64_t *list, int c, uint64_t mine)
{
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < c; j += 2) {
        const ulonglong2 q = *reinterpret_cast<const ulonglong2 *>(list + j);
        above += (q.x > mine) + (q.y > mine);
    }
    return above;
}

// ---- rows of up to 1024 logits: a warp each ----
constexpr int kShortList = 128;

template <typename T, int E, bool TOP>
__global__ void __launch_bounds__(256) short_kernel(const T *x, int64_t ldx, int64_t N, int V, Row o)
{
    __shared__ __align__(16) uint64_t lists[TOP ? 8 : 1][kShortList];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + warp;
    if (n >= N) return;
    const T *xr = x + n * ldx;
    float f[E];
    float top = neg_inf();
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = lane + 32 * i < V ? row::to_f32(xr[lane + 32 * i]) : neg_inf();
#pragma unroll
    for (int i = 0; i < E; ++i) top = fmaxf(top, f[i]);
    Running run{neg_inf(), {0ull, 0ull}, {0ull, 0ull}};
    raise_to(run, top);
    add<false>(run, f);
    const Sums a = moved(warp_joined(sums_of(run)), warp_max(top));
    const Result r = finish(a);
    if (lane == 0) write_row(o, n, xr, V, a, r);
    if constexpr (TOP) {
        // the k-th largest of the lanes' maxima: k elements reach it
        int above = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float other = __shfl_sync(0xffffffffu, top, j);
            above += other > top || (other == top && j < lane);
        }
        const uint32_t at = __ballot_sync(0xffffffffu, above == o.k - 1);
        const float bar = __shfl_sync(0xffffffffu, top, __ffs(at) - 1);  // maxima are no NaN
        auto reaches = [&](int i) { return f[i] >= bar && lane + 32 * i < V; };
        auto key_at = [&](int i) { return key_of(f[i], static_cast<uint32_t>(lane + 32 * i)); };
        int have = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) have += reaches(i);
        // places in the list: those of the lanes before
        int off = have;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, off, s);
            if (lane >= s) off += v;
        }
        const int c = __shfl_sync(0xffffffffu, off, 31);
        off -= have;
        if (c <= kShortList) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (reaches(i)) lists[warp][off++] = key_at(i);
            if (lane == 0 && (c & 1)) lists[warp][c] = 0ull;
            __syncwarp();
            for (int i = lane; i < c; i += 32) {
                const uint64_t mine = lists[warp][i];
                const int rank = count_above(lists[warp], c, mine);
                if (rank < o.k) write_top(o, n, rank, mine, r);
            }
            for (int i = c + lane; i < o.k; i += 32) write_top(o, n, i, 0ull, r);
        } else {
            // k times the best key below the last one
            uint64_t last = ~0ull;
            for (int k = 0; k < o.k; ++k) {
                uint64_t best = 0;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const uint64_t key = reaches(i) ? key_at(i) : 0ull;
                    if (key < last && key > best) best = key;
                }
                last = warp_best(best);
                if (lane == 0) write_top(o, n, k, last, r);
            }
        }
    }
}

// ---- longer rows: a block, or a cluster of `parts` of them ----
// logits that reach the k-th run's maximum: as many as the runs give when drawn one by one, at least
constexpr int kList = kMaxTop * (kMaxTop + 1) / 2 + 48;
static_assert(kList % 2 == 0, "read in pairs");

template <int kWarps>
struct Shared {
    alignas(16) uint64_t list[kList];
    alignas(16) uint64_t best[kWarps * kMaxTop];        // each warp's first k runs: maximum, inverted slot
    alignas(16) uint64_t join[kWarps < 8 ? kMaxTop : 8 * kMaxTop];  // first block of a cluster: the parts' lists
    Sums part[8];                                   // and their sums
    Sums warp[kWarps];
    int run[kMaxTop];  // the k first runs: warp << 16 | slot (of 4096 at most), -1 past the last
    uint32_t bar;      // order of the k-th run's maximum (0: fewer runs)
    int count;
    Result result;
};

// order of a logit alone (NaN is not asked)
__device__ __forceinline__ uint32_t order_of(float x) { return static_cast<uint32_t>(key_of(x, 0u) >> 32); }

// largest of the elements of a load.  bf16 pairs are compared as they are
template <typename T, int V>
__device__ __forceinline__ float raw_max(const row::Raw<T, V> &r, const float *f)
{
    if constexpr (sizeof(T) == 4) {
        float m = f[0];
#pragma unroll
        for (int j = 1; j < V; ++j) m = fmaxf(m, f[j]);
        return m;
    } else {
        uint32_t m = r.w[0].x;
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[0].y));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[0].z));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[0].w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
}

// the elements of a load as fp32; bf16 ones that lie below `low` (two bf16) raised to it, NaN kept
template <typename T, int V>
__device__ __forceinline__ void unpack_floored(row::Raw<T, V> r, uint32_t low, float *f)
{
    if constexpr (sizeof(T) == 2) {
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[0].x) : "r"(low));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[0].y) : "r"(low));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[0].z) : "r"(low));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[0].w) : "r"(low));
    }
    row::unpack<T, V>(r, f);
}

// whether a load holds a number (not NaN alone)
template <typename T, int V>
__device__ __forceinline__ bool has_number(const row::Raw<T, V> &r)
{
    float f[V];
    row::unpack<T, V>(r, f);
    bool any = false;
#pragma unroll
    for (int j = 0; j < V; ++j) any |= f[j] == f[j];
    return any;
}

// RUN: logits of a run (512: an iteration of a warp; fewer: a part of one load of it)
template <typename T, int kThreads, int RUN, bool TOP>
__global__ void __launch_bounds__(kThreads, kThreads == 32 ? 28 : 1024 / kThreads)
    row_kernel(const T *x, int64_t ldx, int V, Row o, int parts, int run_slots)
{
    constexpr int kV = 16 / sizeof(T), kE = 16, kU = kE / kV;  // elements of a load, of an iteration; loads of one
    constexpr int kWarps = kThreads / 32, kIter = 32 * kU;     // words of a warp's iteration
    constexpr int kRunWords = RUN / kV, kGroup = RUN == 512 ? 32 : kRunWords;  // lanes of a run
    __shared__ Shared<kWarps> sh;
    extern __shared__ __align__(16) uint32_t maxima[];  // [kWarps][run_slots], 0: no such run
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = static_cast<int>(blockIdx.x) % parts;
    const int64_t n = blockIdx.x / parts;
    const T *xr = x + n * ldx;
    // a head of single elements up to the first 16-byte word (first part), whole words, a tail (last part)
    const int to_word = static_cast<int>((16 - reinterpret_cast<uintptr_t>(xr) % 16) % 16 / sizeof(T));
    const int head = to_word < V ? to_word : V, words = (V - head) / kV;
    const int w0 = static_cast<int>(static_cast<int64_t>(words) * rank / parts);
    const int nw = static_cast<int>(static_cast<int64_t>(words) * (rank + 1) / parts) - w0;
    // consecutive words for every warp: the same number of whole iterations, the last ones fewer
    const int per_warp = ((nw + kWarps - 1) / kWarps + kIter - 1) / kIter * kIter;
    auto first_word = [&](int q) { return w0 + (q * per_warp < nw ? q * per_warp : nw); };
    const int ws = first_word(warp), we = first_word(warp + 1);
    const T *xw = xr + head;
    uint32_t *own = maxima + warp * run_slots;
    if constexpr (TOP) {
        for (int i = lane; i < run_slots; i += 32) own[i] = 0u;
        if (tid < kMaxTop) sh.run[tid] = -1;
        if (tid == 0) {
            sh.bar = 0u;
            sh.count = 0;
        }
        __syncwarp();
    }
    if (parts > 1) cg::this_cluster().barrier_arrive();  // the wait for it: every block of the cluster runs
    Running a{neg_inf(), {0ull, 0ull}, {0ull, 0ull}};
    row::Raw<T, kV> raw[kU];
    const T *next = xw + static_cast<int64_t>(ws + lane) * kV;  // this lane's words of the iteration to load
#pragma unroll
    for (int u = 0; u < kU; ++u)
        if (ws + u * 32 + lane < we) raw[u] = row::load_once<T, kV>(next + u * 32 * kV);
    // an iteration of the warp at word w; FULL: all of its words lie in the warp's share
    auto iteration = [&](int w, auto full) {
        constexpr bool FULL = decltype(full)::value;
        float f[kE];
        float top = neg_inf();
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const bool in = FULL || w + u * 32 + lane < we;
            float m = neg_inf();
            if (in) {
                if constexpr (sizeof(T) == 4) row::unpack<T, kV>(raw[u], f + u * kV);
                m = raw_max<T, kV>(raw[u], f + u * kV);
            } else {
#pragma unroll
                for (int j = 0; j < kV; ++j) f[u * kV + j] = neg_inf();
            }
            top = fmaxf(top, m);
            if constexpr (TOP && RUN != 512) {
                uint32_t q = in ? order_of(fmaxf(m, neg_inf())) : 0u;
                // a vote, so that the rare look at a load without a larger number is a branch
                if (__any_sync(0xffffffffu, in && !(m > neg_inf()))) q = in && has_number<T, kV>(raw[u]) ? q : 0u;
#pragma unroll
                for (int s = kGroup / 2; s > 0; s >>= 1) q = max(q, __shfl_xor_sync(0xffffffffu, q, s));
                if (lane % kGroup == 0) own[((w - ws) + u * 32 + lane) / kRunWords] = q;
            }
        }
        top = lanes_max(top);
        if constexpr (TOP && RUN == 512) {
            uint32_t q = order_of(top);
            if (!(top > neg_inf())) {  // the rare look at loads without a larger number
                bool any = false;
#pragma unroll
                for (int u = 0; u < kU; ++u) any |= (FULL || w + u * 32 + lane < we) && has_number<T, kV>(raw[u]);
                q = __any_sync(0xffffffffu, any) ? q : 0u;
            }
            if (lane == 0) own[(w - ws) / kIter] = q;
        }
        raise_to(a, top);
        // bf16: two elements at a time are raised to a floor, instead of one exponent at a time
        bool clamped = false;
        uint32_t low = 0u;
        if constexpr (sizeof(T) == 2) {
            const float fl = floor_of(a.m);
            low = row::bf16x2(fl, fl);
            clamped = FULL && fl > -3.38e38f;
            if (!clamped) low = 0xff80ff80u;  // -inf
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (FULL || w + u * 32 + lane < we) unpack_floored<T, kV>(raw[u], low, f + u * kV);
        }
        // the next iteration's loads
        next += kIter * kV;
#pragma unroll
        for (int u = 0; u < kU; ++u)
            if (w + kIter + u * 32 + lane < we) raw[u] = row::load_once<T, kV>(next + u * 32 * kV);
        if (clamped)
            add<true>(a, f);
        else
            add<false>(a, f);
    };
    int w = ws;
    for (; w + kIter <= we; w += kIter) iteration(w, std::true_type{});
    if (w < we) iteration(w, std::false_type{});
    // head and tail: fewer than 2 kV single elements, in the first warp
    float edge = neg_inf();
    int edge_at = -1;
    if (warp == 0) {
        const int tail0 = head + words * kV;
        if (rank == 0 && lane < head)
            edge_at = lane;
        else if (rank == parts - 1 && lane >= kV && lane - kV < V - tail0)
            edge_at = tail0 + lane - kV;
        if (edge_at >= 0) edge = row::to_f32(xr[edge_at]);
        add1(a, edge);
    }

    // the block's sums, to every thread of its first warp
    Sums sum = warp_joined(sums_of(a));
    if (lane == 0) sh.warp[warp] = sum;
    // each warp's first k runs, where its lanes hold two at most
    const bool few = run_slots <= 64;
    if constexpr (TOP) {
        if (few) {
            __syncwarp();
            uint64_t mine[2];
            int above[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at = lane + 32 * i;
                const uint32_t m = at < run_slots ? own[at] : 0u;
                mine[i] = m ? static_cast<uint64_t>(m) << 32 | static_cast<uint32_t>(~(warp << 16 | at)) : 0ull;
            }
            if (run_slots <= 32) {
#pragma unroll 4
                for (int j = 0; j < run_slots; ++j) above[0] += __shfl_sync(0xffffffffu, mine[0], j) > mine[0];
            } else {
#pragma unroll 4
                for (int j = 0; j < 32; ++j) {
                    const uint64_t p = __shfl_sync(0xffffffffu, mine[0], j), q = __shfl_sync(0xffffffffu, mine[1], j);
                    above[0] += (p > mine[0]) + (q > mine[0]);
                    above[1] += (p > mine[1]) + (q > mine[1]);
                }
            }
            uint64_t *best = sh.best + warp * o.k;
            if (lane < o.k) best[lane] = 0ull;
            if (warp == kWarps - 1 && lane == 0 && (kWarps * o.k & 1)) best[o.k] = 0ull;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (mine[i] && above[i] < o.k) best[above[i]] = mine[i];
        }
    }
    __syncthreads();
    if (warp == 0) sum = warp_joined(lane < kWarps ? sh.warp[lane] : Sums{neg_inf(), 0.f, 0.f});
    if (parts > 1) cg::this_cluster().barrier_wait();
    Shared<kWarps> *root = parts > 1 ? cg::this_cluster().map_shared_rank(&sh, 0) : &sh;
    if constexpr (TOP) {
        // the first k runs
        if (few) {
            const int c = kWarps * o.k;
            for (int i = tid; i < c; i += kThreads) {
                const uint64_t mine = sh.best[i];
                if (mine == 0ull) continue;
                const int above = count_above(sh.best, c, mine);
                if (above < o.k) {
                    sh.run[above] = static_cast<int>(~static_cast<uint32_t>(mine));
                    if (above == o.k - 1) sh.bar = static_cast<uint32_t>(mine >> 32);
                }
            }
        } else {
            const int slots = kWarps * run_slots;
            for (int i = tid; i < slots; i += kThreads) {
                const uint32_t mine = maxima[i];
                if (mine == 0u) continue;
                int above = 0;
                for (int j = 0; j < slots; j += 4) {
                    const uint4 other = *reinterpret_cast<const uint4 *>(maxima + j);
                    const uint32_t q[4] = {other.x, other.y, other.z, other.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) above += q[e] >= mine + (j + e < i ? 0u : 1u);
                }
                if (above < o.k) {
                    sh.run[above] = i / run_slots << 16 | i % run_slots;
                    if (above == o.k - 1) sh.bar = mine;
                }
            }
        }
        __syncthreads();
        const uint32_t bar = sh.bar;
        // element e of a run, as a key (0: none, or no number)
        auto run_key = [&](int run, int e) -> uint64_t {
            const int q = run >> 16, word = first_word(q) + (run & 0xffff) * kRunWords + e / kV;
            if (word >= first_word(q + 1)) return 0ull;
            const int at = head + word * kV + e % kV;
            const float v = row::to_f32(xr[at]);
            return v == v ? key_of(v, static_cast<uint32_t>(at)) : 0ull;
        };
        auto list = [&](uint64_t key) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < kList) sh.list[at] = key;
        };
        const uint64_t edge_key = edge_at >= 0 && edge == edge ? key_of(edge, static_cast<uint32_t>(edge_at)) : 0ull;
        if (edge_key) list(edge_key);
        // a warp reads one run of 32 words or more, or several shorter ones side by side
        constexpr int kSide = kRunWords < 32 ? 32 / kRunWords : 1, kPer = kRunWords < 32 ? 1 : kRunWords / 32;
        const float least = bar ? logit_of(static_cast<uint64_t>(bar) << 32) : neg_inf();
        constexpr int kLanes = kRunWords < 32 ? kRunWords : 32;  // of a run
        for (int r0 = warp * kSide; r0 < o.k; r0 += kWarps * kSide) {
            const int r = r0 + (kSide > 1 ? lane / kLanes : 0);
            const int run = r < o.k ? sh.run[r] : -1;
            const int q = run < 0 ? 0 : run >> 16;
            const int from = first_word(q) + (run & 0xffff) * kRunWords, to = run < 0 ? from : first_word(q + 1);
            row::Raw<T, kV> word[kPer];
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int at = from + u * 32 + lane % kLanes;
                if (at < to) word[u] = row::load<T, kV>(xw + static_cast<int64_t>(at) * kV);
            }
            int ties_left = o.k - r;  // of the run of rank r, the first k - r that equal the bar
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
                const int at = from + u * 32 + lane % kLanes;
                float v[kV];
                int ties = 0;
#pragma unroll
                for (int j = 0; j < kV; ++j) v[j] = __int_as_float(0x7fc00000);  // NaN is never listed
                float m = neg_inf();
                if (at < to) {
                    row::unpack<T, kV>(word[u], v);
                    m = raw_max<T, kV>(word[u], v);
                }
                // most loads hold none (8 x 131072 fp32, 20 alternatives: 12.4 us when every element is looked at, 11.8
                // so; many rows 1 % the other way)
                if (!__any_sync(0xffffffffu, at < to && m >= least)) continue;
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    ties += v[j] == least;
                    if (v[j] > least) list(key_of(v[j], static_cast<uint32_t>(head + at * kV + j)));
                }
                if (__any_sync(0xffffffffu, ties)) {
                    int upto = ties;  // ties of the run's lanes up to this one
#pragma unroll
                    for (int s = 1; s < kLanes; s <<= 1) {
                        const int before = __shfl_up_sync(0xffffffffu, upto, s, kLanes);
                        if (lane % kLanes >= s) upto += before;
                    }
                    int place = upto - ties;
#pragma unroll
                    for (int j = 0; j < kV; ++j)
                        if (v[j] == least && place++ < ties_left)
                            list(key_of(v[j], static_cast<uint32_t>(head + at * kV + j)));
                    ties_left -= __shfl_sync(0xffffffffu, upto, kLanes - 1, kLanes);
                }
            }
        }
        __syncthreads();
        if (sh.count > kList) {
            __syncthreads();
            if (tid == 0) sh.count = 0;
            __syncthreads();
            if (edge_key) list(edge_key);
            for (int r = warp; r < o.k && sh.run[r] >= 0; r += kWarps) {
                uint64_t key[RUN / 32], last = ~0ull;
#pragma unroll
                for (int e = 0; e < RUN / 32; ++e) key[e] = run_key(sh.run[r], e * 32 + lane);
                for (int k = r; k < o.k && last; ++k) {
                    uint64_t best = 0;
#pragma unroll
                    for (int e = 0; e < RUN / 32; ++e)
                        if (key[e] < last && key[e] > best) best = key[e];
                    last = warp_best(best);
                    if (lane == 0 && last) list(last);
                }
            }
            __syncthreads();
        }
        const int c = sh.count;
        if (tid == 0 && (c & 1)) sh.list[c] = 0ull;
        __syncthreads();
        for (int i = tid; i < c; i += kThreads) {
            const uint64_t mine = sh.list[i];
            const int above = count_above(sh.list, c, mine);
            if (above < o.k) root->join[rank * o.k + above] = mine;
        }
        for (int i = c + tid; i < o.k; i += kThreads) root->join[rank * o.k + i] = 0ull;
    }
    if (parts > 1) {
        if (tid == 0) root->part[rank] = sum;
        cg::this_cluster().sync();
        if (rank != 0) return;
        if (warp == 0) sum = warp_joined(lane < parts ? sh.part[lane] : Sums{neg_inf(), 0.f, 0.f});
    }
    if (tid == 0) {
        sh.result = finish(sum);
        write_row(o, n, xr, V, sum, sh.result);
    }
    if constexpr (TOP) {
        __syncthreads();
        const int c = parts * o.k;
        for (int i = tid; i < c; i += kThreads) {
            const uint64_t mine = sh.join[i];
            int above = i;  // one part: in order already
            if (parts > 1) {
                // places without a number come last, in any order among themselves
                above = count_above(sh.join, c, mine);  // parts > 1 is even
                if (mine == 0ull)
                    for (int j = 0; j < i; ++j) above += sh.join[j] == 0ull;
            }
            if (above < o.k) write_top(o, n, above, mine, sh.result);
        }
    }
}

// ---- backward: each block takes a run of one row ----
constexpr int kRun = 8192;  // elements of a run

template <typename T>
__global__ void __launch_bounds__(256)
    backward_kernel(const T *x, int64_t ldx, int64_t V, const float *stats, const int64_t *tokens, int64_t ignore,
                    const float *dlogp, const float *entropy, const float *dentropy, T *dx, int64_t lddx, int runs,
                    uint32_t *status)
{
    constexpr int kV = 16 / sizeof(T);
    const int64_t n = blockIdx.x / runs;
    const int run = static_cast<int>(blockIdx.x % runs);
    const int64_t c0 = static_cast<int64_t>(run) * kRun, c1 = c0 + kRun < V ? c0 + kRun : V;
    const T *xr = x + n * ldx;
    T *dr = dx + n * lddx;
    const float m = stats[2 * n], log2_s = stats[2 * n + 1] * kLog2e;
    const bool empty = m == neg_inf() && log2_s == 0.f;
    const float ref = ref_of(m);
    int64_t token = tokens ? tokens[n] : -1;
    float g = dlogp ? dlogp[n] : 0.f;
    if (token == ignore || !dlogp) {
        token = -1;
        g = 0.f;
    } else if (token < 0 || token >= V) {
        report(status, CCI_ERR_INDEX);
        token = -1;
        g = 0.f;
    }
    const float ge = dentropy ? dentropy[n] : 0.f, h = dentropy ? entropy[n] : 0.f;
    auto grad = [&](float xv, int64_t v) {
        const float l2 = fmaf(xv - ref, kLog2e, -log2_s), p = ex2(l2);
        float d = -g * p;
        if (ge != 0.f) d -= ge * p * fmaf(fmaxf(l2, -200.f), kLn2, h);
        if (v == token) d += g;
        return empty ? 0.f : d;
    };
    // 16-byte words where both rows have them at the same place
    const uintptr_t off_x = reinterpret_cast<uintptr_t>(xr + c0) % 16, off_d = reinterpret_cast<uintptr_t>(dr + c0) % 16;
    const int64_t to_word = off_x == off_d ? static_cast<int64_t>((16 - off_x) % 16 / sizeof(T)) : c1 - c0;
    const int64_t b0 = c0 + to_word < c1 ? c0 + to_word : c1, b1 = b0 + (c1 - b0) / kV * kV;
    for (int64_t v = c0 + threadIdx.x; v < b0; v += 256) {
        const float d = grad(row::to_f32(xr[v]), v);
        row::store<T, 1>(dr + v, &d);
    }
    constexpr int kU = kRun / (256 * kV);  // words of a thread
    row::Raw<T, kV> raw[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int64_t v = b0 + (u * 256 + static_cast<int>(threadIdx.x)) * kV;
        if (v < b1) raw[u] = row::load_once<T, kV>(xr + v);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int64_t v = b0 + (u * 256 + static_cast<int>(threadIdx.x)) * kV;
        if (v < b1) {
            float f[kV];
            row::unpack<T, kV>(raw[u], f);
#pragma unroll
            for (int j = 0; j < kV; ++j) f[j] = grad(f[j], v + j);
            row::store<T, kV>(dr + v, f);
        }
    }
    if (b1 + threadIdx.x < c1) {
        const int64_t v = b1 + threadIdx.x;
        const float d = grad(row::to_f32(xr[v]), v);
        row::store<T, 1>(dr + v, &d);
    }
}

template <typename T, int E>
cudaError_t launch_short(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, cudaStream_t stream)
{
    const unsigned blocks = static_cast<unsigned>((N + 7) / 8);
    if (o.k)
        short_kernel<T, E, true><<<blocks, 256, 0, stream>>>(x, ldx, N, static_cast<int>(V), o);
    else
        short_kernel<T, E, false><<<blocks, 256, 0, stream>>>(x, ldx, N, static_cast<int>(V), o);
    return cudaGetLastError();
}

template <typename T, int kThreads, int RUN, bool TOP>
cudaError_t launch_rows(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, int parts, cudaStream_t stream)
{
    // runs of a warp: its share of the words in whole iterations
    constexpr int64_t kV = 16 / sizeof(T), kIter = 512 / kV, kWarps = kThreads / 32;
    const int64_t words = (V / kV + parts - 1) / parts, per_warp = ((words + kWarps - 1) / kWarps + kIter - 1) / kIter * kIter;
    const int slots = static_cast<int>((per_warp / (RUN / kV) + 3) / 4 * 4);  // read four at a time
    const size_t bytes = TOP ? static_cast<size_t>(kWarps) * slots * sizeof(uint32_t) : 0;
    if (bytes > 32 * 1024) {
        static SmemAttrCache attr_cache;
        const cudaError_t attr = smem_attr_once(row_kernel<T, kThreads, RUN, TOP>, kMaxMaxima, attr_cache);
        if (attr != cudaSuccess) return attr;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(N * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = static_cast<unsigned>(parts);
    la[0].val.clusterDim.y = 1;
    la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    const cudaError_t e =
        cudaLaunchKernelEx(&cfg, row_kernel<T, kThreads, RUN, TOP>, x, ldx, static_cast<int>(V), o, parts, slots);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// rows of 1025 to 8192 logits: runs as long as leave 32 of them, for up to 32 alternatives
template <typename T, int kThreads>
cudaError_t launch_middle(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, cudaStream_t stream)
{
    if (!o.k) return launch_rows<T, kThreads, 512, false>(x, ldx, N, V, o, 1, stream);
    if (V < 2048) return launch_rows<T, kThreads, 32, true>(x, ldx, N, V, o, 1, stream);
    if (V < 4096) return launch_rows<T, kThreads, 64, true>(x, ldx, N, V, o, 1, stream);
    return launch_rows<T, kThreads, 128, true>(x, ldx, N, V, o, 1, stream);
}

template <typename T>
cudaError_t launch(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, cudaStream_t stream)
{
    // a warp a row, in its registers (bf16, against the kernel below, which reads whole words, with a warp a row:
    // 65536 x 600 54.9 us and 57.6, 65536 x 1000 66.5 and 59.8; that kernel has no runs short enough for alternatives here)
    if (V <= 128) return launch_short<T, 4>(x, ldx, N, V, o, stream);
    if (V <= 512) return launch_short<T, 16>(x, ldx, N, V, o, stream);
    if (V <= 1024) return launch_short<T, 32>(x, ldx, N, V, o, stream);
    if (V <= 8192) {
        // a warp a row where the rows fill the SMs, else four (bf16: 2432 x 4000 8.3 us and 10.9, 16384 x 8192 55 and
        // 76; with 5 alternatives 14.4 and 18.5, 106 and 140)
        if (N >= 16 * row::sm_count()) return launch_middle<T, 32>(x, ldx, N, V, o, stream);
        return launch_middle<T, 128>(x, ldx, N, V, o, stream);
    }
    // parts of a row where the rows alone leave SMs idle (each holds four blocks).  A part keeps 16384 logits
    // (32 runs).  More parts than that, to fill the last round of blocks, cost more than they save: the
    // alternatives' work at a row's end is per part (1024 x 131072 bf16, 5 alternatives: 145 us in four parts and
    // 101 in one, with the kernel of that time)
    int parts = 1;
    while (parts < 8 && N * parts * 2 <= 4 * row::sm_count() && V >= 2 * parts * 16384) parts *= 2;
    // where the rows fill the SMs: blocks of four warps, eight of an SM, which share the rows out more evenly
    // (bf16: 1024 x 131072 55 us in blocks of eight warps, 51 so; 4096 x 20000 47 and 40; with 5 alternatives 66 and 62,
    // 76 and 64).  Past 131072 logits
    // their warps' runs would not fit two a lane
    if (N >= 4 * row::sm_count() && V <= 131072) {
        if (!o.k) return launch_rows<T, 128, 512, false>(x, ldx, N, V, o, 1, stream);
        return V <= 16384 ? launch_rows<T, 128, 128, true>(x, ldx, N, V, o, 1, stream)
                          : launch_rows<T, 128, 512, true>(x, ldx, N, V, o, 1, stream);
    }
    if (!o.k) return launch_rows<T, 256, 512, false>(x, ldx, N, V, o, parts, stream);
    return V <= 16384 ? launch_rows<T, 256, 128, true>(x, ldx, N, V, o, parts, stream)
                      : launch_rows<T, 256, 512, true>(x, ldx, N, V, o, parts, stream);
}

template <typename T>
cudaError_t launch_backward(const T *x, int64_t ldx, int64_t N, int64_t V, const float *stats, const int64_t *tokens,
                            int64_t ignore, const float *dlogp, const float *entropy, const float *dentropy, T *dx,
                            int64_t lddx, uint32_t *status, cudaStream_t stream)
{
    const int64_t runs = (V + kRun - 1) / kRun;
    backward_kernel<T><<<static_cast<unsigned>(N * runs), 256, 0, stream>>>(
        x, ldx, V, stats, tokens, ignore, dlogp, entropy, dentropy, dx, lddx, static_cast<int>(runs), status);
    return cudaGetLastError();
}

}  // namespace lp

cudaError_t launch_token_logprobs(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldx,
                                  const int64_t *tokens, int64_t ignore, int top, float *logp, float *entropy,
                                  float *stats, float *top_logp, int32_t *top_idx, uint32_t *status,
                                  cudaStream_t stream)
{
    const lp::Row o{tokens, ignore, logp, entropy, stats, top_logp, top_idx, top, status};
    return dtype == CCI_F32 ? lp::launch(static_cast<const float *>(logits), ldx, N, V, o, stream)
                            : lp::launch(static_cast<const uint16_t *>(logits), ldx, N, V, o, stream);
}

cudaError_t launch_token_logprobs_backward(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldx,
                                           const float *stats, const int64_t *tokens, int64_t ignore,
                                           const float *dlogp, const float *entropy, const float *dentropy, void *dx,
                                           int64_t lddx, uint32_t *status, cudaStream_t stream)
{
    return dtype == CCI_F32
               ? lp::launch_backward(static_cast<const float *>(logits), ldx, N, V, stats, tokens, ignore, dlogp,
                                     entropy, dentropy, static_cast<float *>(dx), lddx, status, stream)
               : lp::launch_backward(static_cast<const uint16_t *>(logits), ldx, N, V, stats, tokens, ignore, dlogp,
                                     entropy, dentropy, static_cast<uint16_t *>(dx), lddx, status, stream);
}

}  // namespace cci
