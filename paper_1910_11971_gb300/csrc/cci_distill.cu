// cci_distill.cu -- distillation from a teacher's top logits: the cross entropy of what a teacher
// says of a row's k listed tokens against the student's softmax, and its gradient to the student's logits.
//
// z = x / T, p = softmax(z).  The teacher's q_j: softmax over the listed t_j / T, or (tail) exp(t_j), which leave
// q_rest = 1 - sum q to all that is not listed, whose probability is p_rest = sum of p over it:
//   loss  = - sum q_j log p_j  (- q_rest log p_rest)
//   dz_v  = p_v Q - q_v for the listed, Q = sum q + q_rest, else p_v Q - q_rest r_v, r the softmax over the unlisted
//
// Memory bound: one read of the logits forward, one read and one write backward.  The sum over the unlisted
// is taken by leaving the listed out, not as a difference: p_rest keeps its accuracy where the listed
// tokens have nearly all.  A bit per logit in shared memory says which are listed; it costs a byte's load for eight
// logits, and setting it finds an index that is listed twice.  The difference from the maximum comes before
// the factor log2(e) / T, which would overflow at the type's lowest value.
//
// Rows are walked in groups of eight logits on 16-byte words, whatever their first logit's place; the group at
// either end is read one by one.  Forward, all rows' groups are cut evenly over as many blocks as the SMs hold, each with eight
// warps that walk and one that sets the next row's bits, joins the last row's sums and leaves them for a second launch,
// where a warp a row adds its listed tokens; that launch has read them before the first has ended.  Rows of up to 2048 logits
// take a warp each, which does all of it, and few longer ones a cluster of blocks each, which joins in the first block's shared
// memory.
#include <cooperative_groups.h>

#include "cci_kernels.h"
#include "cci_rowops.cuh"
#include "cci_tc_common.cuh"

namespace cci {
namespace distill {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxListed = 128;
constexpr int kPiece = 32768;    // groups that a block has bits for at a time (32 KB, twice)
// logits of a row that a warp takes by itself, and where there are rows enough for all SMs' warps
constexpr int kShort = 2048, kShortOfMany = 32768;

// beyond it fp32 rounds a number by 2^-18 and more, and as much of its exponential: those maxima and normalisers are not taken from
// their quotients by T
constexpr float kFar = 64.f;

struct Args {
    const void *x;
    int64_t ldx, N;
    int V, k, tail;
    const int32_t *idx;   // [N][k]
    const float *value;   // [N][k]
    float T;
    float *loss, *stats;  // backward: stats is read
    uint32_t *status;
    const float *dloss;
    void *dx;
    int64_t lddx;
    // forward: a row's units of 32 groups, blocks that share all rows' units evenly, places for a row's sums
    int units, blocks, places;
    float2 *sums;         // [N][places]
    int parts;            // few rows: blocks of each
    int chunks, steps;    // warps of a row, backward, and their steps of 1024 logits
};

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }
__device__ __forceinline__ float ref_of(float m) { return m == neg_inf() ? 0.f : m; }  // -inf - -inf would be NaN

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// logits that the first group of a row lacks: group g holds logits 8 g - s .. 8 g - s + 7
template <typename T>
__device__ __forceinline__ int shift_of(const T *row)
{
    return static_cast<int>(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (16 / sizeof(T) - 1);
}

// eight logits from e on as they lie in memory; -inf outside of the row
template <typename T>
__device__ __forceinline__ row::Raw<T, 8> load_group(const T *row, int e, int V)
{
    if (e >= 0 && e + 8 <= V) return row::load_once<T, 8>(row + e);
    row::Raw<T, 8> raw;
    uint32_t w[2 * sizeof(T)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bool in = e + j >= 0 && e + j < V;
        if constexpr (sizeof(T) == 4) {
            w[j] = in ? __float_as_uint(row[e + j]) : 0xff800000u;
        } else {
            const uint32_t v = in ? row[e + j] : 0xff80u;
            w[j / 2] = j % 2 ? w[j / 2] | v << 16 : v;
        }
    }
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) raw.w[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    return raw;
}

struct Sums {
    float m, s;  // maximum of the logits; sum of exp((x - m) / T)
};

__device__ __forceinline__ Sums joined(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m), from = ref_of(m);
    // nothing is 0 whatever its maximum; NaN stays
    const float u = a.s == 0.f ? 0.f : a.s * ex2((a.m - from) * c), v = b.s == 0.f ? 0.f : b.s * ex2((b.m - from) * c);
    return Sums{m, u + v};
}

// what a row's list says: the largest listed logit and the sum of exp((x - top) / T) but for the largest's own 1; the teacher's
// sum or its normaliser's logarithm, as in stats; and - sum q_j (x_j - top) / T with the sum of those q_j
struct Listed {
    float top, others, given, norm, off, share;
    bool nothing;  // no index but -1
};

// a lane's part of a row's list: indices (-1: none), the teacher's values
constexpr int kOwn = kMaxListed / 32;

__device__ __forceinline__ void read_list(const Args &a, int64_t n, int lane, int (&at)[kOwn])
{
#pragma unroll
    for (int i = 0; i < kOwn; ++i) at[i] = lane + 32 * i < a.k ? a.idx[n * a.k + lane + 32 * i] : -1;
}

// the listed logits and the teacher's values
template <typename T>
__device__ __forceinline__ void read_listed(const Args &a, int64_t n, const T *x, int lane, const int (&at)[kOwn],
                                            float (&z)[kOwn], float (&q)[kOwn])
{
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        q[i] = lane + 32 * i < a.k ? a.value[n * a.k + lane + 32 * i] : 0.f;
        z[i] = at[i] >= 0 && at[i] < a.V ? row::to_f32(x[at[i]]) : neg_inf();
    }
}

// what they say, by a warp, to all its lanes
__device__ __forceinline__ Listed listed_of(const Args &a, const int (&at)[kOwn], float (&z)[kOwn], float (&q)[kOwn])
{
    float top = neg_inf(), best = neg_inf();
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        top = fmaxf(top, z[i]);
        if (at[i] >= 0) best = fmaxf(best, q[i]);
    }
    top = row::warp_max(top);
    best = row::warp_max(best);
    Listed r{top, 0.f, 0.f, 0.f, 0.f, 0.f, false};
    const float from = ref_of(top), best_from = ref_of(best);
    int largest = 0;  // how many are
    bool some = false;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        q[i] = at[i] < 0 ? 0.f : (a.tail ? expf(q[i]) : expf((q[i] - best_from) / a.T));
        z[i] = (z[i] - from) / a.T;
        r.given += q[i];
        some = some || at[i] != -1;
        if (z[i] == 0.f)
            ++largest;
        else if (at[i] >= 0)
            r.others += expf(z[i]);
    }
    largest = __reduce_add_sync(0xffffffffu, largest);
    r.nothing = !__any_sync(0xffffffffu, some);
    r.given = row::warp_sum(r.given);
    r.others = row::warp_sum(r.others) + (largest > 1 ? static_cast<float>(largest - 1) : 0.f);
    const float unit = a.tail || r.given == 0.f ? 1.f : 1.f / r.given;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const float share = q[i] * unit;
        r.share += share;
        if (share != 0.f) r.off -= share * z[i];
    }
    r.off = row::warp_sum(r.off);
    r.share = row::warp_sum(r.share);
    r.norm = a.tail ? r.given : (r.given == 0.f ? neg_inf() : logf(r.given) + best_from / a.T);
    return r;
}

// the bits of a row's listed logits in groups [g0, g1), by a warp; true: an index that is none, or that is listed twice
__device__ __forceinline__ bool set_bits(uint32_t *bits, const Args &a, const int (&at)[kOwn], int s, int g0, int g1, int lane)
{
    for (int i = lane; i < (g1 - g0 + 15) / 16; i += 32) reinterpret_cast<uint4 *>(bits)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int v = at[i];
        if (v < -1 || v >= a.V) bad = true;
        const int b = v + s - 8 * g0;
        if (v >= 0 && v < a.V && b >= 0 && b < 8 * (g1 - g0)) {
            const uint32_t bit = 1u << (b & 31);
            if (atomicOr(&bits[b >> 5], bit) & bit) bad = true;
        }
    }
    __syncwarp();
    return __any_sync(0xffffffffu, bad);
}

// the largest of U groups as they lie in memory (NaN is no maximum)
template <typename T, int U>
__device__ __forceinline__ float largest(const row::Raw<T, 8> (&raw)[U])
{
    if constexpr (sizeof(T) == 2) {
        uint32_t m = 0xff80ff80u;  // two at a time
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t w[4] = {raw[u].w[0].x, raw[u].w[0].y, raw[u].w[0].z, raw[u].w[0].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[j]));
        }
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    } else {
        float m = neg_inf();
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 w = raw[u].w[i];
                asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(w.x)), "f"(__uint_as_float(w.y)));
                asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(w.z)), "f"(__uint_as_float(w.w)));
            }
        return m;
    }
}

// A warp's sums while it walks, c = log2(e) / T: s = sum of 2^(x c - r) with r the product m c as it is rounded.  One fused
// operation takes a logit to its exponent, and its only rounding is that of the exponent, as if the difference x - m were
// taken first: that r is not quite m c (`off` is what it lacks) is one factor for all, put right when the maximum moves and at the end.
// Far from 0 (a row that is masked by large negative numbers) that factor would leave the range, and the difference does come first
struct Walk {
    float m, s, r, off;
    __device__ __forceinline__ Walk() : m(neg_inf()), s(0.f), r(0.f), off(0.f) {}
    __device__ __forceinline__ bool far() const { return !(fabsf(r) < 16777216.f); }  // below, off is 1/2 at most
    __device__ __forceinline__ Sums sums() const { return Sums{m, s == 0.f ? 0.f : s * ex2(-off)}; }
    __device__ __forceinline__ void raise(float top, float c)
    {
        s = s == 0.f ? 0.f : s * ex2(-off) * ex2((m - top) * c);
        m = top;
        r = top * c;
        off = far() ? 0.f : fmaf(top, c, -r);
        s *= ex2(off);
    }
};

// adds U groups a lane to a warp's sums, without their listed logits (a bit each)
template <typename T, int U>
__device__ __forceinline__ void add_groups(Walk &walk, row::Raw<T, 8> (&raw)[U], const uint32_t (&listed)[U], float c)
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (listed[u]) {
            constexpr int kEach = 4 / static_cast<int>(sizeof(T));
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) {
                uint32_t w[4] = {raw[u].w[i].x, raw[u].w[i].y, raw[u].w[i].z, raw[u].w[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t m = listed[u] >> (4 * i + j) * kEach;
                    if constexpr (sizeof(T) == 4) {
                        w[j] = m & 1u ? 0xff800000u : w[j];
                    } else {
                        w[j] = m & 1u ? (w[j] & 0xffff0000u) | 0xff80u : w[j];
                        w[j] = m & 2u ? (w[j] & 0xffffu) | 0xff800000u : w[j];
                    }
                }
                raw[u].w[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    float top = largest<T, U>(raw);
    asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
    if (top > walk.m) walk.raise(top, c);
    float e[4] = {};
    if (!walk.far()) {
        const float minus = -walk.r;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[8];
            row::unpack<T, 8>(raw[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j & 3] += ex2(fmaf(f[j], c, minus));
        }
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[8];
            row::unpack<T, 8>(raw[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j & 3] += ex2((f[j] - walk.m) * c);
        }
    }
    walk.s += (e[0] + e[1]) + (e[2] + e[3]);
}

__device__ __forceinline__ Sums warp_joined(Sums a, float c)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a = joined(a, Sums{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o)}, c);
    return a;
}

// a row's loss and stats from the sums over what is not listed, and its list (one lane)
__device__ __forceinline__ void finish(const Args &a, int64_t n, const Sums &sums, const Listed &mine, float c, bool bad)
{
    const float m = fmaxf(sums.m, mine.top), from = ref_of(m);
    float rest = sums.s == 0.f ? 0.f : sums.s * ex2((sums.m - from) * c);
    // The largest's own is 1, which its approximate exponentials (of Walk) miss by some 2^-24 for many maxima: where the others add less,
    // the logarithm below would come out below 0, and its sign says how the maximum is held.  NaN stays
    if (sums.m == m && m != neg_inf() && rest < 1.f) rest = 1.f;
    const bool some = mine.top != neg_inf();
    const float listed = some ? (1.f + mine.others) * ex2((mine.top - from) * c) : mine.others, sum = rest + listed;
    const bool empty = m == neg_inf() && sum == 0.f;
    // A sure student's loss is what others add to the 1 of a listed token, a small rest's what the listed add to it: neither
    // is left to the rounding of a sum that is mostly something else.  No term below is negative: nothing cancels
    const float log_s = empty ? 0.f : (some && mine.top >= sums.m ? log1pf(mine.others + rest) : logf(sum));
    // far below the listed, the rest's share is no number of 32 bits, or one of few digits, but its logarithm is
    const bool others = sums.s != 0.f;
    const float down = (sums.m - from) / a.T, log_own = logf(sums.s < 1.f ? 1.f : sums.s);
    const float log_rest = !others ? neg_inf() : (down > -kFar ? logf(rest) : log_own + down);
    float loss = mine.off + (mine.share == 0.f ? 0.f : mine.share * (log_s - (ref_of(mine.top) - from) / a.T));
    if (a.tail) {
        const float left = others ? fmaxf(1.f - mine.given, 0.f) : 0.f;
        if (left > 0.f) loss += left * (listed < rest ? log1pf(listed / rest) : log_s - log_rest);
    }
    if (bad) report(a.status, CCI_ERR_INDEX);
    // a sum that is NaN (of such logits, of +inf, or of a wrong list, as sums_kernel hands it on) is the loss' too, where the teacher gives
    // nothing any weight as well
    a.loss[n] = bad ? nan_f() : (mine.nothing ? 0.f : (sum != sum ? sum : loss));
    if (mine.nothing && !bad && !(sum < -neg_inf())) {  // a pad row's logits may be anything: its gradient is 0 by these
        reinterpret_cast<float4 *>(a.stats)[n] = make_float4(0.f, 0.f, 0.f, mine.norm);
        return;
    }
    // The gradient takes differences from the maximum.  Where the rounding of m / T says too little of it (a masked row's, say),
    // it is left as it is, and the logarithm, which is 0 at least (of 1 and more, by either way above), has its sign set
    const float high = m / a.T;
    const bool as_is = fabsf(high) >= kFar && high * a.T != m;
    // Nor does the rounding of log_rest say enough of a rest that lies as far below: the largest of it as it is, and in the
    // place of the teacher's sum, which is at least 0 and taken from the list again, the logarithm of its own sum with the sign set
    const bool apart = a.tail && others && log_rest <= -kFar;
    reinterpret_cast<float4 *>(a.stats)[n] = make_float4(bad ? nan_f() : (as_is ? m : high), as_is ? -log_s : log_s,
                                                         apart ? sums.m : log_rest, apart ? -log_own : mine.norm);
}

// ---- short rows, or many: a warp each.  The argument: bytes of a row's bits ----
template <typename T>
__global__ void __launch_bounds__(256, 4) short_kernel(const Args a, int bytes)
{
    constexpr int kU = 8 / sizeof(T);
    extern __shared__ __align__(16) unsigned char shared[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + warp;
    if (n >= a.N) return;
    unsigned char *bits = shared + warp * bytes;
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    const float c = kLog2e / a.T;
    const int s = shift_of(x), groups = (a.V + s + 7) / 8;
    int at[kOwn];
    float z[kOwn], q[kOwn];
    read_list(a, n, lane, at);
    row::Raw<T, 8> next[kU];
    auto load = [&](int g) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int i = g + 32 * u + lane;
            next[u] = load_group(x, i < groups ? 8 * i - s : a.V, a.V);
        }
    };
    load(0);
    read_listed(a, n, x, lane, at, z, q);
    const bool bad = set_bits(reinterpret_cast<uint32_t *>(bits), a, at, s, 0, groups, lane);
    Walk walk;
    for (int g = 0; g < groups; g += 32 * kU) {
        row::Raw<T, 8> raw[kU];
        uint32_t listed[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int i = g + 32 * u + lane;
            raw[u] = next[u];
            listed[u] = i < groups ? bits[i] : 0u;
        }
        if (g + 32 * kU < groups) load(g + 32 * kU);
        add_groups<T, kU>(walk, raw, listed, c);
    }
    const Listed mine = listed_of(a, at, z, q);
    const Sums sums = warp_joined(walk.sums(), c);
    if (lane == 0) finish(a, n, sums, mine, c, bad);
}

// ---- few longer rows: a cluster each (8 x 131072 fp32, k = 32: 7.5 us, 9.0 by the two launches below, and one launch
// less to queue).  `bytes`: groups of a block ----
constexpr int kMaxParts = 8;

template <typename T>
__global__ void __launch_bounds__(256) cluster_kernel(const Args a, int bytes)
{
    constexpr int kU = 8 / sizeof(T), kStep = 256;
    extern __shared__ __align__(16) unsigned char bits[];
    __shared__ Sums warps[8];
    __shared__ float4 parts[kMaxParts];  // maximum, sum, whether an index is bad
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = blockIdx.x / a.parts;
    const int part = static_cast<int>(blockIdx.x % a.parts);
    // the wait for this arrival, before the store into the first block, sees that every block of the cluster runs
    if (a.parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    const float c = kLog2e / a.T;
    const int s = shift_of(x), all = (a.V + s + 7) / 8;
    const int g0 = part * bytes < all ? part * bytes : all, g1 = g0 + bytes < all ? g0 + bytes : all;
    row::Raw<T, 8> next[kU];
    auto load = [&](int g) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int q = g + u * kStep + lane;
            next[u] = load_group(x, q < g1 ? 8 * q - s : a.V, a.V);
        }
    };
    if (g0 + 32 * warp < g1) load(g0 + 32 * warp);
    bool bad = false;
    Listed mine{};
    int at[kOwn];
    float z[kOwn], q[kOwn];
    if (warp == 0) {
        read_list(a, n, lane, at);
        if (part == 0) read_listed(a, n, x, lane, at, z, q);
        bad = set_bits(reinterpret_cast<uint32_t *>(bits), a, at, s, g0, g0 + bytes, lane);
    }
    __syncthreads();
    if (warp == 0 && part == 0) mine = listed_of(a, at, z, q);
    Walk walk;
    for (int g = g0 + 32 * warp; g < g1; g += kU * kStep) {
        row::Raw<T, 8> raw[kU];
        uint32_t listed[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int q = g + u * kStep + lane;
            raw[u] = next[u];
            listed[u] = q < g1 ? bits[q - g0] : 0u;
        }
        if (g + kU * kStep < g1) load(g + kU * kStep);
        add_groups<T, kU>(walk, raw, listed, c);
    }
    Sums sums = warp_joined(walk.sums(), c);
    if (lane == 0) warps[warp] = sums;
    __syncthreads();
    if (warp == 0) sums = warp_joined(lane < 8 ? warps[lane] : Sums{neg_inf(), 0.f}, c);
    if (a.parts > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        cg::cluster_group cluster = cg::this_cluster();
        if (threadIdx.x == 0) *cluster.map_shared_rank(&parts[part], 0) = make_float4(sums.m, sums.s, bad ? 1.f : 0.f, 0.f);
        cluster.sync();
        if (part != 0 || warp != 0) return;
        const float4 p = lane < a.parts ? parts[lane] : make_float4(neg_inf(), 0.f, 0.f, 0.f);
        bad = __any_sync(0xffffffffu, p.z != 0.f);
        sums = warp_joined(Sums{p.x, p.y}, c);
    }
    if (threadIdx.x == 0) finish(a, n, sums, mine, c, bad);
}

// ---- other rows: the sums over what is not listed ----
// of `all` units cut evenly over `blocks`, the block that holds unit u
__device__ __forceinline__ int holder(int64_t u, int64_t all, int blocks)
{
    int b = static_cast<int>(u * blocks / all);
    while (all * (b + 1) / blocks <= u) ++b;
    return b;
}

// a block's units [u, end), piece by piece: groups [g0, g1) of row n
struct Pieces {
    int64_t u, end, n;
    int unit;  // of the row, where the next piece begins
    int g0, g1;
    __device__ __forceinline__ Pieces(const Args &a, int64_t begin, int64_t end_) : u(begin), end(end_), n(begin / a.units)
    {
        unit = static_cast<int>(begin - n * a.units);
        g1 = 0;
    }
    // the next piece (the first after a row's last is the next row's); false: there is none
    __device__ __forceinline__ bool next(const Args &a)
    {
        if (u >= end) return false;
        if (unit == a.units) {
            unit = 0;
            ++n;
        }
        int count = a.units - unit;
        if (count > end - u) count = static_cast<int>(end - u);
        if (count > kPiece / 32) count = kPiece / 32;
        g0 = 32 * unit;
        g1 = g0 + 32 * count;
        unit += count;
        u += count;
        return true;
    }
};

constexpr int kWalkers = 8;

// The last argument: bytes of a piece's bits, of which there are two
template <typename T>
__global__ void __launch_bounds__(32 * (kWalkers + 1), 3) sums_kernel(const Args a, int bytes)
{
    constexpr int kU = 8 / sizeof(T), kStep = 32 * kWalkers;  // groups that a lane sums at a time
    extern __shared__ __align__(16) unsigned char bits[];
    __shared__ Sums warps[2][kWalkers];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t all = a.N * a.units;
    const int64_t begin = all * blockIdx.x / a.blocks, end = all * (blockIdx.x + 1) / a.blocks;
    const float c = kLog2e / a.T;
    const T *rows = static_cast<const T *>(a.x);
    tc::launch_next_grid();  // the second launch, which waits for this one's end
    Pieces p(a, begin, end);
    if (warp < kWalkers) {
        row::Raw<T, 8> next[kU];
        const T *x = rows;
        int s = 0;
        auto load = [&](int g) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int q = g + u * kStep + lane;
                next[u] = load_group(x, q < p.g1 ? 8 * q - s : a.V, a.V);
            }
        };
        auto enter = [&]() {
            if (!p.next(a)) return false;
            x = rows + p.n * a.ldx;
            s = shift_of(x);
            if (p.g0 + 32 * warp < p.g1) load(p.g0 + 32 * warp);
            return true;
        };
        enter();
        for (int k = 0;; ++k) {
            tc::named_sync(1, 32 * (kWalkers + 1));  // this piece's bits are set
            const unsigned char *mask = bits + (k & 1) * bytes;
            Walk walk;
            // the bounds are the same for a warp's lanes, so that they find their common maximum together; the next groups
            // are on their way while these are summed
            for (int g = p.g0 + 32 * warp; g < p.g1; g += kU * kStep) {
                row::Raw<T, 8> raw[kU];
                uint32_t listed[kU];
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    const int q = g + u * kStep + lane;
                    raw[u] = next[u];
                    listed[u] = q < p.g1 ? mask[q - p.g0] : 0u;
                }
                if (g + kU * kStep < p.g1) load(g + kU * kStep);
                add_groups<T, kU>(walk, raw, listed, c);
            }
            const bool more = enter();
            const Sums sums = warp_joined(walk.sums(), c);
            if (lane == 0) warps[k & 1][warp] = sums;
            if (!more) break;
        }
        tc::named_sync(1, 32 * (kWalkers + 1));
    } else {
        // the warp beside them: two pieces ahead with the list, one with its bits, one behind with the sums
        int at[kOwn];
        Pieces list = p, last = p;
        bool bad = false, next_bad = false;
        bool more = list.next(a);
        read_list(a, list.n, lane, at);
        Sums sums{neg_inf(), 0.f};
        auto prepare = [&](int k) {  // the bits of the piece whose list is at hand, then the next list
            p = list;
            next_bad = set_bits(reinterpret_cast<uint32_t *>(bits + (k & 1) * bytes), a, at, shift_of(rows + p.n * a.ldx), p.g0, p.g1, lane);
            more = list.next(a);
            if (more) read_list(a, list.n, lane, at);
        };
        auto join = [&](int k, bool final) {
            sums = joined(sums, warp_joined(lane < kWalkers ? warps[k & 1][lane] : Sums{neg_inf(), 0.f}, c), c);
            if (final || last.g1 == 32 * a.units) {
                if (lane == 0) {
                    // a row that begins here is the first block's
                    const int64_t first = last.n * a.units;
                    const int place = first >= begin ? 0 : static_cast<int>(blockIdx.x) - holder(first, all, a.blocks);
                    a.sums[last.n * a.places + place] = make_float2(sums.m, bad ? nan_f() : sums.s);
                    if (bad) report(a.status, CCI_ERR_INDEX);
                }
                sums = Sums{neg_inf(), 0.f};
                bad = false;
            }
        };
        prepare(0);
        for (int k = 0;; ++k) {
            const Pieces now = p;
            const bool now_bad = next_bad, left = more;
            tc::named_sync(1, 32 * (kWalkers + 1));
            if (k > 0) join(k - 1, false);
            bad = bad || now_bad;  // of the row that `now` is of
            last = now;
            if (left) {
                prepare(k + 1);
            } else {
                tc::named_sync(1, 32 * (kWalkers + 1));
                join(k, true);
                break;
            }
        }
    }
}

// a row's loss from its sums and its list, a warp a row.  The list is read while the sums are taken
template <typename T>
__global__ void __launch_bounds__(256) loss_kernel(const Args a)
{
    const int lane = threadIdx.x & 31;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5), all = a.N * a.units;
    if (n >= a.N) return;
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    const float c = kLog2e / a.T;
    int at[kOwn];
    float z[kOwn], q[kOwn];
    read_list(a, n, lane, at);
    read_listed(a, n, x, lane, at, z, q);
    const Listed mine = listed_of(a, at, z, q);
    const int count = holder(n * a.units + a.units - 1, all, a.blocks) - holder(n * a.units, all, a.blocks) + 1;
    tc::wait_prior_grid();
    Sums sums{neg_inf(), 0.f};
    for (int i = lane; i < count; i += 32) {
        const float2 part = a.sums[n * a.places + i];
        sums = joined(sums, Sums{part.x, part.y}, c);
    }
    sums = warp_joined(sums, c);
    if (lane == 0) finish(a, n, sums, mine, c, false);
}

// ---- gradient: a warp takes one to four steps of 128 groups of a row by itself; the next step's logits are on their way while
// it finds its listed ones, once for all steps (4096 x 50001 bf16, k = 64: 224 us where a block of 256 threads waited for
// them, 180 with one step a warp) ----
template <typename T>
__global__ void __launch_bounds__(256) gradient_kernel(const Args a)
{
    constexpr int kU = 4, kOwn = kMaxListed / 32;
    const int lane = threadIdx.x & 31;
    const int64_t w = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5), n = w / a.chunks;
    if (n >= a.N) return;
    const int chunk = static_cast<int>(w - n * a.chunks);
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    T *dx = static_cast<T *>(a.dx) + n * a.lddx;
    const int s = shift_of(x), V = a.V, lo = chunk * a.steps * 256 * kU - s;
    const int hi = lo + a.steps * 256 * kU < V ? lo + a.steps * 256 * kU : V;
    const float unit = 1.f / a.T, c = kLog2e / a.T;
    row::Raw<T, 8> next[kU];
    bool none = false;  // of what is not listed: -inf for it, whatever the logits
    auto load = [&](int e0) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int e = e0 + 8 * (32 * u + lane);
            next[u] = load_group(x, e < V && !none ? e : V, V);
        }
    };
    load(lo);
    // the listed logits among these, read before any of them is written (dx may be x), and what the teacher says of them
    int at[kOwn];
    float z[kOwn], own[kOwn];
    bool listed = false;  // anything at all: a pad row has no gradient, whatever its loss has
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int j = lane + i * 32;
        at[i] = j < a.k ? a.idx[n * a.k + j] : -1;
        listed = listed || at[i] != -1;
        if (at[i] < lo || at[i] >= hi) at[i] = -1;
        if (at[i] >= 0) {
            z[i] = row::to_f32(x[at[i]]);
            own[i] = a.value[n * a.k + j];
        }
    }
    const float4 st = reinterpret_cast<const float4 *>(a.stats)[n];
    const float weight = a.dloss[n] / a.T, log_s = fabsf(st.y), log_rest = st.z;
    const float m = ref_of(signbit(st.y) ? st.x : st.x * a.T);
    const bool apart = a.tail && signbit(st.w), some = a.tail && (apart || log_rest != neg_inf());
    float whole, left = 0.f;        // Q, q_rest
    float best = 0.f, norm = st.w;  // of the teacher's values: q_j = exp((t_j - best) / T - norm)
    if (a.tail) {
        float given = st.w;
        if (apart) {
            given = 0.f;
            for (int j = lane; j < a.k; j += 32)
                if (a.idx[n * a.k + j] >= 0) given += expf(a.value[n * a.k + j]);
            given = row::warp_sum(given);
        }
        if (some) left = fmaxf(1.f - given, 0.f);
        whole = given + left;
    } else {
        if (fabsf(norm) >= kFar) {
            best = neg_inf();
            for (int j = lane; j < a.k; j += 32)
                if (a.idx[n * a.k + j] >= 0) best = fmaxf(best, a.value[n * a.k + j]);
            best = ref_of(row::warp_max(best));
            norm = 0.f;
            for (int j = lane; j < a.k; j += 32)
                if (a.idx[n * a.k + j] >= 0) norm += expf((a.value[n * a.k + j] - best) / a.T);
            norm = logf(row::warp_sum(norm));
        }
        whole = norm == neg_inf() ? 0.f : 1.f;  // nothing listed
    }
    const bool lost = st.x != st.x || st.y != st.y;  // a wrong list, logits that are no numbers
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        if (at[i] >= 0) {
            const float q = a.tail ? expf(own[i]) : (whole == 0.f ? 0.f : expf((own[i] - best) * unit - norm));
            const float p = expf((z[i] - m) * unit - log_s);
            own[i] = weight == 0.f || (st.x == neg_inf() && !lost) ? 0.f : (p * whole - q) * (lost ? nan_f() : weight);
        }
    }
    // off the list: coef exp((x - base) / T - shift).  With a tail, relative to the sum over the unlisted
    float base = apart ? log_rest : m;
    const float shift = apart ? fabsf(st.w) : (some ? log_rest : log_s);
    const float log_p = (apart ? (base - m) / a.T + shift : log_rest) - log_s;  // of the rest
    float coef = (some ? whole * expf(log_p) - left : whole) * weight, minus = -shift * kLog2e;
    if (lost) coef = nan_f();
    none = weight == 0.f || coef == 0.f || !__any_sync(0xffffffffu, listed);
    if (none) {
        coef = minus = base = 0.f;
        load(lo);
    }
    const unsigned long long c2 = pack2(c, c), neg = pack2(-base, -base), coef2 = pack2(coef, coef);
    const bool words = shift_of(dx) == s;
    __syncwarp();
    for (int e0 = lo; e0 < hi; e0 += 256 * kU) {
        row::Raw<T, 8> raw[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) raw[u] = next[u];
        if (e0 + 256 * kU < hi) load(e0 + 256 * kU);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int e = e0 + 8 * (32 * u + lane);
            if (e >= V) continue;
            unsigned long long p[4];
            row::unpack2<T, 8>(raw[u], p);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned long long y = pack2(minus, minus);
                ffma2(y, row::add2(p[j], neg), c2);
                p[j] = row::mul2(pack2(ex2(lo_of(y)), ex2(hi_of(y))), coef2);
            }
            if (words && e >= 0 && e + 8 <= V) {
                row::store2<T, 8>(dx + e, p);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float v = j % 2 ? hi_of(p[j / 2]) : lo_of(p[j / 2]);
                    if (e + j >= 0 && e + j < V) row::store<T, 1>(dx + e + j, &v);
                }
            }
        }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
        if (at[i] >= 0) row::store<T, 1>(dx + at[i], own + i);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// a warp a row (bf16 8192 x 4096: 25 us, 62 where eight warps share each; 8192 x 16384: 58 and 88)
bool by_warps(int64_t N, int64_t V)
{
    return V <= kShort || (V <= kShortOfMany && N >= 24 * static_cast<int64_t>(row::sm_count()));
}

// a cluster a row: so few that their blocks are all resident, of up to 32768 groups each
bool by_clusters(int64_t N, int64_t V)
{
    return N * kMaxParts <= 3 * static_cast<int64_t>(row::sm_count()) && V <= static_cast<int64_t>(kMaxParts) * 8 * (kPiece - 32);
}

// how a forward call's rows are cut otherwise
struct Cut {
    int units, blocks, places;
};

Cut cut_of(int64_t N, int64_t V)
{
    Cut c{};
    if (N < 1 || by_warps(N, V) || by_clusters(N, V)) return c;
    const int64_t units = ((V + 14) / 8 + 31) / 32, most = 3 * static_cast<int64_t>(row::sm_count());
    int64_t blocks = N * units / kWalkers;  // a unit for each warp at least
    if (blocks > most) blocks = most;
    c.units = static_cast<int>(units);
    c.blocks = static_cast<int>(blocks < 1 ? 1 : blocks);
    c.places = static_cast<int>((c.blocks + N - 1) / N) + 1;  // blocks that a row's units lie with
    return c;
}

template <typename T>
cudaError_t launch_loss(Args a, float2 *workspace, cudaStream_t stream)
{
    if (by_warps(a.N, a.V)) {
        const int bytes = ((a.V + 14) / 8 + 15) / 16 * 16;
        short_kernel<T><<<static_cast<unsigned>((a.N + 7) / 8), 256, static_cast<size_t>(8 * bytes), stream>>>(a, bytes);
        return cudaGetLastError();
    }
    if (by_clusters(a.N, a.V)) {
        a.parts = 1;  // each with 4096 logits or more
        while (a.parts < kMaxParts && a.V / (2 * a.parts) >= 4096) a.parts *= 2;
        const int groups = ((a.V + 14) / 8 + a.parts - 1) / a.parts, bytes = (groups + 31) / 32 * 32;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(a.N * a.parts));
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = static_cast<size_t>(bytes);
        cfg.stream = stream;
        cudaLaunchAttribute la[1];
        la[0].id = cudaLaunchAttributeClusterDimension;
        la[0].val.clusterDim.x = static_cast<unsigned>(a.parts);
        la[0].val.clusterDim.y = 1;
        la[0].val.clusterDim.z = 1;
        cfg.attrs = la;
        cfg.numAttrs = a.parts > 1 ? 1 : 0;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, cluster_kernel<T>, static_cast<const Args>(a), bytes);
        return e == cudaSuccess ? cudaGetLastError() : e;
    }
    const Cut cut = cut_of(a.N, a.V);
    a.units = cut.units;
    a.blocks = cut.blocks;
    a.places = cut.places;
    a.sums = cut.places <= 2 ? reinterpret_cast<float2 *>(a.stats) : workspace;  // two fit where the stats come later
    const int bits = 32 * a.units < kPiece ? 32 * a.units : kPiece;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(sums_kernel<T>, 2 * kPiece, attr_cache);
    if (attr != cudaSuccess) return attr;
    sums_kernel<T><<<static_cast<unsigned>(a.blocks), 32 * (kWalkers + 1), static_cast<size_t>(2 * bits), stream>>>(a, bits);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((a.N + 7) / 8));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, loss_kernel<T>, static_cast<const Args>(a));
    return e == cudaSuccess ? cudaGetLastError() : e;
}

template <typename T>
cudaError_t launch_gradient(Args a, cudaStream_t stream)
{
    // four steps a warp where that leaves several rounds of warps
    const int64_t all = (a.V + 7 + 1023) / 1024;
    a.steps = 4;
    while (a.steps > 1 && a.N * ((all + a.steps - 1) / a.steps) < 4 * 24 * static_cast<int64_t>(row::sm_count())) a.steps /= 2;
    a.chunks = static_cast<int>((all + a.steps - 1) / a.steps);
    const int64_t blocks = (a.N * a.chunks + 7) / 8;
    if (blocks >= (int64_t(1) << 31)) return cudaErrorInvalidValue;
    gradient_kernel<T><<<static_cast<unsigned>(blocks), 256, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace distill

size_t distillation_workspace(int64_t N, int64_t V)
{
    const distill::Cut c = distill::cut_of(N, V);
    return c.places <= 2 ? 0 : static_cast<size_t>(N) * c.places * sizeof(float2);
}

cudaError_t launch_distillation(const void *x, int dtype, int64_t N, int64_t V, int64_t ldx, const int32_t *idx,
                                const float *value, int k, float T, int tail, float *loss, float *stats,
                                uint32_t *status, void *workspace, cudaStream_t stream)
{
    using namespace distill;
    Args a{};
    a.x = x;
    a.ldx = ldx;
    a.N = N;
    a.V = static_cast<int>(V);
    a.k = k;
    a.tail = tail;
    a.idx = idx;
    a.value = value;
    a.T = T;
    a.loss = loss;
    a.stats = stats;
    a.status = status;
    float2 *w = static_cast<float2 *>(workspace);
    return dtype == CCI_F32 ? launch_loss<float>(a, w, stream) : launch_loss<uint16_t>(a, w, stream);
}

cudaError_t launch_distillation_backward(const float *dloss, const void *x, int dtype, int64_t N, int64_t V, int64_t ldx,
                                         const int32_t *idx, const float *value, int k, float T, int tail,
                                         const float *stats, void *dx, int64_t lddx, cudaStream_t stream)
{
    using namespace distill;
    Args a{};
    a.x = x;
    a.ldx = ldx;
    a.N = N;
    a.V = static_cast<int>(V);
    a.k = k;
    a.tail = tail;
    a.idx = idx;
    a.value = value;
    a.T = T;
    a.stats = const_cast<float *>(stats);
    a.dloss = dloss;
    a.dx = dx;
    a.lddx = lddx;
    return dtype == CCI_F32 ? launch_gradient<float>(a, stream) : launch_gradient<uint16_t>(a, stream);
}

}  // namespace cci
