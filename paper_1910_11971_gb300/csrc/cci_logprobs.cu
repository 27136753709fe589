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
// at the type's lowest value.
//
// Top alternatives in the same pass: the elements of an iteration are in registers; those above the
// k-th largest key known so far are appended to a list in shared memory, which is cut back to
// its k largest (each entry counts the entries above it) when it fills.  A first threshold comes from
// the first iteration: of 32 groups of threads, the k-th largest of the groups' maxima is at most the
// k-th largest element.  A key is the logit's order and the inverted index, so ties fall to the
// lower index by themselves.
//
// Rows of up to 1024 logits take a warp each and stay in its registers.  Longer ones take a block,
// or, where the rows alone would not fill the SMs, a cluster of 2, 4 or 8 blocks that each read a
// part of the row and join in the first block's shared memory.
#include <cooperative_groups.h>

#include "cci_kernels.h"
#include "cci_rowops.cuh"

namespace cci {
namespace lp {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxTop = 32;  // a warp's lanes

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

// running sums of a part of a row: maximum m, s = sum 2^y, t = sum 2^y y with y = (x - m) log2(e).
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

// adds n elements (-inf: nothing) to the sums
template <int n>
__device__ __forceinline__ void add(Sums &a, const float (&x)[n])
{
    float top = x[0];
#pragma unroll
    for (int i = 1; i < n; ++i) top = fmaxf(top, x[i]);
    if (top > a.m) a = moved(a, top);
    const float m = ref_of(a.m);
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float y = (x[i] - m) * kLog2e, e = ex2(y);
        a.s += e;
        a.t = fmaf(e, fmaxf(y, -200.f), a.t);  // 2^-200 is 0: no 0 * inf
    }
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

// ---- rows of up to 1024 logits: a warp each ----
template <typename T, int E, bool TOP>
__global__ void __launch_bounds__(256) short_kernel(const T *x, int64_t ldx, int64_t N, int V, Row o)
{
    const int lane = threadIdx.x & 31;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (n >= N) return;
    const T *xr = x + n * ldx;
    float f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = lane + 32 * i < V ? row::to_f32(xr[lane + 32 * i]) : neg_inf();
    Sums a{neg_inf(), 0.f, 0.f};
    add(a, f);
    a = warp_joined(a);
    const Result r = finish(a);
    if (lane == 0) write_row(o, n, xr, V, a, r);
    if constexpr (TOP) {
        // k times the largest key below the last one
        uint64_t last = ~0ull;
        for (int k = 0; k < o.k; ++k) {
            uint64_t best = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const uint64_t key = key_of(f[i], static_cast<uint32_t>(lane + 32 * i));
                if (lane + 32 * i < V && f[i] == f[i] && key < last && key > best) best = key;
            }
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) {
                const uint64_t other = __shfl_xor_sync(0xffffffffu, best, s);
                best = other > best ? other : best;
            }
            if (lane == 0) write_top(o, n, k, best, r);
            last = best;
        }
    }
}

// ---- longer rows: a block of T threads, or a cluster of `parts` of them ----
constexpr int kList = 1024;  // candidates held

struct Shared {
    uint64_t list[2][kList];
    uint64_t join[8 * kMaxTop];  // first block of a cluster: the parts' lists
    Sums part[8];                // and their sums
    Sums warp[32];
    float group[32];
    int count;
    int cur;  // which list is in use
};

// cuts the list (its first `c` entries) back to its k largest, in order; every thread of the block
// calls it after a barrier.  Returns the k-th largest key (0 while there are fewer)
template <int kThreads>
__device__ uint64_t cut(Shared &sh, int k)
{
    const int c = sh.count < kList ? sh.count : kList;
    const uint64_t *in = sh.list[sh.cur];
    uint64_t *out = sh.list[sh.cur ^ 1];
    for (int i = threadIdx.x; i < c; i += kThreads) {
        const uint64_t mine = in[i];
        int above = 0;
        for (int j = 0; j < c; ++j) above += in[j] > mine;
        if (above < k) out[above] = mine;  // keys differ: every place is taken once
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        sh.count = c < k ? c : k;
        sh.cur ^= 1;
    }
    __syncthreads();
    return sh.count < k ? 0ull : sh.list[sh.cur][k - 1];
}

// what a block's threads know of the list
struct Threshold {
    uint64_t kth;  // k-th largest key so far (0: fewer)
    float bar;     // logits below it need not be looked at
    bool first;    // no iteration has been offered
};

// offers an iteration's elements (element i of a thread is logit place(i) of the row; `have`: those
// that exist) to the list of the k largest; every thread of the block calls it
template <int kThreads, int kE, typename Place>
__device__ __forceinline__ void offer(Shared &sh, Threshold &th, int k, const float (&f)[kE], uint32_t have,
                                      Place place)
{
    float top = neg_inf();
#pragma unroll
    for (int i = 0; i < kE; ++i) top = fmaxf(top, f[i]);
    if (th.first) {
        // a bound from the first iteration: the k-th largest of 32 groups' maxima
        constexpr int kGroup = kThreads / 32;  // threads of a group
        const int lane = threadIdx.x & 31;
        float g = top;
#pragma unroll
        for (int s = kGroup / 2; s > 0; s >>= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, s));
        if (threadIdx.x % kGroup == 0) sh.group[threadIdx.x / kGroup] = g;
        __syncthreads();
        const float mine = sh.group[lane];
        int above = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float other = __shfl_sync(0xffffffffu, mine, j);
            above += other > mine || (other == mine && j < lane);
        }
        const uint32_t at = __ballot_sync(0xffffffffu, above == k - 1);
        th.bar = __shfl_sync(0xffffffffu, mine, __ffs(at) - 1);  // maxima are no NaN: one lane has each place
        th.first = false;
    }
    uint32_t want = 0;
    if (top >= th.bar) {
#pragma unroll
        for (int i = 0; i < kE; ++i)
            if (f[i] >= th.bar && key_of(f[i], place(i)) > th.kth) want |= 1u << i;
        want &= have;
    }
    while (true) {
        bool full = false;
#pragma unroll
        for (int i = 0; i < kE; ++i) {
            if (want >> i & 1) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kList) {
                    sh.list[sh.cur][at] = key_of(f[i], place(i));
                    want &= ~(1u << i);
                }
                full |= at >= kList / 2;
            }
        }
        if (!__syncthreads_or(full)) break;
        th.kth = cut<kThreads>(sh, k);
        if (th.kth) th.bar = logit_of(th.kth);
#pragma unroll
        for (int i = 0; i < kE; ++i)
            if ((want >> i & 1) && !(key_of(f[i], place(i)) > th.kth)) want &= ~(1u << i);
    }
}

template <typename T, int kThreads, bool TOP>
__global__ void __launch_bounds__(kThreads) row_kernel(const T *x, int64_t ldx, int64_t V, Row o, int parts)
{
    constexpr int kV = 16 / sizeof(T), kU = 4, kE = kV * kU;  // elements of a load, loads and elements of an iteration
    constexpr int kWarps = kThreads / 32;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = static_cast<int>(blockIdx.x) % parts;
    const int64_t n = blockIdx.x / parts;
    const T *xr = x + n * ldx;
    // a head of single elements up to the first 16-byte word (first part), whole words, a tail (last part)
    const int64_t to_word = static_cast<int64_t>((16 - reinterpret_cast<uintptr_t>(xr) % 16) % 16 / sizeof(T));
    const int64_t head = to_word < V ? to_word : V, words = (V - head) / kV;
    const int64_t w0 = words * rank / parts, w1 = words * (rank + 1) / parts;
    const T *xw = xr + head;
    if (TOP && tid == 0) sh.count = sh.cur = 0;
    Sums a{neg_inf(), 0.f, 0.f};
    Threshold th{0ull, neg_inf(), true};

    if constexpr (TOP) __syncthreads();

    for (int64_t w = w0; w < w1; w += kThreads * kU) {
        row::Raw<T, kV> raw[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int64_t i = w + u * kThreads + tid;
            if (i < w1) raw[u] = row::load_once<T, kV>(xw + i * kV);
        }
        float f[kE];
        uint32_t have = 0;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int64_t i = w + u * kThreads + tid;
            if (i < w1) {
                row::unpack<T, kV>(raw[u], f + u * kV);
                have |= ((1u << kV) - 1u) << (u * kV);
            } else {
#pragma unroll
                for (int j = 0; j < kV; ++j) f[u * kV + j] = neg_inf();
            }
        }
        add(a, f);
        if constexpr (TOP)
            offer<kThreads>(sh, th, o.k, f, have, [=](int i) {
                return static_cast<uint32_t>(head + (w + (i / kV) * kThreads + tid) * kV + i % kV);
            });
    }
    // head and tail: fewer than 2 kV single elements
    const int64_t tail0 = head + words * kV;
    if ((rank == 0 && head > 0) || (rank == parts - 1 && tail0 < V) || w0 == w1) {
        float f[kE];
        uint32_t have = 0, at = 0;
#pragma unroll
        for (int i = 0; i < kE; ++i) f[i] = neg_inf();
        if (rank == 0 && tid < head) {
            at = tid;
            have = 1;
        } else if (rank == parts - 1 && tid >= kV && tid - kV < V - tail0) {
            at = static_cast<uint32_t>(tail0 + tid - kV);
            have = 1;
        }
        if (have) f[0] = row::to_f32(xr[at]);
        add(a, f);
        if constexpr (TOP) offer<kThreads>(sh, th, o.k, f, have, [=](int) { return at; });
    }

    // the block's sums, to every thread of its first warp
    a = warp_joined(a);
    if (lane == 0) sh.warp[warp] = a;
    __syncthreads();
    if (warp == 0) a = warp_joined(lane < kWarps ? sh.warp[lane] : Sums{neg_inf(), 0.f, 0.f});
    if constexpr (TOP) cut<kThreads>(sh, o.k);
    if (parts > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();  // every block of the cluster runs
        Shared *root = cluster.map_shared_rank(&sh, 0);
        if (tid == 0) root->part[rank] = a;
        if (TOP && tid < o.k) root->join[rank * o.k + tid] = tid < sh.count ? sh.list[sh.cur][tid] : 0ull;
        cluster.sync();
        if (rank != 0) return;
        if (warp == 0) a = warp_joined(lane < parts ? sh.part[lane] : Sums{neg_inf(), 0.f, 0.f});
    }
    if (warp != 0 && !TOP) return;
    __shared__ Result result;
    if (tid == 0) {
        result = finish(a);
        write_row(o, n, xr, V, a, result);
    }
    if constexpr (TOP) {
        __syncthreads();
        if (parts == 1) {
            if (tid < o.k) write_top(o, n, tid, tid < sh.count ? sh.list[sh.cur][tid] : 0ull, result);
        } else {
            // places without a number come last, in any order among themselves
            const int c = parts * o.k;
            for (int i = tid; i < c; i += kThreads) {
                const uint64_t mine = sh.join[i];
                int above = 0;
                for (int j = 0; j < c; ++j) above += sh.join[j] > mine || (sh.join[j] == mine && j < i);
                if (above < o.k) write_top(o, n, above, mine, result);
            }
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

template <typename T, int kThreads, bool TOP>
cudaError_t launch_rows(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, int parts, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(N * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = static_cast<unsigned>(parts);
    la[0].val.clusterDim.y = 1;
    la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, row_kernel<T, kThreads, TOP>, x, ldx, V, o, parts);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t launch(const T *x, int64_t ldx, int64_t N, int64_t V, const Row &o, cudaStream_t stream)
{
    if (V <= 128) return launch_short<T, 4>(x, ldx, N, V, o, stream);
    if (V <= 512) return launch_short<T, 16>(x, ldx, N, V, o, stream);
    if (V <= 1024) return launch_short<T, 32>(x, ldx, N, V, o, stream);
    // blocks of 128 threads up to 8192 logits: the list's first bound needs elements in every thread
    if (V <= 8192) return o.k ? launch_rows<T, 128, true>(x, ldx, N, V, o, 1, stream)
                              : launch_rows<T, 128, false>(x, ldx, N, V, o, 1, stream);
    // a part keeps at least one iteration's 8192 elements
    int parts = 1;
    while (parts < 8 && N * parts < 304 && V >= 2 * parts * 8192) parts *= 2;
    return o.k ? launch_rows<T, 512, true>(x, ldx, N, V, o, parts, stream)
               : launch_rows<T, 512, false>(x, ldx, N, V, o, parts, stream);
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
