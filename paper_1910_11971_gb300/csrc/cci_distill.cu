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
// either end is read one by one.  Where the rows alone would not fill the SMs, a cluster of blocks shares one
// and joins in the first block's shared memory.
#include <cooperative_groups.h>

#include "cci_kernels.h"
#include "cci_rowops.cuh"

namespace cci {
namespace distill {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxListed = 128;
constexpr int kBits = 262144;    // logits that a block has bits for at a time (32 KB)

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
    int parts;            // blocks of a row, forward
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

// what a block knows of its part
struct Part {
    Sums sums;
    int bad;
};

// what a row's list says: the largest listed logit and the sum of exp((x - top) / T); the teacher's sum or its normaliser's
// logarithm, as in stats; and - sum q_j (x_j - top) / T with the sum of those q_j
struct Listed {
    float top, sum, given, norm, off, share;
};

// by a warp, a lane's results those of all
template <typename T>
__device__ __forceinline__ Listed listed_of(const Args &a, const T *x, const int32_t *idx, const float *value, int lane)
{
    constexpr int kOwn = kMaxListed / 32;
    int at[kOwn];
    float z[kOwn], q[kOwn];
    float top = neg_inf(), best = neg_inf();
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int j = lane + 32 * i;
        at[i] = j < a.k ? idx[j] : -1;
        q[i] = j < a.k ? value[j] : 0.f;
        z[i] = at[i] >= 0 && at[i] < a.V ? row::to_f32(x[at[i]]) : neg_inf();
        top = fmaxf(top, z[i]);
        if (at[i] >= 0) best = fmaxf(best, q[i]);
    }
    top = row::warp_max(top);
    best = row::warp_max(best);
    Listed r{top, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float from = ref_of(top), best_from = ref_of(best);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        q[i] = at[i] < 0 ? 0.f : (a.tail ? expf(q[i]) : expf((q[i] - best_from) / a.T));
        z[i] = (z[i] - from) / a.T;
        r.given += q[i];
        if (at[i] >= 0) r.sum += expf(z[i]);
    }
    r.given = row::warp_sum(r.given);
    r.sum = row::warp_sum(r.sum);
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

template <typename T, int TPB>
__global__ void __launch_bounds__(TPB) loss_kernel(const Args a)
{
    constexpr int kU = 4;  // groups on their way a thread
    extern __shared__ __align__(16) uint32_t bits[];
    __shared__ Part warps[TPB / 32];
    __shared__ Part parts[8];
    __shared__ int bad_flag;
    const int t = threadIdx.x, lane = t & 31;
    const int64_t n = blockIdx.x / a.parts;
    const int part = static_cast<int>(blockIdx.x % a.parts);
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    const int32_t *idx = a.idx + n * a.k;
    const float c = kLog2e / a.T;
    const int s = shift_of(x), V = a.V;
    const int groups = static_cast<int>((static_cast<int64_t>(V) + s + 7) / 8);
    const int each = ((groups + a.parts - 1) / a.parts + 31) / 32 * 32;
    const int first = part * each < groups ? part * each : groups, last = first + each < groups ? first + each : groups;
    Sums sums{neg_inf(), 0.f};
    Listed mine{};
    if (t == 0) bad_flag = 0;
    for (int g0 = first; g0 < last || g0 == first; g0 += kBits / 8) {
        const int g1 = g0 + kBits / 8 < last ? g0 + kBits / 8 : last;
        // the first groups are on their way while the bits are set
        row::Raw<T, 8> raw[kU];
        auto load = [&](int g) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int q = g + u * TPB + lane;
                raw[u] = load_group(x, q < g1 ? 8 * q - s : V, V);
            }
        };
        int g = g0 + (t & ~31);
        if (g < g1) load(g);
        __syncthreads();
        for (int i = t; i < (g1 - g0 + 3) / 4; i += TPB) bits[i] = 0u;
        __syncthreads();
        for (int j = t; j < a.k; j += TPB) {
            const int32_t v = idx[j];
            if (v < -1 || v >= V) bad_flag = 1;
            const int64_t b = static_cast<int64_t>(v) + s - 8 * static_cast<int64_t>(g0);
            if (v >= 0 && v < V && b >= 0 && b < 8 * static_cast<int64_t>(g1 - g0)) {
                const uint32_t bit = 1u << (b & 31);
                if (atomicOr(&bits[b >> 5], bit) & bit) bad_flag = 1;
            }
        }
        __syncthreads();
        const uint8_t *mask = reinterpret_cast<const uint8_t *>(bits);
        if (g0 == first && part == 0 && t < 32) mine = listed_of(a, x, idx, a.value + n * a.k, lane);
        // the bounds are the same for a warp's lanes, so that they find their common maximum together; the next groups
        // are on their way while these are summed
        for (; g < g1; g += kU * TPB) {
            float f[kU][8];
#pragma unroll
            for (int u = 0; u < kU; ++u) row::unpack<T, 8>(raw[u], f[u]);
            if (g + kU * TPB < g1) load(g + kU * TPB);
            float top = neg_inf();
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int q = g + u * TPB + lane;
                const uint32_t m = q < g1 ? mask[q - g0] : 0u;
                if (m) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[u][j] = m >> j & 1u ? neg_inf() : f[u][j];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, f[u][j]);
            }
            asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
            if (top > sums.m) {
                sums.s = sums.s == 0.f ? 0.f : sums.s * ex2((sums.m - top) * c);
                sums.m = top;
            }
            const float from = ref_of(sums.m);
            const unsigned long long neg = pack2(-from, -from), c2 = pack2(c, c);
            unsigned long long e[2] = {};
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const unsigned long long y = row::mul2(row::add2(pack2(f[u][j], f[u][j + 1]), neg), c2);
                    e[j / 2 & 1] = row::add2(e[j / 2 & 1], pack2(ex2(lo_of(y)), ex2(hi_of(y))));
                }
            const unsigned long long both = row::add2(e[0], e[1]);
            sums.s += lo_of(both) + hi_of(both);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        sums = joined(sums, Sums{__shfl_xor_sync(0xffffffffu, sums.m, o), __shfl_xor_sync(0xffffffffu, sums.s, o)}, c);
    if (lane == 0) warps[t >> 5].sums = sums;
    __syncthreads();
    if (t < 32) {
        sums = lane < TPB / 32 ? warps[lane].sums : Sums{neg_inf(), 0.f};
#pragma unroll
        for (int o = 4; o > 0; o >>= 1)
            sums = joined(sums, Sums{__shfl_xor_sync(0xffffffffu, sums.m, o), __shfl_xor_sync(0xffffffffu, sums.s, o)}, c);
    }
    int bad = bad_flag;
    if (a.parts > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        if (t == 0) *cluster.map_shared_rank(&parts[part], 0) = Part{sums, bad};
        cluster.sync();
        if (part != 0) return;
        if (t < 32) {
            const Part p = lane < a.parts ? parts[lane] : Part{{neg_inf(), 0.f}, 0};
            sums = p.sums;
            bad = __any_sync(0xffffffffu, p.bad);
#pragma unroll
            for (int o = 4; o > 0; o >>= 1)
                sums = joined(sums, Sums{__shfl_xor_sync(0xffffffffu, sums.m, o), __shfl_xor_sync(0xffffffffu, sums.s, o)}, c);
        }
    }
    if (t > 0) return;
    // the listed join, and the teacher has its say
    const float m = fmaxf(sums.m, mine.top), from = ref_of(m);
    const float rest = sums.s == 0.f ? 0.f : sums.s * ex2((sums.m - from) * c);
    const float sum = rest + (mine.sum == 0.f ? 0.f : mine.sum * ex2((mine.top - from) * c));
    const bool empty = m == neg_inf() && sum == 0.f;
    const float log_s = empty ? 0.f : logf(sum), log_rest = logf(rest);
    // no term is below 0: nothing cancels
    float loss = mine.off + (mine.share == 0.f ? 0.f : mine.share * (log_s - (ref_of(mine.top) - from) / a.T));
    if (a.tail) {
        const float left = rest == 0.f ? 0.f : fmaxf(1.f - mine.given, 0.f);
        if (left > 0.f) loss += left * (log_s - log_rest);
    }
    if (bad) report(a.status, CCI_ERR_INDEX);
    a.loss[n] = bad ? nan_f() : loss;
    reinterpret_cast<float4 *>(a.stats)[n] = make_float4(bad ? nan_f() : m / a.T, log_s, log_rest, mine.norm);
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
    const float c = 1.f / a.T;
    row::Raw<T, 8> next[kU];
    auto load = [&](int e0) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int e = e0 + 8 * (32 * u + lane);
            next[u] = load_group(x, e < V ? e : V, V);
        }
    };
    load(lo);
    const float4 st = reinterpret_cast<const float4 *>(a.stats)[n];
    const float weight = a.dloss[n] / a.T, m = ref_of(st.x), log_s = st.y, log_rest = st.z;
    float whole, left = 0.f;  // Q, q_rest
    if (a.tail) {
        left = log_rest == neg_inf() ? 0.f : fmaxf(1.f - st.w, 0.f);
        whole = st.w + left;
    } else {
        whole = st.w == neg_inf() ? 0.f : 1.f;  // nothing listed
    }
    // the listed logits among these, read before any of them is written: dx may be x
    int at[kOwn];
    float own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int j = lane + i * 32;
        at[i] = j < a.k ? a.idx[n * a.k + j] : -1;
        if (at[i] < lo || at[i] >= hi) at[i] = -1;
        if (at[i] >= 0) {
            const float v = a.value[n * a.k + j];
            const float q = a.tail ? expf(v) : (whole == 0.f ? 0.f : expf(v * c - st.w));
            const float p = expf(fmaf(row::to_f32(x[at[i]]), c, -m) - log_s);
            own[i] = st.x == neg_inf() ? 0.f : (p * whole - q) * weight;
        }
    }
    // off the list: coef exp(z - m - shift).  With a tail, relative to the sum over the unlisted
    const bool some = a.tail && log_rest != neg_inf();
    const float shift = some ? log_rest : log_s;
    const float coef = (some ? whole * expf(log_rest - log_s) - left : whole) * weight;
    const unsigned long long c2 = pack2(c, c), neg = pack2(-m, -m), l2 = pack2(kLog2e, kLog2e), coef2 = pack2(coef, coef);
    const float minus = -shift * kLog2e;
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
                unsigned long long d = neg, y = pack2(minus, minus);
                ffma2(d, p[j], c2);
                ffma2(y, d, l2);
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

constexpr int kShort = 2048;  // rows of up to so many logits take two warps

template <typename T, int TPB>
cudaError_t launch_loss(Args a, cudaStream_t stream)
{
    // blocks of a row: about 1024 blocks in all, each with 4096 logits or more
    int parts = 1;
    while (parts < 8 && a.N * parts < 1024 && a.V / (2 * parts) >= 4096) parts *= 2;
    a.parts = parts;
    const int64_t groups = (static_cast<int64_t>(a.V) + 14) / 8;
    const int64_t each = ((groups + parts - 1) / parts + 31) / 32 * 32;
    const size_t bytes = static_cast<size_t>(each < kBits / 8 ? each : kBits / 8) + 16;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.N * parts));
    cfg.blockDim = dim3(TPB);
    cfg.dynamicSmemBytes = (bytes + 15) / 16 * 16;
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = static_cast<unsigned>(parts);
    la[0].val.clusterDim.y = 1;
    la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, loss_kernel<T, TPB>, static_cast<const Args>(a));
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

cudaError_t launch_distillation(const void *x, int dtype, int64_t N, int64_t V, int64_t ldx, const int32_t *idx,
                                const float *value, int k, float T, int tail, float *loss, float *stats,
                                uint32_t *status, cudaStream_t stream)
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
    if (dtype == CCI_F32) return V <= kShort ? launch_loss<float, 64>(a, stream) : launch_loss<float, 256>(a, stream);
    return V <= kShort ? launch_loss<uint16_t, 64>(a, stream) : launch_loss<uint16_t, 256>(a, stream);
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
