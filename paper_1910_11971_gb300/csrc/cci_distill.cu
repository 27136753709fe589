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
    int parts, chunks;    // blocks of a row, forward and backward
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

// eight logits from e on; -inf outside of the row
template <typename T>
__device__ __forceinline__ void load_group(const T *row, int e, int V, float (&f)[8])
{
    if (e >= 0 && e + 8 <= V) {
        row::unpack<T, 8>(row::load_once<T, 8>(row + e), f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = e + j >= 0 && e + j < V ? row::to_f32(row[e + j]) : neg_inf();
    }
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
    const float *value = a.value + n * a.k;
    const float c = kLog2e / a.T;
    const int s = shift_of(x), V = a.V;
    const int groups = static_cast<int>((static_cast<int64_t>(V) + s + 7) / 8);
    const int each = ((groups + a.parts - 1) / a.parts + 31) / 32 * 32;
    const int first = part * each < groups ? part * each : groups, last = first + each < groups ? first + each : groups;
    // the first block's: the listed logits and the teacher's values, on their way meanwhile
    constexpr int kOwn = kMaxListed / 32;
    int32_t at[kOwn];
    float said[kOwn], listed[kOwn];
    if (part == 0 && t < 32) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int j = lane + 32 * i;
            at[i] = j < a.k ? idx[j] : -1;
            said[i] = j < a.k ? value[j] : 0.f;
            listed[i] = at[i] >= 0 && at[i] < V ? row::to_f32(x[at[i]]) : neg_inf();
        }
    }
    Sums sums{neg_inf(), 0.f};
    if (t == 0) bad_flag = 0;
    for (int g0 = first; g0 < last || g0 == first; g0 += kBits / 8) {
        const int g1 = g0 + kBits / 8 < last ? g0 + kBits / 8 : last;
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
        // the bounds are the same for a warp's lanes, so that they find their common maximum together
        for (int g = g0 + (t & ~31); g < g1; g += kU * TPB) {
            float f[kU][8];
            float top = neg_inf();
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int q = g + u * TPB + lane;
                if (q < g1) {
                    load_group(x, 8 * q - s, V, f[u]);
                    const uint32_t m = mask[q - g0];
                    if (m) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[u][j] = m >> j & 1u ? neg_inf() : f[u][j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[u][j] = neg_inf();
                }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, f[u][j]);
            asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
            if (top > sums.m) {
                sums.s = sums.s == 0.f ? 0.f : sums.s * ex2((sums.m - top) * c);
                sums.m = top;
            }
            const float from = ref_of(sums.m);
            float e[4] = {};
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j & 3] += ex2((f[u][j] - from) * c);
            sums.s += (e[0] + e[1]) + (e[2] + e[3]);
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
            sums.m = __shfl_sync(0xffffffffu, sums.m, 0);
            sums.s = __shfl_sync(0xffffffffu, sums.s, 0);
        }
    }
    if (t >= 32) return;
    // the first warp: the listed join, and the teacher has its say
    sums.m = __shfl_sync(0xffffffffu, sums.m, 0);
    sums.s = __shfl_sync(0xffffffffu, sums.s, 0);
    float top = neg_inf(), best = neg_inf();  // of the listed logits, of the teacher's values
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        top = fmaxf(top, listed[i]);
        if (at[i] >= 0) best = fmaxf(best, said[i]);
    }
    top = row::warp_max(top);
    best = row::warp_max(best);
    const float m = fmaxf(sums.m, top), from = ref_of(m), best_from = ref_of(best);
    float of_listed = 0.f, given = 0.f;
    float q[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        q[i] = 0.f;
        if (at[i] >= 0) {
            of_listed += expf((listed[i] - from) / a.T);
            q[i] = a.tail ? expf(said[i]) : expf((said[i] - best_from) / a.T);
            given += q[i];
        }
    }
    of_listed = row::warp_sum(of_listed);
    given = row::warp_sum(given);
    const float rest = sums.s == 0.f ? 0.f : sums.s * ex2((sums.m - from) * c);
    const float sum = rest + of_listed;
    const bool empty = m == neg_inf() && sum == 0.f;
    const float log_s = empty ? 0.f : logf(sum), log_rest = logf(rest);
    const float unit = a.tail || given == 0.f ? 1.f : 1.f / given;
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
        if (at[i] >= 0 && q[i] != 0.f) loss -= q[i] * unit * ((listed[i] - from) / a.T - log_s);
    loss = row::warp_sum(loss);
    if (a.tail) {
        const float left = rest == 0.f ? 0.f : fmaxf(1.f - given, 0.f);
        if (left > 0.f) loss += left * (log_s - log_rest);
    }
    if (lane == 0) {
        if (bad) report(a.status, CCI_ERR_INDEX);
        float *o = a.stats + 4 * n;
        a.loss[n] = bad ? nan_f() : loss;
        o[0] = bad ? nan_f() : m / a.T;
        o[1] = log_s;
        o[2] = log_rest;
        o[3] = a.tail ? given : (given == 0.f ? neg_inf() : logf(given) + best_from / a.T);
    }
}

// ---- gradient: a block takes kU groups a thread of a row ----
template <typename T, int TPB>
__global__ void __launch_bounds__(TPB) gradient_kernel(const Args a)
{
    constexpr int kU = 4;
    const int t = threadIdx.x;
    const int64_t n = blockIdx.x / a.chunks;
    const int chunk = static_cast<int>(blockIdx.x % a.chunks);
    const T *x = static_cast<const T *>(a.x) + n * a.ldx;
    T *dx = static_cast<T *>(a.dx) + n * a.lddx;
    const int s = shift_of(x), V = a.V, g0 = chunk * kU * TPB;
    const int64_t lo = 8 * static_cast<int64_t>(g0) - s, hi = lo + 8 * kU * TPB;
    const float c = 1.f / a.T;
    float f[kU][8];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int64_t e = lo + 8 * (u * TPB + t);
        if (e < V) load_group(x, static_cast<int>(e), V, f[u]);
    }
    const float4 st = reinterpret_cast<const float4 *>(a.stats)[n];
    const float weight = a.dloss[n] / a.T, m = ref_of(st.x), log_s = st.y, log_rest = st.z;
    // the listed logits of this block
    constexpr int kOwn = kMaxListed / TPB < 1 ? 1 : kMaxListed / TPB;
    int32_t at[kOwn];
    float own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        const int j = t + i * TPB;
        at[i] = j < a.k ? a.idx[n * a.k + j] : -1;
        if (at[i] < lo || at[i] >= hi || at[i] >= V) at[i] = -1;
    }
    float whole, left = 0.f;  // Q, q_rest
    if (a.tail) {
        left = log_rest == neg_inf() ? 0.f : fmaxf(1.f - st.w, 0.f);
        whole = st.w + left;
    } else {
        whole = st.w == neg_inf() ? 0.f : 1.f;  // nothing listed
    }
    const bool empty = st.x == neg_inf();
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        if (at[i] >= 0) {
            const float v = a.value[n * a.k + t + i * TPB];
            const float q = a.tail ? expf(v) : (whole == 0.f ? 0.f : expf(v * c - st.w));
            const float p = expf(fmaf(row::to_f32(x[at[i]]), c, -m) - log_s);
            own[i] = empty ? 0.f : (p * whole - q) * weight;
        }
    }
    // off the list: coef exp(z - m - shift).  With a tail, relative to the sum over the unlisted
    const bool some = a.tail && log_rest != neg_inf();
    const float shift = some ? log_rest : log_s;
    const float coef = (some ? whole * expf(log_rest - log_s) - left : whole) * weight;
    const float minus = -shift * kLog2e;
    __syncthreads();  // dx may be x: every listed logit has been read
    const bool words = shift_of(dx) == s;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const int64_t e64 = lo + 8 * (u * TPB + t);
        if (e64 >= V) continue;
        const int e = static_cast<int>(e64);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = ex2(fmaf(fmaf(f[u][j], c, -m), kLog2e, minus)) * coef;
            f[u][j] = empty ? 0.f : d;
        }
        if (words && e >= 0 && e + 8 <= V) {
            row::store<T, 8>(dx + e, f[u]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j >= 0 && e + j < V) row::store<T, 1>(dx + e + j, f[u] + j);
        }
    }
    __syncthreads();
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

template <typename T, int TPB>
cudaError_t launch_gradient(Args a, cudaStream_t stream)
{
    constexpr int64_t kLogits = 8 * 4 * TPB;
    a.chunks = static_cast<int>((static_cast<int64_t>(a.V) + 7 + kLogits - 1) / kLogits);
    if (a.N * a.chunks >= (int64_t(1) << 31)) return cudaErrorInvalidValue;
    gradient_kernel<T, TPB><<<static_cast<unsigned>(a.N * a.chunks), TPB, 0, stream>>>(a);
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
    if (dtype == CCI_F32)
        return V <= kShort ? launch_gradient<float, 64>(a, stream) : launch_gradient<float, 256>(a, stream);
    return V <= kShort ? launch_gradient<uint16_t, 64>(a, stream) : launch_gradient<uint16_t, 256>(a, stream);
}

}  // namespace cci
