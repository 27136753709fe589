// cci_norm.cu -- layer norm of rows, forward and backward.
//
//   y[n][c]  = (x[n][c] - mean[n]) * rstd[n] * w[c] + b[c],   rstd = 1 / sqrt(var + eps)
//   dx       = rstd * (g - mean(g) - xh * mean(g * xh)),      g = dy * w, xh = (x - mean) * rstd
//   dw[c]    = sum over n of dy * xh,  db[c] = sum over n of dy
//
// Memory bound in both directions (two or three row reads and writes, a dozen operations an
// element).  A row belongs to a group of 32 to 1024 threads that holds it in registers: the
// variance is the mean square of the differences from the mean, not a difference of sums, and
// nothing is read twice.  The backward pass keeps each thread's columns of dw and db in
// registers over all rows of its block; the blocks' sums go to the workspace and a second
// launch adds them in block order, so the result does not depend on what finishes first.
// All sums are fp32.
#include "cci_kernels.h"
#include "cci_rowops.cuh"

namespace cci {
namespace norm {

// threads of a block with row groups of TPR threads
constexpr int block_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

// blocks of an SM that the register limit leaves room for
constexpr int forward_residents(int TPR) { return TPR <= 256 ? 3 : (TPR == 512 ? 2 : 1); }
constexpr int backward_residents(int TPR) { return TPR <= 256 ? 2 : 1; }

// V consecutive fp32 parameters from p[c] on, or `missing` where there are none
template <int V>
__device__ __forceinline__ void params_at(const float *p, int c, float missing, float *v)
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = missing;
    } else if constexpr (V == 1) {
        v[0] = __ldg(p + c);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(p + c + j));
            v[j] = q.x;
            v[j + 1] = q.y;
            v[j + 2] = q.z;
            v[j + 3] = q.w;
        }
    }
}

// a thread's columns of a row: vector i at (i * TPR + t) * V
template <typename T, int V, int NV, int TPR>
__device__ __forceinline__ void load_row(row::Raw<T, V> (&raw)[NV], const T *x, int t, int D)
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * V;
        if (c < D) raw[i] = row::load_once<T, V>(x + c);
    }
}

// ---- forward: E columns per thread, in vectors of V.  Groups walk the rows; the next row's loads are on
// their way while this one is reduced.  Rows of up to 4096 keep weight and bias in registers ----
template <typename T, int V, int E, int TPR>
__global__ void __launch_bounds__(block_threads(TPR), forward_residents(TPR))
    norm_kernel(const T *x, int64_t ldx, int64_t N, int D, const float *w, const float *b, float eps, T *y, float *mean,
                float *rstd)
{
    constexpr int kGroups = block_threads(TPR) / TPR, kNV = E / V;
    constexpr bool kHold = TPR <= 256;
    __shared__ float buf[kGroups][2][TPR / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float width = static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    int64_t n = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    float wv[kHold ? E : V], bv[kHold ? E : V];
    row::Raw<T, V> raw[kNV];
    if (n < N) load_row<T, V, kNV, TPR>(raw, x + n * ldx, t, D);
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (i * TPR + t) * V;
            if (c < D) {
                params_at<V>(w, c, 1.f, wv + i * V);
                params_at<V>(b, c, 0.f, bv + i * V);
            }
        }
    }
    for (; n < N; n += step) {
        float f[E];
        float s[1] = {0.f}, q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            if ((i * TPR + t) * V < D) {
                row::unpack<T, V>(raw[i], f + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) s[0] += f[i * V + j];
            }
        }
        if (n + step < N) load_row<T, V, kNV, TPR>(raw, x + (n + step) * ldx, t, D);
        row::group_sum<TPR>(s, buf[group][0], group, t);
        const float mu = s[0] / width;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            if ((i * TPR + t) * V < D) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    f[i * V + j] -= mu;
                    q[0] += f[i * V + j] * f[i * V + j];
                }
            }
        }
        row::group_sum<TPR>(q, buf[group][1], group, t);
        const float r = 1.f / sqrtf(q[0] / width + eps);
        if (t == 0) {
            mean[n] = mu;
            rstd[n] = r;
        }
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (i * TPR + t) * V, h = kHold ? i * V : 0;
            if (c < D) {
                if constexpr (!kHold) {
                    params_at<V>(w, c, 1.f, wv);
                    params_at<V>(b, c, 0.f, bv);
                }
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = f[i * V + j] * r * wv[h + j] + bv[h + j];
                row::store<T, V>(y + n * D + c, o);
            }
        }
    }
}

// ---- forward, rows too long for registers: three passes over the row ----
template <typename T>
__global__ void __launch_bounds__(1024)
    norm_long_kernel(const T *x, int64_t ldx, int64_t N, int64_t D, const float *w, const float *b, float eps, T *y,
                     float *mean, float *rstd)
{
    __shared__ float buf[2][32];
    const int t = threadIdx.x;
    for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
        const T *xr = x + n * ldx;
        float s[1] = {0.f}, q[1] = {0.f};
        for (int64_t c = t; c < D; c += 1024) s[0] += row::to_f32(xr[c]);
        row::group_sum<1024>(s, buf[0], 0, t);
        const float mu = s[0] / static_cast<float>(D);
        for (int64_t c = t; c < D; c += 1024) {
            const float d = row::to_f32(xr[c]) - mu;
            q[0] += d * d;
        }
        row::group_sum<1024>(q, buf[1], 0, t);
        const float r = 1.f / sqrtf(q[0] / static_cast<float>(D) + eps);
        if (t == 0) {
            mean[n] = mu;
            rstd[n] = r;
        }
        for (int64_t c = t; c < D; c += 1024) {
            const float o = (row::to_f32(xr[c]) - mu) * r * (w ? w[c] : 1.f) + (b ? b[c] : 0.f);
            row::store<T, 1>(y + n * D + c, &o);
        }
    }
}

// ---- backward: dx, and this block's sums of dw and db into part[block][2][D] ----
template <typename T, int V, int E, int TPR>
__global__ void __launch_bounds__(block_threads(TPR), backward_residents(TPR))
    norm_backward_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx, const float *mean, const float *rstd,
                         const float *w, int64_t N, int D, T *dx, float *part)
{
    constexpr int kGroups = block_threads(TPR) / TPR, kNV = E / V;
    // 1024 threads leave no registers to hold x and dy besides dw and db: they are read again
    // (from L1) for dx
    constexpr bool kAgain = TPR == 1024;
    __shared__ float buf[kGroups][2][2 * TPR / 32];
    __shared__ float comb[kGroups > 1 ? 2 * E * TPR : 1];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float width = static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    float dw[E], db[E], wv[kAgain ? V : E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
    int64_t n = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    row::Raw<T, V> rx[kAgain ? 1 : kNV], rd[kAgain ? 1 : kNV];
    float mu = 0.f, r = 0.f;
    if constexpr (!kAgain) {
        if (n < N) {
            load_row<T, V, kNV, TPR>(rx, x + n * ldx, t, D);
            load_row<T, V, kNV, TPR>(rd, dy + n * lddy, t, D);
            mu = __ldg(mean + n);
            r = __ldg(rstd + n);
        }
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if ((i * TPR + t) * V < D) params_at<V>(w, (i * TPR + t) * V, 1.f, wv + i * V);
    }
    int k = 0;
    for (; n < N; n += step, k ^= 1) {
        constexpr int kHold = kAgain ? V : E;
        float xh[kHold], g[kHold];
        float s[2] = {0.f, 0.f};
        if constexpr (kAgain) {
            mu = __ldg(mean + n);
            r = __ldg(rstd + n);
        }
        const float rn = r;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (i * TPR + t) * V, h = kAgain ? 0 : i * V;
            if (c < D) {
                if constexpr (kAgain) {
                    rx[0] = row::load<T, V>(x + n * ldx + c);
                    rd[0] = row::load<T, V>(dy + n * lddy + c);
                    params_at<V>(w, c, 1.f, wv);
                }
                row::unpack<T, V>(rx[kAgain ? 0 : i], xh + h);
                row::unpack<T, V>(rd[kAgain ? 0 : i], g + h);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    xh[h + j] = (xh[h + j] - mu) * rn;
                    dw[i * V + j] += g[h + j] * xh[h + j];
                    db[i * V + j] += g[h + j];
                    g[h + j] *= wv[h + j];
                    s[0] += g[h + j];
                    s[1] += g[h + j] * xh[h + j];
                }
            }
        }
        if constexpr (!kAgain) {
            if (n + step < N) {
                load_row<T, V, kNV, TPR>(rx, x + (n + step) * ldx, t, D);
                load_row<T, V, kNV, TPR>(rd, dy + (n + step) * lddy, t, D);
                mu = __ldg(mean + n + step);
                r = __ldg(rstd + n + step);
            }
        }
        row::group_sum<TPR>(s, buf[group][k], group, t);
        const float a = s[0] / width, bq = s[1] / width;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (i * TPR + t) * V, h = kAgain ? 0 : i * V;
            if (c < D) {
                if constexpr (kAgain) {
                    row::unpack<T, V>(row::load<T, V>(x + n * ldx + c), xh);
                    row::unpack<T, V>(row::load<T, V>(dy + n * lddy + c), g);
                    params_at<V>(w, c, 1.f, wv);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        xh[j] = (xh[j] - mu) * rn;
                        g[j] *= wv[j];
                    }
                }
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = (g[h + j] - a - xh[h + j] * bq) * rn;
                row::store<T, V>(dx + n * D + c, o);
            }
        }
    }
    // the groups' sums, added in group order
    if constexpr (kGroups > 1) {
        for (int q = 1; q < kGroups; ++q) {
            __syncthreads();
            if (group == q) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    comb[(2 * e) * TPR + t] = dw[e];
                    comb[(2 * e + 1) * TPR + t] = db[e];
                }
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    dw[e] += comb[(2 * e) * TPR + t];
                    db[e] += comb[(2 * e + 1) * TPR + t];
                }
            }
        }
    }
    if (group == 0) {
        float *pw = part + static_cast<int64_t>(blockIdx.x) * 2 * D;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (i * TPR + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (c < D) {
                    pw[c + j] = dw[i * V + j];
                    pw[D + c + j] = db[i * V + j];
                }
            }
        }
    }
}

// ---- backward, rows too long for registers: dx in two passes over the row ----
template <typename T>
__global__ void __launch_bounds__(1024)
    norm_long_dx_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx, const float *mean, const float *rstd,
                        const float *w, int64_t N, int64_t D, T *dx)
{
    __shared__ float buf[2][64];
    const int t = threadIdx.x;
    int k = 0;
    for (int64_t n = blockIdx.x; n < N; n += gridDim.x, k ^= 1) {
        const T *xr = x + n * ldx, *dr = dy + n * lddy;
        const float mu = mean[n], r = rstd[n];
        float s[2] = {0.f, 0.f};
        for (int64_t c = t; c < D; c += 1024) {
            const float g = row::to_f32(dr[c]) * (w ? w[c] : 1.f);
            s[0] += g;
            s[1] += g * (row::to_f32(xr[c]) - mu) * r;
        }
        row::group_sum<1024>(s, buf[k], 0, t);
        const float a = s[0] / static_cast<float>(D), bq = s[1] / static_cast<float>(D);
        for (int64_t c = t; c < D; c += 1024) {
            const float g = row::to_f32(dr[c]) * (w ? w[c] : 1.f);
            const float o = (g - a - (row::to_f32(xr[c]) - mu) * r * bq) * r;
            row::store<T, 1>(dx + n * D + c, &o);
        }
    }
}

// the sums of dw and db over the rows of one of gridDim.y parts, for such rows
template <typename T>
__global__ void __launch_bounds__(256)
    norm_long_params_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx, const float *mean, const float *rstd,
                            int64_t N, int64_t D, float *part)
{
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= D) return;
    float dw = 0.f, db = 0.f;
    for (int64_t n = blockIdx.y; n < N; n += gridDim.y) {
        const float g = row::to_f32(dy[n * lddy + c]);
        dw += g * (row::to_f32(x[n * ldx + c]) - __ldg(mean + n)) * __ldg(rstd + n);
        db += g;
    }
    float *pw = part + static_cast<int64_t>(blockIdx.y) * 2 * D;
    pw[c] = dw;
    pw[D + c] = db;
}

// dw and db: the sums of the parts (32 columns and 32 interleaved shares of the parts a block, the
// shares added in order)
__global__ void __launch_bounds__(1024)
    norm_params_kernel(const float *part, int parts, int64_t D, float *dw, float *db)
{
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, q = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float s = 0.f;
    if (c < 2 * D) {
#pragma unroll 8
        for (int p = q; p < parts; p += 32) s += part[static_cast<int64_t>(p) * 2 * D + c];
    }
    sh[q][lane] = s;
    __syncthreads();
    // warp q adds column q's shares
    s = row::warp_sum(sh[lane][q]);
    const int64_t d = static_cast<int64_t>(blockIdx.x) * 32 + q;
    if (lane == 0 && d < 2 * D) {
        if (d < D) {
            if (dw) dw[d] = s;
        } else if (db) {
            db[d - D] = s;
        }
    }
}

constexpr int64_t kRegisterColumns = 16384;  // widest row that a block holds

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

struct Args {
    const void *dy, *x;
    int64_t lddy, ldx, N, D;
    const float *w, *b, *mean_in, *rstd_in;
    float eps;
    void *y;
    float *mean, *rstd, *part;
    int *parts;  // written: parts of the sums
    cudaStream_t stream;
};

// columns of a thread: two 16-byte words, or 8 single elements; twice that past 8192 columns, which 1024
// threads share
template <typename T, int V>
constexpr int thread_columns()
{
    return V == 8 ? 16 : 8;
}

// threads of a row group with `e` columns each, a warp at least
int group_threads(int e, int64_t D)
{
    int t = 32;
    while (t < 1024 && static_cast<int64_t>(t) * e < D) t *= 2;
    return t;
}

// blocks of the backward pass' main launch (and parts of its sums)
int64_t backward_blocks(int e, int64_t N, int64_t D)
{
    if (D > kRegisterColumns) return least(N, 16);
    const int tpr = group_threads(e, D), groups = block_threads(tpr) / tpr;
    return least((N + groups - 1) / groups, static_cast<int64_t>(row::sm_count()) * backward_residents(tpr));
}

// the most parts of any form of a call
int64_t most_parts(int64_t N, int64_t D)
{
    const int64_t a = backward_blocks(8, N, D), b = backward_blocks(16, N, D);
    return a > b ? a : b;
}

template <typename T, int V, int E, int TPR>
cudaError_t forward_one(const Args &a)
{
    constexpr int kT = block_threads(TPR), kGroups = kT / TPR;
    const int64_t blocks = least((a.N + kGroups - 1) / kGroups, static_cast<int64_t>(row::sm_count()) * forward_residents(TPR));
    norm_kernel<T, V, E, TPR><<<static_cast<unsigned>(blocks), kT, 0, a.stream>>>(
        static_cast<const T *>(a.x), a.ldx, a.N, static_cast<int>(a.D), a.w, a.b, a.eps, static_cast<T *>(a.y), a.mean,
        a.rstd);
    return cudaGetLastError();
}

template <typename T, int V, int E, int TPR>
cudaError_t backward_one(const Args &a)
{
    *a.parts = static_cast<int>(backward_blocks(thread_columns<T, V>(), a.N, a.D));
    norm_backward_kernel<T, V, E, TPR><<<static_cast<unsigned>(*a.parts), block_threads(TPR), 0, a.stream>>>(
        static_cast<const T *>(a.dy), a.lddy, static_cast<const T *>(a.x), a.ldx, a.mean_in, a.rstd_in, a.w, a.N,
        static_cast<int>(a.D), static_cast<T *>(a.y), a.part);
    return cudaGetLastError();
}

template <typename T, int V, bool BACKWARD, int TPR>
cudaError_t launch_group(const Args &a)
{
    constexpr int E = thread_columns<T, V>();
    if constexpr (BACKWARD)
        return backward_one<T, V, E, TPR>(a);
    else
        return forward_one<T, V, E, TPR>(a);
}

template <typename T, int V, bool BACKWARD>
cudaError_t launch_rows(const Args &a)
{
    constexpr int E = thread_columns<T, V>();
    if (E == 8 && a.D > 8192) {
        if constexpr (BACKWARD)
            return backward_one<T, V, 16, 1024>(a);
        else
            return forward_one<T, V, 16, 1024>(a);
    }
    switch (group_threads(E, a.D)) {
        case 32: return launch_group<T, V, BACKWARD, 32>(a);
        case 64: return launch_group<T, V, BACKWARD, 64>(a);
        case 128: return launch_group<T, V, BACKWARD, 128>(a);
        case 256: return launch_group<T, V, BACKWARD, 256>(a);
        case 512: return launch_group<T, V, BACKWARD, 512>(a);
        default: return launch_group<T, V, BACKWARD, 1024>(a);
    }
}

// whole 16-byte words: every row of every array starts on one, and D ends on one
template <typename T>
bool whole_words(const Args &a)
{
    constexpr int64_t v = 16 / sizeof(T);
    auto at16 = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    return a.D % v == 0 && a.ldx % v == 0 && at16(a.x) && at16(a.y) && at16(a.w) && at16(a.b) &&
           (!a.dy || (a.lddy % v == 0 && at16(a.dy)));
}

template <typename T>
cudaError_t forward(const Args &a)
{
    if (a.D > kRegisterColumns) {
        norm_long_kernel<T><<<static_cast<unsigned>(least(a.N, 2 * row::sm_count())), 1024, 0, a.stream>>>(
            static_cast<const T *>(a.x), a.ldx, a.N, a.D, a.w, a.b, a.eps, static_cast<T *>(a.y), a.mean, a.rstd);
        return cudaGetLastError();
    }
    return whole_words<T>(a) ? launch_rows<T, 16 / sizeof(T), false>(a) : launch_rows<T, 1, false>(a);
}

template <typename T>
cudaError_t backward(const Args &a)
{
    if (a.D > kRegisterColumns) {
        norm_long_dx_kernel<T><<<static_cast<unsigned>(least(a.N, 2 * row::sm_count())), 1024, 0, a.stream>>>(
            static_cast<const T *>(a.dy), a.lddy, static_cast<const T *>(a.x), a.ldx, a.mean_in, a.rstd_in, a.w, a.N,
            a.D, static_cast<T *>(a.y));
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess || !a.part) return e;
        *a.parts = static_cast<int>(backward_blocks(8, a.N, a.D));
        const dim3 grid(static_cast<unsigned>((a.D + 255) / 256), static_cast<unsigned>(*a.parts));
        norm_long_params_kernel<T><<<grid, 256, 0, a.stream>>>(static_cast<const T *>(a.dy), a.lddy,
                                                               static_cast<const T *>(a.x), a.ldx, a.mean_in,
                                                               a.rstd_in, a.N, a.D, a.part);
        return cudaGetLastError();
    }
    return whole_words<T>(a) ? launch_rows<T, 16 / sizeof(T), true>(a) : launch_rows<T, 1, true>(a);
}

}  // namespace norm

size_t layer_norm_workspace(int64_t N, int64_t D)
{
    return static_cast<size_t>(norm::most_parts(N, D)) * 2 * static_cast<size_t>(D) * sizeof(float);
}

cudaError_t launch_layer_norm(const void *x, int dtype, int64_t N, int64_t D, int64_t ldx, const float *w,
                              const float *b, float eps, void *y, float *mean, float *rstd, cudaStream_t stream)
{
    norm::Args a{};
    a.x = x;
    a.ldx = ldx;
    a.N = N;
    a.D = D;
    a.w = w;
    a.b = b;
    a.eps = eps;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.stream = stream;
    return dtype == CCI_F32 ? norm::forward<float>(a) : norm::forward<uint16_t>(a);
}

cudaError_t launch_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, int dtype, int64_t N,
                                       int64_t D, const float *mean, const float *rstd, const float *w, void *dx,
                                       float *dw, float *db, float *part, cudaStream_t stream)
{
    norm::Args a{};
    a.dy = dy;
    a.lddy = lddy;
    a.x = x;
    a.ldx = ldx;
    a.N = N;
    a.D = D;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.w = w;
    a.y = dx;
    int parts = 0;
    a.part = part;
    a.parts = &parts;
    a.stream = stream;
    if (N > 0) {
        const cudaError_t e = dtype == CCI_F32 ? norm::backward<float>(a) : norm::backward<uint16_t>(a);
        if (e != cudaSuccess) return e;
    }
    if (!dw && !db) return cudaSuccess;
    norm::norm_params_kernel<<<static_cast<unsigned>((2 * D + 31) / 32), 1024, 0, stream>>>(
        part, parts, D, dw, db);
    return cudaGetLastError();
}

}  // namespace cci
