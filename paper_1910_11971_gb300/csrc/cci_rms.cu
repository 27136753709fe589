// cci_rms.cu -- root-mean-square norm of rows with the residual's addition, its form with an output in 8
// bits, and its backward pass.
//
//   s = x + residual,  h = s rounded,  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w
//   8 bits: per row or per 128 columns, scale = max(max|y| / 448, 2^-126), q = e4m3(y / scale)
//   dx = rstd (g - xh mean(g xh)) + dh,  dw = sum over n of dy xh,   g = dy w, xh = h rstd
//
// y is taken from the unrounded sum: one rounding each for y and h.  Memory bound: two reads and two writes of a row
// forward (one and one without a residual), three reads and a write backward.  A row belongs to a
// group of 32 to 1024 threads, which read it from memory once, into registers, and while they reduce it
// the next row is on its way.  The backward pass keeps each thread's columns of dw in registers over
// all rows of its block; the blocks' sums go to the workspace and a second launch adds them in block order.  All
// sums are fp32.  h may be the residual or x itself: a thread has read its columns of a row before it writes them.
#include "cci_kernels.h"
#include "cci_rowops.cuh"
#include "cci_tc_common.cuh"

namespace cci {
namespace rms {

constexpr float kE4m3Max = 448.f, kLeastScale = 1.17549435e-38f;

struct Forward {
    const void *x, *residual;
    int64_t ldx, ldr, N;
    int D;
    const float *w;
    float eps;
    void *y, *h;   // y: e4m3 where the scales are asked for
    float *rstd, *scales;
    int groups;    // scales of a row
};

struct Backward {
    const void *dy, *h, *dh;
    int64_t lddy, ldh, lddh, N;
    int D;
    const float *rstd, *w;
    void *dx;
    float *part;   // [blocks][D]
};

constexpr int block_threads(int TPR) { return TPR < 256 ? 256 : TPR; }
// blocks of an SM that the registers leave room for
constexpr int residents(int TPR) { return TPR <= 256 ? 3 : (TPR <= 512 ? 2 : 1); }

// a thread's columns of a row: vector i at (i * TPR + t) * V; zeros past D
template <typename T, int V, int NV, int TPR>
__device__ __forceinline__ void load_row(row::Raw<T, V> (&raw)[NV], const T *x, int t, int D)
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * V;
        raw[i] = c < D ? row::load_once<T, V>(x + c) : row::Raw<T, V>{};
    }
}

template <int V>
__device__ __forceinline__ void weight_at(const float *w, int c, int D, float (&v)[V])
{
    if (!w || c >= D) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = 1.f;
    } else if constexpr (V == 1) {
        v[0] = __ldg(w + c);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(w + c + j));
            v[j] = q.x;
            v[j + 1] = q.y;
            v[j + 2] = q.z;
            v[j + 3] = q.w;
        }
    }
}

// the larger; NaN if either is
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// four values as e4m3, to the nearest, ties to even; NaN stays
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n.reg .b16 lo, hi;\n"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        "mov.b32 %0, {lo, hi};\n}\n"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// the scale of values of up to `most`.  2^-126 at least, so that its reciprocal is finite: smaller values would be
// subnormal in fp32 themselves
__device__ __forceinline__ float scale_of(float most) { return max_nan(most / kE4m3Max, kLeastScale); }

// N values by their scale, each as the division rounds it.  The reciprocal is held in two fp32 numbers, the second what the first
// lacks of it (a double-length quotient: Dekker, "A floating-point technique for extending the available precision", 1971), so that
// one rounding is left, of a quotient 2^-30 off at most: a value at the middle of two codes stays there, which the product with the first
// alone moves now and then.  One operation a value more than that; divisions took 4000 x 8192 bf16 from 38.4 us to 44.6
template <int N>
__device__ __forceinline__ void by_scale(float (&y)[N], float scale)
{
    // of an infinite scale the second is 0, too
    const float high = 1.f / scale, low = fmaf(-high, fminf(scale, 3.402823466e38f), 1.f) * high;
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = fmaf(y[j], high, y[j] * low);
}

template <typename T, int V, int NV, int TPR, bool SUM, bool FP8>
__global__ void __launch_bounds__(block_threads(TPR), residents(TPR)) rms_kernel(const Forward p)
{
    constexpr int kGroups = block_threads(TPR) / TPR;
    constexpr bool kHold = TPR <= 256;  // the weight in registers
    __shared__ float buf[kGroups][2][TPR / 32], most_buf[kGroups][2][TPR / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = p.D;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    const T *x = static_cast<const T *>(p.x), *res = static_cast<const T *>(p.residual);
    row::Raw<T, V> raw[NV], rres[SUM ? NV : 1];
    if (n0 < p.N) {
        load_row<T, V, NV, TPR>(raw, x + n0 * p.ldx, t, D);
        if constexpr (SUM) load_row<T, V, NV, TPR>(rres, res + n0 * p.ldr, t, D);
    }
    float w[kHold ? NV : 1][V];
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < NV; ++i) weight_at<V>(p.w, (i * TPR + t) * V, D, w[i]);
    }
    int turn = 0;
    for (int64_t n = n0; n < p.N; n += step, turn ^= 1) {
        float f[NV][V], s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            row::unpack<T, V>(raw[i], f[i]);
            if constexpr (SUM) {
                float r[V];
                row::unpack<T, V>(rres[i], r);
#pragma unroll
                for (int j = 0; j < V; ++j) f[i][j] += r[j];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] = fmaf(f[i][j], f[i][j], s[0]);
        }
        if (n + step < p.N) {
            load_row<T, V, NV, TPR>(raw, x + (n + step) * p.ldx, t, D);
            if constexpr (SUM) load_row<T, V, NV, TPR>(rres, res + (n + step) * p.ldr, t, D);
        }
        if (SUM && p.h) {
            T *h = static_cast<T *>(p.h) + n * D;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * V;
                if (c < D) row::store<T, V>(h + c, f[i]);
            }
        }
        row::group_sum<TPR>(s, buf[group][turn], group, t);
        const float rstd = 1.f / sqrtf(s[0] / static_cast<float>(D) + p.eps);
        if (t == 0 && p.rstd) p.rstd[n] = rstd;
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * V;
            if constexpr (!kHold) weight_at<V>(p.w, c, D, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[i][j] = f[i][j] * rstd * w[kHold ? i : 0][j];
                if constexpr (FP8) most = max_nan(most, fabsf(f[i][j]));
            }
            if constexpr (!FP8) {
                if (c < D) row::store<T, V>(static_cast<T *>(p.y) + n * D + c, f[i]);
            }
        }
        if constexpr (FP8) {
            static_assert(!FP8 || V == 8, "sixteen lanes hold 128 columns");
            uint8_t *q = static_cast<uint8_t *>(p.y) + n * D;
            float scale = 1.f;
            if (p.groups == 1 && D > 128) {  // of the whole row
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
                if constexpr (TPR > 32) {
                    if ((t & 31) == 0) most_buf[group][turn][t >> 5] = most;
                    row::group_sync<TPR>(group);
                    most = (t & 31) < TPR / 32 ? most_buf[group][turn][t & 31] : 0.f;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
                }
                scale = scale_of(most);
                if (t == 0) p.scales[n] = scale;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * V;
                if (p.groups != 1 || D <= 128) {
                    float m = 0.f;
#pragma unroll
                    for (int j = 0; j < V; ++j) m = max_nan(m, fabsf(f[i][j]));
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                    scale = scale_of(m);
                    if (c < D && (t & 15) == 0) p.scales[n * p.groups + c / 128] = scale;
                }
                by_scale<V>(f[i], scale);
                if (c < D) {
                    uint2 b;
                    b.x = e4m3x4(f[i][0], f[i][1], f[i][2], f[i][3]);
                    b.y = e4m3x4(f[i][4], f[i][5], f[i][6], f[i][7]);
                    *reinterpret_cast<uint2 *>(q + c) = b;
                }
            }
        }
    }
}

// rows too long for registers: two passes, the second from L2 or memory.  Elements one by one
template <typename T, bool FP8>
__global__ void __launch_bounds__(1024) rms_long_kernel(const Forward p)
{
    __shared__ float buf[2][32];
    const int t = threadIdx.x, D = p.D;
    const int64_t n = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + n * p.ldx;
    const T *res = p.residual ? static_cast<const T *>(p.residual) + n * p.ldr : nullptr;
    T *h = res && p.h ? static_cast<T *>(p.h) + n * D : nullptr;
    auto at = [&](int c) { return row::to_f32(x[c]) + (res ? row::to_f32(res[c]) : 0.f); };
    float s[1] = {0.f};
    for (int c = t; c < D; c += 1024) {
        const float v = at(c);
        s[0] = fmaf(v, v, s[0]);
    }
    row::group_sum<1024>(s, buf[0], 0, t);
    const float rstd = 1.f / sqrtf(s[0] / static_cast<float>(D) + p.eps);
    if (t == 0 && p.rstd) p.rstd[n] = rstd;
    auto norm = [&](float v, int c) { return v * rstd * (p.w ? __ldg(p.w + c) : 1.f); };
    if constexpr (!FP8) {
        for (int c = t; c < D; c += 1024) {
            const float v = at(c), y = norm(v, c);
            if (h) row::store<T, 1>(h + c, &v);
            row::store<T, 1>(static_cast<T *>(p.y) + n * D + c, &y);
        }
    } else {
        uint8_t *q = static_cast<uint8_t *>(p.y) + n * D;
        float scale = 1.f;
        if (p.groups == 1) {
            float most = 0.f;
            for (int c = t; c < D; c += 1024) most = max_nan(most, fabsf(norm(at(c), c)));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
            if ((t & 31) == 0) buf[1][t >> 5] = most;
            __syncthreads();
            most = buf[1][t & 31];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
            scale = scale_of(most);
            if (t == 0) p.scales[n] = scale;
        }
        // a warp takes 128 columns at a time, four a lane
        for (int g = t >> 5; g < (D + 127) / 128; g += 32) {
            float v[4], y[4], most = 0.f;
            const int c0 = g * 128 + (t & 31) * 4;  // D is a multiple of 8
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = c0 < D ? at(c0 + j) : 0.f;
                y[j] = c0 < D ? norm(v[j], c0 + j) : 0.f;
                most = max_nan(most, fabsf(y[j]));
            }
            if (p.groups != 1) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
                scale = scale_of(most);
                if ((t & 31) == 0) p.scales[n * p.groups + g] = scale;
            }
            by_scale<4>(y, scale);
            if (c0 < D) {
                *reinterpret_cast<uint32_t *>(q + c0) = e4m3x4(y[0], y[1], y[2], y[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (h) row::store<T, 1>(h + c0 + j, v + j);
            }
        }
    }
}

// ---- backward ----
// a block's columns of dw: each thread's, or the sum of its groups' in their order
template <int V, int NV, int TPR>
__device__ __forceinline__ void write_columns(const float (&dw)[NV][V], float *part, float *sums, int group, int t, int D)
{
    constexpr int kGroups = block_threads(TPR) / TPR;
    if constexpr (kGroups > 1) {
        __syncthreads();  // sums may lie where rows were
        for (int g = 0; g < kGroups; ++g) {
            if (group == g) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (i * TPR + t) * V;
                    if (c < D) {
#pragma unroll
                        for (int j = 0; j < V; ++j) sums[c + j] = g == 0 ? dw[i][j] : sums[c + j] + dw[i][j];
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < D; c += block_threads(TPR)) part[c] = sums[c];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * V;
            if (c < D) row::store<float, V>(part + c, dw[i]);
        }
    }
}

// 16 bytes to shared memory, not through registers; `left`: the newest copies that are not waited for
__device__ __forceinline__ void copy_word(void *to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// Rows on 16-byte words: each thread copies its own columns of dy, h and dh of the next rows into places of its own
// in shared memory and reads them there, so that rows are on their way without registers and nobody waits for
// anybody's copies but their own (16384 x 4096 bf16: 94 us with the next row in registers)
template <typename T, int NV, int TPR, bool MORE>
struct Ring {
    static constexpr int kGroups = block_threads(TPR) / TPR, kArrays = MORE ? 3 : 2;
    static constexpr int kWords = static_cast<int>(sizeof(T)) / 2;  // of eight elements
    static constexpr int kBlocks = NV == 1 ? 3 : (TPR <= 256 ? 2 : 1);  // of an SM
    static constexpr int kStage = kArrays * NV * kWords * TPR * 16; // a row of a group
    static constexpr int kFit = 212 * 1024 / kBlocks / (kStage * kGroups);
    static constexpr int kStages = kFit < 1 ? 1 : (kFit < 4 ? kFit : 4);
    static constexpr int kBytes = kStages * kStage * kGroups;
    static_assert(kBytes <= static_cast<int>(kMaxSmemPerBlock) - 1024 && kBytes >= NV * 8 * TPR * 4, "the groups' sums fit");
};

template <typename T, int NV, int TPR, bool MORE>
__global__ void __launch_bounds__(block_threads(TPR), Ring<T, NV, TPR, MORE>::kBlocks) rms_backward_kernel(const Backward p)
{
    using R = Ring<T, NV, TPR, MORE>;
    constexpr int kGroups = R::kGroups, kStages = R::kStages, kWords = R::kWords;
    constexpr bool kHold = TPR < 1024;  // the weight, and a row's values between its two passes, in registers
    extern __shared__ __align__(16) unsigned char ring_raw[];
    __shared__ float buf[kGroups][2][TPR / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = p.D;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    // word `w` of this thread's eight i of array a in stage k
    uint4 *ring = reinterpret_cast<uint4 *>(ring_raw + group * kStages * R::kStage) + t;
    auto place = [&](int k, int a, int i, int w) { return ring + (((k * R::kArrays + a) * NV + i) * kWords + w) * TPR; };
    auto copy = [&](int64_t n, int k) {
#pragma unroll
        for (int a = 0; a < R::kArrays; ++a) {
            const T *x = a == 0 ? static_cast<const T *>(p.dy) + n * p.lddy
                                : (a == 1 ? static_cast<const T *>(p.h) + n * p.ldh : static_cast<const T *>(p.dh) + n * p.lddh);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * 8;
                if (c < D) {
#pragma unroll
                    for (int w = 0; w < kWords; ++w) copy_word(place(k, a, i, w), reinterpret_cast<const uint4 *>(x + c) + w);
                }
            }
        }
    };
    auto take = [&](int k, int a, int i, float (&f)[8]) {
        row::Raw<T, 8> raw{};
        if ((i * TPR + t) * 8 < D) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) raw.w[w] = *place(k, a, i, w);
        }
        row::unpack<T, 8>(raw, f);
    };
#pragma unroll
    for (int k = 0; k < kStages; ++k) {
        if (n0 + k * step < p.N) copy(n0 + k * step, k);
        copies_end();
    }
    float next_r = n0 < p.N ? p.rstd[n0] : 0.f;
    float w[kHold ? NV : 1][8], dw[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (kHold) weight_at<8>(p.w, (i * TPR + t) * 8, D, w[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
    }
    int turn = 0, k = 0;
    for (int64_t n = n0; n < p.N; n += step, turn ^= 1) {
        const float r = next_r;
        if (n + step < p.N) next_r = p.rstd[n + step];
        copies_wait<kStages - 1>();
        float g[kHold ? NV : 1][8], v[kHold ? NV : 1][8], s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            constexpr bool H = kHold;
            const int at = H ? i : 0;
            take(k, 0, i, g[at]);
            take(k, 1, i, v[at]);
            if constexpr (!kHold) weight_at<8>(p.w, (i * TPR + t) * 8, D, w[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[at][j] *= r;
                dw[i][j] = fmaf(g[at][j], v[at][j], dw[i][j]);
                g[at][j] *= w[at][j];
                s[0] = fmaf(g[at][j], v[at][j], s[0]);
            }
        }
        row::group_sum<TPR>(s, buf[group][turn], group, t);
        const float minus = -s[0] / static_cast<float>(D);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * 8, at = kHold ? i : 0;
            if constexpr (!kHold) {
                take(k, 0, i, g[0]);
                take(k, 1, i, v[0]);
                weight_at<8>(p.w, c, D, w[0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[0][j] *= r;
                    g[0][j] *= w[0][j];
                }
            }
            float o[8];
            if constexpr (MORE) take(k, 2, i, o);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = fmaf(v[at][j], minus, g[at][j]) * r;
                o[j] = MORE ? o[j] + d : d;
            }
            if (c < D) row::store<T, 8>(static_cast<T *>(p.dx) + n * D + c, o);
        }
        if (n + kStages * step < p.N) copy(n + kStages * step, k);  // what this thread has read
        copies_end();
        k = k + 1 == kStages ? 0 : k + 1;
    }
    copies_wait<0>();
    write_columns<8, NV, TPR>(dw, p.part + static_cast<int64_t>(blockIdx.x) * D, reinterpret_cast<float *>(ring_raw), group, t, D);
}

// fp32 rows on words, of which shared memory holds too few (8000 x 4096: 85 us, 135 through it), and all rows off
// them, element by element: the next row in registers.  dh is a row ahead for the latter alone (20000 x 777 bf16: 39 us, 63
// with dh and rstd loaded when they are needed; fp32 on words has no registers left, 109)
template <typename T, int V, int NV, int TPR, bool MORE>
__global__ void __launch_bounds__(block_threads(TPR), TPR <= 256 ? 2 : 1) rms_backward_registers_kernel(const Backward p)
{
    constexpr int kGroups = block_threads(TPR) / TPR;
    constexpr bool kHold = TPR < 1024, kAhead = V == 1;  // the weight in registers; dh a row ahead
    __shared__ float buf[kGroups][2][TPR / 32];
    extern __shared__ __align__(16) float sums[];  // [D] where a block has several groups
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = p.D;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    const T *dy = static_cast<const T *>(p.dy), *h = static_cast<const T *>(p.h), *dh = static_cast<const T *>(p.dh);
    row::Raw<T, V> rdy[NV], rh[NV], more[MORE && kAhead ? NV : 1];
    float next_r = 0.f;
    auto load = [&](int64_t n) {
        next_r = p.rstd[n];
        load_row<T, V, NV, TPR>(rdy, dy + n * p.lddy, t, D);
        load_row<T, V, NV, TPR>(rh, h + n * p.ldh, t, D);
        if constexpr (MORE && kAhead) load_row<T, V, NV, TPR>(more, dh + n * p.lddh, t, D);
    };
    if (n0 < p.N) load(n0);
    float w[kHold ? NV : 1][V], dw[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (kHold) weight_at<V>(p.w, (i * TPR + t) * V, D, w[i]);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = 0.f;
    }
    int turn = 0;
    for (int64_t n = n0; n < p.N; n += step, turn ^= 1) {
        const float r = next_r;
        float g[NV][V], v[NV][V], s[1] = {0.f};
        row::Raw<T, V> now[MORE ? NV : 1];
        if constexpr (MORE && kAhead) {
#pragma unroll
            for (int i = 0; i < NV; ++i) now[i] = more[i];
        } else if constexpr (MORE) {
            load_row<T, V, NV, TPR>(now, dh + n * p.lddh, t, D);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            row::unpack<T, V>(rdy[i], g[i]);
            row::unpack<T, V>(rh[i], v[i]);
            if constexpr (!kHold) weight_at<V>(p.w, (i * TPR + t) * V, D, w[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i][j] *= r;
                dw[i][j] = fmaf(g[i][j], v[i][j], dw[i][j]);
                g[i][j] *= w[kHold ? i : 0][j];
                s[0] = fmaf(g[i][j], v[i][j], s[0]);
            }
        }
        if (n + step < p.N) load(n + step);
        row::group_sum<TPR>(s, buf[group][turn], group, t);
        const float minus = -s[0] / static_cast<float>(D);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * V;
            float o[V];
            if constexpr (MORE) row::unpack<T, V>(now[i], o);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = fmaf(v[i][j], minus, g[i][j]) * r;
                o[j] = MORE ? o[j] + d : d;
            }
            if (c < D) row::store<T, V>(static_cast<T *>(p.dx) + n * D + c, o);
        }
    }
    write_columns<V, NV, TPR>(dw, p.part + static_cast<int64_t>(blockIdx.x) * D, sums, group, t, D);
}

// rows too long for registers: dx by two passes over each, dw's parts by columns (rows blockIdx.y, + parts, ...)
template <typename T>
__global__ void __launch_bounds__(1024) rms_backward_long_kernel(const Backward p)
{
    __shared__ float buf[32];
    const int t = threadIdx.x, D = p.D;
    const int64_t n = blockIdx.x;
    const T *dy = static_cast<const T *>(p.dy) + n * p.lddy, *h = static_cast<const T *>(p.h) + n * p.ldh;
    const T *dh = p.dh ? static_cast<const T *>(p.dh) + n * p.lddh : nullptr;
    const float r = p.rstd[n];
    float s[1] = {0.f};
    for (int c = t; c < D; c += 1024) s[0] = fmaf(row::to_f32(dy[c]) * (p.w ? __ldg(p.w + c) : 1.f), row::to_f32(h[c]) * r, s[0]);
    row::group_sum<1024>(s, buf, 0, t);
    const float minus = -s[0] / static_cast<float>(D);
    for (int c = t; c < D; c += 1024) {
        const float g = row::to_f32(dy[c]) * (p.w ? __ldg(p.w + c) : 1.f);
        float o = fmaf(row::to_f32(h[c]) * r, minus, g) * r;
        if (dh) o += row::to_f32(dh[c]);
        row::store<T, 1>(static_cast<T *>(p.dx) + n * D + c, &o);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) rms_columns_kernel(const Backward p)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.D) return;
    float s = 0.f;
    for (int64_t n = blockIdx.y; n < p.N; n += gridDim.y)
        s = fmaf(row::to_f32(static_cast<const T *>(p.dy)[n * p.lddy + c]),
                 row::to_f32(static_cast<const T *>(p.h)[n * p.ldh + c]) * p.rstd[n], s);
    p.part[static_cast<int64_t>(blockIdx.y) * p.D + c] = s;
}

// dw from the blocks' sums, in block order over 32 shares, whose sums are added in order.  A block takes 32 columns
__global__ void __launch_bounds__(1024) weight_kernel(const float *part, int parts, int D, float *dw)
{
    __shared__ float share[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float s = 0.f;
    tc::wait_prior_grid();
    if (c < D) {
#pragma unroll 8
        for (int i = y; i < parts; i += 32) s += part[static_cast<int64_t>(i) * D + c];
    }
    share[y][x] = s;
    __syncthreads();
    if (y == 0 && c < D) {
#pragma unroll
        for (int i = 1; i < 32; ++i) s += share[i][x];
        dw[c] = s;
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// columns that a row's registers hold: on words, and off them (backward 749 x 10523 bf16: 57 us element by element in
// registers, 46 by two passes)
constexpr int kLongest = 16384, kLongestOff = 8192;

// f(V, NV, TPR): vectors of V, NV of them a thread, TPR threads a row
template <typename Fn>
cudaError_t with_layout(bool words, int64_t D, Fn f)
{
    using std::integral_constant;
#define CCI_RMS_CASE(most, v, nv, tpr) \
    if (D <= most) return f(integral_constant<int, v>{}, integral_constant<int, nv>{}, integral_constant<int, tpr>{});
    if (words) {
        CCI_RMS_CASE(256, 8, 1, 32)
        CCI_RMS_CASE(512, 8, 2, 32)
        CCI_RMS_CASE(1024, 8, 1, 128)
        CCI_RMS_CASE(2048, 8, 2, 128)
        CCI_RMS_CASE(4096, 8, 2, 256)
        CCI_RMS_CASE(6144, 8, 2, 384)
        CCI_RMS_CASE(8192, 8, 2, 512)
        CCI_RMS_CASE(12288, 8, 2, 768)
        CCI_RMS_CASE(16384, 8, 2, 1024)
    } else {
        CCI_RMS_CASE(256, 1, 8, 32)
        CCI_RMS_CASE(1024, 1, 8, 128)
        CCI_RMS_CASE(2048, 1, 8, 256)
        CCI_RMS_CASE(4096, 1, 8, 512)
        CCI_RMS_CASE(8192, 1, 8, 1024)
    }
#undef CCI_RMS_CASE
    return cudaErrorInvalidValue;
}

unsigned blocks_of(int64_t N, int groups, int resident)
{
    const int64_t need = (N + groups - 1) / groups, most = static_cast<int64_t>(row::sm_count()) * resident;
    return static_cast<unsigned>(need < most ? need : most);
}

bool on_words(const void *p, int64_t ld, int es)
{
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0);
}

template <typename T, bool FP8>
cudaError_t forward(const Forward &p, cudaStream_t stream)
{
    constexpr int es = sizeof(T);
    const bool words = p.D % 8 == 0 && on_words(p.x, p.ldx, es) && on_words(p.residual, p.ldr, es) && on_words(p.w, 4, 4) &&
                       on_words(p.y, p.D, FP8 ? 2 : es) && on_words(p.h, p.D, es);
    if (FP8 && !words) return cudaErrorInvalidValue;
    if (p.D > (words ? kLongest : kLongestOff)) {
        rms_long_kernel<T, FP8><<<static_cast<unsigned>(p.N), 1024, 0, stream>>>(p);
        return cudaGetLastError();
    }
    return with_layout(words, p.D, [&](auto v, auto nv, auto tpr) {
        constexpr int V = decltype(v)::value, NV = decltype(nv)::value, TPR = decltype(tpr)::value;
        if constexpr (!FP8 || V == 8) {
            const unsigned blocks = blocks_of(p.N, block_threads(TPR) / TPR, residents(TPR));
            if (p.residual)
                rms_kernel<T, V, NV, TPR, true, FP8><<<blocks, block_threads(TPR), 0, stream>>>(p);
            else
                rms_kernel<T, V, NV, TPR, false, FP8><<<blocks, block_threads(TPR), 0, stream>>>(p);
            return cudaGetLastError();
        } else {
            return cudaErrorInvalidValue;
        }
    });
}

// blocks of the backward pass at most: their sums lie in the workspace
int64_t most_parts(int64_t N) { return N < 3 * row::sm_count() ? N : 3 * row::sm_count(); }

template <typename T, int NV, int TPR, bool MORE>
cudaError_t launch_ring(const Backward &p, unsigned blocks, cudaStream_t stream)
{
    using R = Ring<T, NV, TPR, MORE>;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(rms_backward_kernel<T, NV, TPR, MORE>, R::kBytes, attr_cache);
    if (attr != cudaSuccess) return attr;
    rms_backward_kernel<T, NV, TPR, MORE><<<blocks, block_threads(TPR), R::kBytes, stream>>>(p);
    return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const Backward &p, float *dw, cudaStream_t stream)
{
    constexpr int es = sizeof(T);
    unsigned parts = 0;
    cudaError_t e = cudaSuccess;
    const bool words = p.D % 8 == 0 && on_words(p.dy, p.lddy, es) && on_words(p.h, p.ldh, es) && on_words(p.dh, p.lddh, es) &&
                       on_words(p.w, 4, 4) && on_words(p.dx, p.D, es);
    if (p.D > (words ? kLongest : kLongestOff)) {
        const int64_t most = most_parts(p.N);
        parts = static_cast<unsigned>(most < 32 ? most : 32);
        rms_columns_kernel<T><<<dim3(static_cast<unsigned>((p.D + 255) / 256), parts), 256, 0, stream>>>(p);
        rms_backward_long_kernel<T><<<static_cast<unsigned>(p.N), 1024, 0, stream>>>(p);
        e = cudaGetLastError();
    } else {
        e = with_layout(words, p.D, [&](auto v, auto nv, auto tpr) {
            constexpr int V = decltype(v)::value, NV = decltype(nv)::value, TPR = decltype(tpr)::value;
            constexpr int kGroups = block_threads(TPR) / TPR;
            if constexpr (V == 8 && sizeof(T) == 2) {
                parts = blocks_of(p.N, kGroups, Ring<T, NV, TPR, true>::kBlocks);
                return p.dh ? launch_ring<T, NV, TPR, true>(p, parts, stream) : launch_ring<T, NV, TPR, false>(p, parts, stream);
            } else {
                parts = blocks_of(p.N, kGroups, TPR <= 256 ? 2 : 1);
                const size_t bytes = kGroups > 1 ? static_cast<size_t>(p.D) * sizeof(float) : 0;
                if (p.dh)
                    rms_backward_registers_kernel<T, V, NV, TPR, true><<<parts, block_threads(TPR), bytes, stream>>>(p);
                else
                    rms_backward_registers_kernel<T, V, NV, TPR, false><<<parts, block_threads(TPR), bytes, stream>>>(p);
                return cudaGetLastError();
            }
        });
    }
    if (e != cudaSuccess || !dw) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((p.D + 31) / 32));
    cfg.blockDim = dim3(1024);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, weight_kernel, const_cast<const float *>(p.part), static_cast<int>(parts), p.D, dw);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

}  // namespace rms

size_t rms_norm_workspace(int64_t N, int64_t D)
{
    return static_cast<size_t>(rms::most_parts(N)) * static_cast<size_t>(D) * sizeof(float);
}

cudaError_t launch_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, int dtype, int64_t N, int64_t D,
                            const float *w, float eps, void *y, void *h, float *rstd, float *scales, int groups,
                            cudaStream_t stream)
{
    rms::Forward p{x, residual, ldx, ldr, N, static_cast<int>(D), w, eps, y, h, rstd, scales, groups};
    if (dtype == CCI_F32) return scales ? rms::forward<float, true>(p, stream) : rms::forward<float, false>(p, stream);
    return scales ? rms::forward<uint16_t, true>(p, stream) : rms::forward<uint16_t, false>(p, stream);
}

cudaError_t launch_rms_norm_backward(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dh, int64_t lddh,
                                     int dtype, int64_t N, int64_t D, const float *rstd, const float *w, void *dx, float *dw,
                                     float *part, cudaStream_t stream)
{
    if (N == 0)  // no rows to sum over
        return dw ? cudaMemsetAsync(dw, 0, static_cast<size_t>(D) * sizeof(float), stream) : cudaSuccess;
    rms::Backward p{dy, h, dh, lddy, ldh, lddh, N, static_cast<int>(D), rstd, w, dx, part};
    return dtype == CCI_F32 ? rms::backward<float>(p, dw, stream) : rms::backward<uint16_t>(p, dw, stream);
}

}  // namespace cci
