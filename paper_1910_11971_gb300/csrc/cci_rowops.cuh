// cci_rowops.cuh -- helpers of the kernels that walk the rows of a matrix (layer norm,
// token log probabilities): typed loads and stores as fp32, sums over a group of threads.
#pragma once

#include "cci_common.cuh"

namespace cci {
namespace row {

// SMs of the current device (1 when it cannot be asked)
inline int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 1;
    return n;
}

// element types: float, or uint16_t for the bits of a bf16
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return bf16_bits_to_f32(v); }

// two fp32 values as bf16 bits (lo in the low half), to the nearest, ties to even
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// V consecutive elements as they lie in memory: 16-byte words (V = 8 and, for fp32, 4) or one element
template <typename T, int V>
struct Raw {
    static_assert(V * sizeof(T) % 16 == 0, "whole 16-byte words");
    uint4 w[V * sizeof(T) / 16];
};
template <typename T>
struct Raw<T, 1> {
    T w;
};

template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load(const T *p)
{
    Raw<T, V> r;
    if constexpr (V == 1) {
        r.w = *p;
    } else {
#pragma unroll
        for (int i = 0; i < static_cast<int>(V * sizeof(T) / 16); ++i) r.w[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    return r;
}

// the same for data read once: not kept in L1
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_once(const T *p)
{
    Raw<T, V> r;
    if constexpr (V == 1) {
        r.w = *p;
    } else {
#pragma unroll
        for (int i = 0; i < static_cast<int>(V * sizeof(T) / 16); ++i) {
            const uint4 *q = reinterpret_cast<const uint4 *>(p) + i;
            asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w)
                         : "l"(q));
        }
    }
    return r;
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const Raw<T, V> &r, float *f)
{
    if constexpr (V == 1) {
        f[0] = to_f32(r.w);
    } else {
#pragma unroll
        for (int i = 0; i < static_cast<int>(V * sizeof(T) / 16); ++i) {
            const uint32_t w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    f[4 * i + j] = __uint_as_float(w[j]);
                } else {
                    f[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                    f[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            }
        }
    }
}

template <typename T, int V>
__device__ __forceinline__ void store(T *p, const float *f)
{
    if constexpr (sizeof(T) == 4 && V == 1) {
        *p = f[0];
    } else if constexpr (V == 1) {
        *p = static_cast<uint16_t>(bf16x2(f[0], 0.f));
    } else {
#pragma unroll
        for (int i = 0; i < static_cast<int>(V * sizeof(T) / 16); ++i) {
            uint4 w;
            if constexpr (sizeof(T) == 4)
                w = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]),
                               __float_as_uint(f[4 * i + 3]));
            else
                w = make_uint4(bf16x2(f[8 * i], f[8 * i + 1]), bf16x2(f[8 * i + 2], f[8 * i + 3]),
                               bf16x2(f[8 * i + 4], f[8 * i + 5]), bf16x2(f[8 * i + 6], f[8 * i + 7]));
            reinterpret_cast<uint4 *>(p)[i] = w;
        }
    }
}

// two fp32 at a time (one instruction for both; ffma2 of cci_common.cuh is the third of them)
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// the elements of a vector (V > 1) as V / 2 pairs; pairs to memory
template <typename T, int V>
__device__ __forceinline__ void unpack2(const Raw<T, V> &r, unsigned long long *p)
{
    float f[V];
    unpack<T, V>(r, f);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) p[j] = pack2(f[2 * j], f[2 * j + 1]);
}

template <typename T, int V>
__device__ __forceinline__ void store2(T *to, const unsigned long long *p)
{
    float f[V];
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        f[2 * j] = lo_of(p[j]);
        f[2 * j + 1] = hi_of(p[j]);
    }
    store<T, V>(to, f);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// barrier over the TPR threads of row group `group` of a block (whole warps)
template <int TPR>
__device__ __forceinline__ void group_sync(int group)
{
    if constexpr (TPR == 32)
        __syncwarp();
    else
        asm volatile("barrier.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
}

// sum of each of v[0..N) over the TPR threads of a group, to every thread of it.  `buf`:
// the group's N * TPR / 32 floats, not in use by an earlier sum that some thread may
// still read (two buffers taken in turn are enough: a thread enters the sum after next
// only when all have left this one)
template <int TPR, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float *buf, int group, int t)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if constexpr (TPR > 32) {
        constexpr int kW = TPR / 32;
        if ((t & 31) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) buf[i * kW + (t >> 5)] = v[i];
        }
        group_sync<TPR>(group);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = (t & 31) < kW ? buf[i * kW + (t & 31)] : 0.f;
            v[i] = warp_sum(s);
        }
    }
}

// the same for four values at once, which share the steps: a lane carries one of them from the third on (13
// exchanges in all, 40 for four sums apart)
template <int TPR>
__device__ __forceinline__ void group_sum4(float (&v)[4], float *buf, int group, int t)
{
    const int lane = t & 31;
    const bool hi = lane & 16, up = lane & 8;
    float a = hi ? v[2] : v[0], b = hi ? v[3] : v[1];
    a += __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
    b += __shfl_xor_sync(0xffffffffu, hi ? v[1] : v[3], 16);
    float s = up ? b : a;
    s += __shfl_xor_sync(0xffffffffu, up ? a : b, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if constexpr (TPR > 32) {
        constexpr int kW = TPR / 32;
        const int mine = lane >> 3, j = lane & 7;
        if (j == 0) buf[mine * kW + (t >> 5)] = s;
        group_sync<TPR>(group);
        s = j < kW ? buf[mine * kW + j] : 0.f;
#pragma unroll
        for (int w = 8; w < kW; w += 8) s += buf[mine * kW + w + j];
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xffffffffu, s, 8 * i);
}

}  // namespace row
}  // namespace cci
