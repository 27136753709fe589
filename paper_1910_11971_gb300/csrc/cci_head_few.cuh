// cci_head_few.cuh -- the cross entropy of up to 32 tokens from a head's fp32 inputs.
//
// The head's weights are all that is read, once, as they are: writing W's planes first, as for more tokens
// (cci_head.cu), moves four times its bytes (2 tokens, 3392 x 4076: 96 us, 26 so; 16 tokens, 4096 x 65536 fp32 240 us of
// 158 at the copy rate).  A warp takes 32 entries of the vocabulary and an eighth of the reduction, straight from memory into
// the fragments of mma.sync: 32 elements of a row lie with four lanes, eight each, and X is read in the same order, so that the
// order of the reduction within a step does not matter.  Values become three bf16 planes in registers, cut to eight
// bits each; the six products of planes are those of cci_gated.cuh.  The warps' sums meet in shared memory, where each
// token's maximum and sum of exponentials are taken.  bf16 tokens, however few, go by the tiles of cci_head.cu, whose copies
// keep more on its way (1 token, 4096 x 131072: 203 us through here, 166 so).
#pragma once

#include "cci_kernels.h"
#include "cci_rowops.cuh"
#include "cci_tc_common.cuh"

namespace cci {
namespace head {

constexpr int kFewTokens = 32, kFewRows = 32, kFewWarps = 8;

struct FewParams {
    const uint16_t *x;   // three planes [N][D]
    const float *w;      // [V][D]
    int N, D;
    int64_t V;
    int groups;          // of 32 entries, a block
    const int64_t *targets;
    int64_t ignore;
    float2 *parts;       // [blocks][N]
    float *at_target;    // [N]
};

// the upper halves of a and b as bf16 (a in the low half), which become what that leaves.  Cut, not rounded: eight
// bits a plane, so that three hold all 24 (4 operations a value; to the nearest, with its care for the ends, took a 256 x 256
// tile's output 15 us more)
__device__ __forceinline__ uint32_t next_planes(float &a, float &b)
{
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    a -= __uint_as_float(x & 0xffff0000u);
    b -= __uint_as_float(y & 0xffff0000u);
    return __byte_perm(x, y, 0x7632);
}

// d += a b: 16 rows of a, 8 columns of b, 16 indices
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// NT: eights of tokens, and tokens that a warp sums up
template <int NT>
__global__ void __launch_bounds__(kFewWarps * 32, NT <= 2 ? 2 : 1) few_kernel(const FewParams p)
{
    constexpr int kPlanes = 3, kPitch = 8 * NT + 1;
    __shared__ float sums[kFewWarps][kFewRows][kPitch];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const float *w = p.w;
    const int steps = (p.D + 31) / 32, from = steps * warp / kFewWarps, to = steps * (warp + 1) / kFewWarps;
    const int64_t plane = static_cast<int64_t>(p.N) * p.D;
    // tokens NT warp + i: what their entries so far say
    float most[NT], total[NT] = {};
#pragma unroll
    for (int i = 0; i < NT; ++i) most[i] = __int_as_float(0xff800000);
    tc::launch_next_grid();  // which waits for this one's end
    for (int group = 0; group < p.groups; ++group) {
        const int64_t v0 = (static_cast<int64_t>(blockIdx.x) * p.groups + group) * kFewRows;
        if (v0 >= p.V) break;
        float acc[2][NT][4] = {}, sum[2][NT][4] = {};
        for (int b = from; b < to; ++b) {
            const int k = 32 * b + 8 * q;
            uint4 a[2][2][2] = {};  // 16 rows, the first or the last eight of them, 16 of the 32 indices
            uint4 x[kPlanes][NT] = {};
            if (k < p.D) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t v = v0 + 16 * m + 8 * h + g;
                        if (v < p.V) {
                            const row::Raw<float, 8> r = row::load_once<float, 8>(w + v * p.D + k);
                            a[m][h][0] = r.w[0];
                            a[m][h][1] = r.w[1];
                        }
                    }
#pragma unroll
                for (int s = 0; s < kPlanes; ++s)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (8 * n + g < p.N)
                            x[s][n] = __ldg(reinterpret_cast<const uint4 *>(p.x + s * plane + static_cast<int64_t>(8 * n + g) * p.D + k));
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int half = 0; half < 2; ++half) {  // 16 of the 32 indices
                    uint32_t f[kPlanes][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 word = a[m][h][half];
                        float e[4] = {__uint_as_float(word.x), __uint_as_float(word.y), __uint_as_float(word.z), __uint_as_float(word.w)};
#pragma unroll
                        for (int s = 0; s < kPlanes; ++s) {
                            f[s][h] = next_planes(e[0], e[1]);
                            f[s][2 + h] = next_planes(e[2], e[3]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        auto add = [&](int s, int t) {  // planes s of W, t of X
                            mma16816(acc[m][n], f[s], half ? x[t][n].z : x[t][n].x, half ? x[t][n].w : x[t][n].y);
                        };
                        add(2, 0);  // the smallest first
                        add(1, 1);
                        add(0, 2);
                        add(1, 0);
                        add(0, 1);
                        add(0, 0);
                    }
                }
            if ((b - from) % 16 == 15) {  // no more than 512 indices in one running sum, which is cut at every addition
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sum[m][n][j] += acc[m][n][j];
                            acc[m][n][j] = 0.f;
                        }
            }
        }
        __syncthreads();  // the group before has been read
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sums[warp][16 * m + 8 * (j >> 1) + g][8 * n + 2 * q + (j & 1)] = sum[m][n][j] + acc[m][n][j];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = NT * warp + i;
            if (n >= p.N) continue;
            float z = 0.f;
#pragma unroll
            for (int s = 0; s < kFewWarps; ++s) z += sums[s][lane][n];
            const int64_t v = v0 + lane, token = p.targets[n];
            if (v < p.V && v == token && token != p.ignore) p.at_target[n] = z;
            if (v >= p.V) z = __int_as_float(0xff800000);
            const float top = fmaxf(most[i], row::warp_max(z)), base = top == __int_as_float(0xff800000) ? 0.f : top;
            const float e = row::warp_sum(__expf(z - base));
            total[i] = (total[i] == 0.f ? 0.f : total[i] * __expf(most[i] - base)) + e;
            most[i] = top;
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
        if (lane == 0 && NT * warp + i < p.N)
            p.parts[static_cast<int64_t>(blockIdx.x) * p.N + NT * warp + i] = make_float2(most[i], total[i]);
}

// groups of 32 entries that a block takes: four blocks an SM or more where there are as many
inline int few_groups(int64_t V, int sms)
{
    int groups = 8;
    while (groups > 1 && (V + kFewRows * groups - 1) / (kFewRows * groups) < 4 * sms) groups /= 2;
    return groups;
}

inline int64_t few_blocks(int64_t V, int sms)
{
    const int64_t rows = kFewRows * few_groups(V, sms);
    return (V + rows - 1) / rows;
}

inline cudaError_t launch_few(FewParams p, int sms, cudaStream_t stream)
{
    p.groups = few_groups(p.V, sms);
    const unsigned blocks = static_cast<unsigned>(few_blocks(p.V, sms));
    switch ((p.N + 7) / 8) {
        case 1: few_kernel<1><<<blocks, kFewWarps * 32, 0, stream>>>(p); break;
        case 2: few_kernel<2><<<blocks, kFewWarps * 32, 0, stream>>>(p); break;
        case 3: few_kernel<3><<<blocks, kFewWarps * 32, 0, stream>>>(p); break;
        default: few_kernel<4><<<blocks, kFewWarps * 32, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace head
}  // namespace cci
