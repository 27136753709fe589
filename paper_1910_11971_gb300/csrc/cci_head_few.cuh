// cci_head_few.cuh -- the cross entropy of up to 32 tokens from a head's fp32 inputs, and its gradients.
//
// The head's weights are all that is read, once, as they are: writing W's planes first, as for more tokens
// (cci_head.cu), moves four times its bytes (2 tokens, 3392 x 4076: 96 us, 26 so; 16 tokens, 4096 x 65536 fp32 240 us of
// 158 at the copy rate).  A warp takes 32 entries of the vocabulary and an eighth of the reduction, straight from memory into
// the fragments of mma.sync: 32 elements of a row lie with four lanes, eight each, and X is read in the same order, so that the
// order of the reduction within a step does not matter.  Values become three bf16 planes in registers, cut to eight
// bits each; the six products of planes are those of cci_gated.cuh.  The warps' sums meet in shared memory, where each
// token's maximum and sum of exponentials are taken.  bf16 tokens, however few, go by the tiles of cci_head.cu, whose copies
// keep more on its way (1 token, 4096 x 131072: 203 us through here, 166 so).
//
// Backward the same walk gives P [V][tokens] in fp32, and one pass over the weights takes both gradients from it with
// fused multiply-adds: a thread holds its columns of X and of dX for all tokens, reads a weight, adds P times it to dX and writes
// P^T X in its place of dW.  dX's parts over slices of the vocabulary are added in order.  7 tokens, 2752 x 34448,
// both passes: 845 us with planes of W and products of tiles, 330 so, of 224 to read W three times and write dW.  What bounds
// that pass is P, a broadcast load from shared memory for four multiply-adds of each gradient.  17 to about 80 tokens are past what this,
// or planes, do well: 25 tokens 777 us, where elementary fp32 products take 591.
#pragma once

#include "cci_kernels.h"
#include "cci_rowops.cuh"
#include "cci_tc_common.cuh"

namespace cci {
namespace head {

constexpr int kFewTokens = 32, kFewRows = 32, kFewWarps = 8;

__device__ __forceinline__ bool is_kept(int64_t token, int64_t ignore, int64_t V)
{
    return token != ignore && token >= 0 && token < V;
}

struct FewParams {
    const uint16_t *x;   // three planes [N][D]
    const float *w;      // [V][D]
    int N, D;
    int64_t V;
    int groups;          // of 32 entries, a block
    const int64_t *targets;
    int64_t ignore;
    // forward
    float2 *parts;       // [blocks][N]
    float *at_target;    // [N]
    // backward
    const float *stats, *dloss;
    float *probs;        // [V][8, 16 or 32: few_pitch]
    uint32_t *status;
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

// NT: eights of tokens, and tokens that a warp sums up.  PROBS: P instead
template <int NT, bool PROBS>
__global__ void __launch_bounds__(kFewWarps * 32, NT <= 2 ? 2 : 1) few_kernel(const FewParams p)
{
    // steps in one running sum of the matrix unit, which is cut at every addition (24 tokens, 4096 x 65536: 428 us, 512 with one)
    constexpr int kPlanes = 3, kPitch = 8 * NT + 1, kChunk = NT <= 2 ? 1 : 4;
    __shared__ float sums[kFewWarps][kFewRows][kPitch];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const float *w = p.w;
    const int steps = (p.D + 31) / 32, from = steps * warp / kFewWarps, to = steps * (warp + 1) / kFewWarps;
    const int64_t plane = static_cast<int64_t>(p.N) * p.D;
    // tokens NT warp + i: what their entries so far say
    float most[NT], total[NT] = {};
#pragma unroll
    for (int i = 0; i < NT; ++i) most[i] = __int_as_float(0xff800000);
    // backward: what is subtracted from their logits, the probabilities' factors, the targets (-1: left out)
    float base[NT], log_s[NT], weight[NT];
    int64_t target[NT];
    if constexpr (PROBS) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int n = NT * warp + i;
            const int64_t token = n < p.N ? p.targets[n] : p.ignore;
            const bool kept = is_kept(token, p.ignore, p.V);
            target[i] = kept ? token : -1;
            weight[i] = kept ? p.dloss[n] : 0.f;
            const float m = n < p.N ? p.stats[2 * n] : 0.f;
            base[i] = m == __int_as_float(0xff800000) ? 0.f : m;
            log_s[i] = n < p.N ? p.stats[2 * n + 1] : 0.f;
            if (!kept && token != p.ignore && blockIdx.x == 0 && lane == 0) report(p.status, CCI_ERR_INDEX);
        }
    } else {
        tc::launch_next_grid();  // which waits for this one's end
    }
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
            if ((b - from) % kChunk == kChunk - 1) {
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
            if (!PROBS && n >= p.N) continue;
            float z = 0.f;
#pragma unroll
            for (int s = 0; s < kFewWarps; ++s) z += sums[s][lane][n];
            const int64_t v = v0 + lane;
            if constexpr (PROBS) {
                const float x = (z - base[i]) - log_s[i], e = v == target[i] ? expm1f(x) : __expf(x);
                if (v < p.V) p.probs[v * (8 * NT) + n] = weight[i] == 0.f ? 0.f : e * weight[i];
                continue;
            }
            const int64_t token = p.targets[n];
            if (v < p.V && v == token && token != p.ignore) p.at_target[n] = z;
            if (v >= p.V) z = __int_as_float(0xff800000);
            const float top = fmaxf(most[i], row::warp_max(z)), from = top == __int_as_float(0xff800000) ? 0.f : top;
            const float e = row::warp_sum(__expf(z - from));
            total[i] = (total[i] == 0.f ? 0.f : total[i] * __expf(most[i] - from)) + e;
            most[i] = top;
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
        if (!PROBS && lane == 0 && NT * warp + i < p.N)
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

template <bool PROBS>
cudaError_t launch_few(FewParams p, int sms, cudaStream_t stream)
{
    p.groups = few_groups(p.V, sms);
    const unsigned blocks = static_cast<unsigned>(few_blocks(p.V, sms));
    switch ((p.N + 7) / 8) {
        case 1: few_kernel<1, PROBS><<<blocks, kFewWarps * 32, 0, stream>>>(p); break;
        case 2: few_kernel<2, PROBS><<<blocks, kFewWarps * 32, 0, stream>>>(p); break;
        default: few_kernel<4, PROBS><<<blocks, kFewWarps * 32, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

// ---- both gradients from P ----
constexpr int kFewTile = 64;  // entries whose P is in shared memory at a time

struct FewGradients {
    const float *x, *w, *probs;
    int N, D;
    int64_t V, slice;  // entries of a slice, a multiple of kFewTile
    float *dw, *parts; // dW, dX's parts [slices][N][D]; each may be null
    const int64_t *targets;
    int64_t ignore;
    const float *dloss;
};

constexpr int kFewAhead = 4;           // batches of weights on their way
constexpr int kFewBatch = 16 * 1024;   // bytes of one, of all threads

// NP: P's row length; C = 32 / NP columns a thread, so that its share of X and dX takes 64 registers.  Weights come through
// places of the thread's own in shared memory, several rows ahead.  blockIdx.x: columns, .y: slice
template <int NP, int C>
__global__ void __launch_bounds__(256, 2) few_gradients_kernel(const FewGradients p)
{
    constexpr int kRows = kFewBatch / (256 * C * 4);  // of a batch
    static_assert(kFewTile % kRows == 0, "a tile holds whole batches");
    struct __align__(4 * C) Columns {
        float f[C];
    };
    extern __shared__ __align__(16) unsigned char ring_raw[];
    Columns *ring = reinterpret_cast<Columns *>(ring_raw) + threadIdx.x;
    __shared__ __align__(16) float probs[kFewTile][NP];
    const int d = (static_cast<int>(blockIdx.x) * 256 + static_cast<int>(threadIdx.x)) * C;
    const bool mine = d < p.D;  // D is a multiple of 8
    const int64_t from = p.slice * blockIdx.y, to = from + p.slice < p.V ? from + p.slice : p.V;
    auto copy = [&](int64_t v0, int k) {  // rows v0 .. of a batch
        if (mine && p.parts) {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (v0 + r < to)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(tc::smem_u32(ring + (k * kRows + r) * 256)),
                                 "l"(p.w + (v0 + r) * p.D + d), "n"(4 * C)
                                 : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kFewAhead; ++k) copy(from + k * kRows, k);
    // left-out tokens' X are zeros, whatever they hold
    const int lane = threadIdx.x & 31;
    const unsigned kept = __ballot_sync(0xffffffffu, lane < p.N && is_kept(p.targets[lane], p.ignore, p.V) && p.dloss[lane] != 0.f);
    float x[NP][C], dx[NP][C];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        const Columns q = mine && (kept >> n & 1u) ? *reinterpret_cast<const Columns *>(p.x + static_cast<int64_t>(n) * p.D + d) : Columns{};
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[n][j] = q.f[j];
            dx[n][j] = 0.f;
        }
    }
    int k = 0;
    for (int64_t v0 = from; v0 < to; v0 += kFewTile) {
        const int count = to - v0 < kFewTile ? static_cast<int>(to - v0) : kFewTile;
        __syncthreads();
        for (int i = threadIdx.x; i < count * NP / 4; i += 256)
            reinterpret_cast<float4 *>(&probs[0][0])[i] = reinterpret_cast<const float4 *>(p.probs + v0 * NP)[i];
        __syncthreads();
        for (int r0 = 0; r0 < count; r0 += kRows) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kFewAhead - 1) : "memory");
            if (mine) {
#pragma unroll 4
                for (int r = 0; r < kRows; ++r) {
                    if (r0 + r >= count) break;
                    const Columns w = p.parts ? ring[(k * kRows + r) * 256] : Columns{};
                    Columns dw{};
#pragma unroll
                    for (int n = 0; n < NP; n += 4) {
                        const float4 q = *reinterpret_cast<const float4 *>(&probs[r0 + r][n]);
                        const float f[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int j = 0; j < C; ++j) {
                                dx[n + i][j] = fmaf(f[i], w.f[j], dx[n + i][j]);
                                dw.f[j] = fmaf(f[i], x[n + i][j], dw.f[j]);
                            }
                    }
                    if (p.dw) *reinterpret_cast<Columns *>(p.dw + (v0 + r0 + r) * p.D + d) = dw;
                }
            }
            copy(v0 + r0 + kFewAhead * kRows, k);  // where this thread has read
            k = k + 1 == kFewAhead ? 0 : k + 1;
        }
    }
    if (!p.parts || !mine) return;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        if (n >= p.N) break;
        Columns q;
#pragma unroll
        for (int j = 0; j < C; ++j) q.f[j] = dx[n][j];
        *reinterpret_cast<Columns *>(p.parts + (static_cast<int64_t>(blockIdx.y) * p.N + n) * p.D + d) = q;
    }
}

// dX: its parts in order, n elements
__global__ void __launch_bounds__(256) few_join_kernel(const float *parts, int slices, int64_t n, float *dx)
{
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    tc::wait_prior_grid();
    if (i >= n) return;  // a multiple of 8
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = 0; k < slices; ++k) {
        const float4 q = *reinterpret_cast<const float4 *>(parts + k * n + i);
        s.x += q.x;
        s.y += q.y;
        s.z += q.z;
        s.w += q.w;
    }
    *reinterpret_cast<float4 *>(dx + i) = s;
}

inline int few_pitch(int64_t N) { return N <= 8 ? 8 : (N <= 16 ? 16 : 32); }

// slices of the vocabulary: about four blocks an SM, of kFewTile entries or more
inline int64_t few_slice(int64_t N, int64_t D, int64_t V, int sms)
{
    const int64_t columns = (D + 256 * 32 / few_pitch(N) - 1) / (256 * 32 / few_pitch(N));
    int64_t slices = 4 * sms / columns;
    if (slices < 1) slices = 1;
    return ((V + slices - 1) / slices + kFewTile - 1) / kFewTile * kFewTile;
}

inline int64_t few_slices(int64_t N, int64_t D, int64_t V, int sms)
{
    const int64_t slice = few_slice(N, D, V, sms);
    return (V + slice - 1) / slice;
}

template <int NP, int C>
cudaError_t launch_few_columns(const FewGradients &p, const dim3 &grid, cudaStream_t stream)
{
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(few_gradients_kernel<NP, C>, kFewAhead * kFewBatch, attr_cache);
    if (attr != cudaSuccess) return attr;
    few_gradients_kernel<NP, C><<<grid, 256, kFewAhead * kFewBatch, stream>>>(p);
    return cudaGetLastError();
}

inline cudaError_t launch_few_gradients(FewGradients p, int sms, float *dx, cudaStream_t stream)
{
    const int pitch = few_pitch(p.N);
    p.slice = few_slice(p.N, p.D, p.V, sms);
    const int64_t slices = few_slices(p.N, p.D, p.V, sms);
    const int columns = 256 * 32 / pitch;
    const dim3 grid(static_cast<unsigned>((p.D + columns - 1) / columns), static_cast<unsigned>(slices));
    cudaError_t e = pitch == 8 ? launch_few_columns<8, 4>(p, grid, stream)
                               : (pitch == 16 ? launch_few_columns<16, 2>(p, grid, stream) : launch_few_columns<32, 1>(p, grid, stream));
    if (e != cudaSuccess || !dx) return e;
    const int64_t n = static_cast<int64_t>(p.N) * p.D;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((n / 4 + 255) / 256));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, few_join_kernel, const_cast<const float *>(p.parts), static_cast<int>(slices), n, dx);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

}  // namespace head
}  // namespace cci
