// cci_gated.cu -- the gated feed-forward block: what surrounds its tensor-core products
// (cci_gated.cuh).
//
//   planes    fp32 matrices as three bf16 planes, once per call (memory bound: 4 bytes read and 6
//             written an element)
//   expand    both packed weight matrices (values, idx) to dense bf16, or to those planes; few tokens (cci_gated_few.cu)
//             read the packed bf16 weights themselves, and dense fp32 ones
//   slopes    dg = dh u act'(g), du = dh act(g) from the saved fp32 g and u, rounded to bf16 (or split
//             into planes), the operands of the gradients' products (memory bound: 14 bytes an
//             element in bf16).  g and u are saved in fp32, not rounded to bf16: with them rounded too
//             the gradients would carry three roundings to 8 bits where one is unavoidable (it makes a bf16
//             training pass 0.0023 of its norm off, where the output's rounding alone is 0.0017)
#include "cci_gated.cuh"
#include "cci_rowops.cuh"

namespace cci {
namespace gated {

constexpr size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// eight values to their places in one plane or three, `plane` elements apart
template <int P>
__device__ __forceinline__ void store_planes(uint16_t *out, int64_t plane, const float (&v)[8])
{
    if constexpr (P == 1) {
        row::store<uint16_t, 8>(out, v);
    } else {
        uint32_t w[3][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t a[3], b[3];
            split3(v[2 * j], a);
            split3(v[2 * j + 1], b);
#pragma unroll
            for (int q = 0; q < 3; ++q) w[q][j] = a[q] | b[q] << 16;
        }
#pragma unroll
        for (int q = 0; q < 3; ++q)
            *reinterpret_cast<uint4 *>(out + q * plane) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
}

// up to three matrices in one launch: blockIdx.y is the matrix
struct PlaneJobs {
    const float *in[3];
    uint16_t *out[3];
    int64_t n[3];  // elements, a multiple of 8
};

__global__ void __launch_bounds__(256) planes_kernel(PlaneJobs j)
{
    const float *in = j.in[blockIdx.y];
    uint16_t *out = j.out[blockIdx.y];
    const int64_t n = j.n[blockIdx.y];
    for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n;
         i += static_cast<int64_t>(gridDim.x) * 2048) {
        float v[8];
        row::unpack<float, 8>(row::load_once<float, 8>(in + i), v);
        store_planes<3>(out + i, n, v);
    }
}

// ---- packed weights -> dense, one group of G rows and `cols` columns a block; blockIdx.y: gate, up ----
struct ExpandJob {
    const void *values[2];
    const uint8_t *idx[2];
    uint16_t *out[2];
    int64_t F, D;
    int G, K, cols, col_blocks;
    int whole;  // fp32: [F][D] fp32 instead of planes
    uint32_t *status;
};

// The usual shapes (G a power of two up to 128; K 1, 2, 4 or 8): a thread holds the run of eight indices of a
// group and writes all G rows of it, 16 bytes at a time, neighbours next to each other.  4096 x 4096 twice at G = 8,
// K = 2: 65 us through shared memory (below), 18 so, with 67 MB written
template <int K>
__global__ void __launch_bounds__(256) expand_bf16_kernel(ExpandJob j)
{
    const int which = blockIdx.y, words = static_cast<int>(j.D / 8);
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, group = i / words;
    if (group * j.G >= j.F) return;
    const int64_t d = (i - group * words) * 8, at = (group * j.D + d) * K;
    Run<K> run;
#pragma unroll
    for (int q = 0; q < K; ++q) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(j.values[which]) + at) + q);
        run.v[4 * q] = v.x;
        run.v[4 * q + 1] = v.y;
        run.v[4 * q + 2] = v.z;
        run.v[4 * q + 3] = v.w;
        const uint2 x = __ldg(reinterpret_cast<const uint2 *>(j.idx[which] + at) + q);
        run.i[2 * q] = x.x;
        run.i[2 * q + 1] = x.y;
    }
    if (ws::pk::bad_sets<K>(run.i, j.G)) report(j.status, CCI_ERR_INDEX);
    uint16_t *out = j.out[which] + group * j.G * j.D + d;
    for (int r = 0; r < j.G; ++r)
        *reinterpret_cast<uint4 *>(out + r * j.D) = pick(run, static_cast<uint32_t>(r) * 0x01010101u);
}

// fp32, likewise: whole values or planes
template <int K>
__global__ void __launch_bounds__(256) expand_f32_kernel(ExpandJob j)
{
    const int which = blockIdx.y, words = static_cast<int>(j.D / 8);
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, group = i / words;
    if (group * j.G >= j.F) return;
    const int64_t d = (i - group * words) * 8, at = (group * j.D + d) * K;
    float v[8 * K];
    uint32_t idx[2 * K];
#pragma unroll
    for (int q = 0; q < 2 * K; ++q) row::unpack<float, 4>(row::load<float, 4>(static_cast<const float *>(j.values[which]) + at + 4 * q), v + 4 * q);
#pragma unroll
    for (int q = 0; q < K; ++q) {
        const uint2 x = __ldg(reinterpret_cast<const uint2 *>(j.idx[which] + at) + q);
        idx[2 * q] = x.x;
        idx[2 * q + 1] = x.y;
    }
    if (ws::pk::bad_sets<K>(idx, j.G)) report(j.status, CCI_ERR_INDEX);
    for (int r = 0; r < j.G; ++r) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = 0.f;
#pragma unroll
            for (int s = 0; s < K; ++s) {
                const int slot = e * K + s;
                if ((idx[slot / 4] >> (8 * (slot % 4)) & 0xffu) == static_cast<uint32_t>(r)) o[e] = v[slot];
            }
        }
        const int64_t to = (group * j.G + r) * j.D + d;
        if (j.whole)
            row::store<float, 8>(reinterpret_cast<float *>(j.out[which]) + to, o);
        else
            store_planes<3>(j.out[which] + to, j.F * j.D, o);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) expand_kernel(ExpandJob j)
{
    extern __shared__ __align__(16) unsigned char tile_raw[];
    T *tile = reinterpret_cast<T *>(tile_raw);  // [G][cols]
    const int which = blockIdx.y, G = j.G, K = j.K, cols = j.cols;
    const int64_t group = blockIdx.x / j.col_blocks, d0 = static_cast<int64_t>(blockIdx.x % j.col_blocks) * cols;
    const int n = j.D - d0 < cols ? static_cast<int>(j.D - d0) : cols;
    for (int i = threadIdx.x; i < G * cols * static_cast<int>(sizeof(T)) / 16; i += 256)
        reinterpret_cast<uint4 *>(tile)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    const int64_t at = (group * j.D + d0) * K;
    const T *values = static_cast<const T *>(j.values[which]) + at;
    const uint8_t *idx = j.idx[which] + at;
    bool bad = false;
    for (int i = threadIdx.x; i < n * K; i += 256) {
        const int c = i / K, k = i - c * K, r = idx[i];
        bad |= r >= G || (k > 0 && r <= idx[i - 1]);
        if (r < G) tile[r * cols + c] = values[i];
    }
    if (bad) report(j.status, CCI_ERR_INDEX);
    __syncthreads();
    uint16_t *out = j.out[which] + group * G * j.D + d0;
    const int words = n / 8;  // D is a multiple of 8
    for (int i = threadIdx.x; i < G * words; i += 256) {
        const int r = i / words, c = (i - r * words) * 8;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(out + r * j.D + c) = *reinterpret_cast<const uint4 *>(tile + r * cols + c);
        } else {
            float v[8];
            row::unpack<float, 8>(row::load<float, 8>(reinterpret_cast<const float *>(tile) + r * cols + c), v);
            if (j.whole)
                row::store<float, 8>(reinterpret_cast<float *>(j.out[which]) + (group * G + r) * j.D + d0 + c, v);
            else
                store_planes<3>(out + r * j.D + c, j.F * j.D, v);
        }
    }
}

// ---- dg and du ----
template <typename T, int P>
__global__ void __launch_bounds__(256)
    slopes_kernel(const T *dh, const float *g, const float *u, int64_t n, int act, uint16_t *dg, uint16_t *du)
{
    for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n;
         i += static_cast<int64_t>(gridDim.x) * 2048) {
        float h[8], gv[8], uv[8];
        row::unpack<T, 8>(row::load_once<T, 8>(dh + i), h);
        row::unpack<float, 8>(row::load_once<float, 8>(g + i), gv);
        row::unpack<float, 8>(row::load_once<float, 8>(u + i), uv);
        with_act(act, [&](auto code) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float a;
                const float s = slope_of<decltype(code)::value>(gv[j], a);
                gv[j] = h[j] * uv[j] * s;
                uv[j] = h[j] * a;
            }
        });
        store_planes<P>(dg + i, n, gv);
        store_planes<P>(du + i, n, uv);
    }
}

unsigned grid_of(int64_t n)
{
    const int64_t blocks = (n / 8 + 255) / 256, most = static_cast<int64_t>(ws::sm_count()) * 8;
    return static_cast<unsigned>(blocks < 1 ? 1 : (blocks < most ? blocks : most));
}

// places in the workspace (bytes from its start; 0 sized where a call does not need one)
struct Layout {
    size_t x, wg, wu, dg, du, parts, total;
};

Layout layout(int dtype, int64_t N, int64_t D, int64_t F, int call)
{
    const bool f32 = dtype == CCI_F32;
    const size_t planes = f32 ? 3 : 1;
    const bool dense = f32 || call == CCI_GATED_PACKED;  // weights laid out here
    Layout l{};
    size_t at = 0;
    auto take = [&](bool need, int64_t n) {
        const size_t here = at;
        if (need) at += round256(static_cast<size_t>(n) * 2 * planes);
        return here;
    };
    l.x = take(f32, N * D);
    l.wg = take(dense, F * D);
    l.wu = take(dense, F * D);
    l.dg = take(call == CCI_GATED_BACKWARD, N * F);
    l.du = take(call == CCI_GATED_BACKWARD, N * F);
    l.parts = at;
    const int terms = f32 ? 6 : 1;
    if (call != CCI_GATED_BACKWARD) {
        at += round256(plan(kForward, N, F, D, terms).part_bytes);
    } else {  // the products follow each other: one place for both
        const size_t dx = plan(kDx, N, D, F, terms).part_bytes, dw = plan(kDw, F, D, N, terms).part_bytes;
        at += round256(dx > dw ? dx : dw);
    }
    l.total = at;
    return l;
}

template <int K>
void launch_expand_k(const ExpandJob &j, bool f32, cudaStream_t stream)
{
    const dim3 grid(static_cast<unsigned>((j.F / j.G * (j.D / 8) + 255) / 256), 2);
    if (f32)
        expand_f32_kernel<K><<<grid, 256, 0, stream>>>(j);
    else
        expand_bf16_kernel<K><<<grid, 256, 0, stream>>>(j);
}

// both matrices to j.out
cudaError_t expand(ExpandJob &j, bool f32, cudaStream_t stream)
{
    auto at8 = [](const void *q) { return reinterpret_cast<uintptr_t>(q) % 8 == 0; };
    const bool usual = j.G <= 128 && (j.G & (j.G - 1)) == 0 && at8(j.idx[0]) && at8(j.idx[1]);
    if (usual && (j.K == 1 || j.K == 2 || j.K == 4 || j.K == 8)) {
        if (j.F / j.G * (j.D / 8) / 256 >= 0x7fffffff) return cudaErrorInvalidValue;
        switch (j.K) {
            case 1: launch_expand_k<1>(j, f32, stream); break;
            case 2: launch_expand_k<2>(j, f32, stream); break;
            case 4: launch_expand_k<4>(j, f32, stream); break;
            default: launch_expand_k<8>(j, f32, stream);
        }
        return cudaGetLastError();
    }
    // a tile of at most 32 KB
    j.cols = j.G <= 32 ? 256 : (j.G <= 64 ? 128 : (j.G <= 128 ? 64 : 32));
    j.col_blocks = static_cast<int>((j.D + j.cols - 1) / j.cols);
    const int64_t blocks = j.F / j.G * j.col_blocks;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks), 2);
    const size_t bytes = static_cast<size_t>(j.G) * j.cols * (f32 ? 4 : 2);
    if (f32)
        expand_kernel<float><<<grid, 256, bytes, stream>>>(j);
    else
        expand_kernel<uint16_t><<<grid, 256, bytes, stream>>>(j);
    return cudaGetLastError();
}

cudaError_t split(const float *const *in, uint16_t *const *out, const int64_t *n, int jobs, cudaStream_t stream)
{
    PlaneJobs j{};
    int64_t most = 0;
    for (int i = 0; i < jobs; ++i) {
        j.in[i] = in[i];
        j.out[i] = out[i];
        j.n[i] = n[i];
        most = n[i] > most ? n[i] : most;
    }
    planes_kernel<<<dim3(grid_of(most), static_cast<unsigned>(jobs)), 256, 0, stream>>>(j);
    return cudaGetLastError();
}

}  // namespace gated

size_t gated_workspace(int dtype, int64_t N, int64_t D, int64_t F, int call)
{
    return gated::layout(dtype, N, D, F, call).total;
}

cudaError_t launch_gated(const GatedArgs &a, cudaStream_t stream)
{
    using namespace gated;
    const bool f32 = a.dtype == CCI_F32, packed = a.gate_idx != nullptr, few = few_tokens(a.dtype, a.N, a.F);
    if (packed ? few_packed(a) : few) return launch_few(a, a.Wg, a.Wu, packed, stream);
    const Layout l = layout(a.dtype, a.N, a.D, a.F, packed ? CCI_GATED_PACKED : CCI_GATED_FORWARD);
    char *base = static_cast<char *>(a.workspace);
    const void *x = a.X, *wg = a.Wg, *wu = a.Wu;
    if (packed) {
        ExpandJob j{};
        j.values[0] = a.Wg;
        j.values[1] = a.Wu;
        j.idx[0] = a.gate_idx;
        j.idx[1] = a.up_idx;
        j.out[0] = reinterpret_cast<uint16_t *>(base + l.wg);
        j.out[1] = reinterpret_cast<uint16_t *>(base + l.wu);
        j.F = a.F;
        j.D = a.D;
        j.G = a.G;
        j.K = a.K;
        j.whole = few;
        j.status = a.status;
        const cudaError_t e = expand(j, f32, stream);
        if (e != cudaSuccess) return e;
        wg = base + l.wg;
        wu = base + l.wu;
        if (few) return launch_few(a, wg, wu, false, stream);
    }
    if (f32) {
        const float *in[3] = {static_cast<const float *>(a.X), static_cast<const float *>(a.Wg),
                              static_cast<const float *>(a.Wu)};
        uint16_t *out[3] = {reinterpret_cast<uint16_t *>(base + l.x), reinterpret_cast<uint16_t *>(base + l.wg),
                            reinterpret_cast<uint16_t *>(base + l.wu)};
        const int64_t n[3] = {a.N * a.D, a.F * a.D, a.F * a.D};
        const cudaError_t e = split(in, out, n, packed ? 1 : 3, stream);
        if (e != cudaSuccess) return e;
        x = base + l.x;
        wg = base + l.wg;
        wu = base + l.wu;
    }
    const int planes = f32 ? 3 : 1;
    Job j{};
    j.a[0] = Operand{x, a.N, a.D, planes};
    j.b[0] = Operand{wg, a.F, a.D, planes};
    j.b[1] = Operand{wu, a.F, a.D, planes};
    j.out[0] = a.H;
    j.save[0] = a.g;
    j.save[1] = a.u;
    j.parts = reinterpret_cast<float *>(base + l.parts);
    j.M = a.N;
    j.N = a.F;
    j.K = a.D;
    j.terms = f32 ? 6 : 1;
    j.act = a.act;
    j.out_f32 = f32;
    j.status = a.status;
    return launch_forward(j, stream);
}

cudaError_t launch_gated_backward(const GatedArgs &a, cudaStream_t stream)
{
    using namespace gated;
    const bool f32 = a.dtype == CCI_F32;
    if (a.N == 0) {  // no rows to sum over
        const size_t bytes = static_cast<size_t>(a.F) * a.D * (f32 ? 4 : 2);
        cudaError_t e = a.dWg ? cudaMemsetAsync(a.dWg, 0, bytes, stream) : cudaSuccess;
        if (e == cudaSuccess && a.dWu) e = cudaMemsetAsync(a.dWu, 0, bytes, stream);
        return e;
    }
    const Layout l = layout(a.dtype, a.N, a.D, a.F, CCI_GATED_BACKWARD);
    char *base = static_cast<char *>(a.workspace);
    uint16_t *dg = reinterpret_cast<uint16_t *>(base + l.dg), *du = reinterpret_cast<uint16_t *>(base + l.du);
    const int64_t n = a.N * a.F;
    if (f32)
        slopes_kernel<float, 3><<<grid_of(n), 256, 0, stream>>>(static_cast<const float *>(a.dH), a.g, a.u, n, a.act,
                                                                dg, du);
    else
        slopes_kernel<uint16_t, 1><<<grid_of(n), 256, 0, stream>>>(static_cast<const uint16_t *>(a.dH), a.g, a.u, n,
                                                                   a.act, dg, du);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const void *x = a.X, *wg = a.Wg, *wu = a.Wu;
    if (f32) {
        // only what a gradient asked for needs (dW alone of 1000 tokens, 1024 -> 2048: 66.4 us with all three, 59.9 so)
        const float *in[3] = {};
        uint16_t *out[3] = {};
        int64_t count[3] = {};
        int jobs = 0;
        auto need = [&](const void *v, size_t at, int64_t elements) {
            in[jobs] = static_cast<const float *>(v);
            out[jobs] = reinterpret_cast<uint16_t *>(base + at);
            count[jobs++] = elements;
        };
        if (a.dWg) need(a.X, l.x, a.N * a.D);
        if (a.dX) {
            need(a.Wg, l.wg, a.F * a.D);
            need(a.Wu, l.wu, a.F * a.D);
        }
        if (jobs) e = split(in, out, count, jobs, stream);
        if (e != cudaSuccess) return e;
        x = base + l.x;
        wg = base + l.wg;
        wu = base + l.wu;
    }
    const int planes = f32 ? 3 : 1;
    Job j{};
    j.terms = f32 ? 6 : 1;
    j.out_f32 = f32;
    j.status = a.status;
    j.parts = reinterpret_cast<float *>(base + l.parts);
    j.a[0] = Operand{dg, a.N, a.F, planes};
    j.a[1] = Operand{du, a.N, a.F, planes};
    if (a.dX) {
        j.b[0] = Operand{wg, a.F, a.D, planes};
        j.b[1] = Operand{wu, a.F, a.D, planes};
        j.out[0] = a.dX;
        j.M = a.N;
        j.N = a.D;
        j.K = a.F;
        e = launch_dx(j, stream);
        if (e != cudaSuccess) return e;
    }
    if (a.dWg) {
        j.b[0] = Operand{x, a.N, a.D, planes};
        j.out[0] = a.dWg;
        j.out[1] = a.dWu;
        j.M = a.F;
        j.N = a.D;
        j.K = a.N;
        e = launch_dw(j, stream);
    }
    return e;
}

}  // namespace cci
