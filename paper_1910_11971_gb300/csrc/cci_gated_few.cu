// cci_gated_few.cu -- the gated block for few tokens (decoding): h = act(X Wg^T) * (X Wu^T).
//
// What bounds it: every weight is read once and multiplied with a handful of tokens, so the time is
// that of the weights' bytes.  The tile kernel (cci_gated.cuh) reads a row in 128-byte pieces, one per
// stage, with as many tiles as SMs at best (4096 -> 8192 bf16, one token: 25.3 us, here 22.0, the
// bytes' time 19.7).  Here a block of eight warps takes eight hidden channels, and its warps read
// neighbouring 64-byte pieces of the same sixteen rows (gate and up), 512 bytes of a row at a time,
// straight into registers.
//
// bf16: mma.sync m16n8k16.  The tensor core's rate does not matter here, but its fragment layout does: a
// lane's 16 bytes of a row are eight consecutive indices, and as the tokens' fragment is read the
// same way, the two products they make just take the indices in another order.  Rows 0-7 of the
// fragment are the gate's channels, 8-15 the up projection's, so a lane ends with both for its outputs.
// Packed weights (values, idx) become fragments in registers: the lanes of a group's rows read the
// same run, copied to shared memory in bulk, and each keeps the values whose index is its row.
//
// fp32: fused multiply-adds, 16 rows by up to eight tokens a warp.  Twice the bytes and no products of planes.
// A token stays at the memory's time (4096 -> 8192: 1 token 39.5 us of 39.5, 4 52, 8 73, 16 142).  What bounds more
// is not the multiply-adds (8 tokens 13 us of them, 16 27) but the tokens' own reads, which every block makes: past
// four tokens 2048 blocks of four channels read 268 MB of them out of L2, as much as the weights, and past
// eight the weights are read twice.
//
// The warps' sums are joined in shared memory in warp order: the same bits at every call.
#include "cci_gated.cuh"
#include "cci_rowops.cuh"

namespace cci {
namespace gated {
namespace few {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kF = 8;  // hidden channels of a block

struct Args {
    const void *X, *Wg, *Wu;  // Wg, Wu: dense, or the packed values
    const uint8_t *gate_idx, *up_idx;
    void *H;
    float *g, *u;
    int N, D, F, log_g, act;
    uint32_t *status;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
        "%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// g and u of one output from the warps' sums at red[warp][at] and red[warp][at + 2]
__device__ __forceinline__ void finish(const Args &p, const float *red, int stride, int at, int up, int n, int f,
                                       bool f32)
{
    float g = 0.f, u = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        g += red[w * stride + at];
        u += red[w * stride + at + up];
    }
    const int64_t o = static_cast<int64_t>(n) * p.F + f;
    if (p.g) {
        p.g[o] = g;
        p.u[o] = u;
    }
    float h = 0.f;
    with_act(p.act, [&](auto act) { h = act_of<decltype(act)::value>(g) * u; });
    if (f32)
        static_cast<float *>(p.H)[o] = h;
    else
        row::store<uint16_t, 1>(static_cast<uint16_t *>(p.H) + o, &h);
}

// eight weights of one row (bf16) as a lane's fragment words
__device__ __forceinline__ uint4 load_weights(const uint16_t *w) { return row::load_once<uint16_t, 8>(w).w[0]; }

// from shared memory; the lanes of a group read the same words
template <int K>
__device__ __forceinline__ void load_run(Run<K> &r, const unsigned char *values, const unsigned char *idx)
{
#pragma unroll
    for (int q = 0; q < K; ++q) {
        const uint4 v = reinterpret_cast<const uint4 *>(values)[q];
        r.v[4 * q] = v.x;
        r.v[4 * q + 1] = v.y;
        r.v[4 * q + 2] = v.z;
        r.v[4 * q + 3] = v.w;
        const uint2 i = reinterpret_cast<const uint2 *>(idx)[q];
        r.i[2 * q] = i.x;
        r.i[2 * q + 1] = i.y;
    }
}

// whether the index set of K at `idx` is not strictly increasing below G
template <int K>
__device__ __forceinline__ bool bad_set(const unsigned char *idx, int G)
{
    int last = -1;
    bool bad = false;
#pragma unroll
    for (int s = 0; s < K; ++s) {
        const int i = idx[s];
        bad |= i <= last;
        last = i;
    }
    return bad || last >= G;
}

// A warp's share of a row: 128 indices (four 32-index steps, 256 bytes of a dense row) in turn with the other
// warps', whatever the weights' form: packed weights give the bits that their dense form gives here
constexpr int kSteps = 4, kRound = kSteps * kWarps * 32;

// this lane's sums c[m][i] of each set of eight channels and eight tokens, from every warp: channel g of the
// set, tokens 2 t and 2 t + 1 of the eight; the gate's first, then the up projection's
template <int MT, int NT>
__device__ __forceinline__ void join(const Args &p, float *red, const float (&c)[MT][NT][4], int f0)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kSums = MT * NT * 128;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < NT; ++i)
            *reinterpret_cast<float4 *>(red + warp * kSums + (m * NT + i) * 128 + lane * 4) =
                make_float4(c[m][i][0], c[m][i][1], c[m][i][2], c[m][i][3]);
    __syncthreads();
    for (int o = threadIdx.x; o < MT * NT * 64; o += kThreads) {
        const int ch = o % (MT * 8), n = o / (MT * 8);
        if (n < p.N && f0 + ch < p.F)
            finish(p, red, kSums, ((ch >> 3) * NT + (n >> 3)) * 128 + ((ch & 7) * 4 + ((n & 7) >> 1)) * 4 + (n & 1), 2, n,
                   f0 + ch, false);
    }
}

// eight indices of each of NT eights of tokens, as this lane's fragment words
template <int NT>
__device__ __forceinline__ void load_tokens(uint4 (&x)[NT], const Args &p, int g, int k)
{
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (k < p.D && 8 * i + g < p.N)
            x[i] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.X) +
                                                         static_cast<int64_t>(8 * i + g) * p.D + k));
    }
}

// ---- dense weights.  NT: tokens by eights; as many sets of eight channels a block, which share the tokens' loads ----
template <int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 4 : 3) bf16_kernel(Args p)
{
    constexpr int kAhead = NT == 1 ? 4 : 2, MT = NT;  // steps whose weights are on their way
    __shared__ __align__(16) float red[kWarps * MT * NT * 128];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int f0 = blockIdx.x * kF * MT;
    const int64_t D = p.D;
    // the last block's second set of channels may lie past F: it reads the first set's and writes nothing
    const uint16_t *wg[MT], *wu[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int f = (f0 + m * kF < p.F ? f0 + m * kF : f0) + g;
        wg[m] = static_cast<const uint16_t *>(p.Wg) + f * D;
        wu[m] = static_cast<const uint16_t *>(p.Wu) + f * D;
    }
    float c[MT][NT][4] = {};
    for (int kw = warp * kSteps * 32; kw < p.D; kw += kRound) {
#pragma unroll
        for (int q = 0; q < kSteps; q += kAhead) {
            const int k0 = kw + q * 32 + t * 8;
            uint4 a[kAhead][MT], b[kAhead][MT], x[kAhead][NT];
#pragma unroll
            for (int s = 0; s < kAhead; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const int k = k0 + s * 32;
                    a[s][m] = b[s][m] = make_uint4(0u, 0u, 0u, 0u);
                    if (k < p.D) {  // D is a multiple of 8
                        a[s][m] = load_weights(wg[m] + k);
                        b[s][m] = load_weights(wu[m] + k);
                    }
                }
#pragma unroll
            for (int s = 0; s < kAhead; ++s) load_tokens<NT>(x[s], p, g, k0 + s * 32);
#pragma unroll
            for (int s = 0; s < kAhead; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        mma_bf16(c[m][i], a[s][m].x, b[s][m].x, a[s][m].y, b[s][m].y, x[s][i].x, x[s][i].y);
                        mma_bf16(c[m][i], a[s][m].z, b[s][m].z, a[s][m].w, b[s][m].w, x[s][i].z, x[s][i].w);
                    }
        }
    }
    join<MT, NT>(p, red, c, f0);
}

// ---- packed weights ----
// A block takes a group (two of G = 4) of each projection: MT sets of eight channels.  Their runs of a round
// of 1024 indices are contiguous, and bulk copies bring them to shared memory, as many rounds ahead as it
// holds: registers hold no weights that are on their way.  What bounds it is taking each row's weights out of the
// runs, each row by itself, on the integer pipe: work that grows with G K where the bytes grow with K (60 % of that pipe; 16 tokens,
// 4096 -> 4096, G = 8, K = 2: 21.3 us of 3.7 for the bytes; its 512 blocks are 1.1 rounds of 456 places).  So
// packed weights save memory, and time with K = 1 alone; against dense weights of the same block, us:
//                            1 token              8                16
//   4096 -> 4096  dense      11.7                 12.8             16.3
//     G = 8, K = 1, 2        11.9, 19.8           12.1, 20.1       15.1, 21.7
//     G = 4, K = 2           24.8                 26.5             28.1
//     G = 32, K = 8          35.7                 36.6             39.2
//   4096 -> 8192  dense      21.6                 23.5             26.9
//     G = 8, K = 1, 2        18.2, 33.2           18.9, 33.3       24.0, 36.5
//     G = 4, K = 2           39.3                 40.6             43.4
//     G = 32, K = 8          72.5                 74.2             78.5
constexpr int kMaxStages = 8;

struct PackedSmem {
    uint64_t full[kMaxStages], empty[kMaxStages];
    int abort;
};

// untiled bulk copy of `bytes` (a multiple of 16) to shared memory, completing on `bar`; both addresses on 16 bytes
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(tc::smem_u32(bar))
                 : "memory");
}

// a stage: [gate, up][group][1024 K values, then 1024 K indices]
constexpr int stage_bytes(int K, int groups) { return 2 * groups * kRound * K * 3; }

// blocks of an SM that registers and shared memory are shared out to.  Sets of eight channels: four with K = 1
// (G = 8, 4096 -> 4096, 16 tokens: 18.5 us with two, 14.8 so), three with K = 2 (4096 -> 8192, 16 tokens: 39.3 us with
// two, 36.3 so, 38.6 with four)
constexpr int packed_blocks(int K, int MT) { return K > 2 ? 1 : (MT > 1 ? 2 : (K == 1 ? 4 : 3)); }

template <int K, int NT, int MT>
__global__ void __launch_bounds__(kThreads, packed_blocks(K, MT)) packed_kernel(Args p, int stages)
{
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ PackedSmem S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = 1 << p.log_g, groups = G < kF ? kF / G : 1;  // of a block
    const int f0 = blockIdx.x * kF * MT, group0 = f0 >> p.log_g;
    const int rounds = (p.D + kRound - 1) / kRound;
    constexpr int kValues = kRound * K * 2, kHalf = kRound * K * 3;  // bytes of a group's values; with its indices
    const int stage = 2 * groups * kHalf;
    volatile int *abort = &S.abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            tc::mbar_init(&S.full[s], 1);
            tc::mbar_init(&S.empty[s], kWarps);
        }
        S.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    // copies round r into stage s (one thread)
    auto copy = [&](int r, int s) {
        const int n = p.D - r * kRound < kRound ? p.D - r * kRound : kRound;
        tc::mbar_arrive_expect_tx(&S.full[s], static_cast<uint32_t>(2 * groups * n * K * 3));
        for (int q = 0; q < 2; ++q)
            for (int j = 0; j < groups; ++j) {
                const int64_t at = (static_cast<int64_t>(group0 + j) * p.D + r * kRound) * K;
                const uint32_t dst = tc::smem_u32(smem) + static_cast<uint32_t>(s * stage + (q * groups + j) * kHalf);
                bulk_load(dst, static_cast<const uint16_t *>(q ? p.Wu : p.Wg) + at, static_cast<uint32_t>(n * K * 2), &S.full[s]);
                bulk_load(dst + kValues, (q ? p.up_idx : p.gate_idx) + at, static_cast<uint32_t>(n * K), &S.full[s]);
            }
    };
    int copied = 0;  // rounds
    if (threadIdx.x == 0)
        for (; copied < rounds && copied < stages; ++copied) copy(copied, copied);
    // this lane's group of a set of G = 4, and its row of the first set's group in every byte
    const int my = G < kF ? g >> p.log_g : 0;
    const uint32_t row0 = static_cast<uint32_t>(g & (G - 1));
    // the rows of a group (four or eight here) share the check of its eight index sets
    const int sharing = G < kF ? G : kF;
    bool bad = false, ok = true;
    float c[MT][NT][4] = {};
    int s = 0;
    uint32_t ph = 0u;
    // the tokens of a step are loaded a step ahead: their way from L2 is the length of one
    uint4 x[NT];
    load_tokens<NT>(x, p, g, warp * kSteps * 32 + t * 8);
    for (int r = 0; r < rounds; ++r) {
        ok = tc::mbar_wait(&S.full[s], ph, abort, p.status);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const unsigned char *gate = smem + s * stage + my * kHalf, *up = gate + groups * kHalf;
#pragma unroll
        for (int q = 0; q < kSteps; ++q) {
            const int at = warp * kSteps * 32 + q * 32 + t * 8, k = r * kRound + at;
            uint4 next[NT];
            load_tokens<NT>(next, p, g, k + (q < kSteps - 1 ? 32 : kRound - (kSteps - 1) * 32));
            uint4 a[MT], b[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) a[m] = b[m] = make_uint4(0u, 0u, 0u, 0u);
            if (k < p.D) {
                Run<K> run;
                load_run(run, gate + at * K * 2, gate + kValues + at * K);
#pragma unroll
                for (int m = 0; m < MT; ++m) a[m] = pick(run, (row0 + 8 * m) * 0x01010101u);
                load_run(run, up + at * K * 2, up + kValues + at * K);
#pragma unroll
                for (int m = 0; m < MT; ++m) b[m] = pick(run, (row0 + 8 * m) * 0x01010101u);
                for (int e = g & (sharing - 1); e < 8; e += sharing)
                    bad |= bad_set<K>(gate + kValues + (at + e) * K, G) || bad_set<K>(up + kValues + (at + e) * K, G);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    mma_bf16(c[m][i], a[m].x, b[m].x, a[m].y, b[m].y, x[i].x, x[i].y);
                    mma_bf16(c[m][i], a[m].z, b[m].z, a[m].w, b[m].w, x[i].z, x[i].w);
                }
#pragma unroll
            for (int i = 0; i < NT; ++i) x[i] = next[i];
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&S.empty[s]);
        // the stage that this round leaves, once every warp has (a wait that expires sets the abort flag, on which
        // the warps stop together)
        if (threadIdx.x == 0 && copied < rounds && !*abort && tc::mbar_wait(&S.empty[s], ph, abort, p.status))
            copy(copied++, s);
        __syncwarp();
        if (++s == stages) {
            s = 0;
            ph ^= 1u;
        }
    }
    if (bad) report(p.status, CCI_ERR_INDEX);
    // no copy is in flight when the block ends or the sums take the stages' place, also after an abort
    if (threadIdx.x == 0) {
        int no_abort = 0;
        for (int r = copied > stages ? copied - stages : 0; r < copied; ++r)
            tc::mbar_wait(&S.full[r % stages], (r / stages) & 1, &no_abort, p.status);
    }
    __syncthreads();
    join<MT, NT>(p, reinterpret_cast<float *>(smem), c, f0);
}

// NT: tokens of a block (blockIdx.y takes the next NT), CH: its channels
template <int NT, int CH>
__global__ void __launch_bounds__(kThreads, 2) f32_kernel(Args p)
{
    constexpr int kRows = 2 * CH;
    __shared__ float red[kWarps][NT * kRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int f0 = blockIdx.x * CH, n0 = blockIdx.y * NT;
    const int64_t D = p.D;
    const float *X = static_cast<const float *>(p.X) + n0 * D;
    const float *wg = static_cast<const float *>(p.Wg) + f0 * D, *wu = static_cast<const float *>(p.Wu) + f0 * D;
    float c[kRows][NT];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int i = 0; i < NT; ++i) c[r][i] = 0.f;
    for (int k = (warp * 32 + lane) * 4; k < p.D; k += kThreads * 4) {
        float4 x[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i)
            x[i] = n0 + i < p.N ? __ldg(reinterpret_cast<const float4 *>(X + i * D + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
        float w[kRows][4];
#pragma unroll
        for (int r = 0; r < CH; ++r) {
            row::unpack<float, 4>(row::load_once<float, 4>(wg + r * D + k), w[r]);
            row::unpack<float, 4>(row::load_once<float, 4>(wu + r * D + k), w[CH + r]);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                c[r][i] = fmaf(w[r][0], x[i].x, c[r][i]);
                c[r][i] = fmaf(w[r][1], x[i].y, c[r][i]);
                c[r][i] = fmaf(w[r][2], x[i].z, c[r][i]);
                c[r][i] = fmaf(w[r][3], x[i].w, c[r][i]);
            }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float s = row::warp_sum(c[r][i]);
            if (lane == 0) red[warp][i * kRows + r] = s;
        }
    __syncthreads();
    for (int o = threadIdx.x; o < NT * CH; o += kThreads) {
        const int ch = o % CH, n = o / CH;
        if (n0 + n < p.N) finish(p, &red[0][0], NT * kRows, n * kRows + ch, CH, n0 + n, f0 + ch, true);
    }
}

cudaError_t launch_bf16(const Args &p, cudaStream_t stream)
{
    const unsigned sets = static_cast<unsigned>(p.F / kF);
    if (p.N <= 8)
        bf16_kernel<1><<<sets, kThreads, 0, stream>>>(p);
    else
        bf16_kernel<2><<<(sets + 1) / 2, kThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

template <int K, int NT, int MT>
cudaError_t launch_packed(const Args &p, cudaStream_t stream)
{
    const int groups = (1 << p.log_g) < kF ? kF >> p.log_g : 1, stage = stage_bytes(K, groups);
    constexpr int sums = kWarps * MT * NT * 128 * static_cast<int>(sizeof(float));
    constexpr int blocks = packed_blocks(K, MT), budget = (blocks == 4 ? 54 : (blocks > 1 ? 72 : 192)) * 1024;
    const int rounds = (p.D + kRound - 1) / kRound;
    int stages = budget / stage < kMaxStages ? budget / stage : kMaxStages;
    if (stages > rounds) stages = rounds;
    const int bytes = stages * stage > sums ? stages * stage : sums;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(packed_kernel<K, NT, MT>, 200 * 1024, attr_cache);
    if (attr != cudaSuccess) return attr;
    packed_kernel<K, NT, MT><<<static_cast<unsigned>(p.F / (kF * MT)), kThreads, static_cast<size_t>(bytes), stream>>>(p, stages);
    return cudaGetLastError();
}

template <int K, int NT>
cudaError_t launch_packed_sets(const Args &p, cudaStream_t stream)
{
    if (p.log_g == 5) return launch_packed<K, NT, 4>(p, stream);
    if (p.log_g == 4) return launch_packed<K, NT, 2>(p, stream);
    if constexpr (K <= 4) return launch_packed<K, NT, 1>(p, stream);
    return cudaErrorInvalidValue;
}

template <int K>
cudaError_t launch_packed_tokens(const Args &p, cudaStream_t stream)
{
    return p.N <= 8 ? launch_packed_sets<K, 1>(p, stream) : launch_packed_sets<K, 2>(p, stream);
}

cudaError_t launch_f32(const Args &p, cudaStream_t stream)
{
    const unsigned sets = static_cast<unsigned>(p.F / 8);
    if (p.N == 1)
        f32_kernel<1, 8><<<sets, kThreads, 0, stream>>>(p);
    else if (p.N == 2)
        f32_kernel<2, 8><<<sets, kThreads, 0, stream>>>(p);
    else if (p.N <= 4)
        f32_kernel<4, 8><<<sets, kThreads, 0, stream>>>(p);
    else
        f32_kernel<8, 4><<<dim3(2 * sets, static_cast<unsigned>((p.N + 7) / 8)), kThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace few

// Up to 16 tokens, but for 9 to 16 of bf16 only where the tile kernel has no tile (32 channels) for each SM: past 8
// tokens the tokens' own reads, which every block makes, weigh as much as the weights.
//   bf16, here against tiles:  4096 -> 8192: 1 token 22.0 us and 25.3, 8 22.7 and 25.3, 16 32.1 and 25.5;
//                              1024 -> 8192: 16 tokens 11.3 and 9.3;  4096 -> 4096: 16 tokens 15.8 and 16.6;
//                              1024 -> 2048: 1 token 3.2 and 6.5, 16 4.2 and 6.5
//   fp32 (tiles work on planes made in a launch of their own):
//                              4096 -> 8192: 1 token 39.5 us and 246, 8 73 and 246, 16 142 and 246;
//                              1024 -> 2048: 1 token 3.8 and 30, 16 18 and 30
bool few_tokens(int dtype, int64_t N, int64_t F)
{
    return N <= 8 || (N <= 16 && (dtype == CCI_F32 || F < 32 * static_cast<int64_t>(row::sm_count())));
}

// Packed weights read as they are, against expanded and multiplied by tiles (4096 -> 8192): G = 8, K = 2 1 token
// 33.2 us and 62.7, 16 36.5 and 62.7; G = 32, K = 8 1 token 72.5 and 89, 16 78.5 and 89.  fp32 is always expanded: G = 8,
// K = 2, 4096 -> 4096 1 token 57 us and 21 with dense weights, 16 109 and 73, 500 205 and 218
bool few_packed(const GatedArgs &a)
{
    auto at16 = [](const void *q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
    return a.dtype == CCI_BF16 && a.N <= 16 && (a.G == 4 || a.G == 8 || a.G == 16 || a.G == 32) &&
           (a.K == 1 || a.K == 2 || a.K == 4 || a.K == 8) && 2 * a.K <= a.G && a.D * a.K % 16 == 0 && a.F % 8 == 0 &&
           at16(a.gate_idx) && at16(a.up_idx);
}

cudaError_t launch_few(const GatedArgs &a, const void *wg, const void *wu, bool packed, cudaStream_t stream)
{
    few::Args p{};
    p.X = a.X;
    p.Wg = wg;
    p.Wu = wu;
    p.gate_idx = a.gate_idx;
    p.up_idx = a.up_idx;
    p.H = a.H;
    p.g = a.g;
    p.u = a.u;
    p.N = static_cast<int>(a.N);
    p.D = static_cast<int>(a.D);
    p.F = static_cast<int>(a.F);
    p.act = a.act;
    p.status = a.status;
    if (a.dtype == CCI_F32) return few::launch_f32(p, stream);
    if (!packed) return few::launch_bf16(p, stream);
    while ((1 << p.log_g) < a.G) ++p.log_g;
    switch (a.K) {
        case 1: return few::launch_packed_tokens<1>(p, stream);
        case 2: return few::launch_packed_tokens<2>(p, stream);
        case 4: return few::launch_packed_tokens<4>(p, stream);
        default: return few::launch_packed_tokens<8>(p, stream);
    }
}

}  // namespace gated
}  // namespace cci
