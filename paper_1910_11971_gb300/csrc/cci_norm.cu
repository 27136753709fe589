// cci_norm.cu -- layer norm of rows, forward and backward.
//
//   y[n][c]  = (x[n][c] - mean[n]) * rstd[n] * w[c] + b[c],   rstd = 1 / sqrt(var + eps)
//   dx       = rstd * (g - mean(g) - xh * mean(g * xh)),      g = dy * w, xh = (x - mean) * rstd
//   dw[c]    = sum over n of dy * xh,  db[c] = sum over n of dy
//
// Memory bound in both directions (two or three row reads and writes, a dozen operations an
// element).  A row of up to 16384 columns belongs to a group of 32 to 1024 threads and is read
// from memory once: forward into registers, the next row while this one is reduced; backward by bulk copies into
// shared memory where it lies on whole 16-byte words, else likewise.  The variance is the mean square of the
// differences from the mean, not a difference
// of sums.  The backward pass takes its sums and then dx from shared memory, and keeps each
// thread's columns of dw and db in registers over all rows of its block; the blocks' sums go to the
// workspace and a second launch adds them in block order (a single block's go straight to dw and
// db), so the result does not depend on what finishes first.  Longer rows are read again for each pass.
// All sums are fp32.
#include "cci_rowops.cuh"
#include "cci_tc_common.cuh"

namespace cci {
namespace norm {

// threads of a block with row groups of TPR threads
constexpr int block_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

// blocks of an SM that the registers leave room for
constexpr int residents(int TPR, bool words, bool backward) { return TPR <= 256 ? (words && !backward ? 3 : 2) : 1; }

// Backward, rows on whole 16-byte words come by bulk copies into a ring of rows per group, as many ahead as shared
// memory holds; the copies of a row are counted in bytes on its stage's barrier.  Loads into registers, which
// other rows take, keep less of two wide rows on its way (bf16 16384 x 4096: 76 us, 71 so, 4000 x 16384 136 and 105;
// narrow rows lose, 60000 x 256 29 and 33).  Forward, with one row and no sums to keep, they are as good or better
// (bf16 16384 x 4096 50.8 us by copies, 48.8 so, 16000 x 2048 30.0 and 26.4, 8000 x 8192 81 and 73) and wait for nothing
constexpr int kMaxStages = 6;

struct Ring {
    uint64_t full[kMaxStages];
    int64_t lost;  // after an expired wait: the first row of the set at which the group's first thread stopped copying
};

// untiled bulk copy of `bytes` (a multiple of 16) to shared memory, completing on `bar`; both addresses on 16 bytes
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     tc::smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(tc::smem_u32(bar))
                 : "memory");
}

// A wait that expires sets the block's abort flag and the status word, and its rows come out as NaN.  The group's
// first thread copies no row into a stage whose last one it did not see land, and before the block ends, or its ring
// takes other values, waits (again with a limit) for the last copy to each stage.  Not inlined, and everything made again
// from the block's place: the rows' loop keeps its registers (4000 x 12288 bf16: 97.5 us inlined, 90.5 so)
template <int STAGES, int ROWS, int TPR>
__device__ __noinline__ void drain(Ring *rings, int64_t N, uint32_t *status)
{
    constexpr int kGroups = block_threads(TPR) / TPR;
    const int group = threadIdx.x / TPR;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups, n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    Ring &ring = rings[group];
    // a set of ROWS rows brings its last stages' copies only once it is summed
    const int64_t row = (ring.lost - n0) / step, rows = (N - n0 + step - 1) / step;
    int64_t issued = row > 0 ? row + STAGES - ROWS : STAGES;
    if (issued > rows) issued = rows;
    int no_abort = 0;
    for (int64_t r = issued > STAGES ? issued - STAGES : 0; r < issued; ++r)
        tc::mbar_wait(&ring.full[r % STAGES], static_cast<uint32_t>(r / STAGES) & 1u, &no_abort, status);
}

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }

// stages of a group's ring: `bytes` a stage, `groups` rings in a block, `blocks` blocks in an SM
constexpr int stages_of(int bytes, int groups, int blocks)
{
    const int fit = (200 * 1024 / blocks) / (bytes * groups);
    return fit < kMaxStages ? fit : kMaxStages;
}

// Parameters of wide rows, which no registers are left for, lie in shared memory; backward beside the ring, where that
// keeps two stages or more: bytes of them, and the ring's stages then.  From L2 they are 8 bytes an element again for
// every row (forward bf16 8000 x 8192 78.8 us, 73.3 so; fp32 16384 x 4096 126 and 121; backward bf16 4000 x 16384 184 and
// 105).  Not where a block has few rows (forward bf16 100 x 8192: 3.6 us, 4.2 with them), nor in the backward pass of
// fp32 rows (8000 x 8192: 6 % slower with it)
constexpr int kWideBudget = 224 * 1024;
constexpr int shared_params(int bytes, int stage) { return (kWideBudget - bytes) / stage >= 2 ? bytes : 0; }
constexpr int stages_beside(int params, int stage)
{
    const int fit = (kWideBudget - params) / stage;
    return fit < kMaxStages ? fit : kMaxStages;
}

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
        if (c < D)
            raw[i] = row::load_once<T, V>(x + c);
        else
            raw[i] = row::Raw<T, V>{};
    }
}

// pairs of a thread's columns: kP of them from kStep vectors at a time, vectors i .. i + kStep - 1
template <int V>
struct Pairs {
    static constexpr int kStep = V == 1 ? 2 : 1, kP = V == 1 ? 1 : V / 2;
    unsigned long long p[kP];
};

template <typename T, int V>
__device__ __forceinline__ Pairs<V> pairs_of(const row::Raw<T, V> *raw)
{
    Pairs<V> r;
    if constexpr (V == 1)
        r.p[0] = pack2(row::to_f32(raw[0].w), row::to_f32(raw[1].w));
    else
        row::unpack2<T, V>(raw[0], r.p);
    return r;
}

// the same from a row in memory: global (columns past D: zeros), or a stage of a ring, which holds zeros there
template <typename T, int V, int TPR, bool RING>
__device__ __forceinline__ Pairs<V> pairs_at(const T *x, int i, int t, int D)
{
    row::Raw<T, V> raw[Pairs<V>::kStep];
#pragma unroll
    for (int j = 0; j < Pairs<V>::kStep; ++j) {
        const int c = ((i + j) * TPR + t) * V;
        raw[j] = RING || c < D ? row::load<T, V>(x + c) : row::Raw<T, V>{};
    }
    return pairs_of<T, V>(raw);
}

// zeros in the columns past D of `rows` rows of a ring, which no copy writes (one group's threads)
template <typename T, int V, int E, int TPR>
__device__ __forceinline__ void zero_tails(unsigned char *ring, int rows, int t, int D)
{
    constexpr int kWidth = E * TPR;
    for (int r = 0; r < rows; ++r)
        for (int c = D + t * V; c < kWidth; c += TPR * V)
            *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(ring) + r * kWidth + c) = make_uint4(0u, 0u, 0u, 0u);
}

template <int V, int TPR>
__device__ __forceinline__ Pairs<V> params2(const float *w, int i, int t, int D, float missing)
{
    float f[2 * Pairs<V>::kP] = {};
#pragma unroll
    for (int j = 0; j < Pairs<V>::kStep; ++j) {
        const int c = ((i + j) * TPR + t) * V;
        if (c < D) params_at<V>(w, c, missing, f + j * V);
    }
    Pairs<V> r;
#pragma unroll
    for (int j = 0; j < Pairs<V>::kP; ++j) r.p[j] = pack2(f[2 * j], f[2 * j + 1]);
    return r;
}

// parameters in shared memory: the words of four of every V columns together, so that neighbours read neighbours
template <int V, int E, int TPR>
__device__ __forceinline__ void keep_params(float *to, const float *w, int t, int D, float missing)
{
    constexpr int kVectors = E * TPR / V;
    for (int z = t; z < kVectors; z += TPR) {
        float f[V] = {};
        if (z * V < D) params_at<V>(w, z * V, missing, f);
#pragma unroll
        for (int j = 0; j < V / 4; ++j)
            *reinterpret_cast<float4 *>(to + (j * kVectors + z) * 4) =
                make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
    }
}

template <int V, int E, int TPR>
__device__ __forceinline__ Pairs<V> kept_params(const float *from, int i, int t)
{
    constexpr int kVectors = E * TPR / V;
    Pairs<V> r;
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
        const float4 q = *reinterpret_cast<const float4 *>(from + (j * kVectors + i * TPR + t) * 4);
        r.p[2 * j] = pack2(q.x, q.y);
        r.p[2 * j + 1] = pack2(q.z, q.w);
    }
    return r;
}

template <typename T, int V, int TPR>
__device__ __forceinline__ void store_pairs(T *y, int i, int t, int D, const Pairs<V> &o)
{
    const int c = (i * TPR + t) * V;
    if constexpr (V == 1) {
        const float a = lo_of(o.p[0]), b = hi_of(o.p[0]);
        if (c < D) row::store<T, 1>(y + c, &a);
        if (c + TPR < D) row::store<T, 1>(y + c + TPR, &b);
    } else if (c < D) {
        row::store2<T, V>(y + c, o.p);
    }
}

// ---- forward: E columns per thread, in vectors of V.  Groups walk the rows; the next row is on its way while
// one is reduced.  Groups of up to 256 threads keep weight and bias in registers: bf16 rows of whole words up to 4096
// columns, others up to 2048 ----
// bytes of shared memory: weight and bias, where they are kept there (KEEP: rows enough for it)
template <int V, int E, int TPR, bool KEEP>
constexpr int kForwardBytes = KEEP && V > 1 && TPR > 256 ? 2 * E * TPR * static_cast<int>(sizeof(float)) : 0;

template <typename T, int V, int E, int TPR, bool KEEP>
__global__ void __launch_bounds__(block_threads(TPR), residents(TPR, (V > 1), false))
    norm_kernel(const T *x, int64_t ldx, int64_t N, int D, const float *w, const float *b, float eps, T *y, float *mean,
                float *rstd)
{
    constexpr int kGroups = block_threads(TPR) / TPR, kNV = E / V;
    constexpr bool kHold = TPR <= 256, kKept = kForwardBytes<V, E, TPR, KEEP> > 0;
    extern __shared__ __align__(16) float kept[];  // weight, then bias
    __shared__ float buf[kGroups][2][TPR / 32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float width = static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    row::Raw<T, V> raw[kNV];
    if (n0 < N) load_row<T, V, kNV, TPR>(raw, x + n0 * ldx, t, D);
    if constexpr (kKept) {
        keep_params<V, E, TPR>(kept, w, t, D, 1.f);
        keep_params<V, E, TPR>(kept + E * TPR, b, t, D, 0.f);
        __syncthreads();
    }
    constexpr int kStep = Pairs<V>::kStep, kP = Pairs<V>::kP;
    Pairs<V> wv[kHold ? E / 2 / kP : 1], bv[kHold ? E / 2 / kP : 1];
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < kNV; i += kStep) {
            wv[i / kStep] = params2<V, TPR>(w, i, t, D, 1.f);
            bv[i / kStep] = params2<V, TPR>(b, i, t, D, 0.f);
        }
    }
    for (int64_t n = n0; n < N; n += step) {
        Pairs<V> f[E / 2 / kP];
        float s[1], q[1];
        unsigned long long s2 = 0ull, q2 = 0ull;
#pragma unroll
        for (int i = 0; i < kNV; i += kStep) {
            f[i / kStep] = pairs_of<T, V>(raw + i);
#pragma unroll
            for (int j = 0; j < kP; ++j) s2 = row::add2(s2, f[i / kStep].p[j]);
        }
        s[0] = lo_of(s2) + hi_of(s2);
        if (n + step < N) load_row<T, V, kNV, TPR>(raw, x + (n + step) * ldx, t, D);
        row::group_sum<TPR>(s, buf[group][0], group, t);
        const float mu = s[0] / width;
        const unsigned long long minus_mu = pack2(-mu, -mu);
#pragma unroll
        for (int i = 0; i < kNV; i += kStep) {
#pragma unroll
            for (int j = 0; j < kP; ++j) {
                unsigned long long &v = f[i / kStep].p[j];
                v = row::add2(v, minus_mu);
                // columns past D add nothing
                const int c = (i * TPR + t) * V;
                unsigned long long sq = v;
                if (c >= D) sq = 0ull;
                if (V == 1 && c + TPR >= D) sq = pack2(lo_of(sq), 0.f);
                ffma2(q2, sq, sq);
            }
        }
        q[0] = lo_of(q2) + hi_of(q2);
        row::group_sum<TPR>(q, buf[group][1], group, t);
        const float r = 1.f / sqrtf(q[0] / width + eps);
        if (t == 0) {
            mean[n] = mu;
            rstd[n] = r;
        }
        const unsigned long long r2 = pack2(r, r);
#pragma unroll
        for (int i = 0; i < kNV; i += kStep) {
            if constexpr (kKept) {
                wv[0] = kept_params<V, E, TPR>(kept, i, t);
                bv[0] = kept_params<V, E, TPR>(kept + E * TPR, i, t);
            } else if constexpr (!kHold) {
                wv[0] = params2<V, TPR>(w, i, t, D, 1.f);
                bv[0] = params2<V, TPR>(b, i, t, D, 0.f);
            }
            Pairs<V> o;
#pragma unroll
            for (int j = 0; j < kP; ++j) {
                o.p[j] = bv[kHold ? i / kStep : 0].p[j];
                ffma2(o.p[j], row::mul2(f[i / kStep].p[j], r2), wv[kHold ? i / kStep : 0].p[j]);
            }
            store_pairs<T, V, TPR>(y + n * D, i, t, D, o);
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

// one row's share of dw and db, and of the sums of g = dy w and g xh (columns past D: dy is 0)
template <int V>
__device__ __forceinline__ void add_columns(const Pairs<V> &x, const Pairs<V> &dy, const Pairs<V> &w,
                                            unsigned long long minus_m, unsigned long long r, unsigned long long *dw,
                                            unsigned long long *db, unsigned long long &s0, unsigned long long &s1)
{
#pragma unroll
    for (int j = 0; j < Pairs<V>::kP; ++j) {
        const unsigned long long xh = row::mul2(row::add2(x.p[j], minus_m), r);
        ffma2(dw[j], dy.p[j], xh);
        db[j] = row::add2(db[j], dy.p[j]);
        const unsigned long long g = row::mul2(dy.p[j], w.p[j]);
        s0 = row::add2(s0, g);
        ffma2(s1, g, xh);
    }
}

// dx = (dy w - a - xh b) r
template <int V>
__device__ __forceinline__ Pairs<V> input_gradient(const Pairs<V> &x, const Pairs<V> &dy, const Pairs<V> &w,
                                                   unsigned long long minus_m, unsigned long long r,
                                                   unsigned long long minus_a, unsigned long long minus_b)
{
    Pairs<V> o;
#pragma unroll
    for (int j = 0; j < Pairs<V>::kP; ++j) {
        const unsigned long long xh = row::mul2(row::add2(x.p[j], minus_m), r);
        unsigned long long q = minus_a;
        ffma2(q, dy.p[j], w.p[j]);
        ffma2(q, xh, minus_b);
        o.p[j] = row::mul2(q, r);
    }
    return o;
}

// ---- backward: dx, and this block's sums of dw and db to pw and pb, each block 2 D further ----
// its shared memory: the ring, then the weight; after the rows, the groups' sums
template <typename T, int V, int E, int TPR>
struct Backward {
    static constexpr int kGroups = block_threads(TPR) / TPR;
    static constexpr bool kHold = TPR < 1024;  // the weight in registers
    static constexpr int kRow = E * TPR * static_cast<int>(sizeof(T)), kStage = 2 * kRow;  // a stage: x, then dy
    static constexpr int kParams = V > 1 && !kHold && sizeof(T) == 2 ? shared_params(E * TPR * 4, kStage) : 0;
    static constexpr int kStages = kParams ? stages_beside(kParams, kStage) : stages_of(kStage, kGroups, residents(TPR, (V > 1), true));
    static constexpr bool kBulk = V > 1 && kStages >= 2;
    // rows at a time, so that their sums share the exchanges and the barrier; a ring has one more such set at least
    static constexpr int kRows = kStages % 2 == 0 && kStages > 2 ? 2 : 1;
    static constexpr int kRing = kBulk ? kStages * kStage * kGroups + kParams : 0;
    static constexpr int kSums = kGroups > 1 ? 2 * E * TPR * static_cast<int>(sizeof(float)) : 0;
    static constexpr int kBytes = kRing > kSums ? kRing : kSums;
};

template <typename T, int V, int E, int TPR>
__global__ void __launch_bounds__(block_threads(TPR), residents(TPR, (V > 1), true))
    norm_backward_kernel(const T *dy, int64_t lddy, const T *x, int64_t ldx, const float *mean, const float *rstd,
                         const float *w, int64_t N, int D, T *dx, float *pw, float *pb, uint32_t *status)
{
    using C = Backward<T, V, E, TPR>;
    constexpr int kGroups = C::kGroups, kNV = E / V, kRow = C::kRow, kStage = C::kStage, kStages = C::kStages;
    // two stages at least; else, and for rows off whole words, a row is loaded into registers, or where 1024 threads
    // have none left, both passes over it read global memory, the second from L1
    constexpr bool kBulk = C::kBulk, kKeep = !kBulk && TPR < 1024, kHold = C::kHold, kKept = kBulk && C::kParams > 0;
    extern __shared__ __align__(128) unsigned char ring_raw[];
    __shared__ Ring rings[kGroups];
    __shared__ float buf[kGroups][2][4 * TPR / 32];
    __shared__ int abort_flag;
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float width = static_cast<float>(D);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    unsigned char *ring = ring_raw + group * kStages * kStage;
    float *kept = reinterpret_cast<float *>(ring_raw + kStages * kStage);  // with one group
    Ring &R = rings[group];
    volatile int *abort = &abort_flag;
    const uint32_t bytes = static_cast<uint32_t>(D) * sizeof(T);
    auto copy = [&](int64_t n, int s) {
        tc::mbar_arrive_expect_tx(&R.full[s], 2 * bytes);
        bulk_load(ring + s * kStage, x + n * ldx, bytes, &R.full[s]);
        bulk_load(ring + s * kStage + kRow, dy + n * lddy, bytes, &R.full[s]);
    };
    // the second launch, which adds the blocks' sums, may be scheduled: it waits for this one
    tc::launch_next_grid();
    if constexpr (kBulk) {
        if (threadIdx.x == 0) abort_flag = 0;
        zero_tails<T, V, E, TPR>(ring, 2 * kStages, t, D);
        if constexpr (kKept) keep_params<V, E, TPR>(kept, w, t, D, 1.f);
        if (t == 0) {
            for (int s = 0; s < kStages; ++s) tc::mbar_init(&R.full[s], 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            for (int s = 0; s < kStages; ++s)
                if (n0 + s * step < N) copy(n0 + s * step, s);
        }
        __syncthreads();
    }
    constexpr int kStep = Pairs<V>::kStep, kP = Pairs<V>::kP;
    unsigned long long dw[E / 2], db[E / 2];
    Pairs<V> wv[kHold ? E / 2 / kP : 1];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) dw[e] = db[e] = 0ull;
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < kNV; i += kStep) wv[i / kStep] = params2<V, TPR>(w, i, t, D, 1.f);
    }
    int k = 0;
    if constexpr (kBulk) {
        constexpr int kRows = C::kRows;
        int st = 0;
        uint32_t ph = 0u;
        bool ok = true;
        float mu[kRows], r[kRows];  // of the next rows
        auto stats_of = [&](int64_t n) {
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                mu[q] = n + q * step < N ? __ldg(mean + n + q * step) : 0.f;
                r[q] = n + q * step < N ? __ldg(rstd + n + q * step) : 0.f;
            }
        };
        stats_of(n0);
        for (int64_t n = n0; n < N; n += kRows * step, k ^= 1) {
            float s[4] = {0.f, 0.f, 0.f, 0.f};
            float m[kRows], rn[kRows];
            const T *xr[kRows], *dr[kRows];
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                xr[q] = reinterpret_cast<const T *>(ring + (st + q) * kStage);
                dr[q] = reinterpret_cast<const T *>(ring + (st + q) * kStage + kRow);
                m[q] = mu[q];
                rn[q] = r[q];
            }
            stats_of(n + kRows * step);
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                if (q > 0 && n + step >= N) break;
                // after a wait that expired every thread goes on, none is left at a barrier, with NaN in the row's sums
                // and in its own columns of dw and db from then on
                if (ok && !tc::mbar_wait(&R.full[st + q], ph, abort, status)) {
                    ok = false;
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) dw[e] = db[e] = pack2(nan_f(), nan_f());
                    if (t == 0) R.lost = n;
                }
                const unsigned long long minus_m = pack2(-m[q], -m[q]), rn2 = pack2(rn[q], rn[q]);
                unsigned long long s0 = 0ull, s1 = 0ull;
#pragma unroll
                for (int i = 0; i < kNV; i += kStep) {
                    const Pairs<V> xp = pairs_at<T, V, TPR, true>(xr[q], i, t, D);
                    const Pairs<V> gp = pairs_at<T, V, TPR, true>(dr[q], i, t, D);
                    if constexpr (kKept)
                        wv[0] = kept_params<V, E, TPR>(kept, i, t);
                    else if constexpr (!kHold)
                        wv[0] = params2<V, TPR>(w, i, t, D, 1.f);
                    add_columns<V>(xp, gp, wv[kHold ? i / kStep : 0], minus_m, rn2, dw + i / kStep * kP, db + i / kStep * kP, s0, s1);
                }
                s[2 * q] = ok ? lo_of(s0) + hi_of(s0) : nan_f();
                s[2 * q + 1] = ok ? lo_of(s1) + hi_of(s1) : nan_f();
            }
            row::group_sum4<TPR>(s, buf[group][k], group, t);
            // every thread of the group has left the rows before these: their stages take the rows after these
            if (ok && t == 0 && n > n0) {
#pragma unroll
                for (int q = 0; q < kRows; ++q) {
                    const int64_t next = n + (kStages - kRows + q) * step;
                    if (next < N) copy(next, (st == 0 ? kStages : st) - kRows + q);
                }
            }
            if ((st += kRows) == kStages) {
                st = 0;
                ph ^= 1u;
            }
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                if (q > 0 && n + step >= N) break;
                const unsigned long long minus_m = pack2(-m[q], -m[q]), rn2 = pack2(rn[q], rn[q]);
                const float a = s[2 * q] / width, bq = s[2 * q + 1] / width;
                const unsigned long long minus_a = pack2(-a, -a), minus_b = pack2(-bq, -bq);
#pragma unroll
                for (int i = 0; i < kNV; i += kStep) {
                    const Pairs<V> xp = pairs_at<T, V, TPR, true>(xr[q], i, t, D);
                    const Pairs<V> gp = pairs_at<T, V, TPR, true>(dr[q], i, t, D);
                    if constexpr (kKept)
                        wv[0] = kept_params<V, E, TPR>(kept, i, t);
                    else if constexpr (!kHold)
                        wv[0] = params2<V, TPR>(w, i, t, D, 1.f);
                    store_pairs<T, V, TPR>(dx + (n + q * step) * D, i, t, D,
                                           input_gradient<V>(xp, gp, wv[kHold ? i / kStep : 0], minus_m, rn2, minus_a, minus_b));
                }
            }
        }
        if (!ok && t == 0) drain<kStages, kRows, TPR>(rings, N, status);
    } else {
        float mu = 0.f, r = 0.f;
        row::Raw<T, V> nx[kKeep ? kNV : 1], nd[kKeep ? kNV : 1];  // the next row
        if (n0 < N) {
            mu = __ldg(mean + n0);
            r = __ldg(rstd + n0);
            if constexpr (kKeep) {
                load_row<T, V, kNV, TPR>(nx, x + n0 * ldx, t, D);
                load_row<T, V, kNV, TPR>(nd, dy + n0 * lddy, t, D);
            }
        }
        for (int64_t n = n0; n < N; n += step, k ^= 1) {
            const unsigned long long minus_m = pack2(-mu, -mu), rn2 = pack2(r, r);
            if (n + step < N) {
                mu = __ldg(mean + n + step);
                r = __ldg(rstd + n + step);
            }
            const T *xr = x + n * ldx, *dr = dy + n * lddy;
            row::Raw<T, V> rx[kKeep ? kNV : 1], rd[kKeep ? kNV : 1];
            if constexpr (kKeep) {
#pragma unroll
                for (int i = 0; i < kNV; ++i) {
                    rx[i] = nx[i];
                    rd[i] = nd[i];
                }
                if (n + step < N) {
                    load_row<T, V, kNV, TPR>(nx, x + (n + step) * ldx, t, D);
                    load_row<T, V, kNV, TPR>(nd, dy + (n + step) * lddy, t, D);
                }
            }
            unsigned long long s0 = 0ull, s1 = 0ull;
#pragma unroll
            for (int i = 0; i < kNV; i += kStep) {
                const Pairs<V> xp = kKeep ? pairs_of<T, V>(rx + (kKeep ? i : 0)) : pairs_at<T, V, TPR, false>(xr, i, t, D);
                const Pairs<V> gp = kKeep ? pairs_of<T, V>(rd + (kKeep ? i : 0)) : pairs_at<T, V, TPR, false>(dr, i, t, D);
                if constexpr (!kHold) wv[0] = params2<V, TPR>(w, i, t, D, 1.f);
                add_columns<V>(xp, gp, wv[kHold ? i / kStep : 0], minus_m, rn2, dw + i / kStep * kP, db + i / kStep * kP, s0, s1);
            }
            float s[2] = {lo_of(s0) + hi_of(s0), lo_of(s1) + hi_of(s1)};
            row::group_sum<TPR>(s, buf[group][k], group, t);
            const float a = s[0] / width, bq = s[1] / width;
            const unsigned long long minus_a = pack2(-a, -a), minus_b = pack2(-bq, -bq);
#pragma unroll
            for (int i = 0; i < kNV; i += kStep) {
                const Pairs<V> xp = kKeep ? pairs_of<T, V>(rx + (kKeep ? i : 0)) : pairs_at<T, V, TPR, false>(xr, i, t, D);
                const Pairs<V> gp = kKeep ? pairs_of<T, V>(rd + (kKeep ? i : 0)) : pairs_at<T, V, TPR, false>(dr, i, t, D);
                if constexpr (!kHold) wv[0] = params2<V, TPR>(w, i, t, D, 1.f);
                store_pairs<T, V, TPR>(dx + n * D, i, t, D,
                                       input_gradient<V>(xp, gp, wv[kHold ? i / kStep : 0], minus_m, rn2, minus_a, minus_b));
            }
        }
    }
    // the rings are done with (every copy was waited for, after a wait that expired by drain): the groups' sums take
    // their place
    float *comb = reinterpret_cast<float *>(ring_raw);
    const bool pw_ok = pw != nullptr, pb_ok = pb != nullptr;
    // the groups' sums, added in group order
    if constexpr (kGroups > 1) {
        unsigned long long *cp = reinterpret_cast<unsigned long long *>(comb);
        for (int q = 1; q < kGroups; ++q) {
            __syncthreads();
            if (group == q) {
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    cp[(2 * e) * TPR + t] = dw[e];
                    cp[(2 * e + 1) * TPR + t] = db[e];
                }
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    dw[e] = row::add2(dw[e], cp[(2 * e) * TPR + t]);
                    db[e] = row::add2(db[e], cp[(2 * e + 1) * TPR + t]);
                }
            }
        }
    }
    if (group == 0) {
        pw += static_cast<int64_t>(blockIdx.x) * 2 * D;
        pb += static_cast<int64_t>(blockIdx.x) * 2 * D;
        if (V > 1 && (reinterpret_cast<uintptr_t>(pw) | reinterpret_cast<uintptr_t>(pb)) % 16 == 0) {
#pragma unroll
            for (int e = 0; e < E / 2; e += 2) {  // four neighbouring columns
                const int c = (e / kP * kStep * TPR + t) * V + e % kP * 2;
                if (c < D) {
                    if (pw_ok) *reinterpret_cast<float4 *>(pw + c) = make_float4(lo_of(dw[e]), hi_of(dw[e]), lo_of(dw[e + 1]), hi_of(dw[e + 1]));
                    if (pb_ok) *reinterpret_cast<float4 *>(pb + c) = make_float4(lo_of(db[e]), hi_of(db[e]), lo_of(db[e + 1]), hi_of(db[e + 1]));
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const int c = (e / kP * kStep * TPR + t) * V + e % kP * 2, d = V == 1 ? c + TPR : c + 1;
                if (c < D) {
                    if (pw_ok) pw[c] = lo_of(dw[e]);
                    if (pb_ok) pb[c] = lo_of(db[e]);
                }
                if (d < D) {
                    if (pw_ok) pw[d] = hi_of(dw[e]);
                    if (pb_ok) pb[d] = hi_of(db[e]);
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
                            int64_t N, int64_t D, float *pw, float *pb)
{
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= D) return;
    float dw = 0.f, db = 0.f;
    for (int64_t n = blockIdx.y; n < N; n += gridDim.y) {
        const float g = row::to_f32(dy[n * lddy + c]);
        dw += g * (row::to_f32(x[n * ldx + c]) - __ldg(mean + n)) * __ldg(rstd + n);
        db += g;
    }
    const int64_t part = static_cast<int64_t>(blockIdx.y) * 2 * D;
    if (pw) pw[part + c] = dw;
    if (pb) pb[part + c] = db;
}

// dw and db: the sums of the parts.  A block takes 32 columns; V of them a thread (4 where D is even, so that every
// part starts on 16 bytes), the parts in 32 V interleaved shares, so that all loads of a thread are on their way
// at once; the shares are added in order
template <int V>
__global__ void __launch_bounds__(1024)
    norm_params_kernel(const float *part, int parts, int64_t D, float *dw, float *db)
{
    constexpr int kLanes = 32 / V, kShares = 32 * V;
    __shared__ float sh[kShares][33];
    tc::wait_prior_grid();
    const int q = threadIdx.x % kLanes, share = threadIdx.x / kLanes;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + q * V;
    float s[V] = {};
    if (c < 2 * D) {
#pragma unroll 4
        for (int p = share; p < parts; p += kShares) {
            const float *at = part + static_cast<int64_t>(p) * 2 * D + c;
            if constexpr (V == 4) {
                const float4 v = *reinterpret_cast<const float4 *>(at);
                s[0] += v.x;
                s[1] += v.y;
                s[2] += v.z;
                s[3] += v.w;
            } else {
                s[0] += *at;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sh[share][q * V + j] = s[j];
    __syncthreads();
    // warp w adds column w's shares
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) sum += sh[lane + 32 * j][w];
    sum = row::warp_sum(sum);
    const int64_t d = static_cast<int64_t>(blockIdx.x) * 32 + w;
    if (lane == 0 && d < 2 * D) {
        if (d < D) {
            if (dw) dw[d] = sum;
        } else if (db) {
            db[d - D] = sum;
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
    float *mean, *rstd;
    float *dw, *db, *part;
    int *parts;  // written: parts of the sums
    uint32_t *status;
    cudaStream_t stream;
};

// where the first part of the sums goes: to the gradients themselves if it is the only one
float *first_dw(const Args &a) { return *a.parts == 1 ? a.dw : a.part; }
float *first_db(const Args &a) { return *a.parts == 1 ? a.db : a.part + a.D; }

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
int64_t backward_blocks(int e, bool words, int64_t N, int64_t D)
{
    if (D > kRegisterColumns) return least(N, 16);
    const int tpr = group_threads(e, D), groups = block_threads(tpr) / tpr;
    return least((N + groups - 1) / groups, static_cast<int64_t>(row::sm_count()) * residents(tpr, words, true));
}

// the most parts of any form of a call
int64_t most_parts(int64_t N, int64_t D)
{
    const int64_t a = backward_blocks(8, true, N, D), b = backward_blocks(16, true, N, D);  // off whole words: fewer
    return a > b ? a : b;
}

template <typename T, int V, int E, int TPR, bool KEEP>
cudaError_t forward_as(const Args &a, int64_t blocks)
{
    constexpr int kT = block_threads(TPR), bytes = kForwardBytes<V, E, TPR, KEEP>;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(norm_kernel<T, V, E, TPR, KEEP>, bytes, attr_cache);
    if (attr != cudaSuccess) return attr;
    norm_kernel<T, V, E, TPR, KEEP><<<static_cast<unsigned>(blocks), kT, bytes, a.stream>>>(
        static_cast<const T *>(a.x), a.ldx, a.N, static_cast<int>(a.D), a.w, a.b, a.eps, static_cast<T *>(a.y), a.mean,
        a.rstd);
    return cudaGetLastError();
}

template <typename T, int V, int E, int TPR>
cudaError_t forward_one(const Args &a)
{
    constexpr int kGroups = block_threads(TPR) / TPR;
    const int64_t blocks = least((a.N + kGroups - 1) / kGroups, static_cast<int64_t>(row::sm_count()) * residents(TPR, (V > 1), false));
    if constexpr (kForwardBytes<V, E, TPR, true> > 0)
        if (a.N > 4 * blocks) return forward_as<T, V, E, TPR, true>(a, blocks);  // rows enough for it
    return forward_as<T, V, E, TPR, false>(a, blocks);
}

template <typename T, int V, int E, int TPR>
cudaError_t backward_one(const Args &a)
{
    constexpr int kT = block_threads(TPR), bytes = Backward<T, V, E, TPR>::kBytes;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(norm_backward_kernel<T, V, E, TPR>, bytes, attr_cache);
    if (attr != cudaSuccess) return attr;
    *a.parts = static_cast<int>(backward_blocks(thread_columns<T, V>(), V > 1, a.N, a.D));
    norm_backward_kernel<T, V, E, TPR><<<static_cast<unsigned>(*a.parts), kT, bytes, a.stream>>>(
        static_cast<const T *>(a.dy), a.lddy, static_cast<const T *>(a.x), a.ldx, a.mean_in, a.rstd_in, a.w, a.N,
        static_cast<int>(a.D), static_cast<T *>(a.y), first_dw(a), first_db(a), a.status);
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
        if (e != cudaSuccess || (!a.dw && !a.db)) return e;
        *a.parts = static_cast<int>(backward_blocks(8, true, a.N, a.D));
        const dim3 grid(static_cast<unsigned>((a.D + 255) / 256), static_cast<unsigned>(*a.parts));
        norm_long_params_kernel<T><<<grid, 256, 0, a.stream>>>(static_cast<const T *>(a.dy), a.lddy,
                                                               static_cast<const T *>(a.x), a.ldx, a.mean_in,
                                                               a.rstd_in, a.N, a.D, first_dw(a), first_db(a));
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
                                       float *dw, float *db, float *part, uint32_t *status, cudaStream_t stream)
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
    a.dw = dw;
    a.db = db;
    a.part = part;
    a.parts = &parts;
    a.status = status;
    a.stream = stream;
    if (N > 0) {
        const cudaError_t e = dtype == CCI_F32 ? norm::backward<float>(a) : norm::backward<uint16_t>(a);
        if (e != cudaSuccess) return e;
    }
    if (parts == 1 || (!dw && !db)) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((2 * D + 31) / 32));
    cfg.blockDim = dim3(1024);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    const cudaError_t e = D % 2 == 0
                              ? cudaLaunchKernelEx(&cfg, norm::norm_params_kernel<4>, const_cast<const float *>(part), parts, D, dw, db)
                              : cudaLaunchKernelEx(&cfg, norm::norm_params_kernel<1>, const_cast<const float *>(part), parts, D, dw, db);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace cci
