// cci_head.cu -- softmax cross entropy from a head's inputs: the logits z = X W^T of N tokens over V
// entries are computed tile by tile and never kept.
//
//   forward   m = max z, s = sum exp(z - m), loss = log s - (z_t - m): the product's output warps take
//             their columns' maximum and sum where they lie, in registers, and write two numbers per
//             token and 128 columns; a second launch joins them in order.
//   backward  P = dloss (softmax(z) - 1[t]) in pieces of the vocabulary: the product again, its output
//             warps write P's piece in bf16 (fp32: three planes, as every operand; cci_gated.cuh), and
//             two more products take dX += P W and dW = P^T X from it.  dX's sum over the pieces is
//             fp32, rounded once.
//
// What bounds it: 2 N D V operations forward and 6 N D V backward on the tensor cores for many tokens, one read of W
// forward for few.  P is rounded to bf16 (2^-8 of each of its values at most) because it is an operand of the tensor core.
//
// The tensor core cuts its running sum at every addition, always towards zero: 256 of them, at D = 4096, leave a logit
// of 12 about 6e-5 off, and a confident token's loss, a difference of such logits, as much of itself and more.  So the
// forward pass adds about eight stages (512 reduction indices, 704 at most) at a time there and the chunks in registers, to the nearest, as
// fp32 does throughout (1999 x 4096 x 50257 bf16: 421 us with one running sum, 437 so, 579 with chunks of 256).  That takes
// eight output warps, each 32 tokens by half of a tile's columns.  The backward pass adds as the forward pass does: a sure token's
// gradient, p - 1, is the difference of its logit from what the forward pass made of the same sums (with one running
// sum a p of 0.999 was 2 % of its 1 - p off).
//
// Tiles: 256 tokens x 256 columns over a CTA pair, or for few tokens or columns 128 x 256 and 128 x 128 on one CTA.
// Sixteen M tiles at a time pass over the vocabulary, so that W is read once for up to 4096 tokens.
// Every wait is bounded, as in the gated block's products.
#include "cci_gated.cuh"
#include "cci_head_few.cuh"

namespace cci {
namespace head {

using gated::load_3d;
using gated::Operand;
using gated::operand_map;
using gated::stage_mma;
using gated::term_planes;
using gated::tile_desc;

// stages that the tensor core adds up by itself, of a tile's n: about eight of many, up to eleven of up to 33, where the output
// warps are what a tile waits for (4096 x 2048 x 131072 bf16 both passes: 5235 us with eight, 5084 so; 4096 tokens by 32768, forward:
// 1280 wide 194 and 171, 1408 212 and 192, 1792 275 and 248, 2112 309 and 302; widths between 1408 and 1792, and from 2176 on, are cut alike by
// both)
inline int chunk_of(int n)
{
    const int chunks = n <= 33 ? (n + 10) / 11 : (n + 4) / 8;
    return (n + chunks - 1) / chunks;
}
constexpr int kMTilesAtOnce = 16;

// one launch: a piece of the vocabulary
struct Params {
    int64_t M, N;       // tokens; columns of the piece
    int64_t col0, V;    // the piece's first column; columns of the whole
    int k_stages, terms, chunk;
    int a_rows;         // rows of A's box
    int m_tiles, n_tiles, tiles;
    const int64_t *targets;
    int64_t ignore;
    // forward
    float2 *parts;      // [2 n_tiles][M]: maximum and sum of half a tile's columns
    float *at_target;   // [M]: the target's logit
    // backward
    const float *stats, *dloss;
    uint32_t *status;
};

struct Maps {
    CUtensorMap a, b, out[3];  // out: P, its planes
};

template <int CG, int BN, bool PROBS>
struct Cfg {
    static constexpr int kM = 128, kBRows = BN / CG;
    static constexpr int kABytes = kM * 128, kBBytes = kBRows * 128, kStage = kABytes + kBBytes;
    // buffers of 64 columns for each four output warps: two where five stages or more are left beside them
    static constexpr int kOut = kM * 128, kBufs = 5 * kStage + 4 * kOut + 2048 <= static_cast<int>(kMaxSmemPerBlock) ? 2 : 1;
    static constexpr int kOuts = PROBS ? 2 * kBufs : 0;
    static constexpr int kFit = (static_cast<int>(kMaxSmemPerBlock) - 2048 - kOuts * kOut) / kStage;
    static constexpr int kStages = kFit < 8 ? kFit : 8;
    static constexpr int kTmem = 2 * BN;
    static constexpr int kThreads = 384;  // a warp for copies, one for products, one for tensor memory, one idle, eight for output
    static constexpr int kCols = BN / 2;  // of an output warp
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStage + kOuts * kOut + 1024;
    static_assert(kStage % 1024 == 0 && kStages >= 4 && kSmem <= kMaxSmemPerBlock, "stages");
    static_assert(kTmem == 256 || kTmem == 512, "tensor memory comes in powers of two");
};

struct Smem {
    uint64_t full[8], empty[8];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};
static_assert(sizeof(Smem) <= 1024, "barriers");

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// exp(x) for x <= 0 or so: the difference from the maximum is taken before, in fp32
__device__ __forceinline__ float exp_of(float x) { return __expf(x); }

// z to z log2(e) - r with r the product m log2(e) as it is rounded: one fused operation, whose only rounding is that of the
// exponent, as if the difference z - m were taken first.  What r lacks of m log2(e) is returned, one factor for all, 1/2 at most:
// for larger logits than that leaves, the difference does come first
template <int N>
__device__ __forceinline__ float to_exponents(float (&z)[N], float m)
{
    const float r = m * kLog2e;
    if (!(fabsf(r) < 16777216.f)) {
#pragma unroll
        for (int j = 0; j < N; ++j) z[j] = (z[j] - m) * kLog2e;
        return 0.f;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) z[j] = fmaf(z[j], kLog2e, -r);
    return fmaf(m, kLog2e, -r);
}

// sixteen columns of this warp's TMEM lanes, without waiting for them
__device__ __forceinline__ void tmem_ld16_begin(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr));
}

// and waited for: they are operands, so that nothing takes them before
__device__ __forceinline__ void tmem_ld16_end(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

__device__ __forceinline__ void tile_at(const Params &p, int tile, int &mt, int &nt)
{
    const int per = kMTilesAtOnce * p.n_tiles, g = tile / per, r = tile - g * per;
    const int left = p.m_tiles - kMTilesAtOnce * g, gm = left < kMTilesAtOnce ? left : kMTilesAtOnce;
    nt = r / gm;
    mt = kMTilesAtOnce * g + r - nt * gm;
}

template <int CG, int BN, bool PROBS>
__global__ void __launch_bounds__(Cfg<CG, BN, PROBS>::kThreads, 1)
    head_kernel(const Params p, const __grid_constant__ Maps maps)
{
    using C = Cfg<CG, BN, PROBS>;
    constexpr int kStages = C::kStages;
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(BN >> 3) << 17) |
                                (static_cast<uint32_t>((C::kM * CG) >> 4) << 24);
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const uint32_t raw = tc::smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t outs = base + kStages * C::kStage;
    Smem *S = reinterpret_cast<Smem *>(smem_raw + (outs - raw) + C::kOuts * C::kOut);
    volatile int *abort = &S->abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? ws::cluster_rank() : 0u;
    const int first = static_cast<int>(blockIdx.x) / CG, step = static_cast<int>(gridDim.x) / CG;
    const int per_tile = p.terms * p.k_stages;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&S->full[s], 1);
            tc::mbar_init(&S->empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            tc::mbar_init(&S->acc_full[a], 1);
            tc::mbar_init(&S->acc_empty[a], 8 * CG);
        }
        tc::mbar_init(&S->drain, 1);
        S->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                             tc::smem_u32(&S->tmem_base)),
                         "r"(C::kTmem)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                             tc::smem_u32(&S->tmem_base)),
                         "r"(C::kTmem)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) ws::cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = S->tmem_base;
    if constexpr (!PROBS) tc::launch_next_grid();  // the losses' launch, which waits for this one's end

    // output threads hold up to 128 sums each: 128 threads give up 96 of their 168 registers, and 256 take 48 more
    if (warp < 4) {
        if constexpr (C::kCols == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0) {
            // ---- copies
            if (tc::elect_one()) {
                const uint32_t bytes = CG * (static_cast<uint32_t>(p.a_rows) * 128u + static_cast<uint32_t>(C::kBBytes));
                int s = 0, it = 0;
                uint32_t ph = 1u;  // a fresh barrier's preceding phase counts as complete
                bool ok = true;
                for (int tile = first; ok && tile < p.tiles; tile += step) {
                    int mt, nt, ks = 0, t = 0, pa, pb;
                    tile_at(p, tile, mt, nt);
                    const int m0 = (mt * CG + static_cast<int>(rank)) * C::kM;
                    const int n0 = nt * BN + static_cast<int>(rank) * C::kBRows;
                    term_planes(0, p.terms, pa, pb);
                    for (int i = 0; i < per_tile; ++i, ++it) {
                        ok = tc::mbar_wait(&S->empty[s], ph, abort, p.status);
                        if (!ok) break;
                        const uint32_t sa = base + s * C::kStage;
                        uint32_t bar = tc::smem_u32(&S->full[s]);
                        if (rank == 0) tc::mbar_arrive_expect_tx(&S->full[s], bytes);
                        if constexpr (CG == 2) bar = ws::map_to_rank(bar, 0);
                        load_3d<CG>(sa, &maps.a, ks * 64, m0, pa, bar);
                        load_3d<CG>(sa + C::kABytes, &maps.b, ks * 64, n0, pb, bar);
                        if (++s == kStages) {
                            s = 0;
                            ph ^= 1u;
                        }
                        // all terms of a stage one after the other: what they share comes from L2
                        if (++t == p.terms) {
                            t = 0;
                            ++ks;
                        }
                        term_planes(t, p.terms, pa, pb);
                    }
                }
                // no copy is in flight when the block ends, nor a commit, also after an abort (as in the gated block's products)
                int no_abort = 0;
                if (rank == 0)
                    for (int d = it > kStages ? it - kStages : 0; d < it; ++d)
                        tc::mbar_wait(&S->full[d % kStages], (d / kStages) & 1, &no_abort, p.status);
                no_abort = 0;
                for (int d = it > kStages ? it - kStages : 0; d < it; ++d)
                    tc::mbar_wait(&S->empty[d % kStages], (d / kStages) & 1, &no_abort, p.status);
            }
            __syncwarp();
        } else if (warp == 1 && rank == 0) {
            // ---- products
            if (tc::elect_one()) {
                int s = 0, t = 0;
                uint32_t ph = 0u;
                bool ok = true;
                const uint64_t da0 = tile_desc<false>(base), db0 = tile_desc<false>(base + C::kABytes);
                const uint32_t empty0 = tc::smem_u32(&S->empty[0]);
                for (int tile = first; ok && tile < p.tiles; tile += step) {
                    for (int left = per_tile; left > 0 && ok; left -= p.chunk, ++t) {
                        const int acc = t & 1, n = left < p.chunk ? left : p.chunk;
                        if (t >= 2) ok = tc::mbar_wait<CG == 2>(&S->acc_empty[acc], ((t >> 1) - 1) & 1, abort, p.status);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t d = tmem + static_cast<uint32_t>(acc * BN);
                        for (int i = 0; i < n; ++i) {
                            ok = tc::mbar_wait(&S->full[s], ph, abort, p.status);
                            if (!ok) break;
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            const uint64_t off = static_cast<uint64_t>(s) * (C::kStage >> 4);
                            stage_mma<CG, kIdesc, 2, 2>(d, da0 + off, db0 + off, i > 0 ? 1u : 0u, empty0 + 8u * s);
                            if (++s == kStages) {
                                s = 0;
                                ph ^= 1u;
                            }
                        }
                        if (ok) {
                            if constexpr (CG == 2)
                                ws::mma_commit_pair(&S->acc_full[acc]);
                            else
                                tc::mma_commit(&S->acc_full[acc]);
                        }
                    }
                }
                // every product has ended before the tensor memory is given back
                if constexpr (CG == 2)
                    ws::mma_commit_pair(&S->drain);
                else
                    tc::mma_commit(&S->drain);
                int no_abort = 0;
                tc::mbar_wait(&S->drain, 0, &no_abort, p.status);
            }
            __syncwarp();
        }
    } else {
        if constexpr (C::kCols == 128) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- output: row `m` of the CTA's 128 and kCols columns from c0 of the tile on, per thread
        const int half = (warp - 4) >> 2, m = tid & 127, c0 = half * C::kCols;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t acc_empty0 = CG == 2 ? ws::map_to_rank(tc::smem_u32(&S->acc_empty[0]), 0) : 0u;
        const uint32_t bufs = outs + static_cast<uint32_t>(half * C::kBufs) * C::kOut;
        int t = 0, stored = 0;
        bool ok = true;
        for (int tile = first; ok && tile < p.tiles; tile += step) {
            int mt, nt;
            tile_at(p, tile, mt, nt);
            const int64_t r0 = (static_cast<int64_t>(mt) * CG + rank) * C::kM, r = r0 + m;
            const int64_t n0 = static_cast<int64_t>(nt) * BN + c0;
            const int64_t left_cols = p.N - n0;
            const int count = left_cols < 0 ? 0 : (left_cols < C::kCols ? static_cast<int>(left_cols) : C::kCols);
            // the row's: on their way while the products are, and looked at after them
            const int64_t token = r < p.M ? p.targets[r] : p.ignore;
            float top = 0.f, log_s = 0.f, weight = 0.f;
            if (PROBS && r < p.M) {
                top = p.stats[2 * r];
                log_s = p.stats[2 * r + 1];
                weight = p.dloss[r];
            }
            float z[C::kCols];
            for (int left = per_tile, chunk = 0; left > 0 && ok; left -= p.chunk, ++chunk) {
                ok = tc::mbar_wait(&S->acc_full[t & 1], (t >> 1) & 1, abort, p.status);
                // the output warps that wait for one another below leave together
                ok = PROBS ? tc::named_and(1, 256, ok) : __all_sync(0xffffffffu, ok) != 0;
                if (!ok) break;
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t col = tmem + lanes + static_cast<uint32_t>((t & 1) * BN + c0);
#pragma unroll
                for (int q = 0; q < C::kCols; q += 16) {
                    uint32_t v[16];
                    tmem_ld16_begin(col + q, v);
                    tmem_ld16_end(v);
                    if (chunk == 0) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[q + j] = __uint_as_float(v[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[q + j] += __uint_as_float(v[j]);
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if (CG == 2 && rank != 0)
                        ws::mbar_arrive_remote(acc_empty0 + static_cast<uint32_t>((t & 1) * sizeof(uint64_t)));
                    else
                        tc::mbar_arrive(&S->acc_empty[t & 1]);
                }
                ++t;
            }
            if (!ok) break;
            // the target among these columns, or -1
            const bool kept = is_kept(token, p.ignore, p.V);
            const int64_t at = kept ? token - p.col0 - n0 : -1;
            const int target = at >= 0 && at < count ? static_cast<int>(at) : -1;
            if constexpr (!PROBS) {
                if (count < C::kCols) {
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j) z[j] = j < count ? z[j] : neg_inf();
                }
                if (target >= 0) {
                    float x = 0.f;
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j) x = j == target ? z[j] : x;
                    p.at_target[r] = x;
                }
                float most[2] = {neg_inf(), neg_inf()}, sum[4] = {};
#pragma unroll
                for (int j = 0; j < C::kCols; j += 4) {
                    asm("max.f32 %0, %0, %1, %2;" : "+f"(most[0]) : "f"(z[j]), "f"(z[j + 1]));
                    asm("max.f32 %0, %0, %1, %2;" : "+f"(most[1]) : "f"(z[j + 2]), "f"(z[j + 3]));
                }
                const float high = fmaxf(most[0], most[1]);
                const float off = to_exponents(z, high == neg_inf() ? 0.f : high);  // -inf - -inf would be NaN
#pragma unroll
                for (int j = 0; j < C::kCols; ++j) sum[j & 3] += ex2(z[j]);
                float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                if (high > neg_inf()) {
                    // the largest's own is 1, which its two approximate exponentials miss by some 2^-22, and no loss is below 0
                    total = 1.f + (total - ex2(off)) * ex2(-off);
                    if (total < 1.f) total = 1.f;  // NaN stays
                }
                if (r < p.M) p.parts[(2 * static_cast<int64_t>(nt) + half) * p.M + r] = make_float2(high, total);
            } else {
                if (!kept && token != p.ignore && nt == 0 && half == 0) report(p.status, CCI_ERR_INDEX);
                const bool none = !kept || weight == 0.f;  // left out: 0 whatever the logits
                const float off = to_exponents(z, top == neg_inf() ? 0.f : top), minus = -fmaf(log_s, kLog2e, off);
                float less = 0.f;  // p - 1 of the target
                if (target >= 0) {
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j) less = j == target ? z[j] : less;
                    less = expm1f((less + minus) * kLn2);
                }
#pragma unroll
                for (int j = 0; j < C::kCols; ++j) z[j] = ex2(z[j] + minus);
                if (target >= 0) {
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j) z[j] = j == target ? less : z[j];
                }
#pragma unroll
                for (int j = 0; j < C::kCols; ++j) z[j] = none ? 0.f : z[j] * weight;
                if (r0 < p.M) {  // the odd CTA's rows may all lie past the last token
                    const int planes = p.terms > 1 ? 3 : 1;
#pragma unroll
                    for (int c = 0; c < C::kCols; c += 64) {
                        if (c < count) {
                            for (int plane = 0; plane < planes; ++plane) {
                                const uint32_t buf = bufs + static_cast<uint32_t>(stored % C::kBufs) * C::kOut;
                                ++stored;
                                if (m == 0) tc::bulk_wait_read<C::kBufs - 1>();
                                tc::named_sync(2 + half, 128);
#pragma unroll
                                for (int q = 0; q < 8; ++q) {
                                    uint32_t w[4];
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        float &a = z[c + 8 * q + 2 * j], &b = z[c + 8 * q + 2 * j + 1];
                                        w[j] = planes == 1 ? row::bf16x2(a, b) : next_planes(a, b);
                                    }
                                    ws::st_shared_v4(buf + ws::sw_chunk(m, q), w[0], w[1], w[2], w[3]);
                                }
                                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                                tc::named_sync(2 + half, 128);
                                if (m == 0) {
                                    tc::tma_store_2d(&maps.out[plane], buf, static_cast<int>(n0) + c, static_cast<int>(r0));
                                    tc::bulk_commit();
                                }
                            }
                        }
                    }
                }
            }
        }
        if (m == 0) {
            if constexpr (PROBS) tc::bulk_wait_all();
            if (!ok) {  // accumulators that may be committed all the same: this one and the next
                int no_abort = 0;
                for (int a = t; a < t + 2; ++a) tc::mbar_wait(&S->acc_full[a & 1], (a >> 1) & 1, &no_abort, p.status);
            }
        }
    }

    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) {
        // the last commit signals this CTA's barrier too: it has arrived before either CTA leaves
        if (rank != 0 && tid == 0) {
            int no_abort = 0;
            tc::mbar_wait(&S->drain, 0, &no_abort, p.status);
        }
        __syncwarp();
        ws::cluster_sync();
    }
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmem) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmem) : "memory");
    }
}

// ---- a token's parts, in their order, and its loss.  A block takes 32 tokens, 32 threads each ----
__device__ __forceinline__ float2 joined(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), from = m == neg_inf() ? 0.f : m;
    // a sum of nothing is 0 whatever its maximum, and NaN stays
    const float u = a.y == 0.f ? 0.f : a.y * exp_of(a.x - from), v = b.y == 0.f ? 0.f : b.y * exp_of(b.x - from);
    return make_float2(m, u + v);
}

__global__ void __launch_bounds__(1024) loss_kernel(const float2 *parts, int count, const float *at_target, const int64_t *targets,
                                                    int64_t ignore, int64_t N, int64_t V, float *loss, float *stats,
                                                    uint32_t *status)
{
    __shared__ float2 sums[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + x;
    float2 a = make_float2(neg_inf(), 0.f);
    tc::wait_prior_grid();
    if (n < N) {
#pragma unroll 4
        for (int i = y; i < count; i += 32) a = joined(a, parts[static_cast<int64_t>(i) * N + n]);
    }
    sums[y][x] = a;
    __syncthreads();
    // a warp joins a token's 32
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 32 + y;
    a = sums[x][y];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float2 b = make_float2(__shfl_down_sync(0xffffffffu, a.x, o), __shfl_down_sync(0xffffffffu, a.y, o));
        a = joined(a, b);
    }
    if (x == 0 && row < N) {
        const float log_s = logf(a.y);
        const int64_t token = targets[row];
        float l = 0.f;
        if (token != ignore) {
            if (token >= 0 && token < V) {
                l = log_s - (at_target[row] - a.x);
            } else {
                report(status, CCI_ERR_INDEX);
                l = __int_as_float(0x7fc00000);
            }
        }
        loss[row] = l;
        stats[2 * row] = a.x;
        stats[2 * row + 1] = log_s;
    }
}

// three bf16 planes of n fp32 elements (a multiple of 8), one after the other, cut as P's are: memory bound, where
// planes to the nearest are bound by their conversions (16128 x 1024: 33 us, 21 so)
__global__ void __launch_bounds__(256) cut_kernel(const float *in, uint16_t *out, int64_t n)
{
    const int64_t step = static_cast<int64_t>(gridDim.x) * 2048;
    int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
    row::Raw<float, 8> next{};
    if (i < n) next = row::load_once<float, 8>(in + i);
    for (; i < n; i += step) {
        float v[8];
        row::unpack<float, 8>(next, v);
        if (i + step < n) next = row::load_once<float, 8>(in + i + step);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = next_planes(v[2 * j], v[2 * j + 1]);
            *reinterpret_cast<uint4 *>(out + q * n + i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// X for the gradients' products: left-out tokens' rows are zeros whatever they hold, which would come into every row of dW as 0 times
// it.  fp32: its planes, cut as above.  A warp a row (4096 x 2048 bf16: 6 us of the pass' 3900)
template <typename T>
__global__ void __launch_bounds__(256) kept_rows_kernel(const T *in, uint16_t *out, int64_t N, int D, const int64_t *targets, int64_t ignore,
                                                        int64_t V, const float *dloss)
{
    const int lane = threadIdx.x & 31;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (n >= N) return;
    const bool keep = is_kept(targets[n], ignore, V) && dloss[n] != 0.f;
    for (int c = lane * 8; c < D; c += 256) {
        row::Raw<T, 8> raw{};
        if (keep) raw = row::load_once<T, 8>(in + n * D + c);
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(out + n * D + c) = raw.w[0];
        } else {
            float v[8];
            row::unpack<float, 8>(raw, v);
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = next_planes(v[2 * j], v[2 * j + 1]);
                *reinterpret_cast<uint4 *>(out + q * N * D + n * D + c) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

// dX from its fp32 sums
__global__ void __launch_bounds__(256) round_kernel(const float *in, uint16_t *out, int64_t n)
{
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    float v[8];
    row::unpack<float, 8>(row::load_once<float, 8>(in + i), v);
    row::store<uint16_t, 8>(out + i, v);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

constexpr size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// how a piece's product is tiled: the shape whose rounds over the SMs take the fewest cycles, counted as for the gated
// block's products
struct Shape {
    int cg, bn;
};

Shape shape_of(int64_t M, int64_t N, int64_t D, int terms)
{
    const int64_t sms = ws::sm_count(), stages = (D + 63) / 64 * terms;
    const int64_t a_rows = M > 128 ? 128 : (M + 7) / 8 * 8;
    Shape best{1, 128};
    double least = 0.0;
    const int shapes[3][3] = {{2, 256, 512}, {1, 256, 512}, {1, 128, 256}};
    for (const auto &s : shapes) {
        const int cg = s[0], bn = s[1];
        if (cg > sms) continue;
        const int64_t tiles = (M + 128 * cg - 1) / (128 * cg) * ((N + bn - 1) / bn), units = sms / cg;
        const double copies = static_cast<double>((a_rows + bn / cg) * 128) / 64.0;
        const double cost = static_cast<double>((tiles + units - 1) / units) *
                            (static_cast<double>(stages) * (copies > s[2] ? copies : s[2]) + 4000.0);
        if (least == 0.0 || cost < least) {
            least = cost;
            best = Shape{cg, bn};
        }
    }
    return best;
}

// columns of a piece, at most: what a piece takes in the workspace, `bytes` a column, stays below `budget`, but for
// pieces of 2048 columns, or of a tile of 128 x 128 for each SM, which fewer columns would leave idle.  Pieces are of like
// size
int64_t piece_of(int64_t V, int64_t bytes, int64_t budget, int64_t N)
{
    int64_t most = budget / (bytes < 1 ? 1 : bytes) / 256 * 256, least = 128 * ws::sm_count() / ((N + 127) / 128);
    if (least < 2048) least = 2048;
    if (most < least) most = (least + 255) / 256 * 256;
    const int64_t pieces = (V + most - 1) / most;
    const int64_t each = (V + pieces - 1) / pieces;
    return (each + 255) / 256 * 256;
}

// Forward, fp32: a piece's planes are written and read again at once, so they may as well stay in L2
constexpr int64_t kForwardBudget = int64_t(96) << 20;
// Backward: P's piece (and W's planes)
constexpr int64_t kBackwardBudget = int64_t(256) << 20;

// places in the workspace, in bytes from its start
struct Layout {
    int64_t piece;    // columns of a piece (the last one may be narrower)
    int64_t ldp;      // row stride of P
    size_t x, w;      // planes (fp32); backward: kept_rows_kernel's X
    size_t parts, at_target;  // forward
    size_t p, dx, products;   // backward
    size_t total;
};

// few fp32 tokens read the weights as they are (cci_head_few.cuh)
bool few_tokens(int dtype, int64_t N) { return dtype == CCI_F32 && N <= kFewTokens; }

Layout layout(int dtype, int64_t N, int64_t D, int64_t V, int call)
{
    const bool f32 = dtype == CCI_F32;
    const int terms = f32 ? 6 : 1, planes = f32 ? 3 : 1;
    Layout l{};
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += round256(static_cast<size_t>(bytes));
        return here;
    };
    if (call == CCI_HEAD_FORWARD)
        l.piece = f32 ? piece_of(V, 6 * D, kForwardBudget, N) : V;
    else
        l.piece = piece_of(V, f32 ? 6 * (N + D) : 2 * N, kBackwardBudget, N);
    if (l.piece > V) l.piece = V;
    if (f32 || call == CCI_HEAD_BACKWARD) l.x = take(2 * planes * N * D);
    if (f32 && !few_tokens(dtype, N)) l.w = take(6 * l.piece * D);
    if (few_tokens(dtype, N) && call == CCI_HEAD_BACKWARD) {
        l.p = take(4 * V * few_pitch(N));
        l.products = take(4 * few_slices(N, D, V, ws::sm_count()) * N * D);
    } else if (few_tokens(dtype, N)) {
        l.parts = take(few_blocks(V, ws::sm_count()) * N * static_cast<int64_t>(sizeof(float2)));
        l.at_target = take(N * 4);
    } else if (call == CCI_HEAD_FORWARD) {
        int64_t parts = 0;
        for (int64_t c = 0; c < V; c += l.piece) {
            const int64_t n = V - c < l.piece ? V - c : l.piece;
            const int bn = shape_of(N, n, D, terms).bn;
            parts += 2 * ((n + bn - 1) / bn);
        }
        l.parts = take(parts * N * static_cast<int64_t>(sizeof(float2)));
        l.at_target = take(N * 4);
    } else {
        l.ldp = (l.piece + 63) / 64 * 64;
        l.p = take(2 * planes * N * l.ldp);
        if (!f32 && l.piece < V) l.dx = take(4 * N * D);
        size_t most = 0;
        const int64_t last = V - (V - 1) / l.piece * l.piece;
        for (const int64_t n : {l.piece, last}) {
            const size_t dx = gated::plan(gated::kDxAdd, N, D, n, terms).part_bytes;
            const size_t dw = gated::plan(gated::kDwOne, n, D, N, terms).part_bytes;
            most = dx > most ? dx : most;
            most = dw > most ? dw : most;
        }
        l.products = take(static_cast<int64_t>(most));
    }
    l.total = at;
    return l;
}

template <int CG, int BN, bool PROBS>
cudaError_t launch_tiled(Params p, const Operand &a, const Operand &b, uint16_t *out, int64_t ldp, cudaStream_t stream)
{
    using C = Cfg<CG, BN, PROBS>;
    const int64_t mt = (p.M + CG * 128 - 1) / (CG * 128), nt = (p.N + BN - 1) / BN;
    if (mt * nt > (int64_t(1) << 30)) return cudaErrorInvalidValue;
    p.m_tiles = static_cast<int>(mt);
    p.n_tiles = static_cast<int>(nt);
    p.tiles = static_cast<int>(mt * nt);
    p.a_rows = p.M < C::kM ? static_cast<int>((p.M + 7) / 8 * 8) : C::kM;
    Maps maps{};
    if (!operand_map(&maps.a, a, p.a_rows) || !operand_map(&maps.b, b, C::kBRows)) return cudaErrorInvalidValue;
    if constexpr (PROBS) {
        const int64_t dims[2] = {p.N, p.M}, strides[1] = {ldp * 2};
        const int box[2] = {64, 128};
        for (int i = 0; i < a.planes; ++i)
            if (!ws::make_map_strided(&maps.out[i], out + i * p.M * ldp, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dims,
                                      strides, box))
                return cudaErrorInvalidValue;
    }
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(head_kernel<CG, BN, PROBS>, static_cast<int>(C::kSmem), attr_cache);
    if (attr != cudaSuccess) return attr;
    const int units = ws::sm_count() / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((p.tiles < units ? p.tiles : units) * CG));
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = CG;
    la[0].val.clusterDim.y = 1;
    la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = CG == 2 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, head_kernel<CG, BN, PROBS>, p, maps);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

template <bool PROBS>
cudaError_t launch_piece(const Shape &s, const Params &p, const Operand &a, const Operand &b, uint16_t *out, int64_t ldp,
                         cudaStream_t stream)
{
    if (s.cg == 2) return launch_tiled<2, 256, PROBS>(p, a, b, out, ldp, stream);
    return s.bn == 256 ? launch_tiled<1, 256, PROBS>(p, a, b, out, ldp, stream)
                       : launch_tiled<1, 128, PROBS>(p, a, b, out, ldp, stream);
}

// bf16 planes of n fp32 elements
cudaError_t planes(const void *in, void *out, int64_t n, cudaStream_t stream)
{
    const int64_t blocks = (n / 8 + 255) / 256, most = 8 * static_cast<int64_t>(ws::sm_count());
    cut_kernel<<<static_cast<unsigned>(blocks < most ? blocks : most), 256, 0, stream>>>(static_cast<const float *>(in),
                                                                                     static_cast<uint16_t *>(out), n);
    return cudaGetLastError();
}

// rows [c, c + n) of W [V][D]
const void *rows_at(const HeadArgs &a, int64_t c)
{
    return static_cast<const char *>(a.W) + c * a.D * (a.dtype == CCI_F32 ? 4 : 2);
}

FewParams few_params(const HeadArgs &a, const void *x_planes)
{
    FewParams f{};
    f.x = static_cast<const uint16_t *>(x_planes);
    f.w = static_cast<const float *>(a.W);
    f.N = static_cast<int>(a.N);
    f.D = static_cast<int>(a.D);
    f.V = a.V;
    f.targets = a.targets;
    f.ignore = a.ignore;
    f.status = a.status;
    return f;
}

}  // namespace head

size_t head_workspace(int dtype, int64_t N, int64_t D, int64_t V, int call)
{
    return head::layout(dtype, N, D, V, call).total;
}

cudaError_t launch_head(const HeadArgs &a, cudaStream_t stream)
{
    using namespace head;
    const bool f32 = a.dtype == CCI_F32;
    const Layout l = layout(a.dtype, a.N, a.D, a.V, CCI_HEAD_FORWARD);
    char *base = static_cast<char *>(a.workspace);
    cudaError_t e = cudaSuccess;
    Params p{};
    p.M = a.N;
    p.V = a.V;
    p.k_stages = static_cast<int>((a.D + 63) / 64);
    p.terms = f32 ? 6 : 1;
    p.chunk = chunk_of(p.k_stages * p.terms);
    p.targets = a.targets;
    p.ignore = a.ignore;
    p.at_target = reinterpret_cast<float *>(base + l.at_target);
    p.status = a.status;
    float2 *parts = reinterpret_cast<float2 *>(base + l.parts);
    int64_t count = 0;
    if (f32) e = planes(a.X, base + l.x, a.N * a.D, stream);
    const Operand x{f32 ? base + l.x : a.X, a.N, a.D, f32 ? 3 : 1};
    const bool few = few_tokens(a.dtype, a.N);
    if (few && e == cudaSuccess) {
        FewParams f = few_params(a, x.data);
        f.parts = parts;
        f.at_target = p.at_target;
        e = launch_few<false>(f, ws::sm_count(), stream);
        count = few_blocks(a.V, ws::sm_count());
    }
    for (int64_t c = 0; !few && c < a.V && e == cudaSuccess; c += l.piece) {
        const int64_t n = a.V - c < l.piece ? a.V - c : l.piece;
        const void *w = rows_at(a, c);
        if (f32) {
            e = planes(w, base + l.w, n * a.D, stream);
            if (e != cudaSuccess) break;
            w = base + l.w;
        }
        const Shape s = shape_of(a.N, n, a.D, p.terms);
        p.N = n;
        p.col0 = c;
        p.parts = parts + count * a.N;
        e = launch_piece<false>(s, p, x, Operand{w, n, a.D, x.planes}, nullptr, 0, stream);
        count += 2 * ((n + s.bn - 1) / s.bn);
    }
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((a.N + 31) / 32));
    cfg.blockDim = dim3(1024);
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, loss_kernel, const_cast<const float2 *>(parts), static_cast<int>(count),
                           const_cast<const float *>(p.at_target), a.targets, a.ignore, a.N, a.V, a.loss, a.stats, a.status);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

cudaError_t launch_head_backward(const HeadArgs &a, cudaStream_t stream)
{
    using namespace head;
    const bool f32 = a.dtype == CCI_F32;
    const size_t es = f32 ? 4 : 2;
    if (a.N == 0)  // no rows to sum over
        return a.dW ? cudaMemsetAsync(a.dW, 0, static_cast<size_t>(a.V) * a.D * es, stream) : cudaSuccess;
    if (!a.dX && !a.dW) return cudaSuccess;
    const Layout l = layout(a.dtype, a.N, a.D, a.V, CCI_HEAD_BACKWARD);
    char *base = static_cast<char *>(a.workspace);
    cudaError_t e = cudaSuccess;
    Params p{};
    p.M = a.N;
    p.V = a.V;
    p.k_stages = static_cast<int>((a.D + 63) / 64);
    p.terms = f32 ? 6 : 1;
    p.chunk = chunk_of(p.k_stages * p.terms);  // as forward: a sure token's P is the difference of its logit from those
    p.targets = a.targets;
    p.ignore = a.ignore;
    p.stats = a.stats;
    p.dloss = a.dloss;
    p.status = a.status;
    uint16_t *probs = reinterpret_cast<uint16_t *>(base + l.p);
    const int np = f32 ? 3 : 1;
    const bool sums = !f32 && l.piece < a.V;  // dX in fp32 until the last piece
    const unsigned blocks = static_cast<unsigned>((a.N + 7) / 8);
    uint16_t *kept = reinterpret_cast<uint16_t *>(base + l.x);
    if (f32)
        kept_rows_kernel<float><<<blocks, 256, 0, stream>>>(static_cast<const float *>(a.X), kept, a.N, static_cast<int>(a.D), a.targets,
                                                            a.ignore, a.V, a.dloss);
    else
        kept_rows_kernel<uint16_t><<<blocks, 256, 0, stream>>>(static_cast<const uint16_t *>(a.X), kept, a.N, static_cast<int>(a.D),
                                                               a.targets, a.ignore, a.V, a.dloss);
    e = cudaGetLastError();
    const Operand x{kept, a.N, a.D, np};
    if (few_tokens(a.dtype, a.N)) {
        if (e != cudaSuccess) return e;
        FewParams f = few_params(a, x.data);
        f.stats = a.stats;
        f.dloss = a.dloss;
        f.probs = reinterpret_cast<float *>(base + l.p);
        e = launch_few<true>(f, ws::sm_count(), stream);
        if (e != cudaSuccess) return e;
        const FewGradients g{static_cast<const float *>(a.X), f.w, f.probs, f.N, f.D, a.V, 0, static_cast<float *>(a.dW),
                             a.dX ? reinterpret_cast<float *>(base + l.products) : nullptr, a.targets, a.ignore, a.dloss};
        return launch_few_gradients(g, ws::sm_count(), static_cast<float *>(a.dX), stream);
    }
    for (int64_t c = 0; c < a.V && e == cudaSuccess; c += l.piece) {
        const int64_t n = a.V - c < l.piece ? a.V - c : l.piece;
        const void *w = rows_at(a, c);
        if (f32) {
            e = planes(w, base + l.w, n * a.D, stream);
            if (e != cudaSuccess) break;
            w = base + l.w;
        }
        const Operand rows{w, n, a.D, np};
        p.N = n;
        p.col0 = c;
        e = launch_piece<true>(shape_of(a.N, n, a.D, p.terms), p, x, rows, probs, l.ldp, stream);
        if (e != cudaSuccess) break;
        gated::Job j{};
        j.terms = p.terms;
        j.status = a.status;
        j.parts = reinterpret_cast<float *>(base + l.products);
        j.a[0] = Operand{probs, a.N, n, np, l.ldp};
        if (a.dW) {
            j.b[0] = x;
            j.out[0] = static_cast<char *>(a.dW) + static_cast<size_t>(c) * a.D * es;
            j.out_f32 = f32;
            j.M = n;
            j.N = a.D;
            j.K = a.N;
            e = gated::launch_dw_one(j, stream);
            if (e != cudaSuccess) break;
        }
        if (a.dX) {
            j.b[0] = rows;
            j.out[0] = sums ? static_cast<void *>(base + l.dx) : a.dX;
            j.out_f32 = f32 || sums;
            j.add = c > 0;
            j.M = a.N;
            j.N = a.D;
            j.K = n;
            e = gated::launch_dx_add(j, stream);
        }
    }
    if (e == cudaSuccess && a.dX && sums) {
        const int64_t n = a.N * a.D;
        round_kernel<<<static_cast<unsigned>((n / 8 + 255) / 256), 256, 0, stream>>>(
            reinterpret_cast<const float *>(base + l.dx), static_cast<uint16_t *>(a.dX), n);
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace cci
