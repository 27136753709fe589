// cci_gated.cuh -- the tensor-core products of the gated feed-forward block.
//
//   forward   g = X Wg^T, u = X Wu^T, h = act(g) * u in one kernel: an output tile holds the gate's
//             and the up projection's accumulators of the same channels side by side in tensor
//             memory, and the epilogue joins them.  X [N][D], W [F][D]: both K-major.
//   dX        dg Wg + du Wu: one reduction over both pairs, 2 F long.  dg, du [N][F] K-major; the
//             weights' rows run along the output, so they are read MN-major (no transposed copy).
//   dW        dg^T X and du^T X in one launch, the reduction over the tokens: both operands MN-major.
//
// Operands are bf16 with fp32 accumulators (tcgen05.mma kind::f16).  fp32 tensors come as three bf16
// planes, v = v1 + v2 + v3 with v1 the nearest bf16 of v and so on (each takes 8 bits of the 24): the
// reduction runs over the six products of planes down to 2^-18 of the whole, the smallest
// first; what is left out is below 2^-25 |a||b|.  Six bf16 products beat fp32 on the CUDA cores
// (80 TFLOP/s against 1887 / 6) and keep its accuracy, which one tf32 product would not.
//
// Tiles: 256 x 256 over a CTA pair (each CTA holds its 128 rows of A and half of B; the even CTA
// issues), or 128 x 128 and 128 x 64 on one CTA where there is little to do.  Both operands are copied
// by TMA into 128-byte-swizzled stages 64 deep; two accumulators in tensor memory, so that one tile's
// epilogue runs beside the next one's products; a persistent grid walks the tiles eight M tiles at
// a time, so that what the SMs read at once stays in L2.
//
// Roles: warp 0 copies, warp 1 issues the MMAs, warp 2 holds the tensor memory, warps 4-7 write the
// output through shared memory by TMA, which clips ragged edges.  Every wait is bounded: on expiry
// the status word gets CCI_ERR_TIMEOUT, the other roles stop, and the block leaves when its copies
// and products have ended.
#pragma once

#include "cci_gemm_ws.cuh"

namespace cci {
namespace gated {

enum Mode { kForward = 0, kDx = 1, kDw = 2 };

// everything a launch needs but its tensor maps
struct Params {
    int64_t M, N;        // output rows and columns (forward: N = F)
    int k_stages;        // 64-deep stages of one reduction
    int pairs;           // reductions added up: 2 for dX (gate, up), else 1
    int terms;           // products of planes: 1 (bf16) or 6 (fp32)
    int a_rows;          // rows of A's box (K-major): 128, or fewer where the matrix has fewer
    int m_tiles;         // of one output (dW has two)
    int n_tiles;
    int tiles;
    int act;             // cci_activation
    int out_f32;
    int save;            // forward: g and u are written too (fp32)
    // tiles below `whole` are computed whole, one CTA (pair) after the other; the reductions of the rest, where a
    // last round of tiles would leave most SMs idle, are laid end to end and cut evenly over all of them, their parts
    // written in fp32 and added by join_kernel
    int whole;
    uint32_t *status;
};

// [0] gate, [1] up where an operand or output is one of two
struct Maps {
    CUtensorMap a[2], b[2], out[2];
    CUtensorMap save[2];  // forward: g and u
    CUtensorMap parts;
};

template <int CG, int BN>
struct Cfg {
    static constexpr int kM = 128;            // rows of a CTA
    static constexpr int kBRows = BN / CG;    // rows of B that a CTA holds
    static constexpr int kABytes = kM * 128, kBBytes = kBRows * 128;
    static constexpr int kStage = kABytes + kBBytes;
    static constexpr int kOut = kM * 128;     // an output buffer: 128 rows of 128 bytes
    static constexpr int kOuts = 2;
    static constexpr int kFit = (static_cast<int>(kMaxSmemPerBlock) - 2048 - kOuts * kOut) / kStage;
    static constexpr int kStages = kFit < 8 ? kFit : 8;
    static constexpr int kTmem = 2 * BN;
    static constexpr int kThreads = 256;
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStage + kOuts * kOut + 1024;
    static_assert(kStage % 1024 == 0 && kStages >= 4 && kSmem <= kMaxSmemPerBlock, "stages");
    static_assert(kTmem == 128 || kTmem == 256 || kTmem == 512, "tensor memory comes in powers of two");
};

struct Smem {
    uint64_t full[8], empty[8];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};
static_assert(sizeof(Smem) <= 1024, "barriers");

// ---- activations, in fp32 ----
// exp and the quotient in their fast forms (exp(z) within 2 + 1.17 |z| units of 2^-23, so a tail of SiLU or sigmoid
// at g = -20 is tens of them off): the exact ones branch, and so does a choice
// of activation per element, and one thread's elements then run one after the other.  A 256 x 256 tile's epilogue
// of SiLU took 60 us with both, 19 with the fast forms alone, and takes 4 with the choice made once (prompt of
// 1999 tokens, 4096 -> 8192: 268, 164 and 143 us on the device)
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// the normal distribution's Phi(g), and e^(-g^2 / 2), which it takes on the way.  Phi(-a) = e^(-a^2 / 2) R(a) for
// a >= 0, with R(a) = e^(a^2 / 2) erfc(a / sqrt(2)) / 2 as t Q(t), t = 1 / (1 + 0.282 a), which keeps R's 1 / a
// far out.  Q, of degree 8, is the least maximum of the relative error over all t in (0, 1] (least squares at 4000
// Chebyshev points, weighted anew by the error until it levels, in 64 bits): 1.4e-7, and with its fp32 arithmetic
// R is within 4 units of 2^-23.  So the tail keeps its bits: gelu(g) below 0 is within (10 + g^2) 2^-23 of itself,
// where g's own rounding moves it by g^2 2^-24.  No branch; erfcf has one
__device__ __forceinline__ float normal_cdf(float g, float &e)
{
    const float t = __fdividef(1.f, fmaf(fabsf(g), 0.282f, 1.f));
    e = __expf(-0.5f * g * g);
    float q = fmaf(t, 0.0250037387f, -0.0920643508f);
    q = fmaf(t, q, 0.0868110359f);
    q = fmaf(t, q, -0.00381121482f);
    q = fmaf(t, q, 0.0712975115f);
    q = fmaf(t, q, 0.0840900093f);
    q = fmaf(t, q, 0.103673153f);
    q = fmaf(t, q, 0.112498358f);
    q = fmaf(t, q, 0.11250174f);
    q *= t * e;  // Phi(-|g|)
    return g > 0.f ? 1.f - q : q;
}

template <int ACT>
__device__ __forceinline__ float act_of(float g)
{
    if constexpr (ACT == CCI_ACT_SILU) return g * sigmoid(g);
    if constexpr (ACT == CCI_ACT_GELU) {
        float e;
        return g * normal_cdf(g, e);
    }
    if constexpr (ACT == CCI_ACT_GELU_TANH) return g * sigmoid(1.5957691f * (g + 0.044715f * g * g * g));
    if constexpr (ACT == CCI_ACT_RELU) return g > 0.f ? g : (g != g ? g : 0.f);
    return sigmoid(g);
}

// act'(g), act(g) to a
template <int ACT>
__device__ __forceinline__ float slope_of(float g, float &a)
{
    if constexpr (ACT == CCI_ACT_GELU) {
        float e;
        const float c = normal_cdf(g, e);
        a = g * c;
        return fmaf(g * 0.39894228f, e, c);
    }
    if constexpr (ACT == CCI_ACT_RELU) {
        a = act_of<ACT>(g);
        return g > 0.f ? 1.f : 0.f;
    }
    if constexpr (ACT == CCI_ACT_GELU_TANH) {
        // 0.5 (1 + tanh(z)) = sigmoid(2 z).  Past 16 the second term is 0, which an infinite g^2 must not meet
        const float g2 = g * g, p = sigmoid(1.5957691f * (g + 0.044715f * g2 * g)), c = fminf(fmaxf(g, -16.f), 16.f);
        a = g * p;
        return p + c * p * (1.f - p) * 1.5957691f * (1.f + 3.f * 0.044715f * c * c);
    }
    const float p = sigmoid(g);
    if constexpr (ACT == CCI_ACT_SILU) {
        a = g * p;
        return p * (1.f + g * (1.f - p));
    }
    a = p;
    return p * (1.f - p);
}

// f(activation's code as a constant): one choice for a whole run of elements
template <typename Fn>
__device__ __forceinline__ void with_act(int act, Fn f)
{
    switch (act) {
        case CCI_ACT_SILU: f(std::integral_constant<int, CCI_ACT_SILU>{}); break;
        case CCI_ACT_GELU: f(std::integral_constant<int, CCI_ACT_GELU>{}); break;
        case CCI_ACT_GELU_TANH: f(std::integral_constant<int, CCI_ACT_GELU_TANH>{}); break;
        case CCI_ACT_RELU: f(std::integral_constant<int, CCI_ACT_RELU>{}); break;
        default: f(std::integral_constant<int, CCI_ACT_SIGMOID>{});
    }
}

// ---- packed weights ----
// K kept weights of each of eight indices and their places in the group, as they are packed
template <int K>
struct Run {
    uint32_t v[4 * K], i[2 * K];
};

// the eight weights of the row with index j (rows: j in every byte): each value whose index is j, else zero
template <int K>
__device__ __forceinline__ uint4 pick(const Run<K> &r, uint32_t rows)
{
    using ws::pk::prmt;
    uint32_t m[2 * K];  // bit 7 of a byte: that slot's index is j (indices are below 128)
#pragma unroll
    for (int q = 0; q < 2 * K; ++q) m[q] = 0x80808080u - (r.i[q] ^ rows);
    uint32_t out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // indices 2 e and 2 e + 1
        if constexpr (K == 1) {
            out[e] = r.v[e] & prmt(m[e >> 1], 0u, e & 1 ? 0xbbaau : 0x9988u);
        } else {
            uint32_t x[2];  // both halves of x[h]: what of index 2 e + h's slots is kept
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x[h] = 0u;
#pragma unroll
                for (int s = 0; s < K / 2; ++s) {  // word s of the index: slots 2 s and 2 s + 1
                    const int word = (2 * e + h) * (K / 2) + s;
                    x[h] |= r.v[word] & prmt(m[word >> 1], 0u, word & 1 ? 0xbbaau : 0x9988u);
                }
            }
            out[e] = prmt(x[0], x[1], 0x5410u) | prmt(x[0], x[1], 0x7632u);
        }
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// ---- tensor core ----
// shared-memory descriptor of a tile with the 128-byte swizzle.  K-major: rows of 128 bytes, 8-row
// atoms of 1024 (stride offset).  MN-major: rows of 64 outputs (128 bytes) for one k, 8 k to an atom
// (stride offset 1024), the next 64 outputs 64 rows further (leading offset 8192)
template <bool MN>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((addr & 0x3ffff) >> 4);
    d |= static_cast<uint64_t>(MN ? 8192 >> 4 : 1) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}

// the four 16-deep products of a 64-deep stage, and the commit that frees the stage (in both CTAs of a
// pair).  kA, kB: descriptor steps of 16 reduction indices (32 bytes K-major, 16 rows MN-major)
template <int CG, uint32_t kIdesc, int kA, int kB>
__device__ __forceinline__ void stage_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t acc, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile(
            "{\n.reg .pred pa, pt;\n.reg .b64 x, y;\n"
            "setp.ne.b32 pa, %3, 0;\nsetp.eq.b32 pt, 0, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %4, pa;\n"
            "add.s64 x, %1, %7;\nadd.s64 y, %2, %8;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], x, y, %4, pt;\n"
            "add.s64 x, x, %7;\nadd.s64 y, y, %8;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], x, y, %4, pt;\n"
            "add.s64 x, x, %7;\nadd.s64 y, y, %8;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], x, y, %4, pt;\n"
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], %6;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(acc), "n"(kIdesc), "r"(bar), "h"(static_cast<uint16_t>(3)), "n"(kA), "n"(kB)
            : "memory");
    else
        asm volatile(
            "{\n.reg .pred pa, pt;\n.reg .b64 x, y;\n"
            "setp.ne.b32 pa, %3, 0;\nsetp.eq.b32 pt, 0, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %4, pa;\n"
            "add.s64 x, %1, %6;\nadd.s64 y, %2, %7;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, pt;\n"
            "add.s64 x, x, %6;\nadd.s64 y, y, %7;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, pt;\n"
            "add.s64 x, x, %6;\nadd.s64 y, y, %7;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, pt;\n"
            "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(acc), "n"(kIdesc), "r"(bar), "n"(kA), "n"(kB)
            : "memory");
}

// 3-D tile load (inner element, row, plane); the inner coordinate is a multiple of 64.  CG = 2:
// completes on the even CTA's barrier (a cluster address)
template <int CG>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, "
            "{%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, "
            "%4}], [%5];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
            : "memory");
}

// 32 columns of this warp's TMEM lanes, without waiting for them
__device__ __forceinline__ void tmem_ld32_begin(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr));
}

// products of planes (of A, of B) by term, the smallest first
__device__ __forceinline__ void term_planes(int term, int terms, int &pa, int &pb)
{
    // 0 2, 1 1, 2 0, 0 1, 1 0, 0 0: two bits a term
    pa = terms == 1 ? 0 : (0x124 >> (2 * term)) & 3;
    pb = terms == 1 ? 0 : (0x046 >> (2 * term)) & 3;
}

// tile -> M tile (with which output, for dW) and N tile: eight M tiles at a time
__device__ __forceinline__ void tile_at(const Params &p, int tile, int mt_all, int &mt, int &nt)
{
    const int per = 8 * p.n_tiles, g = tile / per, r = tile - g * per;
    const int gm = mt_all - 8 * g < 8 ? mt_all - 8 * g : 8;
    nt = r / gm;
    mt = 8 * g + r - nt * gm;
}

// SPLIT (fp32, CG = 1): the tensor core cuts, not rounds, its running sum at every addition, an error
// that grows with the length of the sum (1.9e-5 of the result at 4096 indices and six terms, measured).
// So it adds kChunk stages at a time, and the output warps add the chunks in registers, to the nearest.  bf16 keeps
// one running sum: K / 16 additions, each cutting half a unit of 2^-23 in the mean, are 1.5e-5 of the sum at 4096
// indices and 2.4e-4 at 65536, under the 2e-3 that its output is rounded by
constexpr int kChunk = 8;

// a CTA's (or pair's) work: stages s0 .. s0 + n - 1 of a tile's reduction; part: -1 if that is all of it, else where
// its sums go (parts of CG 128 rows)
struct Work {
    int tile, s0, n, part;
};

// unit `unit` of `units`, its j-th piece of work; false: there is none.  per: stages of a tile
__device__ __forceinline__ bool work_at(const Params &p, int unit, int units, int per, int j, Work &w)
{
    const int count = unit < p.whole ? (p.whole - unit + units - 1) / units : 0;
    if (j < count) {
        w = Work{unit + j * units, 0, per, -1};
        return true;
    }
    const int64_t rest = static_cast<int64_t>(p.tiles - p.whole) * per;
    const int64_t b0 = rest * unit / units, b1 = rest * (unit + 1) / units;
    const int k = j - count, t0 = static_cast<int>(b0 / per);
    const int64_t cut = static_cast<int64_t>(t0 + 1) * per;  // where the next tile begins: a share is shorter than a tile
    const int64_t from = k == 0 ? b0 : cut, to = k == 0 && b1 > cut ? cut : b1;
    if (k > 1 || from >= to) return false;
    const int tile = t0 + k;
    w = Work{p.whole + tile, static_cast<int>(from - static_cast<int64_t>(tile) * per), static_cast<int>(to - from), 2 * unit + k};
    if (w.n == per) w.part = -1;
    return true;
}

template <int MODE, int CG, int BN, bool SPLIT>
__global__ void __launch_bounds__(Cfg<CG, BN>::kThreads, 1)
    product_kernel(const Params p, const __grid_constant__ Maps maps)
{
    using C = Cfg<CG, BN>;
    constexpr bool kAMn = MODE == kDw, kBMn = MODE != kForward;
    constexpr int kStages = C::kStages;
    constexpr int kNOut = MODE == kForward ? BN / 2 : BN;  // output columns of a tile
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kAMn) << 15) |
                                (static_cast<uint32_t>(kBMn) << 16) | (static_cast<uint32_t>(BN >> 3) << 17) |
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
    const int mt_all = MODE == kDw ? 2 * p.m_tiles : p.m_tiles;
    const int per_tile = p.pairs * p.terms * p.k_stages;  // stages of a tile
    const int chunk_len = SPLIT ? kChunk : per_tile;
    Work work;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&S->full[s], 1);
            tc::mbar_init(&S->empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            tc::mbar_init(&S->acc_full[a], 1);
            tc::mbar_init(&S->acc_empty[a], 4 * CG);
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

    if (warp == 0) {
        // ---- copies
        if (tc::elect_one()) {
            const uint32_t a_bytes = kAMn ? static_cast<uint32_t>(C::kABytes) : static_cast<uint32_t>(p.a_rows) * 128u;
            const uint32_t bytes = CG * (a_bytes + static_cast<uint32_t>(C::kBBytes));
            int s = 0, it = 0;
            uint32_t ph = 1u;  // a fresh barrier's preceding phase counts as complete
            bool ok = true;
            for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
                int mt, nt;
                tile_at(p, work.tile, mt_all, mt, nt);
                int which = 0;  // dW: gate or up
                if (MODE == kDw && mt >= p.m_tiles) {
                    which = 1;
                    mt -= p.m_tiles;
                }
                const int m0 = (mt * CG + static_cast<int>(rank)) * C::kM;
                const int n0 = nt * kNOut;
                // the stage within its product of planes, that within its pair
                int ks = work.s0 % p.k_stages, t = work.s0 / p.k_stages % p.terms, pair = work.s0 / (p.k_stages * p.terms);
                int pa, pb;
                term_planes(t, p.terms, pa, pb);
                const CUtensorMap *ma = &maps.a[MODE == kDw ? which : pair];
                for (int i = 0; i < work.n; ++i, ++it) {
                    ok = tc::mbar_wait(&S->empty[s], ph, abort, p.status);
                    if (!ok) break;
                    const uint32_t sa = base + s * C::kStage, sb = sa + C::kABytes;
                    uint32_t bar = tc::smem_u32(&S->full[s]);
                    if (rank == 0) tc::mbar_arrive_expect_tx(&S->full[s], bytes);
                    if constexpr (CG == 2) bar = ws::map_to_rank(bar, 0);
                    const int k0 = ks * 64;
                    if constexpr (kAMn) {
#pragma unroll
                        for (int q = 0; q < C::kM / 64; ++q) load_3d<CG>(sa + q * 8192, ma, m0 + 64 * q, k0, pa, bar);
                    } else {
                        load_3d<CG>(sa, ma, k0, m0, pa, bar);
                    }
                    if constexpr (MODE == kForward) {
                        if constexpr (CG == 2) {
                            // the even CTA holds the gate's rows, the odd one the up projection's
                            load_3d<CG>(sb, &maps.b[rank], k0, n0, pb, bar);
                        } else {
                            load_3d<CG>(sb, &maps.b[0], k0, n0, pb, bar);
                            load_3d<CG>(sb + C::kBBytes / 2, &maps.b[1], k0, n0, pb, bar);
                        }
                    } else {
                        const CUtensorMap *mb = &maps.b[MODE == kDx ? pair & 1 : 0];
                        const int nb = n0 + static_cast<int>(rank) * C::kBRows;
#pragma unroll
                        for (int q = 0; q < C::kBRows / 64; ++q) load_3d<CG>(sb + q * 8192, mb, nb + 64 * q, k0, pb, bar);
                    }
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                    if (++ks == p.k_stages) {
                        ks = 0;
                        if (++t == p.terms) {
                            t = 0;
                            ++pair;
                            if (MODE == kDx) ma = &maps.a[pair & 1];
                        }
                        term_planes(t, p.terms, pa, pb);
                    }
                }
            }
            // no copy is in flight when the block ends, also after an abort: the even CTA's barriers
            // count those of both.  Nor is a commit: each stage's last one arrives at the `empty` of both CTAs, and
            // that a later commit (drain) has arrived does not say that an earlier one has.  After an abort some
            // stages are never committed: the first wait for one expires, and the others give up with it
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
            const uint64_t da0 = tile_desc<kAMn>(base), db0 = tile_desc<kBMn>(base + C::kABytes);
            const uint32_t empty0 = tc::smem_u32(&S->empty[0]);
            for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
                for (int left = work.n; left > 0 && ok; left -= chunk_len, ++t) {
                    const int acc = t & 1, n = left < chunk_len ? left : chunk_len;
                    if (t >= 2) ok = tc::mbar_wait<CG == 2>(&S->acc_empty[acc], ((t >> 1) - 1) & 1, abort, p.status);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + static_cast<uint32_t>(acc * BN);
                    for (int i = 0; i < n; ++i) {
                        ok = tc::mbar_wait(&S->full[s], ph, abort, p.status);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t off = static_cast<uint64_t>(s) * (C::kStage >> 4);
                        stage_mma<CG, kIdesc, kAMn ? 128 : 2, kBMn ? 128 : 2>(d, da0 + off, db0 + off, i > 0 ? 1u : 0u,
                                                                              empty0 + 8u * s);
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
    } else if (warp >= 4) {
        // ---- output: row `m` of the CTA's 128 per thread
        const int m = tid - 128;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t acc_empty0 = CG == 2 ? ws::map_to_rank(tc::smem_u32(&S->acc_empty[0]), 0) : 0u;
        int t = 0, stored = 0;
        bool ok = true;
        // the next buffer, once the store that last read it has; a buffer's store to `map` at (c0, r0)
        auto take = [&]() {
            const uint32_t buf = outs + static_cast<uint32_t>(stored % C::kOuts) * C::kOut;
            ++stored;
            if (m == 0) tc::bulk_wait_read<C::kOuts - 1>();
            tc::named_sync(1, 128);
            return buf;
        };
        auto give = [&](uint32_t buf, const CUtensorMap *map, int c0, int r0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc::named_sync(1, 128);
            if (m == 0) {
                tc::tma_store_2d(map, buf, c0, r0);
                tc::bulk_commit();
            }
        };
        // 128 bytes of every row
        auto put = [&](const uint32_t (&v)[32], const CUtensorMap *map, int c0, int r0) {
            const uint32_t buf = take();
#pragma unroll
            for (int q = 0; q < 8; ++q)
                ws::st_shared_v4(buf + ws::sw_chunk(m, q), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            give(buf, map, c0, r0);
        };
        // 64 bytes of every row (tiles of 32 bf16 columns), rows 64 bytes apart without a swizzle
        auto put_half = [&](const uint32_t (&v)[32], const CUtensorMap *map, int c0, int r0) {
            const uint32_t buf = take();
#pragma unroll
            for (int q = 0; q < 4; ++q)
                ws::st_shared_v4(buf + static_cast<uint32_t>(m) * 64u + 16u * q, v[4 * q], v[4 * q + 1], v[4 * q + 2],
                                 v[4 * q + 3]);
            give(buf, map, c0, r0);
        };
        // accumulator t of this CTA: waited for, and given back once read
        auto acc_wait = [&]() {
            bool done = tc::mbar_wait(&S->acc_full[t & 1], (t >> 1) & 1, abort, p.status);
            done = tc::named_and(1, 128, done);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            return done;
        };
        auto acc_free = [&]() {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (CG == 2 && rank != 0)
                    ws::mbar_arrive_remote(acc_empty0 + static_cast<uint32_t>((t & 1) * sizeof(uint64_t)));
                else
                    tc::mbar_arrive(&S->acc_empty[t & 1]);
            }
            ++t;
        };
        for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
            int mt, nt;
            tile_at(p, work.tile, mt_all, mt, nt);
            int which = 0;
            if (MODE == kDw && mt >= p.m_tiles) {
                which = 1;
                mt -= p.m_tiles;
            }
            const int r0 = (mt * CG + static_cast<int>(rank)) * C::kM, n0 = nt * kNOut;
            const bool rows = r0 < p.M;  // the odd CTA's rows may all lie past the matrix
            const int cols = p.N - n0 < kNOut ? static_cast<int>(p.N - n0) : kNOut;
            uint32_t o[32];
            // 32 finished columns from c on (forward: v the gate's, u the up projection's)
            auto output = [&](int c, uint32_t (&v)[32], const uint32_t (&u)[32]) {
                if ((MODE != kForward || SPLIT) && work.part >= 0) {
                    const int row = (work.part * CG + static_cast<int>(rank)) * C::kM;
                    put(v, &maps.parts, c, row);
                    if constexpr (MODE == kForward) put(u, &maps.parts, kNOut + c, row);
                    return;
                }
                if constexpr (MODE == kForward) {
                    if (p.save) {
                        put(v, &maps.save[0], n0 + c, r0);
                        put(u, &maps.save[1], n0 + c, r0);
                    }
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            v[j] = __float_as_uint(act_of<decltype(act)::value>(__uint_as_float(v[j])) * __uint_as_float(u[j]));
                    });
                }
                if (p.out_f32) {
                    put(v, &maps.out[which], n0 + c, r0);
                } else if constexpr (kNOut == 32) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = ws::bf16x2_rn(v[2 * j], v[2 * j + 1]);
                    put_half(o, &maps.out[which], n0 + c, r0);
                } else if (c & 32) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[16 + j] = ws::bf16x2_rn(v[2 * j], v[2 * j + 1]);
                    put(o, &maps.out[which], n0 + c - 32, r0);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = ws::bf16x2_rn(v[2 * j], v[2 * j + 1]);
                    if (c + 32 >= cols) {
#pragma unroll
                        for (int j = 16; j < 32; ++j) o[j] = 0u;
                        put(o, &maps.out[which], n0 + c, r0);
                    }
                }
            };
            if constexpr (SPLIT) {
                uint32_t sum[BN / 32][32];
#pragma unroll
                for (int q = 0; q < BN / 32; ++q)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[q][j] = 0u;
                for (int left = work.n; left > 0 && ok; left -= chunk_len) {
                    ok = acc_wait();
                    if (!ok) break;
#pragma unroll
                    for (int q = 0; q < BN / 32; ++q) {
                        uint32_t v[32];
                        tmem_ld32_begin(tmem + lanes + static_cast<uint32_t>((t & 1) * BN + 32 * q), v);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            sum[q][j] = __float_as_uint(__uint_as_float(sum[q][j]) + __uint_as_float(v[j]));
                    }
                    acc_free();
                }
                if (!ok) break;
#pragma unroll
                for (int q = 0; q < kNOut / 32; ++q)
                    if (32 * q < cols && rows) output(32 * q, sum[q], sum[(MODE == kForward ? kNOut / 32 : 0) + q]);
            } else {
                ok = acc_wait();
                if (!ok) break;
                const uint32_t col0 = tmem + lanes + static_cast<uint32_t>((t & 1) * BN);
                for (int c = 0; c < cols && rows; c += 32) {
                    uint32_t v[32], u[32];
                    tmem_ld32_begin(col0 + c, v);
                    if constexpr (MODE == kForward) tmem_ld32_begin(col0 + kNOut + c, u);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                    output(c, v, u);
                }
                acc_free();
            }
        }
        if (m == 0) {
            tc::bulk_wait_all();
            if (!ok) {  // accumulators that may be committed all the same: this one and the next
                int no_abort = 0;
                for (int a = t; a < t + 2; ++a) tc::mbar_wait(&S->acc_full[a & 1], (a >> 1) & 1, &no_abort, p.status);
            }
        }
    }

    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) {
        // the last commit signals this CTA's barrier too: it has arrived before either CTA leaves, as those before it
        // have, for which the copying and the output warps have waited
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

// the tiles whose reductions were cut: the sum of a tile's parts, in their order.  A block takes 8 rows of a tile
// (blockIdx.x: tile, then rows), a thread 8 columns of one (forward: of the gate and of the up projection, as many
// threads; out0 is H, out1 g and out2 u, or null)
template <int MODE, int CG, int BN>
__global__ void __launch_bounds__(MODE == kForward ? BN / 2 : BN)
    join_kernel(const Params p, const float *parts, void *out0, void *out1, float *out2, int units)
{
    constexpr int kBlocks = CG * 128 / 8, kNOut = MODE == kForward ? BN / 2 : BN, kSums = MODE == kForward ? 2 : 1;
    const int per = p.pairs * p.terms * p.k_stages;
    const int rest = static_cast<int>(blockIdx.x) / kBlocks, tile = p.whole + rest;
    const int row = static_cast<int>(blockIdx.x) % kBlocks * 8 + static_cast<int>(threadIdx.x) / (kNOut / 8);
    const int col = static_cast<int>(threadIdx.x) % (kNOut / 8) * 8;
    int mt, nt;
    tile_at(p, tile, MODE == kDw ? 2 * p.m_tiles : p.m_tiles, mt, nt);
    void *out = out0;
    if (MODE == kDw && mt >= p.m_tiles) {
        out = out1;
        mt -= p.m_tiles;
    }
    const int64_t r = static_cast<int64_t>(mt) * CG * 128 + row, c = static_cast<int64_t>(nt) * kNOut + col;
    tc::wait_prior_grid();
    if (r >= p.M || c >= p.N) return;  // N is a multiple of 8
    // the units whose shares meet the tile: `unit`, which holds its first stage, to `last`, which holds its last one
    const int64_t all = static_cast<int64_t>(p.tiles - p.whole) * per, t0 = static_cast<int64_t>(rest) * per;
    auto holder = [&](int64_t stage) {
        int q = static_cast<int>(stage * units / all);
        while (all * (q + 1) / units <= stage) ++q;
        return q;
    };
    const int unit = holder(t0), last = holder(t0 + per - 1);
    if (unit == last) return;  // computed whole
    // a unit's part is its first piece, but for one whose share began in the tile before
    const int64_t stride = static_cast<int64_t>(CG * 128) * BN;
    const float *at = parts + static_cast<int64_t>(row) * BN + col;
    const float *first = at + (2 * unit + (all * unit / units < t0 ? 1 : 0)) * stride;
    float v[kSums][8];
#pragma unroll
    for (int w = 0; w < kSums; ++w) {
        *reinterpret_cast<float4 *>(v[w]) = *reinterpret_cast<const float4 *>(first + w * kNOut);
        *reinterpret_cast<float4 *>(v[w] + 4) = *reinterpret_cast<const float4 *>(first + w * kNOut + 4);
    }
    // the loads of four parts are on their way at a time (3 tokens, 192 -> 8072 fp32, dX of 152 parts: 53 us one by
    // one, 33 to 35 so)
#pragma unroll 4
    for (int q = unit + 1; q <= last; ++q)
#pragma unroll
        for (int w = 0; w < kSums; ++w) {
            const float4 *one = reinterpret_cast<const float4 *>(at + 2 * q * stride + w * kNOut);
            const float4 a = one[0], b = one[1];
            v[w][0] += a.x;
            v[w][1] += a.y;
            v[w][2] += a.z;
            v[w][3] += a.w;
            v[w][4] += b.x;
            v[w][5] += b.y;
            v[w][6] += b.z;
            v[w][7] += b.w;
        }
    const int64_t o = r * p.N + c;
    auto store = [&](float *to, const float *from) {
        reinterpret_cast<float4 *>(to)[0] = make_float4(from[0], from[1], from[2], from[3]);
        reinterpret_cast<float4 *>(to)[1] = make_float4(from[4], from[5], from[6], from[7]);
    };
    if constexpr (MODE == kForward) {
        if (p.save) {
            store(static_cast<float *>(out1) + o, v[0]);
            store(out2 + o, v[1]);
        }
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[0][j] = act_of<decltype(act)::value>(v[0][j]) * v[1][j];
        });
    }
    if (p.out_f32) {
        store(static_cast<float *>(out) + o, v[0]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = ws::bf16x2_rn(__float_as_uint(v[0][2 * j]), __float_as_uint(v[0][2 * j + 1]));
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(out) + o) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// one operand: a row-major matrix [rows][cols] of bf16 in `planes` planes, one after the other
struct Operand {
    const void *data;
    int64_t rows, cols;
    int planes;
};

// copies of 64 (swizzled 128-byte rows) x box_rows
inline bool operand_map(CUtensorMap *m, const Operand &o, int box_rows)
{
    const int64_t dims[3] = {o.cols, o.rows, o.planes};
    const int64_t strides[2] = {o.cols * 2, o.cols * o.rows * 2};
    const int box[3] = {64, box_rows, 1};
    return ws::make_map_strided(m, o.data, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, dims, strides, box);
}

// stores of `width` columns x 128 rows into [rows][cols]: 128 swizzled bytes a row, or 64 plain ones
inline bool output_map(CUtensorMap *m, void *data, bool f32, int64_t rows, int64_t cols, int width)
{
    const int es = f32 ? 4 : 2;
    const int64_t dims[2] = {cols, rows}, strides[1] = {cols * es};
    const int box[2] = {width, 128};
    return ws::make_map_strided(m, data, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                                dims, strides, box, width * es == 128);
}

// a launch: `a`, `b` and `out` with two entries where there are two
struct Job {
    Operand a[2], b[2];
    void *out[2];
    float *save[2];   // forward: g and u, or null
    int64_t M, N, K;  // rows and columns of an output, length of a reduction
    int terms, act, out_f32;
    float *parts;     // plan().part_bytes of workspace
    uint32_t *status;
};

// how a product is tiled: CTAs of a tile, its columns, whether its last tiles' reductions are cut, and the bytes
// of their parts
struct Plan {
    int cg, bn;
    bool cut;
    int units;  // CTAs (pairs) that share the cut reductions
    size_t part_bytes;
};

// The tile whose rounds over the SMs take the fewest cycles.  A 64-deep stage takes its products' time, 512 cycles
// in a 256 x 256 pair tile, 256 in a 128 x 128 one and 192 in a 128 x 64 one, or that of its copies at about 64
// bytes a cycle and SM (what L2 gives all SMs at once); a round about 4000 more for the first copies and the last
// output.  Cutting the last tiles' reductions fills the last round, but writes and reads parts and takes a launch:
// about 20000 cycles (dX of 4096 tokens, 4096 -> 8192: 256 tiles over 76 pairs, 394 us whole, 291 cut).  Where
// even eight stages each are too few for all SMs, fewer share them.  The forward pass is cut in fp32 alone, where it has
// a workspace (427 tokens, 4088 -> 648: 122 us whole, 69 cut); its parts hold g and u, which the join then joins
inline Plan plan(Mode mode, int64_t M, int64_t N, int64_t K, int terms)
{
    const int64_t sms = ws::sm_count(), outs = mode == kDw ? 2 : 1;
    const int64_t stages = (K + 63) / 64 * terms * (mode == kDx ? 2 : 1);
    const int64_t a_rows = mode == kDw || M > 128 ? 128 : (M + 7) / 8 * 8;
    Plan best{};
    double least = 0.0;
    const int shapes[3][3] = {{2, 256, 512}, {1, 128, 256}, {1, 64, 192}};
    for (const auto &shape : shapes) {
        const int cg = shape[0], bn = shape[1];
        if (terms > 1 && cg == 2) continue;  // fp32: the output warps hold a tile's sums
        if (cg > sms) continue;              // no device: sizes and refusals are still answered
        const int64_t n = mode == kForward ? bn / 2 : bn, units = sms / cg;
        const int64_t tiles = (M + 128 * cg - 1) / (128 * cg) * outs * ((N + n - 1) / n);
        const double copies = static_cast<double>((a_rows + bn / cg) * 128) / 64.0;
        const double stage = copies > shape[2] ? copies : shape[2], tile = static_cast<double>(stages) * stage;
        const int64_t rounds = (tiles + units - 1) / units, rest = tiles % units;
        const double whole = static_cast<double>(rounds) * (tile + 4000.0);
        // every share has eight stages or more, and is shorter than a tile
        const int64_t shares = tiles < units && tiles * stages / 8 < units ? tiles * stages / 8 : units;
        const bool can = (mode != kForward || terms > 1) && rest > 0 && shares > rest && rest * stages >= 8 * shares;
        double cut = static_cast<double>(tiles) / static_cast<double>(can ? shares : units) * tile +
                     static_cast<double>(rounds) * 4000.0 + 20000.0;
        if (!can) cut = whole;
        const double cost = cut < whole ? cut : whole;
        if (best.cg == 0 || cost < least) {
            least = cost;
            best = Plan{cg, bn, cut < whole, static_cast<int>(shares), 0};
            if (best.cut) best.part_bytes = static_cast<size_t>(shares) * 2 * cg * 128 * bn * sizeof(float);
        }
    }
    return best;
}

template <int MODE, int CG, int BN, bool SPLIT>
cudaError_t launch_tiled(const Job &j, const Plan &plan, cudaStream_t stream)
{
    using C = Cfg<CG, BN>;
    constexpr int kNOut = MODE == kForward ? BN / 2 : BN;
    constexpr int two_a = MODE == kForward ? 1 : 2, two_b = MODE == kDw ? 1 : 2, two_out = MODE == kDw ? 2 : 1;
    Params p{};
    Maps maps{};
    p.M = j.M;
    p.N = j.N;
    p.k_stages = static_cast<int>((j.K + 63) / 64);
    p.pairs = MODE == kDx ? 2 : 1;
    p.terms = j.terms;
    p.a_rows = j.M < C::kM ? static_cast<int>((j.M + 7) / 8 * 8) : C::kM;
    p.act = j.act;
    p.out_f32 = j.out_f32;
    p.save = j.save[0] != nullptr;
    p.status = j.status;
    const int64_t mt = (j.M + CG * C::kM - 1) / (CG * C::kM), nt = (j.N + kNOut - 1) / kNOut;
    if (mt * two_out * nt > (int64_t(1) << 30)) return cudaErrorInvalidValue;
    p.m_tiles = static_cast<int>(mt);
    p.n_tiles = static_cast<int>(nt);
    p.tiles = static_cast<int>(mt * two_out * nt);
    const bool cut = plan.cut;
    const int units = cut ? plan.units : ws::sm_count() / CG;
    p.whole = cut ? p.tiles - p.tiles % units : p.tiles;
    for (int i = 0; i < two_a; ++i)
        if (!operand_map(&maps.a[i], j.a[i], MODE == kDw ? 64 : p.a_rows)) return cudaErrorInvalidValue;
    for (int i = 0; i < two_b; ++i)
        if (!operand_map(&maps.b[i], j.b[i], MODE == kForward ? (CG == 2 ? C::kBRows : C::kBRows / 2) : 64))
            return cudaErrorInvalidValue;
    const int width = j.out_f32 ? 32 : (kNOut < 64 ? kNOut : 64);
    for (int i = 0; i < two_out; ++i)
        if (!output_map(&maps.out[i], j.out[i], j.out_f32, j.M, j.N, width)) return cudaErrorInvalidValue;
    if (p.save)
        for (int i = 0; i < 2; ++i)
            if (!output_map(&maps.save[i], j.save[i], true, j.M, j.N, 32)) return cudaErrorInvalidValue;
    if (cut && !output_map(&maps.parts, j.parts, true, static_cast<int64_t>(units) * 2 * CG * 128, BN, 32))
        return cudaErrorInvalidValue;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(product_kernel<MODE, CG, BN, SPLIT>, static_cast<int>(C::kSmem), attr_cache);
    if (attr != cudaSuccess) return attr;
    const unsigned blocks = static_cast<unsigned>((cut || p.tiles > units ? units : p.tiles) * CG);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
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
    cudaError_t e = cudaLaunchKernelEx(&cfg, product_kernel<MODE, CG, BN, SPLIT>, p, maps);
    if (e == cudaSuccess) e = cudaGetLastError();
    if constexpr (MODE != kForward || SPLIT) {
        if (e != cudaSuccess || !cut) return e;
        cudaLaunchConfig_t jc = {};
        jc.gridDim = dim3(static_cast<unsigned>((p.tiles - p.whole) * (CG * 128 / 8)));
        jc.blockDim = dim3(kNOut);
        jc.stream = stream;
        la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        la[0].val.programmaticStreamSerializationAllowed = 1;
        jc.attrs = la;
        jc.numAttrs = 1;
        void *second = MODE == kForward ? static_cast<void *>(j.save[0]) : j.out[MODE == kDw ? 1 : 0];
        e = cudaLaunchKernelEx(&jc, join_kernel<MODE, CG, BN>, p, const_cast<const float *>(j.parts), j.out[0], second,
                               j.save[1], units);
        if (e == cudaSuccess) e = cudaGetLastError();
    }
    return e;
}

template <int MODE>
cudaError_t launch(const Job &j, cudaStream_t stream)
{
    const Plan pl = plan(static_cast<Mode>(MODE), j.M, j.N, j.K, j.terms);
    if (j.terms > 1)
        return pl.bn == 128 ? launch_tiled<MODE, 1, 128, true>(j, pl, stream)
                            : launch_tiled<MODE, 1, 64, true>(j, pl, stream);
    if (pl.cg == 2) return launch_tiled<MODE, 2, 256, false>(j, pl, stream);
    return pl.bn == 128 ? launch_tiled<MODE, 1, 128, false>(j, pl, stream)
                        : launch_tiled<MODE, 1, 64, false>(j, pl, stream);
}

// few tokens (cci_gated_few.cu): few_tokens, dense weights [F][D] of dtype; few_packed, also the packed ones (wg
// and wu: the values) as they are
bool few_tokens(int dtype, int64_t N, int64_t F);
bool few_packed(const GatedArgs &a);
cudaError_t launch_few(const GatedArgs &a, const void *wg, const void *wu, bool packed, cudaStream_t stream);

cudaError_t launch_forward(const Job &j, cudaStream_t stream);
cudaError_t launch_dx(const Job &j, cudaStream_t stream);
cudaError_t launch_dw(const Job &j, cudaStream_t stream);

}  // namespace gated
}  // namespace cci
