// cci_wide.cuh -- fp32 products of a head's gradients over 256 x 256 tiles of a CTA pair.
//
// Six products of bf16 planes each, as in cci_gated.cuh, whose tiles of one CTA hold a tile's sums in the registers of
// four output warps: 128 x 128 of them, two loads from L2 for each product.  Here eight output warps hold 128 sums a
// thread, so that a pair shares its operands and each load serves two products.  Roles, waits, the
// cut of the last tiles' reductions and their join are those of cci_gated.cuh; the dX product's A lies K-major, the others MN-major.
// 500 tokens, 1024 wide, 16128 entries: dX 87 us with the tiles of one CTA, 68 so; dW 76 and 74; both passes of 1000 tokens,
// 1024 wide, 32000 entries 1311 and 1201.
#pragma once

#include "cci_gated.cuh"

namespace cci {
namespace gated {

struct WideCfg {
    static constexpr int kM = 128, kBN = 256, kABytes = kM * 128, kBBytes = 128 * 128, kStage = kABytes + kBBytes;
    static constexpr int kOut = kM * 128, kBufs = 2, kOuts = 2 * kBufs;  // buffers of 32 columns for each four output warps
    static constexpr int kStages = (static_cast<int>(kMaxSmemPerBlock) - 2048 - kOuts * kOut) / kStage;
    static constexpr int kThreads = 384, kCols = 128;
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStage + kOuts * kOut + 1024;
    static_assert(kStages >= 4 && kStages <= 8 && kSmem <= kMaxSmemPerBlock, "stages");
};

// sixteen columns of this warp's TMEM lanes, waited for: they are operands of the wait, so that nothing takes them before
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

template <int MODE>
__global__ void __launch_bounds__(WideCfg::kThreads, 1) wide_kernel(const Params p, const __grid_constant__ Maps maps)
{
    using C = WideCfg;
    constexpr bool kAMn = is_dw(MODE);
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kAMn) << 15) | (1u << 16) |
                                (static_cast<uint32_t>(C::kBN >> 3) << 17) | (static_cast<uint32_t>((C::kM * 2) >> 4) << 24);
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const uint32_t raw = tc::smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t outs = base + C::kStages * C::kStage;
    Smem *S = reinterpret_cast<Smem *>(smem_raw + (outs - raw) + C::kOuts * C::kOut);
    volatile int *abort = &S->abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = ws::cluster_rank();
    const int first = static_cast<int>(blockIdx.x) / 2, step = static_cast<int>(gridDim.x) / 2;
    const int per_tile = p.terms * p.k_stages;
    Work work;

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            tc::mbar_init(&S->full[s], 1);
            tc::mbar_init(&S->empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            tc::mbar_init(&S->acc_full[a], 1);
            tc::mbar_init(&S->acc_empty[a], 16);
        }
        tc::mbar_init(&S->drain, 1);
        S->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&S->tmem_base)),
                     "r"(2 * C::kBN)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    ws::cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = S->tmem_base;

    // output threads hold 128 sums each: 128 threads give up 96 of their 168 registers, and 256 take 48 more
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0) {
            // ---- copies
            if (tc::elect_one()) {
                const uint32_t a_bytes = kAMn ? static_cast<uint32_t>(C::kABytes) : static_cast<uint32_t>(p.a_rows) * 128u;
                const uint32_t bytes = 2u * (a_bytes + static_cast<uint32_t>(C::kBBytes));
                int s = 0, it = 0;
                uint32_t ph = 1u;  // a fresh barrier's preceding phase counts as complete
                bool ok = true;
                for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
                    int mt, nt;
                    tile_at(p, work.tile, p.m_tiles, mt, nt);
                    const int m0 = (mt * 2 + static_cast<int>(rank)) * C::kM;
                    const int n0 = nt * C::kBN + static_cast<int>(rank) * 128;
                    // all terms of a stage one after the other: what they share comes from L2
                    int ks = work.s0 / p.terms, t = work.s0 % p.terms, pa, pb;
                    term_planes(t, p.terms, pa, pb);
                    for (int i = 0; i < work.n; ++i, ++it) {
                        ok = tc::mbar_wait(&S->empty[s], ph, abort, p.status);
                        if (!ok) break;
                        const uint32_t sa = base + s * C::kStage, sb = sa + C::kABytes;
                        if (rank == 0) tc::mbar_arrive_expect_tx(&S->full[s], bytes);
                        const uint32_t bar = ws::map_to_rank(tc::smem_u32(&S->full[s]), 0);
                        const int k0 = ks * 64;
                        if constexpr (kAMn) {
                            load_3d<2>(sa, &maps.a[0], m0, k0, pa, bar);
                            load_3d<2>(sa + 8192, &maps.a[0], m0 + 64, k0, pa, bar);
                        } else {
                            load_3d<2>(sa, &maps.a[0], k0, m0, pa, bar);
                        }
                        load_3d<2>(sb, &maps.b[0], n0, k0, pb, bar);
                        load_3d<2>(sb + 8192, &maps.b[0], n0 + 64, k0, pb, bar);
                        if (++s == C::kStages) {
                            s = 0;
                            ph ^= 1u;
                        }
                        if (++t == p.terms) {
                            t = 0;
                            ++ks;
                        }
                        term_planes(t, p.terms, pa, pb);
                    }
                }
                // no copy is in flight when the block ends, nor a commit, also after an abort (as in product_kernel)
                int no_abort = 0;
                if (rank == 0)
                    for (int d = it > C::kStages ? it - C::kStages : 0; d < it; ++d)
                        tc::mbar_wait(&S->full[d % C::kStages], (d / C::kStages) & 1, &no_abort, p.status);
                no_abort = 0;
                for (int d = it > C::kStages ? it - C::kStages : 0; d < it; ++d)
                    tc::mbar_wait(&S->empty[d % C::kStages], (d / C::kStages) & 1, &no_abort, p.status);
            }
            __syncwarp();
        } else if (warp == 1 && rank == 0) {
            // ---- products
            if (tc::elect_one()) {
                int s = 0, t = 0;
                uint32_t ph = 0u;
                bool ok = true;
                const uint64_t da0 = tile_desc<kAMn>(base), db0 = tile_desc<true>(base + C::kABytes);
                const uint32_t empty0 = tc::smem_u32(&S->empty[0]);
                for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
                    for (int left = work.n; left > 0 && ok; left -= kChunk, ++t) {
                        const int acc = t & 1, n = left < kChunk ? left : kChunk;
                        if (t >= 2) ok = tc::mbar_wait<true>(&S->acc_empty[acc], ((t >> 1) - 1) & 1, abort, p.status);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t d = tmem + static_cast<uint32_t>(acc * C::kBN);
                        for (int i = 0; i < n; ++i) {
                            ok = tc::mbar_wait(&S->full[s], ph, abort, p.status);
                            if (!ok) break;
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            const uint64_t off = static_cast<uint64_t>(s) * (C::kStage >> 4);
                            stage_mma<2, kIdesc, kAMn ? 128 : 2, 128>(d, da0 + off, db0 + off, i > 0 ? 1u : 0u, empty0 + 8u * s);
                            if (++s == C::kStages) {
                                s = 0;
                                ph ^= 1u;
                            }
                        }
                        if (ok) ws::mma_commit_pair(&S->acc_full[acc]);
                    }
                }
                // every product has ended before the tensor memory is given back
                ws::mma_commit_pair(&S->drain);
                int no_abort = 0;
                tc::mbar_wait(&S->drain, 0, &no_abort, p.status);
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- output: row `m` of the CTA's 128 and 128 columns from c0 of the tile on, per thread
        const int half = (warp - 4) >> 2, m = tid & 127, c0 = half * C::kCols;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t acc_empty0 = ws::map_to_rank(tc::smem_u32(&S->acc_empty[0]), 0);
        const uint32_t bufs = outs + static_cast<uint32_t>(half * C::kBufs) * C::kOut;
        int t = 0, stored = 0;
        bool ok = true;
        for (int j = 0; ok && work_at(p, first, step, per_tile, j, work); ++j) {
            int mt, nt;
            tile_at(p, work.tile, p.m_tiles, mt, nt);
            const int r0 = (mt * 2 + static_cast<int>(rank)) * C::kM, n0 = nt * C::kBN + c0;
            float z[C::kCols];
            bool begun = false;
            for (int left = work.n; left > 0 && ok; left -= kChunk, begun = true) {
                ok = tc::mbar_wait(&S->acc_full[t & 1], (t >> 1) & 1, abort, p.status);
                ok = tc::named_and(1, 256, ok);
                if (!ok) break;
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t col = tmem + lanes + static_cast<uint32_t>((t & 1) * C::kBN + c0);
#pragma unroll
                for (int q = 0; q < C::kCols; q += 16) {
                    uint32_t v[16];
                    tmem_ld16(col + q, v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[q + i] = begun ? z[q + i] + __uint_as_float(v[i]) : __uint_as_float(v[i]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if (rank != 0)
                        ws::mbar_arrive_remote(acc_empty0 + static_cast<uint32_t>((t & 1) * sizeof(uint64_t)));
                    else
                        tc::mbar_arrive(&S->acc_empty[t & 1]);
                }
                ++t;
            }
            if (!ok) break;
            if (r0 >= p.M) continue;  // the odd CTA's rows may all lie past the matrix
#pragma unroll
            for (int c = 0; c < C::kCols; c += 32) {
                if (n0 + c >= p.N) break;
                const uint32_t buf = bufs + static_cast<uint32_t>(stored % C::kBufs) * C::kOut;
                ++stored;
                if (m == 0) tc::bulk_wait_read<C::kBufs - 1>();
                tc::named_sync(2 + half, 128);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    ws::st_shared_v4(buf + ws::sw_chunk(m, q), __float_as_uint(z[c + 4 * q]), __float_as_uint(z[c + 4 * q + 1]),
                                     __float_as_uint(z[c + 4 * q + 2]), __float_as_uint(z[c + 4 * q + 3]));
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc::named_sync(2 + half, 128);
                if (m == 0) {
                    if (work.part >= 0)
                        tc::tma_store_2d(&maps.parts, buf, c0 + c, (work.part * 2 + static_cast<int>(rank)) * C::kM);
                    else if (MODE == kDxAdd && p.add)
                        tma_add_2d(&maps.out[0], buf, n0 + c, r0);
                    else
                        tc::tma_store_2d(&maps.out[0], buf, n0 + c, r0);
                    tc::bulk_commit();
                }
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
    // the last commit signals this CTA's barrier too: it has arrived before either CTA leaves
    if (rank != 0 && tid == 0) {
        int no_abort = 0;
        tc::mbar_wait(&S->drain, 0, &no_abort, p.status);
    }
    __syncwarp();
    ws::cluster_sync();
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * C::kBN) : "memory");
    }
}

template <int MODE>
cudaError_t launch_wide(const Job &j, const Plan &plan, cudaStream_t stream)
{
    using C = WideCfg;
    Params p{};
    Maps maps{};
    p.M = j.M;
    p.N = j.N;
    p.k_stages = static_cast<int>((j.K + 63) / 64);
    p.pairs = 1;
    p.terms = j.terms;
    p.a_rows = j.M < C::kM ? static_cast<int>((j.M + 7) / 8 * 8) : C::kM;
    p.out_f32 = 1;
    p.add = j.add;
    p.status = j.status;
    const int64_t mt = (j.M + 255) / 256, nt = (j.N + C::kBN - 1) / C::kBN;
    if (mt * nt > (int64_t(1) << 30)) return cudaErrorInvalidValue;
    p.m_tiles = static_cast<int>(mt);
    p.n_tiles = static_cast<int>(nt);
    p.tiles = static_cast<int>(mt * nt);
    const bool cut = plan.cut;
    const int units = cut ? plan.units : ws::sm_count() / 2;
    p.whole = cut ? p.tiles - p.tiles % units : p.tiles;
    if (!operand_map(&maps.a[0], j.a[0], is_dw(MODE) ? 64 : p.a_rows) || !operand_map(&maps.b[0], j.b[0], 64) ||
        !output_map(&maps.out[0], j.out[0], true, j.M, j.N, 32))
        return cudaErrorInvalidValue;
    if (cut && !output_map(&maps.parts, j.parts, true, static_cast<int64_t>(units) * 2 * 256, C::kBN, 32))
        return cudaErrorInvalidValue;
    static SmemAttrCache attr_cache;
    const cudaError_t attr = smem_attr_once(wide_kernel<MODE>, static_cast<int>(C::kSmem), attr_cache);
    if (attr != cudaSuccess) return attr;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((cut || p.tiles > units ? units : p.tiles) * 2));
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = 2;
    la[0].val.clusterDim.y = 1;
    la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, wide_kernel<MODE>, p, maps);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess || !cut) return e;
    cudaLaunchConfig_t jc = {};
    jc.gridDim = dim3(static_cast<unsigned>((p.tiles - p.whole) * (256 / 8)));
    jc.blockDim = dim3(C::kBN);
    jc.stream = stream;
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    jc.attrs = la;
    jc.numAttrs = 1;
    e = cudaLaunchKernelEx(&jc, join_kernel<MODE, 2, 256>, p, const_cast<const float *>(j.parts), j.out[0],
                           static_cast<void *>(nullptr), static_cast<float *>(nullptr), units);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

// a head's product: fp32 by the tiles of a pair where the plan takes them
template <int MODE>
cudaError_t launch_one(const Job &j, cudaStream_t stream)
{
    if (j.terms > 1) {
        const Plan pl = plan(static_cast<Mode>(MODE), j.M, j.N, j.K, j.terms);
        if (pl.cg == 2) return launch_wide<MODE>(j, pl, stream);
    }
    return launch<MODE>(j, stream);
}

}  // namespace gated
}  // namespace cci
