// cci_kernels.h -- launchers shared between the libcci translation units.
#pragma once

#include "cci_common.cuh"

namespace cci {

cudaError_t launch_pack(const void *W, int dtype, int64_t Cout, int64_t R, int G, int K, void *values,
                        uint8_t *idx, uint32_t *status, cudaStream_t stream);
cudaError_t launch_td_mask(const void *W, int dtype, int64_t Cout, int64_t R, int G, int K, float rate,
                           const float *u, void *Wout, uint8_t *mask, uint32_t *status, cudaStream_t stream);
// balanced sparsity, the comparison format (cci_bbs.cu)
cudaError_t launch_bbs_pack(const void *W, int dtype, int64_t Cout, int64_t R, int G, int K, void *values,
                            uint8_t *idx, uint32_t *status, cudaStream_t stream);
cudaError_t launch_bbs_decompress(const FwdParams &p, int dtype, int G, int K, cudaStream_t stream);
cudaError_t launch_bbs_gather(const FwdParams &p, int dtype, int G, int K, cudaStream_t stream);
cudaError_t launch_pack_stats(const void *W, int dtype, int64_t Cout, int64_t R, int G, int K,
                              unsigned long long *counts, cudaStream_t stream);
cudaError_t launch_generic(const FwdParams &p, int dtype, int G, int K, cudaStream_t stream);
cudaError_t launch_fma_probe(float *out, int blocks, int threads, int iters, cudaStream_t stream);
// bounded-wait diagnostic (cci_dense_tc.cu): arrive = 0 lets the wait expire
cudaError_t launch_wait_probe(uint32_t *status, int arrive, cudaStream_t stream);

// (G, K) pairs of the workspace tensor-core family
bool dense_tc_supported(int dtype, int G, int K);
// decompress once into p.wdense and copy B tiles from it (bf16: dense [Cout][R];
// fp32: the two operand planes of the split, cci_common.cuh)
cudaError_t launch_dense_tc_ws(const FwdParams &p, int dtype, int G, int K, cudaStream_t stream);
// dense fp32 W[Cout][R] (R % 4 == 0, 16-byte aligned) into the operand planes at planes
cudaError_t launch_dense_split(const uint32_t *W, int64_t Cout, int64_t R, void *planes, cudaStream_t stream);

// dense product on the tensor cores from the decompressed workspace p.wdense
// (cci_gemm_ws_*.cu): bf16 dense [Cout][R], or the fp32 operand planes
cudaError_t launch_gemm_ws(const FwdParams &p, int dtype, cudaStream_t stream);
cudaError_t launch_gemm_ws_bf16(const FwdParams &p, cudaStream_t stream);
cudaError_t launch_gemm_ws_tf32(const FwdParams &p, cudaStream_t stream);

// products of at most 128 columns in one launch (cci_narrow.cu; bf16, no
// workspace): the packed weights (p.values, p.idx, p.G, p.K) expanded and
// multiplied once, the reduction split over a cluster.  N: the columns of the
// whole call (a host-buffer product runs chunks of it, with the bits of the whole).
// launch_narrow returns cudaErrorNotSupported, before any launch, when the activations
// cannot be copied by TMA
bool narrow_ok(const FwdParams &p, int dtype, int64_t N);
cudaError_t launch_narrow(const FwdParams &p, cudaStream_t stream);

// fused tensor-core product (cci_gemm_pk*.cu): the GEMM of the workspace family
// with the packed weights (p.values, p.idx, p.G, p.K) expanded into each B tile
// in shared memory; bf16 only.  gemm_pk_shape_ok: (G, K), packed-array shape and
// alignment allow it; gemm_pk_supported: also the activations are copied by
// TMA; launch_gemm_pk returns cudaErrorNotSupported, before any launch, for a
// layer without it.
bool gemm_pk_shape_ok(const FwdParams &p);
bool gemm_pk_supported(const FwdParams &p);
cudaError_t launch_gemm_pk(const FwdParams &p, cudaStream_t stream);

// layer norm (cci_norm.cu); ld*: row strides in elements.  part: the backward pass' workspace
// of layer_norm_workspace bytes (N >= 1), which the sums of dw and db need
size_t layer_norm_workspace(int64_t N, int64_t D);
cudaError_t launch_layer_norm(const void *x, int dtype, int64_t N, int64_t D, int64_t ldx, const float *w,
                              const float *b, float eps, void *y, float *mean, float *rstd, cudaStream_t stream);
cudaError_t launch_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, int dtype, int64_t N,
                                       int64_t D, const float *mean, const float *rstd, const float *w, void *dx,
                                       float *dw, float *db, float *part, uint32_t *status, cudaStream_t stream);

// token log probabilities (cci_logprobs.cu)
cudaError_t launch_token_logprobs(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldx,
                                  const int64_t *tokens, int64_t ignore, int top, float *logp, float *entropy,
                                  float *stats, float *top_logp, int32_t *top_idx, uint32_t *status,
                                  cudaStream_t stream);
cudaError_t launch_token_logprobs_backward(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldx,
                                           const float *stats, const int64_t *tokens, int64_t ignore,
                                           const float *dlogp, const float *entropy, const float *dentropy, void *dx,
                                           int64_t lddx, uint32_t *status, cudaStream_t stream);

// gated feed-forward block (cci_gated*.cu).  Wg, Wu: dense [F][D], or with gate_idx the packed
// values; g, u: the saved pre-activations (forward: written, or null; backward: read); backward: dX, and
// dWg with dWu, each may be null.  workspace: gated_workspace bytes for the call (a cci_gated_call)
struct GatedArgs {
    const void *X;
    int dtype;
    int64_t N, D, F;
    const void *Wg, *Wu;
    const uint8_t *gate_idx, *up_idx;
    int G, K, act;
    void *H;
    float *g, *u;
    const void *dH;
    void *dX, *dWg, *dWu;
    uint32_t *status;
    void *workspace;
};
size_t gated_workspace(int dtype, int64_t N, int64_t D, int64_t F, int call);
cudaError_t launch_gated(const GatedArgs &a, cudaStream_t stream);
cudaError_t launch_gated_backward(const GatedArgs &a, cudaStream_t stream);

// distillation from a teacher's top logits (cci_distill.cu); workspace: distillation_workspace bytes
size_t distillation_workspace(int64_t N, int64_t V);
cudaError_t launch_distillation(const void *x, int dtype, int64_t N, int64_t V, int64_t ldx, const int32_t *idx,
                                const float *value, int k, float T, int tail, float *loss, float *stats,
                                uint32_t *status, void *workspace, cudaStream_t stream);
cudaError_t launch_distillation_backward(const float *dloss, const void *x, int dtype, int64_t N, int64_t V, int64_t ldx,
                                         const int32_t *idx, const float *value, int k, float T, int tail,
                                         const float *stats, void *dx, int64_t lddx, cudaStream_t stream);

// root-mean-square norm (cci_rms.cu); scales: y is e4m3, with `groups` scales a row (null: y of the rows' type).
// part: the backward pass' workspace of rms_norm_workspace bytes (N >= 1); dw may be null
size_t rms_norm_workspace(int64_t N, int64_t D);
cudaError_t launch_rms_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, int dtype, int64_t N, int64_t D,
                            const float *w, float eps, void *y, void *h, float *rstd, float *scales, int groups,
                            cudaStream_t stream);
cudaError_t launch_rms_norm_backward(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dh, int64_t lddh,
                                     int dtype, int64_t N, int64_t D, const float *rstd, const float *w, void *dx, float *dw,
                                     float *part, cudaStream_t stream);

// softmax cross entropy from a head's inputs (cci_head*.cu).  backward: dX and dW may each be null.  workspace:
// head_workspace bytes for the call (a cci_head_call)
struct HeadArgs {
    const void *X;
    int dtype;
    int64_t N, D, V;
    const void *W;
    const int64_t *targets;
    int64_t ignore;
    float *loss, *stats;  // backward: stats is read
    const float *dloss;
    void *dX, *dW;
    uint32_t *status;
    void *workspace;
};
size_t head_workspace(int dtype, int64_t N, int64_t D, int64_t V, int call);
cudaError_t launch_head(const HeadArgs &a, cudaStream_t stream);
cudaError_t launch_head_backward(const HeadArgs &a, cudaStream_t stream);

// One register-tiled instantiation: (dtype, G, K) -> tile shape and launcher.
struct RegtileEntry {
    int dtype, G, K, MG, T, D;
    const char *name;
    cudaError_t (*launch)(const FwdParams &p, cudaStream_t stream);
};

// all instantiations, terminated by an entry with launch == nullptr
const RegtileEntry *regtile_table();

// channel-warps per CTA (4 or 8) for a layer with this many groups
int regtile_wc(int64_t groups, int MG);

constexpr size_t kMaxSmemPerBlock = 227 * 1024;

}  // namespace cci
