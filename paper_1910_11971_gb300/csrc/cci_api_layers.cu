// cci_api_layers.cu -- the extern "C" entry points of the layers around a pruned projection
// (declared in cci.h): argument checks, all before anything is enqueued, and the launch on the
// caller's stream.
#include "cci_checks.h"
#include "cci_kernels.h"

using namespace cci;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31;
constexpr int64_t kMaxLogits = int64_t(1) << 24;  // of a row: the alternatives' runs fit shared memory

cudaStream_t as_stream(cci_stream_t s) { return reinterpret_cast<cudaStream_t>(s); }

// N rows of D elements, row stride ld: sizes that no index computation can pass
bool rows_ok(int64_t N, int64_t D, int64_t ld) { return N >= 0 && D >= 1 && ld >= D && mul_ok(N, ld); }

}  // namespace

extern "C" {

cci_status cci_layer_norm(const void *x, cci_dtype dtype, int64_t N, int64_t D, int64_t ldx, const float *weight,
                          const float *bias, float eps, void *y, float *mean, float *rstd, cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!x || !y || !mean || !rstd)) return CCI_ERR_NULL;
    if (!rows_ok(N, D, ldx)) return CCI_ERR_SHAPE;
    if (!(eps >= 0.0f)) return CCI_ERR_VALUE;  // also NaN
    const size_t es = elem_size(dtype);
    if (!aligned(x, es) || !aligned(y, es) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) ||
        !aligned(rstd, 4))
        return CCI_ERR_ALIGN;
    if (N == 0) return CCI_OK;
    return to_status(launch_layer_norm(x, dtype, N, D, ldx, weight, bias, eps, y, mean, rstd, as_stream(stream)));
}

size_t cci_layer_norm_workspace_size(int64_t N, int64_t D)
{
    return N < 1 || D < 1 || !mul_ok(N, D) ? 0 : layer_norm_workspace(N, D);
}

cci_status cci_layer_norm_backward_ex(const void *dy, int64_t lddy, const void *x, int64_t ldx, cci_dtype dtype,
                                      int64_t N, int64_t D, const float *mean, const float *rstd, const float *weight,
                                      void *dx, float *dweight, float *dbias, uint32_t *dev_status, void *workspace,
                                      size_t workspace_bytes, cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!dy || !x || !mean || !rstd || !dx)) return CCI_ERR_NULL;
    if (!rows_ok(N, D, ldx) || !rows_ok(N, D, lddy)) return CCI_ERR_SHAPE;
    const size_t es = elem_size(dtype);
    if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return CCI_ERR_ALIGN;
    const size_t need = N > 0 ? layer_norm_workspace(N, D) : 0;
    if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return CCI_ERR_WORKSPACE;
    return to_status(launch_layer_norm_backward(dy, lddy, x, ldx, dtype, N, D, mean, rstd, weight, dx, dweight, dbias,
                                                static_cast<float *>(workspace), dev_status, as_stream(stream)));
}

cci_status cci_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, cci_dtype dtype,
                                   int64_t N, int64_t D, const float *mean, const float *rstd, const float *weight,
                                   void *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                                   cci_stream_t stream)
{
    return cci_layer_norm_backward_ex(dy, lddy, x, ldx, dtype, N, D, mean, rstd, weight, dx, dweight, dbias, nullptr,
                                      workspace, workspace_bytes, stream);
}

cci_status cci_token_logprobs(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                              const int64_t *tokens, int64_t ignore_index, int top, float *logp, float *entropy,
                              float *stats, float *top_logp, int32_t *top_idx, uint32_t *dev_status,
                              cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!logits || !tokens || !logp || !entropy || !stats || (top > 0 && (!top_logp || !top_idx))))
        return CCI_ERR_NULL;
    if (!rows_ok(N, V, ldx) || V > kMaxLogits || N >= kMaxRows || top < 0 || top > CCI_MAX_TOP || top > V)
        return CCI_ERR_SHAPE;
    if (!aligned(logits, elem_size(dtype)) || !aligned(tokens, 8) || !aligned(logp, 4) || !aligned(entropy, 4) ||
        !aligned(stats, 4) || !aligned(top_logp, 4) || !aligned(top_idx, 4))
        return CCI_ERR_ALIGN;
    if (N == 0) return CCI_OK;
    return to_status(launch_token_logprobs(logits, dtype, N, V, ldx, tokens, ignore_index, top, logp, entropy, stats,
                                           top_logp, top_idx, dev_status, as_stream(stream)));
}

cci_status cci_token_logprobs_backward(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                                       const float *stats, const int64_t *tokens, int64_t ignore_index,
                                       const float *dlogp, const float *entropy, const float *dentropy,
                                       void *dlogits, int64_t lddx, uint32_t *dev_status, cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!logits || !stats || !dlogits || (dlogp && !tokens) || (dentropy && !entropy))) return CCI_ERR_NULL;
    // a block takes 8192 logits of a row
    if (!rows_ok(N, V, ldx) || !rows_ok(N, V, lddx) || V > kMaxLogits || N >= kMaxRows ||
        N * ((V + 8191) / 8192) >= kMaxRows)
        return CCI_ERR_SHAPE;
    const size_t es = elem_size(dtype);
    if (!aligned(logits, es) || !aligned(dlogits, es) || !aligned(stats, 4) || !aligned(tokens, 8) ||
        !aligned(dlogp, 4) || !aligned(entropy, 4) || !aligned(dentropy, 4))
        return CCI_ERR_ALIGN;
    if (N == 0) return CCI_OK;
    return to_status(launch_token_logprobs_backward(logits, dtype, N, V, ldx, stats, tokens, ignore_index, dlogp,
                                                    entropy, dentropy, dlogits, lddx, dev_status, as_stream(stream)));
}

}  // extern "C"

namespace {

// sizes and pointers that every call of the gated block has
cci_status check_gated(int dtype, int64_t N, int64_t D, int64_t F, int act, const void *X, const void *Wg,
                       const void *Wu, const void *workspace, size_t bytes, int call)
{
    constexpr int64_t lim = int64_t(1) << 30;  // tile coordinates are 32-bit
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (!Wg || !Wu || (N > 0 && !X)) return CCI_ERR_NULL;
    if (N < 0 || D < 1 || F < 1 || N >= lim || D >= lim || F >= lim) return CCI_ERR_SHAPE;
    if (act < CCI_ACT_SILU || act > CCI_ACT_SIGMOID) return CCI_ERR_VALUE;
    if (D % 8 != 0 || F % 8 != 0) return CCI_ERR_UNSUPPORTED;
    if (!aligned(X, 16) || !aligned(Wg, 16) || !aligned(Wu, 16)) return CCI_ERR_ALIGN;
    const size_t need = N > 0 ? gated_workspace(dtype, N, D, F, call) : 0;
    if (need > 0 && (!workspace || bytes < need || !aligned(workspace, 16))) return CCI_ERR_WORKSPACE;
    return CCI_OK;
}

}  // namespace

extern "C" {

size_t cci_gated_workspace_size(cci_gated_call call, cci_dtype dtype, int64_t N, int64_t D, int64_t F)
{
    constexpr int64_t lim = int64_t(1) << 30;
    if (!valid_dtype(dtype) || N < 1 || D < 1 || F < 1 || N >= lim || D >= lim || F >= lim) return 0;
    if (call < CCI_GATED_FORWARD || call > CCI_GATED_BACKWARD) return 0;
    return gated_workspace(dtype, N, D, F, call);
}

cci_status cci_gated_linear(const void *X, cci_dtype dtype, int64_t N, int64_t D, const void *Wg, const void *Wu,
                            int64_t F, cci_activation act, void *H, float *g, float *u, uint32_t *dev_status,
                            void *workspace, size_t workspace_bytes, cci_stream_t stream)
{
    const cci_status st = check_gated(dtype, N, D, F, act, X, Wg, Wu, workspace, workspace_bytes, CCI_GATED_FORWARD);
    if (st != CCI_OK) return st;
    if (N > 0 && (!H || !g != !u)) return CCI_ERR_NULL;
    if (!aligned(H, 16) || !aligned(g, 16) || !aligned(u, 16)) return CCI_ERR_ALIGN;
    if (N == 0) return CCI_OK;
    GatedArgs a{};
    a.X = X;
    a.dtype = dtype;
    a.N = N;
    a.D = D;
    a.F = F;
    a.Wg = Wg;
    a.Wu = Wu;
    a.act = act;
    a.H = H;
    a.g = g;
    a.u = u;
    a.status = dev_status;
    a.workspace = workspace;
    return to_status(launch_gated(a, as_stream(stream)));
}

cci_status cci_gated_linear_packed(const void *X, cci_dtype dtype, int64_t N, int64_t D, const void *gate_values,
                                   const uint8_t *gate_idx, const void *up_values, const uint8_t *up_idx, int64_t F,
                                   int G, int K, cci_activation act, void *H, uint32_t *dev_status, void *workspace,
                                   size_t workspace_bytes, cci_stream_t stream)
{
    if (!gate_idx || !up_idx) return valid_dtype(dtype) ? CCI_ERR_NULL : CCI_ERR_DTYPE;
    const cci_status st = check_gated(dtype, N, D, F, act, X, gate_values, up_values, workspace, workspace_bytes,
                                      CCI_GATED_PACKED);
    if (st != CCI_OK) return st;
    const cci_status gr = check_group(F, G, K);
    if (gr != CCI_OK) return gr;
    if (N > 0 && !H) return CCI_ERR_NULL;
    if (!aligned(H, 16)) return CCI_ERR_ALIGN;
    if (N == 0) return CCI_OK;
    GatedArgs a{};
    a.X = X;
    a.dtype = dtype;
    a.N = N;
    a.D = D;
    a.F = F;
    a.Wg = gate_values;
    a.Wu = up_values;
    a.gate_idx = gate_idx;
    a.up_idx = up_idx;
    a.G = G;
    a.K = K;
    a.act = act;
    a.H = H;
    a.status = dev_status;
    a.workspace = workspace;
    return to_status(launch_gated(a, as_stream(stream)));
}

cci_status cci_gated_linear_backward(const void *dH, const void *X, cci_dtype dtype, int64_t N, int64_t D,
                                     const void *Wg, const void *Wu, int64_t F, cci_activation act, const float *g,
                                     const float *u, void *dX, void *dWg, void *dWu, uint32_t *dev_status,
                                     void *workspace, size_t workspace_bytes, cci_stream_t stream)
{
    const cci_status st = check_gated(dtype, N, D, F, act, X, Wg, Wu, workspace, workspace_bytes, CCI_GATED_BACKWARD);
    if (st != CCI_OK) return st;
    if (N > 0 && (!dH || !g || !u)) return CCI_ERR_NULL;
    if (!dWg != !dWu) return CCI_ERR_NULL;
    if (!aligned(dH, 16) || !aligned(g, 16) || !aligned(u, 16) || !aligned(dX, 16) || !aligned(dWg, 16) ||
        !aligned(dWu, 16))
        return CCI_ERR_ALIGN;
    GatedArgs a{};
    a.X = X;
    a.dtype = dtype;
    a.N = N;
    a.D = D;
    a.F = F;
    a.Wg = Wg;
    a.Wu = Wu;
    a.act = act;
    a.g = const_cast<float *>(g);
    a.u = const_cast<float *>(u);
    a.dH = dH;
    a.dX = dX;
    a.dWg = dWg;
    a.dWu = dWu;
    a.status = dev_status;
    a.workspace = workspace;
    return to_status(launch_gated_backward(a, as_stream(stream)));
}

}  // extern "C"
