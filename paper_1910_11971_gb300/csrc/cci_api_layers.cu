// cci_api_layers.cu -- the extern "C" entry points of the layers around a pruned projection
// (declared in cci.h): argument checks, all before anything is enqueued, and the launch on the
// caller's stream.
#include "cci_checks.h"
#include "cci_kernels.h"

using namespace cci;

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31;

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

cci_status cci_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, cci_dtype dtype,
                                   int64_t N, int64_t D, const float *mean, const float *rstd, const float *weight,
                                   void *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                                   cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!dy || !x || !mean || !rstd || !dx)) return CCI_ERR_NULL;
    if (!rows_ok(N, D, ldx) || !rows_ok(N, D, lddy)) return CCI_ERR_SHAPE;
    const size_t es = elem_size(dtype);
    if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return CCI_ERR_ALIGN;
    if (N > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < layer_norm_workspace(N, D)))
        return CCI_ERR_WORKSPACE;
    return to_status(launch_layer_norm_backward(dy, lddy, x, ldx, dtype, N, D, mean, rstd, weight, dx, dweight, dbias,
                                                static_cast<float *>(workspace), as_stream(stream)));
}

cci_status cci_token_logprobs(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                              const int64_t *tokens, int64_t ignore_index, int top, float *logp, float *entropy,
                              float *stats, float *top_logp, int32_t *top_idx, uint32_t *dev_status,
                              cci_stream_t stream)
{
    if (!valid_dtype(dtype)) return CCI_ERR_DTYPE;
    if (N > 0 && (!logits || !tokens || !logp || !entropy || !stats || (top > 0 && (!top_logp || !top_idx))))
        return CCI_ERR_NULL;
    if (!rows_ok(N, V, ldx) || V >= kMaxRows || N >= kMaxRows || top < 0 || top > CCI_MAX_TOP || top > V)
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
    if (!rows_ok(N, V, ldx) || !rows_ok(N, V, lddx) || V >= kMaxRows || N >= kMaxRows ||
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
