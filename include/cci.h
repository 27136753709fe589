/*
 * cci.h -- C ABI of libcci.so: forward products of layers with cross-channel
 * intragroup (CCI) sparsity on NVIDIA GB300 (sm_103a), and the layers of a language model
 * around them (layer norm, gated feed-forward block, token log probabilities) in both directions.
 *
 * Method: Yu et al., "Cross-Channel Intragroup Sparsity Neural Network"
 * (arXiv 1910.11971).  For every input feature r of a layer (for a convolution,
 * every tap (kh, kw, ci)), the weights of G neighbouring output channels form a
 * group, and exactly K of the G are kept (Sec. 3.1, Fig. 1).  Every G rows of the
 * weight matrix therefore compress into K rows of (value, index) pairs, each with
 * as many columns as the original matrix; the index is the plain row index
 * inside the group (log2 G bits, Sec. 3.1).  The product H = W x X is then Alg. 2
 * of Sec. 3.2: H(G*i + Idx, j) += Val * X(k, j).
 *
 * Layouts (all row-major, dense, contiguous; element = dtype unless stated):
 *   W       [Cout][R]              dense weights (pack input); R = Cin*KH*KW,
 *                                  r = (kh*KW + kw)*Cin + ci for convolutions
 *                                  (OHWI order)
 *   values  [Cout/G][R][K]         kept weights, per (group, r) in increasing index
 *   idx     [Cout/G][R][K] uint8   index j in [0, G) of each kept weight
 *   X       [N][Cin]               product input: N columns of Cin features
 *                                  (the paper's column-major X)
 *   X       [B][H][W][Cin]         convolution input (NHWC)
 *   Y       [N][Cout] float32      product output (the paper's H, transposed)
 *   Y       [B][P][Q][Cout] float32  convolution output (NHWC),
 *                                  P = (H + 2*pad_h - KH)/stride_h + 1, Q likewise
 *
 * Ownership and execution: the caller allocates every buffer; all data pointers
 * are DEVICE pointers (except the X_host / Y_host of cci_linear_host); the
 * library allocates nothing.  It keeps no state between calls except three
 * per-device caches, filled on a device's first use: the dynamic shared-memory
 * limit set on each kernel that asks for more than the default, the device's number of SMs, and the device
 * address of the static scratch array of cci_linear_dense_tc_static (see there).  Every
 * call is asynchronous on `stream` (NULL = the legacy default stream) and
 * returns once its kernels are enqueued.  Calls on different streams may run
 * concurrently when their outputs do not overlap.
 *
 * Errors:
 *   - Argument errors are detected on the host, before anything is enqueued, and
 *     returned directly (nothing is written).
 *   - A failed launch returns CCI_ERR_CUDA.
 *   - Errors found by the kernels while they run (NaN in a pack input, a packed
 *     index >= G, a token outside its vocabulary, an expired bounded wait) are OR-ed as bits (1u << code) into
 *     the caller's device word `*dev_status`, if it is not NULL; read it after
 *     synchronising the stream and decode it with cci_decode_device_status().
 *     The library never clears that word.  When a kernel reports an error its
 *     outputs are unspecified.
 */
#ifndef CCI_H_
#define CCI_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

struct CUstream_st; /* the same type as cudaStream_t */
typedef struct CUstream_st *cci_stream_t;

typedef enum cci_status {
    CCI_OK = 0,
    CCI_ERR_NULL = 1,         /* a required pointer is NULL */
    CCI_ERR_SHAPE = 2,        /* a size is negative/zero where not allowed, too large,
                                 or the convolution geometry has no output */
    CCI_ERR_GROUP = 3,        /* G not in [1, 256], K not in [1, G], or Cout % G != 0 */
    CCI_ERR_DTYPE = 4,        /* dtype is not a cci_dtype */
    CCI_ERR_ALIGN = 5,        /* a pointer is not aligned to its element size */
    CCI_ERR_VALUE = 6,        /* device: NaN among the weights given to cci_pack */
    CCI_ERR_CUDA = 7,         /* a CUDA launch or runtime call failed */
    CCI_ERR_TIMEOUT = 8,      /* device: a bounded wait inside a kernel expired */
    CCI_ERR_UNSUPPORTED = 9,  /* valid request this build does not implement */
    CCI_ERR_INDEX = 10,       /* device: a packed index >= G given to a product (dense
                                 kernels: also an index set not strictly increasing) */
    CCI_ERR_WORKSPACE = 11    /* the kernel family needs a workspace: missing, too small
                                 or not 16-byte aligned (see cci_workspace_size) */
} cci_status;

typedef enum cci_dtype {
    CCI_F32 = 0,   /* IEEE binary32 */
    CCI_BF16 = 1   /* bfloat16; products accumulate in fp32 on the exact values */
} cci_dtype;

/* Kernel family for cci_linear_ex / cci_conv2d_ex. */
typedef enum cci_algo {
    CCI_ALGO_AUTO = 0,      /* the fastest family this build has for (G, K, dtype, shape): the
                               workspace tensor-core family when a large enough workspace is
                               given (cci_linear_ws); else the fused tensor-core family
                               (CCI_ALGO_DENSE_TC) for bf16 layers that have it; else the
                               CUDA-core families.  Most bf16 products of at most 128
                               columns (K <= 8) run one launch instead of either tensor-core
                               family: it expands the weights inside the product and
                               neither reads nor writes the workspace.  Long reductions
                               are summed there in up to eight parts, so a column's last
                               bits may differ from those it has in a call of more columns */
    CCI_ALGO_GENERIC = 1,   /* generic kernel: any G <= 256, any K, any alignment */
    CCI_ALGO_REGTILE = 2,   /* register-tiled scatter on CUDA cores: Alg. 2 with the output
                               row chosen per (group, r) by a warp-uniform jump;
                               CCI_ERR_UNSUPPORTED when (G, K, dtype, shape) has no tile */
    CCI_ALGO_DENSE_TC = 3,  /* fused tensor-core family, no workspace: inside the GEMM the
                               packed (value, index) runs of each stage are copied by TMA
                               and expanded by producer warps into the dense bf16 weight
                               tile in shared memory (each value to row G*i + Idx of its
                               group, Alg. 2), which tcgen05.mma multiplies with the TMA-
                               copied activations.  bf16; G in {4, 8, 16, 32}, K in
                               {1, 2, 4, 8} with K <= G/2; Cin % 8 == 0, R*K % 16 == 0;
                               16-byte aligned X, Y, values and idx; activations a product
                               or a convolution with strides <= 2 and Cin % 64 == 0 (else
                               CCI_ERR_UNSUPPORTED).  Index sets are checked (strictly
                               increasing, < G; CCI_ERR_INDEX) by the CTAs of the first
                               column tile of every channel tile */
    CCI_ALGO_EXPAND = 4,    /* register-tiled on CUDA cores without jumps: each (group, r)
                               is expanded to its G weights (pruned ones zero) in shared
                               memory and all G rows are updated; same shape rules as
                               CCI_ALGO_REGTILE */
    CCI_ALGO_DENSE_TC_WS = 5  /* decompress the packed weights once per call into a caller
                               workspace and multiply densely on the tensor cores (tcgen05),
                               operands copied by TMA (cp.async.bulk.tensor).  bf16: dense bf16 [Cout][R],
                               Cin % 8 == 0, R % 8 == 0.  fp32: every operand split as
                               hi + lo (hi a tf32 value) and, per 32 indices, the product
                               hi(x) hi(w) on tf32 MMAs plus bf16(x) bf16(lo(w)) +
                               bf16(lo(x)) bf16(hi(w)) on bf16 MMAs (8 MMAs; per term
                               |error| <= 5.7e-6 |w||x| before the fp32 accumulation);
                               workspace: plane 0 [Cout][R] fp32 hi, then plane 1
                               [Cout][ceil(R/32)*64] bf16 (per 32-wide chunk of r, 32
                               bf16(hi(w)) then 32 bf16(lo(w))).  Cin % 4 == 0, R % 4 == 0.
                               Needs cci_workspace_size() bytes */
} cci_algo;

/*
 * cci_pack -- choose and compress the kept weights (Sec. 3.1 format, Sec. 5.1
 * selection: the weights of largest |w| survive).
 *
 * For every group gi in [0, Cout/G) and r in [0, R), the G weights
 * W[gi*G + j][r], j = 0..G-1, are ranked by decreasing |w| (compared in the
 * storage dtype; -0 and +0 are equal, +-inf is largest); equal magnitudes rank by
 * increasing j.  The first K survive and are written in increasing j:
 * values[gi][r][s] = W[gi*G + j_s][r] (bit-exact copy), idx[gi][r][s] = j_s.
 *
 *   W          device, [Cout][R] of dtype, aligned to the element size
 *   values     device, [Cout/G][R][K] of dtype (written)
 *   idx        device, [Cout/G][R][K] uint8 (written)
 *   dev_status device uint32 or NULL; NaN in W sets bit (1u << CCI_ERR_VALUE)
 *              (with NULL, NaN goes unreported and ranks above +inf)
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (Cout or R < 1), CCI_ERR_GROUP,
 *         CCI_ERR_DTYPE, CCI_ERR_ALIGN, CCI_ERR_CUDA.
 */
cci_status cci_pack(const void *W, cci_dtype dtype, int64_t Cout, int64_t R, int G, int K,
                    void *values, uint8_t *idx, uint32_t *dev_status, cci_stream_t stream);

/*
 * cci_linear -- Y = X W-hat^T for a CCI-sparse fully connected layer (Alg. 2 of
 * Sec. 3.2 over all N columns, with the slot loop for K > 1):
 *   Y[n][gi*G + idx[gi][r][s]] += values[gi][r][s] * X[n][r]
 * summed over r and s in fp32, starting from zero.  A repeated index inside one
 * (group, r) adds both values, as Alg. 2 does.
 *
 *   X          device, [N][Cin] of dtype (R = Cin)
 *   values,idx device, as written by cci_pack for (Cout, R = Cin, G, K)
 *   Y          device, [N][Cout] float32 (written, every element)
 *   dev_status device uint32 or NULL; an index >= G sets bit (1u << CCI_ERR_INDEX)
 * N = 0 is valid and enqueues nothing.
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE, CCI_ERR_GROUP, CCI_ERR_DTYPE, CCI_ERR_ALIGN,
 *         CCI_ERR_CUDA.
 */
cci_status cci_linear(const void *X, cci_dtype dtype, int64_t N, int64_t Cin,
                      const void *values, const uint8_t *idx, int64_t Cout, int G, int K,
                      float *Y, uint32_t *dev_status, cci_stream_t stream);

/*
 * cci_conv2d -- CCI-sparse 2-D convolution (Sec. 3.1: the structure applies to
 * convolutional layers with one group per tap (kh, kw, ci)), computed as an
 * implicit product: column n = (b, p, q), reduction index
 * r = (kh*KW + kw)*Cin + ci, and
 *   x[n][r] = X[b][p*stride_h - pad_h + kh][q*stride_w - pad_w + kw][ci]
 * or 0 outside the image (cross-correlation, zero padding, floor output size, no
 * dilation, conv groups or bias).
 *
 *   X          device NHWC [B][H][W][Cin] of dtype
 *   values,idx device, cci_pack output for W[Cout][KH*KW*Cin] (OHWI)
 *   Y          device NHWC [B][P][Q][Cout] float32 (written, every element)
 * B = 0 is valid and enqueues nothing.
 * Errors: as cci_linear; CCI_ERR_SHAPE also when P or Q < 1.
 */
cci_status cci_conv2d(const void *X, cci_dtype dtype, int64_t B, int64_t H, int64_t W,
                      int64_t Cin, const void *values, const uint8_t *idx, int64_t Cout,
                      int KH, int KW, int stride_h, int stride_w, int pad_h, int pad_w, int G,
                      int K, float *Y, uint32_t *dev_status, cci_stream_t stream);

/* As cci_linear / cci_conv2d, with the kernel family chosen by `algo` and no
 * workspace (CCI_ALGO_DENSE_TC_WS returns CCI_ERR_WORKSPACE; AUTO does not pick it,
 * but does pick the fused tensor-core family, which needs none). */
cci_status cci_linear_ex(const void *X, cci_dtype dtype, int64_t N, int64_t Cin,
                         const void *values, const uint8_t *idx, int64_t Cout, int G, int K,
                         float *Y, uint32_t *dev_status, cci_algo algo, cci_stream_t stream);
cci_status cci_conv2d_ex(const void *X, cci_dtype dtype, int64_t B, int64_t H, int64_t W,
                         int64_t Cin, const void *values, const uint8_t *idx, int64_t Cout,
                         int KH, int KW, int stride_h, int stride_w, int pad_h, int pad_w,
                         int G, int K, float *Y, uint32_t *dev_status, cci_algo algo,
                         cci_stream_t stream);

/*
 * cci_workspace_size -- bytes of device workspace that cci_linear_ws /
 * cci_conv2d_ws need for this kernel family and layer (R = Cin for a product,
 * Cin*KH*KW for a convolution): for CCI_ALGO_DENSE_TC_WS Cout*R*2 (bf16) or
 * Cout*(R*4 + ceil(R/32)*128) (fp32: Cout*R*8 when R % 32 == 0), 0 for the
 * families that need none.  For CCI_ALGO_AUTO: the
 * bytes that let AUTO pick its fastest family (the dense tensor-core one).
 */
size_t cci_workspace_size(cci_algo algo, cci_dtype dtype, int64_t Cout, int64_t R);

/*
 * As cci_linear_ex / cci_conv2d_ex with a caller workspace (device, 16-byte
 * aligned, `workspace_bytes` long; NULL / 0 allowed for families that need
 * none).  The call overwrites the workspace (CCI_ALGO_AUTO may leave it as it
 * is); calls that overlap on the GPU must use different workspaces.
 * CCI_ALGO_AUTO uses the dense tensor-core family when the layer has one and the
 * workspace is large enough, else the CUDA-core family.
 */
cci_status cci_linear_ws(const void *X, cci_dtype dtype, int64_t N, int64_t Cin,
                         const void *values, const uint8_t *idx, int64_t Cout, int G, int K,
                         float *Y, uint32_t *dev_status, cci_algo algo, void *workspace,
                         size_t workspace_bytes, cci_stream_t stream);
cci_status cci_conv2d_ws(const void *X, cci_dtype dtype, int64_t B, int64_t H, int64_t W,
                         int64_t Cin, const void *values, const uint8_t *idx, int64_t Cout,
                         int KH, int KW, int stride_h, int stride_w, int pad_h, int pad_w,
                         int G, int K, float *Y, uint32_t *dev_status, cci_algo algo,
                         void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_linear_host -- the product H = W-hat x X of Alg. 2 (Sec. 3.2) with the
 * activations and the output in HOST memory: Y_host[N][Cout] (fp32) =
 * X_host[N][Cin] * Wd^T, Wd the dense matrix of the packed weights (which stay
 * on the device).  The columns are processed in chunks of `chunk_cols`; chunk c
 * is copied in on `copy_in_stream`, multiplied on `stream` (the dense
 * tensor-core family AUTO picks: the fused one from the packed weights, else the
 * workspace one, the weights decompressed once by the first chunk, or for an N
 * of few columns the one-launch product, which expands them in every chunk) and
 * copied out on `copy_out_stream`, so that the copies of neighbouring chunks
 * overlap the product.  The result equals cci_linear_ws with CCI_ALGO_AUTO and a
 * workspace on the same data bit for bit.
 *
 *   X_host, Y_host  host memory; page-locked (cudaHostAlloc / registered) for the
 *                   copies to overlap; pageable memory is correct but serialises
 *   values, idx     device, as cci_linear
 *   chunk_cols      columns per chunk, >= 1 (a multiple of 128 keeps the
 *                   product's tiles full)
 *   device_buffer   device, 256-byte aligned, at least
 *                   cci_linear_host_buffer_size(dtype, Cin, Cout, chunk_cols)
 *                   bytes: the workspace and two staging slots per direction;
 *                   overwritten
 *   copy_in_stream, copy_out_stream  may be NULL: that copy then runs on `stream`
 * Ordering: the copies start after the work enqueued on `stream` before the
 * call; `stream` waits for the last copy-out, so Y_host is complete once `stream`
 * has reached the end of the call's work (synchronise `stream` before reading
 * it).  Calls that overlap on the GPU must use different device buffers.
 * Errors: as cci_linear; CCI_ERR_SHAPE for chunk_cols < 1; CCI_ERR_UNSUPPORTED
 * for layers without the dense tensor-core kernel (it needs Cin % 4 == 0 for
 * fp32, % 8 for bf16, and G in {4, 8, 16, 32} with K <= G/2); CCI_ERR_WORKSPACE for a missing,
 * short or misaligned device buffer; CCI_ERR_CUDA if an event, copy or launch
 * fails (chunks already enqueued still complete on the streams).
 */
size_t cci_linear_host_buffer_size(cci_dtype dtype, int64_t Cin, int64_t Cout, int64_t chunk_cols);
cci_status cci_linear_host(const void *X_host, cci_dtype dtype, int64_t N, int64_t Cin,
                           const void *values, const uint8_t *idx, int64_t Cout, int G, int K,
                           float *Y_host, int64_t chunk_cols, void *device_buffer,
                           size_t device_buffer_bytes, uint32_t *dev_status, cci_stream_t stream,
                           cci_stream_t copy_in_stream, cci_stream_t copy_out_stream);

/*
 * cci_td_mask -- one step of the improved targeted dropout used to train CCI
 * layers (Sec. 5.1).  Per group of G output channels at one input index r the K
 * weights of largest |w| (those cci_pack keeps: same ranking, ties to the lower
 * index) are protected; each other weight is a pruning candidate and is dropped
 * for this training pass when its uniform draw is below `rate`:
 *   W_out[co][r] = 0 if (co is a candidate and uniforms[co][r] < rate) else W[co][r]
 *   mask[co][r]  = 1 if W_out keeps the weight, else 0      (mask may be NULL)
 * The paper starts the candidate drop rate at 0.5 and raises it toward 1 during
 * training (rate is the caller's schedule).  The random numbers are an input:
 * uniforms[Cout][R] fp32 in [0, 1), device.  W, W_out: device [Cout][R] of dtype
 * (W_out may not alias W); mask: device uint8 [Cout][R].  rate outside [0, 1]
 * or NaN: CCI_ERR_VALUE; NaN weights are reported in dev_status as for cci_pack;
 * other argument errors as for cci_pack.
 */
cci_status cci_td_mask(const void *W, cci_dtype dtype, int64_t Cout, int64_t R, int G, int K, float rate,
                       const float *uniforms, void *W_out, uint8_t *mask, uint32_t *dev_status,
                       cci_stream_t stream);

/*
 * cci_td_drop_rate -- the candidate drop rate of the targeted-dropout schedule
 * (Sec. 5.1) at training step `step`: the paper fixes only the end points (start
 * at 50 %, end toward 100 %); this library ramps linearly from `start` to `end`
 * over `ramp_steps` steps and holds `end` afterwards (ramp_steps <= 0: `end` at
 * once; negative steps count as 0).  Host function, no device work.
 */
float cci_td_drop_rate(int64_t step, int64_t ramp_steps, float start, float end);

/*
 * Balanced sparsity (Sec. 3.4), the format the paper compares CCI with: groups
 * run along the INPUT dimension.  Per output channel co and group of G
 * consecutive inputs r in [g*G, g*G + G) (R % G == 0), K weights are kept.
 *
 * cci_bbs_pack -- values[Cout][R/G][K] (dtype) and idx[Cout][R/G][K] (uint8,
 * offsets inside the group): the K of largest |w| per group, ties to the lower
 * index, in increasing index (the selection rule of cci_pack).  Errors as for
 * cci_pack; R % G != 0 is CCI_ERR_GROUP.
 *
 * cci_bbs_linear -- Y[N][Cout] fp32 = sum over groups and slots of
 * values[co][g][k] * X[n][g*G + idx[co][g][k]] (the gather form of the product).
 * algo CCI_ALGO_DENSE_TC_WS: decompression into the workspace and the tensor-core
 * product of the CCI path (Cin % 8 bf16 / % 4 fp32, Cout % 4, 16-byte aligned X,
 * Y and workspace of cci_workspace_size(CCI_ALGO_DENSE_TC_WS, dtype, Cout, Cin)
 * bytes); CCI_ALGO_GENERIC: the CUDA-core gather kernel (32 % G == 0); AUTO: the
 * first when the layer and workspace allow, else the second; other families:
 * CCI_ERR_UNSUPPORTED.  Index sets must be strictly increasing and < G
 * (CCI_ERR_INDEX in dev_status).  Everything else as for cci_linear_ws.
 */
cci_status cci_bbs_pack(const void *W, cci_dtype dtype, int64_t Cout, int64_t R, int G, int K, void *values,
                        uint8_t *idx, uint32_t *dev_status, cci_stream_t stream);
cci_status cci_bbs_linear(const void *X, cci_dtype dtype, int64_t N, int64_t Cin, const void *values,
                          const uint8_t *idx, int64_t Cout, int G, int K, float *Y, uint32_t *dev_status,
                          cci_algo algo, void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_pack_stats -- the allocation error of packing W (Sec. 4, Eq. 1, measured):
 * adds to counts[0] the number of nonzero weights of W[Cout][R] and to counts[1]
 * the number of them that cci_pack with (G, K) cannot keep (per group of G
 * output channels at one input index, the nonzeros beyond K).  counts[1] /
 * counts[0] estimates Eq. 1's P_d when the zeros of W are independent with
 * probability Ps and K = G*(1 - Ps).  A weight is nonzero when its magnitude
 * bits are (-0 counts as zero).  W: device, row-major, dtype bf16 or fp32;
 * counts: device, two 8-byte-aligned unsigned 64-bit counters the caller zeroes
 * and reads after a stream sync.  Argument errors as for cci_pack.
 */
cci_status cci_pack_stats(const void *W, cci_dtype dtype, int64_t Cout, int64_t R, int G, int K,
                          unsigned long long *counts, cci_stream_t stream);

/*
 * cci_linear_fused / cci_conv2d_fused -- the product / convolution of
 * cci_linear_ws / cci_conv2d_ws on a tensor-core family (the fused one where AUTO
 * would pick it or no workspace is given, else CCI_ALGO_DENSE_TC_WS; products of few
 * columns in one launch, where AUTO runs it), followed by the usual output stage of
 * a CNN layer, applied in the kernel's epilogue to each fp32 accumulator y[n][co]
 * (the sum of Alg. 2, Sec. 3.2):
 *   y += bias[co]          when bias != NULL (fp32, Cout entries, 16-byte aligned);
 *   y = max(y, 0)          when relu != 0;
 *   Y[n][co] = y           as fp32 (out_dtype CCI_F32) or rounded to the nearest
 *                          bf16, ties to even (out_dtype CCI_BF16; needs Cout % 8 == 0).
 * The paper defines only the product; bias, ReLU and the bf16 output are the
 * surrounding network's, fused here so that a layer's output is written once at
 * the width the next layer reads.  X and Y must be 16-byte aligned and, for
 * layers without the fused family, the workspace as for CCI_ALGO_DENSE_TC_WS
 * (else CCI_ERR_ALIGN / CCI_ERR_WORKSPACE; the workspace may be NULL otherwise);
 * layers without that family return CCI_ERR_UNSUPPORTED.  Y is [N][Cout] or NHWC
 * [B][P][Q][Cout] of out_dtype; everything else as for cci_linear_ws /
 * cci_conv2d_ws.  NaN accumulators become 0 under the ReLU.
 */
cci_status cci_linear_fused(const void *X, cci_dtype dtype, int64_t N, int64_t Cin,
                            const void *values, const uint8_t *idx, int64_t Cout, int G, int K,
                            const float *bias, int relu, cci_dtype out_dtype, void *Y,
                            uint32_t *dev_status, void *workspace, size_t workspace_bytes,
                            cci_stream_t stream);
cci_status cci_conv2d_fused(const void *X, cci_dtype dtype, int64_t B, int64_t H, int64_t W,
                            int64_t Cin, const void *values, const uint8_t *idx, int64_t Cout,
                            int KH, int KW, int stride_h, int stride_w, int pad_h, int pad_w,
                            int G, int K, const float *bias, int relu, cci_dtype out_dtype,
                            void *Y, uint32_t *dev_status, void *workspace,
                            size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_dense_linear_tc / cci_dense_conv2d_tc -- the tensor-core GEMM of
 * CCI_ALGO_DENSE_TC_WS run on a DENSE weight matrix that the caller provides,
 * with no decompression: Y = X * Wd^T (a convolution: the implicit product of
 * cci_conv2d with Wd in OHWI order).  This is the reference line that isolates
 * what the sparsity buys on this hardware: Sec. 3.2 argues that CCI cuts the
 * work of the product by G/K; timing the same kernel on the unpruned weights
 * shows how much of that a dense tensor-core product keeps.
 *
 *   Wd   device, 16-byte aligned, in the workspace layout of the dense family
 *        (CCI_ALGO_DENSE_TC_WS): bf16 dense [Cout][R]; fp32 the two operand
 *        planes, as cci_dense_planes writes them
 *   X, Y as cci_linear / cci_conv2d, 16-byte aligned; Cin % 8 == 0 (bf16) or
 *        % 4 == 0 (fp32); Cout % 4 == 0
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE, CCI_ERR_DTYPE, CCI_ERR_ALIGN,
 *         CCI_ERR_UNSUPPORTED (shapes the dense kernel lacks), CCI_ERR_CUDA.
 */
cci_status cci_dense_linear_tc(const void *X, cci_dtype dtype, int64_t N, int64_t Cin, const void *Wd,
                               int64_t Cout, float *Y, uint32_t *dev_status, cci_stream_t stream);
cci_status cci_dense_conv2d_tc(const void *X, cci_dtype dtype, int64_t B, int64_t H, int64_t W,
                               int64_t Cin, const void *Wd, int64_t Cout, int KH, int KW,
                               int stride_h, int stride_w, int pad_h, int pad_w, float *Y,
                               uint32_t *dev_status, cci_stream_t stream);

/*
 * cci_dense_planes -- writes a dense weight matrix W[Cout][R] (device, 16-byte
 * aligned, OHWI order for a convolution) in the workspace layout that
 * cci_dense_linear_tc / cci_dense_conv2d_tc read: bf16 copied as is; fp32 split
 * into the two operand planes of CCI_ALGO_DENSE_TC_WS (hi the nearest tf32 value
 * of w, lo = w - hi).  Wd: device, 16-byte aligned, bytes >=
 * cci_workspace_size(CCI_ALGO_DENSE_TC_WS, dtype, Cout, R).  Asynchronous on
 * stream.  Errors: CCI_ERR_DTYPE, CCI_ERR_SHAPE, CCI_ERR_NULL, CCI_ERR_WORKSPACE
 * (bytes too small), CCI_ERR_ALIGN (pointers, or R % 4 (fp32) / % 8 (bf16)),
 * CCI_ERR_CUDA.
 */
cci_status cci_dense_planes(const void *W, cci_dtype dtype, int64_t Cout, int64_t R, void *Wd, size_t bytes,
                            cci_stream_t stream);

/* Largest dense-weight size (Cout*R*2 bytes) that cci_linear_dense_tc_static accepts. */
#define CCI_STATIC_WORKSPACE_BYTES (16u * 1024u * 1024u)

/*
 * cci_linear_dense_tc_static -- the product of cci_linear_ws with
 * CCI_ALGO_DENSE_TC_WS, for callers that cannot allocate device memory
 * themselves: for example a plug-in called by a host framework that owns all
 * device memory and hands it no allocator, or a latency-bound serving loop that
 * forbids allocations after start-up.  Such a caller still passes X, the packed
 * weights and Y, but no workspace: the dense weights are decompressed into a
 * scratch array that lives in the library itself (a static device array of
 * CCI_STATIC_WORKSPACE_BYTES, held by every GPU that loads the library until the
 * process exits).  This entry point calls no allocation routine.  (The paper
 * has no counterpart: this is a deployment convenience of this library.)
 *
 *   arguments  as cci_linear (bf16 only, Cin % 8 == 0, 16-byte aligned X and Y)
 * Rules:
 *   - Cout*Cin*2 > CCI_STATIC_WORKSPACE_BYTES is rejected with CCI_ERR_WORKSPACE;
 *   - the first call on a device looks up the array's device address on that
 *     device (the device current at the call); make that first call before any
 *     stream capture.  The address is cached for the life of the process: after
 *     cudaDeviceReset() on that device the cached address is stale, so do not
 *     call this entry point again on a device that was reset;
 *   - every call shares the one array per device and leaves it holding the last
 *     call's dense weights; each call rewrites the part it reads, so nothing
 *     needs clearing, but calls that overlap on the GPU (other streams, other
 *     threads) race on the array and must be serialised by the caller.
 * Errors: as cci_linear; CCI_ERR_UNSUPPORTED for shapes the dense kernel lacks;
 *         CCI_ERR_CUDA if the address lookup fails.
 */
cci_status cci_linear_dense_tc_static(const void *X, cci_dtype dtype, int64_t N, int64_t Cin,
                                      const void *values, const uint8_t *idx, int64_t Cout, int G,
                                      int K, float *Y, uint32_t *dev_status, cci_stream_t stream);

/*
 * ---- The layers around a pruned projection: norms, the gated block, what a head answers ----
 * (The paper has no counterpart: a language model's feed-forward sub-layer needs them
 * beside its projections.)  Row strides ld* are in elements, at least the row's length.
 */

/*
 * cci_layer_norm -- y[n][c] = (x[n][c] - mean[n]) * rstd[n] * weight[c] + bias[c] for
 * N rows of D, mean the row's mean, rstd = 1 / sqrt(var + eps) with var the mean
 * square of the differences from it (all sums fp32; y rounded once).
 *
 *   x          device, N rows of D of dtype, row stride ldx
 *   weight, bias device fp32 [D] or NULL (1 and 0)
 *   y          device [N][D] of dtype (written)
 *   mean, rstd device fp32 [N] (written; the backward pass reads them)
 * N = 0 is valid and enqueues nothing.  eps must be >= 0 (CCI_ERR_VALUE; NaN too).
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (D < 1, ldx < D), CCI_ERR_DTYPE,
 *         CCI_ERR_ALIGN, CCI_ERR_VALUE, CCI_ERR_CUDA.
 */
cci_status cci_layer_norm(const void *x, cci_dtype dtype, int64_t N, int64_t D, int64_t ldx, const float *weight,
                          const float *bias, float eps, void *y, float *mean, float *rstd, cci_stream_t stream);

/*
 * cci_layer_norm_backward -- the gradients of cci_layer_norm, with g = dy * weight and
 * xh = (x - mean) * rstd:
 *   dx      = rstd * (g - mean over c of g - xh * mean over c of g * xh)
 *   dweight[c] = sum over n of dy * xh,  dbias[c] = sum over n of dy
 * The sums over n are added in a fixed order: the same call gives the same bits.
 *
 *   dy         device, N rows of D of dtype, row stride lddy;  x as in the forward call
 *   mean, rstd as cci_layer_norm wrote them
 *   weight     as in the forward call (NULL: 1)
 *   dx         device [N][D] of dtype (written)
 *   dweight, dbias device fp32 [D] (written; zeros for N = 0), each may be NULL
 *   workspace  device, 16-byte aligned, cci_layer_norm_workspace_size(N, D) bytes (which
 *              depends on the current device's number of SMs); overwritten
 * Errors: as cci_layer_norm; CCI_ERR_WORKSPACE.
 * cci_layer_norm_backward_ex takes a status word too (CCI_ERR_TIMEOUT: the kernel's copies of
 * the rows are waited for with a limit).  With or without one, after an expired wait the rows
 * of dx and the columns of dweight and dbias that it touches are NaN.
 */
size_t cci_layer_norm_workspace_size(int64_t N, int64_t D);
cci_status cci_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, cci_dtype dtype,
                                   int64_t N, int64_t D, const float *mean, const float *rstd, const float *weight,
                                   void *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                                   cci_stream_t stream);
cci_status cci_layer_norm_backward_ex(const void *dy, int64_t lddy, const void *x, int64_t ldx, cci_dtype dtype,
                                      int64_t N, int64_t D, const float *mean, const float *rstd, const float *weight,
                                      void *dx, float *dweight, float *dbias, uint32_t *dev_status, void *workspace,
                                      size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_rms_norm -- with s = x + residual (x alone without one), for N rows of D:
 *   h[n][c] = s,  rstd[n] = 1 / sqrt(mean over c of s^2 + eps),  y[n][c] = s * rstd[n] * weight[c]
 * sums in fp32, y and h each rounded once (y from the unrounded s).
 *
 *   x          device, N rows of D of dtype, row stride ldx
 *   residual   the same with row stride ldr, or NULL
 *   weight     device fp32 [D] or NULL (1)
 *   y          device [N][D] of dtype (written)
 *   h          device [N][D] of dtype (written where there is a residual) or NULL; may be the residual or x
 *              themselves, packed
 *   rstd       device fp32 [N] (written; the backward pass reads it) or NULL
 * N = 0 is valid and enqueues nothing.  eps must be >= 0 (CCI_ERR_VALUE; NaN too).
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (D < 1 or >= 2^30, N >= 2^31, ldx or ldr < D, h in the place of rows that are
 *         not packed), CCI_ERR_DTYPE, CCI_ERR_ALIGN, CCI_ERR_VALUE, CCI_ERR_CUDA.
 */
cci_status cci_rms_norm(const void *x, cci_dtype dtype, int64_t N, int64_t D, int64_t ldx, const void *residual,
                        int64_t ldr, const float *weight, float eps, void *y, void *h, float *rstd,
                        cci_stream_t stream);

/*
 * cci_rms_norm_fp8 -- cci_rms_norm with y in 8 bits (e4m3) for a product in 8 bits:
 *   scale = max(max |y| / 448, 2^-126),  q = e4m3(y / scale), to the nearest, ties to even
 * with a scale for each row (group 0) or for each 128 columns of it (group 128; the last of a row may cover
 * fewer).  y is not rounded before.  NaN in y makes the scale and its columns NaN.
 *
 *   q          device [N][D], one byte each (written)
 *   scales     device fp32 [N] or [N][ceil(D / 128)] (written)
 * D is a multiple of 8 (CCI_ERR_UNSUPPORTED); rows of x and residual, h, weight and q are on 16 bytes.
 * Errors: as cci_rms_norm; CCI_ERR_GROUP (group is neither 0 nor 128).
 */
cci_status cci_rms_norm_fp8(const void *x, cci_dtype dtype, int64_t N, int64_t D, int64_t ldx, const void *residual,
                            int64_t ldr, const float *weight, float eps, int group, void *q, float *scales, void *h,
                            float *rstd, cci_stream_t stream);

/*
 * cci_rms_norm_backward -- the gradients of cci_rms_norm, with g = dy * weight and xh = h * rstd:
 *   dx = rstd * (g - xh * mean over c of g * xh) + dh
 *   dweight[c] = sum over n of dy * xh
 * dx is the gradient of x and of the residual alike; dh is the gradient that h has besides, from where
 * it is added again.  Sums over n are added in a fixed order: the same call gives the same bits.
 *
 *   dy         device, N rows of D of dtype, row stride lddy
 *   h          as the forward call wrote it (x where it had no residual), row stride ldh
 *   dh         the same with row stride lddh, or NULL (0)
 *   rstd, weight as in the forward call
 *   dx         device [N][D] of dtype (written)
 *   dweight    device fp32 [D] (written; zeros for N = 0) or NULL
 *   workspace  device, 16-byte aligned, cci_rms_norm_workspace_size(N, D) bytes (which depends on the
 *              current device's number of SMs); overwritten
 * Errors: as cci_rms_norm; CCI_ERR_WORKSPACE.
 */
size_t cci_rms_norm_workspace_size(int64_t N, int64_t D);
cci_status cci_rms_norm_backward(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dh, int64_t lddh,
                                 cci_dtype dtype, int64_t N, int64_t D, const float *rstd, const float *weight, void *dx,
                                 float *dweight, void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_token_logprobs -- for N rows of V logits x, each with a token t:
 *   logp[n]    = x[t] - log sum exp(x)
 *   entropy[n] = - sum over v of p_v log p_v, p the row's softmax
 *   top_logp[n][j], top_idx[n][j]   the `top` largest logits' log probabilities and
 *                indices, largest first, ties by increasing index
 *   stats[n]   = (m, log sum exp(x - m)), m the row's maximum (the gradient needs them)
 * Masked logits (-inf) have probability 0 and add nothing to the entropy.  A row of -inf
 * alone gives logp -inf, entropy 0, top_logp -inf and stats (-inf, 0).  NaN or +inf in a
 * row makes its logp and entropy NaN; NaN logits are never listed (places that no number
 * fills: index -1, NaN).  A token equal to `ignore_index` gives logp 0; any other token
 * outside [0, V) sets CCI_ERR_INDEX in dev_status and gives NaN.
 *
 *   logits     device, N rows of V of dtype, row stride ldx
 *   tokens     device int64 [N]
 *   logp, entropy device fp32 [N]; stats fp32 [N][2] (written)
 *   top        0 .. min(V, CCI_MAX_TOP); top_logp fp32, top_idx int32 [N][top] (written;
 *              may be NULL for top = 0)
 *   dev_status device uint32 or NULL
 * N = 0 is valid and enqueues nothing.
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (V < 1 or > 2^24, N >= 2^31, ldx < V, top out of
 *         range), CCI_ERR_DTYPE, CCI_ERR_ALIGN, CCI_ERR_CUDA.
 */
#define CCI_MAX_TOP 32
cci_status cci_token_logprobs(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                              const int64_t *tokens, int64_t ignore_index, int top, float *logp, float *entropy,
                              float *stats, float *top_logp, int32_t *top_idx, uint32_t *dev_status,
                              cci_stream_t stream);

/*
 * cci_token_logprobs_backward -- the gradient of logp and entropy to the logits:
 *   dlogits[n][v] = dlogp[n] * (1[v = t] - p_v) - dentropy[n] * p_v * (log p_v + entropy[n])
 * Rows of -inf alone, and for the first term rows whose token is `ignore_index`, get 0.
 *
 *   logits, tokens as in the forward call; stats, entropy as it wrote them
 *   dlogp      device fp32 [N] or NULL (0; tokens may be NULL then)
 *   dentropy   device fp32 [N] or NULL (0; entropy may be NULL then)
 *   dlogits    device, N rows of V of dtype, row stride lddx (written; may be the logits
 *              themselves, with the same stride).  Rows at the same offset from a 16-byte boundary
 *              as the logits' rows are written in whole vectors
 *   dev_status as in the forward call: a token outside [0, V) counts as left out
 * Errors: as cci_token_logprobs; CCI_ERR_SHAPE also for lddx < V.
 */
cci_status cci_token_logprobs_backward(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                                       const float *stats, const int64_t *tokens, int64_t ignore_index,
                                       const float *dlogp, const float *entropy, const float *dentropy,
                                       void *dlogits, int64_t lddx, uint32_t *dev_status, cci_stream_t stream);

/*
 * cci_distillation_loss -- what a student's logits x are off a teacher's word on k tokens of each of N rows,
 * z = x / T and p = softmax(z) over all V:
 *   loss[n] = - sum over j of q_j log p[idx_j]                          (tail 0)
 *             with q = softmax over the listed of t_j / T
 *   loss[n] = - sum over j of q_j log p[idx_j] - q_rest log p_rest      (tail 1)
 *             with q_j = exp(t_j): t are the teacher's log probabilities, at temperature T already,
 *             q_rest = max(1 - sum q, 0) and p_rest = sum of p over what is not listed
 * the teacher's cross entropy against the student: its divergence and the teacher's own entropy, which has no
 * gradient.  The lists are those of cci_token_logprobs on the teacher's logits.  It is not multiplied
 * by T^2: the gradient's dloss is the place for that.
 *   stats[n] = (max z, log sum exp(z - max), log of that sum over what is not listed,
 *               tail: sum q, else: log sum exp(t_j / T));  where |max z| is 64 or more and its rounding loses
 *               something of max x, the first two are max x and the logarithm with its sign set; with a tail, where
 *               the third is -64 or less, the last two are the largest x of what is not listed, and the log of
 *               the sum of exp(z - its z) with its sign set
 * An index of -1 lists nothing, whatever its t; a row that lists nothing has loss 0 and no gradient,
 * whatever its logits (stats 0, 0, 0 where they have no sum).  t_j may
 * be -inf (q_j = 0, and listed).  A listed logit of -inf with q_j > 0 makes the loss inf.  Where no unlisted logit is
 * above -inf, the rest takes no part (q_rest counts as 0).  NaN or +inf in a row makes its loss NaN.  Any other
 * index outside [0, V), or one that a row lists twice, sets CCI_ERR_INDEX in dev_status and makes the row's loss, and
 * its gradient, NaN.
 *
 *   logits     device, N rows of V of dtype, row stride ldx
 *   top_idx    device int32 [N][k]; top_logp device fp32 [N][k]
 *   k          1 .. min(V, CCI_MAX_TEACHER)
 *   temperature T > 0, T and log2(e) / T finite
 *   loss       device fp32 [N]; stats device fp32 [N][4], 16-byte aligned (written)
 *   dev_status device uint32 or NULL
 *   workspace  device, 16-byte aligned, cci_distillation_workspace_size(N, V) bytes (0 for many rows, for few and
 *              for short ones; it depends on the current device's number of SMs); overwritten
 * N = 0 is valid and enqueues nothing.
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (V < 1 or > 2^24, N >= 2^28, N rows of V / 2048 blocks or more than 2^31, ldx < V,
 *         k out of range), CCI_ERR_DTYPE, CCI_ERR_VALUE (temperature), CCI_ERR_ALIGN, CCI_ERR_WORKSPACE, CCI_ERR_CUDA.
 */
#define CCI_MAX_TEACHER 128
size_t cci_distillation_workspace_size(int64_t N, int64_t V);
cci_status cci_distillation_loss(const void *logits, cci_dtype dtype, int64_t N, int64_t V, int64_t ldx,
                                 const int32_t *top_idx, const float *top_logp, int k, float temperature, int tail,
                                 float *loss, float *stats, uint32_t *dev_status, void *workspace,
                                 size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_distillation_loss_backward -- the gradient of cci_distillation_loss to the logits:
 *   dlogits[n][v] = dloss[n] / T * (Q p_v - q_v)            for the listed, Q = sum q + q_rest
 *                   dloss[n] / T * (Q p_v - q_rest r_v)     for others, r_v = p_v / p_rest (tail 0: Q p_v)
 * Rows of -inf alone, rows that list nothing, whatever their dloss, and rows whose dloss is 0 get 0.
 *
 *   dloss      device fp32 [N]; logits, top_idx, top_logp, k, temperature, tail as in the forward call
 *   stats      as it wrote them
 *   dlogits    device, N rows of V of dtype, row stride lddx (written; may be the logits themselves, with
 *              the same stride).  Rows at the same offset from a 16-byte boundary as the logits' are
 *              written in whole vectors
 * Errors: as cci_distillation_loss; CCI_ERR_SHAPE also for lddx < V, and in place with another stride.
 */
cci_status cci_distillation_loss_backward(const float *dloss, const void *logits, cci_dtype dtype, int64_t N, int64_t V,
                                          int64_t ldx, const int32_t *top_idx, const float *top_logp, int k,
                                          float temperature, int tail, const float *stats, void *dlogits, int64_t lddx,
                                          cci_stream_t stream);

/*
 * cci_gated_linear -- the gated feed-forward block's two projections, activation and
 * product in one kernel, for N tokens of D features and F hidden channels:
 *   g = X Wg^T,  u = X Wu^T,  H[n][f] = act(g[n][f]) * u[n][f]
 * with fp32 accumulators and one rounding, to the type of H.  bf16: products of the exact
 * values on the tensor cores.  fp32: every operand as three bf16 planes, the six products
 * of planes down to 2^-18 of the whole (what is left out is below 2^-25 |x||w| a term; an
 * infinite input gives NaN where its products of planes do).  Calls of up to 16 tokens may
 * stream the weights as they are (fp32: fused multiply-adds), with the sums in another order, so
 * a token's last bits may differ from those it has in a call of more tokens.  The activations
 * take the fast exponential and quotient, in fp32 too: act(g) is within n units of 2^-23 of
 * itself, n = 6 + 2.7 |g| for SiLU and sigmoid, 10 + g^2 for GELU at g < 0 (where the rounding of
 * g itself is worth g^2 / 2) and 10 above, 6 + 2.7 z for the tanh form with z = 1.6 |g + 0.045 g^3|;
 * values below 2^-100 may be 0.
 *
 *   X          device [N][D] of dtype
 *   Wg, Wu     device [F][D] of dtype (pruned weights: their dense form, as cci_td_mask
 *              writes it; or cci_gated_linear_packed)
 *   H          device [N][F] of dtype (written)
 *   g, u       device fp32 [N][F] (written, for cci_gated_linear_backward), or both NULL
 *   workspace  device, 16-byte aligned, cci_gated_workspace_size(CCI_GATED_FORWARD, ...)
 *              bytes (0 for bf16, which needs none); overwritten
 *   dev_status device uint32 or NULL (CCI_ERR_TIMEOUT)
 * D and F are multiples of 8; every matrix is 16-byte aligned.  N = 0 is valid and enqueues
 * nothing.
 * Errors: CCI_ERR_NULL (also one of g and u alone), CCI_ERR_SHAPE (N < 0, D or F < 1, sizes
 *         of 2^30 or more), CCI_ERR_UNSUPPORTED (D % 8, F % 8), CCI_ERR_DTYPE,
 *         CCI_ERR_VALUE (act is not a cci_activation), CCI_ERR_ALIGN, CCI_ERR_WORKSPACE,
 *         CCI_ERR_CUDA.
 */
typedef enum cci_activation {
    CCI_ACT_SILU = 0,      /* g / (1 + exp(-g)) */
    CCI_ACT_GELU = 1,      /* g * Phi(g), by the error function */
    CCI_ACT_GELU_TANH = 2, /* g / 2 * (1 + tanh(sqrt(2 / pi) * (g + 0.044715 g^3))) */
    CCI_ACT_RELU = 3,      /* max(g, 0); NaN stays */
    CCI_ACT_SIGMOID = 4    /* 1 / (1 + exp(-g)) */
} cci_activation;

typedef enum cci_gated_call {
    CCI_GATED_FORWARD = 0,
    CCI_GATED_PACKED = 1,
    CCI_GATED_BACKWARD = 2
} cci_gated_call;

/* bytes of workspace of a call (0: none needed, or invalid sizes); the backward pass' depend on the
 * current device's number of SMs */
size_t cci_gated_workspace_size(cci_gated_call call, cci_dtype dtype, int64_t N, int64_t D, int64_t F);

cci_status cci_gated_linear(const void *X, cci_dtype dtype, int64_t N, int64_t D, const void *Wg, const void *Wu,
                            int64_t F, cci_activation act, void *H, float *g, float *u, uint32_t *dev_status,
                            void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_gated_linear_packed -- cci_gated_linear with both weight matrices in the packed format
 * of cci_pack (Cout = F, R = D, the same G and K): any G and K of that format.  The
 * weights are expanded into the workspace (CCI_GATED_PACKED) and multiplied there; up to 16
 * tokens of bf16 read them packed where G is 4, 8, 16 or 32, K a power of two up to G / 2 and 8,
 * D * K a multiple of 16 and the indices are on 16 bytes.  Pruned positions take part as zeros either way
 * (an infinite x gives NaN).  An index set that is not strictly
 * increasing or has an index >= G sets CCI_ERR_INDEX in dev_status.
 * Errors: as cci_gated_linear; CCI_ERR_GROUP.
 */
cci_status cci_gated_linear_packed(const void *X, cci_dtype dtype, int64_t N, int64_t D, const void *gate_values,
                                   const uint8_t *gate_idx, const void *up_values, const uint8_t *up_idx, int64_t F,
                                   int G, int K, cci_activation act, void *H, uint32_t *dev_status, void *workspace,
                                   size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_gated_linear_backward -- the gradients of cci_gated_linear from that of H:
 *   dg = dH * u * act'(g),  du = dH * act(g)      (act' of ReLU at 0 is 0)
 *   dX = dg Wg + du Wu,  dWg = dg^T X,  dWu = du^T X
 * dg and du are rounded to bf16 for the products (fp32: split into planes, as every operand);
 * sums are fp32 in a fixed order, each gradient rounded once to dtype.
 *
 *   dH         device [N][F] of dtype;  X, Wg, Wu as in the forward call
 *   g, u       as the forward call wrote them
 *   dX         device [N][D] of dtype (written), or NULL
 *   dWg, dWu   device [F][D] of dtype (written; zeros for N = 0), or both NULL
 *   workspace  cci_gated_workspace_size(CCI_GATED_BACKWARD, ...) bytes
 * Errors: as cci_gated_linear.
 */
cci_status cci_gated_linear_backward(const void *dH, const void *X, cci_dtype dtype, int64_t N, int64_t D,
                                     const void *Wg, const void *Wu, int64_t F, cci_activation act, const float *g,
                                     const float *u, void *dX, void *dWg, void *dWu, uint32_t *dev_status,
                                     void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_linear_cross_entropy -- the loss of N tokens over a vocabulary of V straight from a head's inputs,
 * z = X W^T, without keeping the logits:
 *   loss[n]  = log sum over v of exp(z_v) - z_t,  t = targets[n]
 *   stats[n] = (m, log sum exp(z - m)), m the row's maximum (the gradient needs them)
 * with fp32 accumulators (bf16: products of the exact values; fp32: three bf16 planes of every
 * operand, as cci_gated_linear).  A target equal to `ignore_index` gives loss 0; any other target
 * outside [0, V) sets CCI_ERR_INDEX in dev_status and gives NaN.  NaN or +inf logits make their row's loss
 * NaN.
 *
 *   X          device [N][D] of dtype
 *   W          device [V][D] of dtype (pruned weights: their dense form, as cci_td_mask writes it)
 *   targets    device int64 [N]
 *   loss       device fp32 [N]; stats fp32 [N][2] (written)
 *   workspace  device, 16-byte aligned, cci_head_workspace_size(CCI_HEAD_FORWARD, ...) bytes;
 *              overwritten.  It depends on the current device's number of SMs
 *   dev_status device uint32 or NULL (CCI_ERR_INDEX, CCI_ERR_TIMEOUT)
 * D is a multiple of 8; X and W are 16-byte aligned.  V may be any size.  N = 0 is valid and enqueues
 * nothing.
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE (N < 0, D or V < 1, sizes of 2^30 or more),
 *         CCI_ERR_UNSUPPORTED (D % 8), CCI_ERR_DTYPE, CCI_ERR_ALIGN, CCI_ERR_WORKSPACE, CCI_ERR_CUDA.
 */
typedef enum cci_head_call {
    CCI_HEAD_FORWARD = 0,
    CCI_HEAD_BACKWARD = 1
} cci_head_call;

/* bytes of workspace of a call (0: none needed, or invalid sizes) */
size_t cci_head_workspace_size(cci_head_call call, cci_dtype dtype, int64_t N, int64_t D, int64_t V);

cci_status cci_linear_cross_entropy(const void *X, cci_dtype dtype, int64_t N, int64_t D, const void *W, int64_t V,
                                    const int64_t *targets, int64_t ignore_index, float *loss, float *stats,
                                    uint32_t *dev_status, void *workspace, size_t workspace_bytes,
                                    cci_stream_t stream);

/*
 * cci_linear_cross_entropy_backward -- the gradients of cci_linear_cross_entropy from that of the loss:
 *   P[n][v] = dloss[n] * (softmax(z)[v] - 1[v = t]),  dX = P W,  dW = P^T X
 * in pieces of the vocabulary, whose logits are computed again.  P is rounded to bf16 for the products (fp32:
 * split into planes); sums are fp32 in a fixed order, each gradient rounded once to dtype.  Rows whose
 * target is `ignore_index`, or outside [0, V) (which sets CCI_ERR_INDEX), or whose dloss is 0 have P = 0 and
 * take no part, whatever their X holds.  Up to 32 tokens of fp32 take the sums in another order than
 * more do.
 *
 *   dloss      device fp32 [N];  X, W, targets as in the forward call
 *   stats      as the forward call wrote them
 *   dX         device [N][D] of dtype (written), or NULL
 *   dW         device [V][D] of dtype (written; zeros for N = 0), or NULL
 *   workspace  cci_head_workspace_size(CCI_HEAD_BACKWARD, ...) bytes: X once more and about 256 MB for a piece, more
 *              only where a piece of 2048 entries, or of 128 times 128 / N for each SM, takes more
 * Errors: as cci_linear_cross_entropy.
 */
cci_status cci_linear_cross_entropy_backward(const float *dloss, const void *X, cci_dtype dtype, int64_t N, int64_t D,
                                             const void *W, int64_t V, const int64_t *targets, int64_t ignore_index,
                                             const float *stats, void *dX, void *dW, uint32_t *dev_status,
                                             void *workspace, size_t workspace_bytes, cci_stream_t stream);

/*
 * cci_kernel_name -- the name of the kernel family that cci_linear_ws /
 * cci_conv2d_ws would run for a layer with these sizes (R = Cin for a product,
 * Cin*KH*KW for a convolution, taken to have strides <= 2) when every pointer is
 * 16-byte aligned and, for CCI_ALGO_AUTO, the workspace is the one
 * cci_workspace_size(CCI_ALGO_AUTO) asks for: a static string, "" when the call
 * would be rejected.  The number of columns is not asked: for CCI_ALGO_AUTO the
 * name is that of the family which runs for many columns.  No device work; used to
 * label results.
 */
const char *cci_kernel_name(cci_dtype dtype, int64_t Cin, int64_t R, int64_t Cout, int G, int K,
                            cci_algo algo);

/* Human-readable text of a status code (static string). */
const char *cci_status_string(cci_status status);

/* The lowest-numbered error among the bits set in a device status word, or
 * CCI_OK when none is set. */
cci_status cci_decode_device_status(uint32_t word);

/* Library version, major*10000 + minor*100 + patch. */
int cci_version(void);

/*
 * cci_fma_probe -- measurement helper, not part of the method: enqueue one
 * kernel of `blocks` x `threads` threads, each running `iters` iterations of 16
 * independent packed fp32 FMAs (fma.rn.f32x2, 2 FMAs each), and write one float
 * per thread to `out` (device, blocks*threads floats) so the work is kept.
 * Flops performed = blocks * threads * iters * 64.  Time it with CUDA events to
 * measure the CUDA-core FMA throughput.
 * Errors: CCI_ERR_NULL, CCI_ERR_SHAPE, CCI_ERR_CUDA.
 */
cci_status cci_fma_probe(float *out, int blocks, int threads, int iters, cci_stream_t stream);

/*
 * cci_wait_probe -- diagnostic of the bounded waits inside the tensor-core
 * kernels (a safety mechanism of this library; the paper has no counterpart).
 * One thread initialises an mbarrier that expects one arrival, arrives on it if
 * `arrive` is nonzero, and waits for the barrier's phase exactly as the kernels
 * wait for their copies and MMAs.  With the arrival the wait returns at once and
 * nothing is reported.  Without it nothing can complete the phase: the wait
 * gives up after 2^31 SM clock cycles (about one second), ORs bit
 * (1u << CCI_ERR_TIMEOUT) into *dev_status and the kernel returns, leaving the
 * context usable.
 *   dev_status  device uint32, required
 * Errors: CCI_ERR_NULL, CCI_ERR_CUDA.
 */
cci_status cci_wait_probe(uint32_t *dev_status, int arrive, cci_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CCI_H_ */
