/*
 * qmm.h -- C ABI of the MI355X (gfx950) quantized-matmul library.
 *
 * The library implements the hot path of "A Metric Driven Approach to Mixed
 * Precision Training" (arXiv 2408.02897): for one matrix multiply,
 *   qmm_scale     step size delta = max|X| / qmax per scale group   (Eq. 1, right half)
 *   qmm_quantize  codes = round(X / delta) onto INT8 / E4M3 / E5M2  (Eq. 1, left half;
 *                 Methodology bullets on saturation, underflow and rounding)
 *   qmm_gemm      8-bit x 8-bit product in a wide accumulator, then
 *                 descale by deltaL * deltaR                        (Methodology, scaling bullet)
 *   qmm_metric    error sums of the result against the high-precision
 *                 product: noise-to-signal ratio, Eq. 2, Eq. 3      (Results, Eq. 2 and Eq. 3)
 * and, for the products of a transformer's feed-forward block, what stands around them
 * (extensions: the paper quantizes the products, it does not say what feeds them):
 *   qmm_rmsnorm_quantize   residual addition, root-mean-square norm, steps 1 and 2 in one pass
 *   qmm_gemm_gated         both projections, activation and product in one kernel
 *   qmm_gated_backward, qmm_rmsnorm_backward   their gradients, the first one quantized
 * and, for layers whose products have a step size for every block of 128 elements (an extension: a finer granularity than the paper's),
 *   qmm_quantize_blocks    steps 1 and 2 block by block, along one axis or along both in one pass
 *   qmm_gemm_blocks        steps 3 and 4 of two such operands
 *   qmm_layernorm_quantize, qmm_layernorm_backward   what a layer has behind a block of products: dropout, residual addition, layer norm
 *                          and its codes, and their gradients
 *   qmm_dropout            dropout alone, from a counter-based generator
 *
 * General rules
 *  - Every pointer named "device" is GPU memory owned by the caller; the
 *    library allocates nothing and frees nothing.  What it keeps between calls:
 *    per GPU, the addresses of arrays of its own device image (the scratch
 *    of qmm_scale_static, and a ring of arrival counters that the single-launch
 *    reductions of qmm_scale / qmm_scale_multi use where a board does not serve
 *    and leave at zero; a call takes the next slot of the ring, 1024 calls would
 *    have to be in flight for two of them to meet on one), two rings of boards
 *    through which the workgroups of one launch exchange values (calls outside
 *    stream capture; a board shared by two calls in flight costs time, never a
 *    result), and which GPUs have had the kernels' LDS limit set.
 *    Descriptor structs (qmm_tensor, qmm_operand, qmm_granularity) are host memory
 *    and are read before the call returns.
 *  - Calls validate their arguments on the host, enqueue kernels on `stream`
 *    (a hipStream_t passed as void*; NULL = the default stream) and return
 *    without synchronising.  Results stay on the device.
 *  - Argument errors are reported before anything is launched and leave the
 *    outputs untouched.  A launch failure returns QMM_ERR_LAUNCH.
 *  - NaN / inf inputs and all-zero groups are not errors; their results are
 *    defined below.
 *  - Arithmetic is IEEE binary32 unless stated, round-to-nearest-even,
 *    subnormals kept.
 *
 * Scale groups.  A tensor is a batch of matrices [batch][rows][cols].  Matrix b
 * belongs to batch group g = (b / batch_inner) % batch_groups (batch_groups = 1:
 * one group for the whole batch, "tensor"/"channel" level; batch_groups = H with
 * the batch laid out [example][head]: one group per head, shared by the
 * examples -- the fine-grained level of the Results section, which adds batch
 * dimensions other than the examples' to the scale's index).  With the batch
 * laid out [outer][mid][inner], batch_groups = mid and batch_inner = inner give
 * one group per index of the middle dimensions, shared over outer and inner:
 * any run of neighbouring batch dimensions can carry the scales.  With
 * per_channel = 1 every index c of the non-contracting axis has its own step
 * size, shared by the matrices of the group: delta[g * C + c], C = extent of
 * the non-contracting axis.  With per_channel = 0: delta[g].
 */
#ifndef QMM_H
#define QMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    QMM_OK = 0,
    QMM_ERR_NULL = 1,        /* a required pointer is NULL                        */
    QMM_ERR_SHAPE = 2,       /* negative extent, stride smaller than extent, ...  */
    QMM_ERR_ENUM = 3,        /* unknown format / dtype / rounding / axis value    */
    QMM_ERR_ALIGN = 4,       /* pointer or extent alignment rule violated         */
    QMM_ERR_UNSUPPORTED = 5, /* valid request this build does not implement       */
    QMM_ERR_WORKSPACE = 6,   /* workspace missing or too small                    */
    QMM_ERR_LAUNCH = 7,      /* the HIP runtime refused a launch                  */
    QMM_ERR_LIMIT = 8        /* input larger than a fixed, documented capacity    */
} qmm_status;

/* 8-bit formats of the paper, plus the un-quantized pass-through used for the
 * high-precision reference product.  Largest magnitudes: 127, 448, 57344. */
typedef enum { QMM_FMT_INT8 = 0, QMM_FMT_E4M3 = 1, QMM_FMT_E5M2 = 2, QMM_FMT_BF16 = 3 } qmm_format;
typedef enum { QMM_DT_BF16 = 0, QMM_DT_F32 = 1 } qmm_dtype;
typedef enum { QMM_ROUND_RTNE = 0, QMM_ROUND_STOCHASTIC = 1 } qmm_round;

/* A batch of row-major matrices in device memory.  Element (b, r, c) is at
 * data[b*batch_stride + r*row_stride + c] (strides in elements, columns are
 * contiguous).  contract_axis names the axis the matrix multiply sums over:
 * 1 = columns (an [M][K] operand), 0 = rows (a [K][M] operand, e.g. the
 * activations and the upstream gradient in a weight-gradient product). */
typedef struct {
    const void* data;        /* device */
    int32_t dtype;           /* qmm_dtype */
    int32_t contract_axis;   /* 0 or 1 */
    int64_t batch, rows, cols;
    int64_t batch_stride, row_stride;
} qmm_tensor;

typedef struct {
    int32_t per_channel;     /* 0: one step size per batch group; 1: one per non-contracting index */
    int32_t batch_inner;     /* >= 0; 0 means 1: consecutive matrices that share a group            */
    int64_t batch_groups;    /* >= 1: group = (b / batch_inner) % batch_groups                      */
} qmm_granularity;

/* Number of step sizes qmm_scale writes / qmm_quantize reads for this tensor. */
int64_t qmm_num_scales(const qmm_tensor* x, const qmm_granularity* g);

/*
 * Step 1 -- step size (Eq. 1: delta = max|X| / (2^(n-1)-1); for FP8 the
 * denominator is the format maximum, last Methodology bullet).
 *   delta_out  device, qmm_num_scales() floats.
 *   workspace  device scratch of at least qmm_scale_workspace_size() bytes,
 *              16-byte aligned; contents on entry are irrelevant.
 * Defined results: the maximum is taken over magnitude bit patterns, so an
 * inf or NaN element makes its group's delta inf / NaN; an all-zero (or
 * empty) group gets delta = 1; a quotient below 2^-126 is raised to 2^-126.
 * fmt must be one of the three 8-bit formats.  batch above 65535: QMM_ERR_UNSUPPORTED.
 * Dense aligned tensors with one step size per matrix or group of matrices take one launch, under stream capture two below 2^24
 * elements and with several groups, as all others do.
 */
size_t qmm_scale_workspace_size(const qmm_tensor* x, const qmm_granularity* g);
qmm_status qmm_scale(const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g,
                     float* delta_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_scale_static -- qmm_scale for callers that cannot allocate device memory or hand over a workspace (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc).  Same arguments, results and errors as
 * qmm_scale without the workspace: the partial maxima go to a scratch array of QMM_SCALE_STATIC_BYTES that is part
 * of the library's device image (one copy per GPU, held until the process ends; its address is looked up once per
 * device on the first call there).  The call allocates and frees nothing.
 *   Limit: qmm_scale_workspace_size(x, g) must not exceed QMM_SCALE_STATIC_BYTES, else QMM_ERR_LIMIT (checked on
 *   the host before anything is launched; 1 MiB covers one step size per tensor for any size, and e.g. one step
 *   size per row for 262144 rows).
 *   Nothing in the array has to be cleared between calls (every word read by the second kernel has been written by
 *   the first of the same call), but all calls on one GPU share it: calls that may overlap on one GPU -- different
 *   streams, or graphs replayed concurrently -- race on it and must be serialised by the caller.
 */
#define QMM_SCALE_STATIC_BYTES (1u << 20)
qmm_status qmm_scale_static(const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g,
                            float* delta_out, void* stream);

/*
 * Step 2 -- quantize (Eq. 1: code = round(X / delta)).  The quotient is formed
 * as t = fl(x * fl(1/delta)): one correctly rounded reciprocal per group, one
 * correctly rounded product per element.
 *   INT8: round half to even, keep [-127, 127], two's complement byte; NaN -> 0.
 *   E4M3 / E5M2 (OCP FP8 value sets): nearest finite value, ties to the even
 *   mantissa, |t| above the maximum (and inf) -> +-maximum, sign of t kept
 *   (negative underflow -> 0x80), NaN -> 0x7F.
 *   QMM_ROUND_STOCHASTIC: with lo <= |t| < hi the neighbouring grid values, the
 *   result is hi iff u < (|t|-lo)/(hi-lo), u = (24 random bits)/2^24.  The bits
 *   of output element p (linear index in codes_out) are the top 24 bits of word
 *   (p+offset)%4 of Philox4x32-10, p+offset modulo 2^64, with counter ((p+offset)/4, 0) as two 32-bit
 *   halves followed by two zero words, and key = seed as two 32-bit halves, so
 *   a tensor quantized in pieces with matching offsets equals the whole.
 *   codes_out  device, [batch][non-contracting][contracting] bytes, dense: the
 *              contracting axis is contiguous whatever contract_axis is.
 *   delta      device, as written by qmm_scale (or supplied by the caller).
 * Uses no workspace.  batch above 65535: QMM_ERR_UNSUPPORTED.
 */
qmm_status qmm_quantize(const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g,
                        const float* delta, qmm_round mode, uint64_t seed, uint64_t offset,
                        uint8_t* codes_out, void* stream);

/*
 * qmm_scale_quantize -- steps 1 and 2 of one tensor in one call: delta_out and codes_out are exactly what qmm_scale and
 * then qmm_quantize with those step sizes write, with fewer launches and passes over x: one step size per row (rows up
 * to 8192 bfloat16 / 4096 binary32 elements, every matrix a batch group of its own) takes a single pass, other tensors that the
 * chip holds one launch that reads the tensor once: rows contracting up to 67 MB (strided rows, stochastic rounding 33 MB), rows
 * contracted up to 50 MB (binary32 33 MB; stochastic 2^23 elements, and not the smallest).  Beyond, and under stream capture, the
 * passes are separate launches, and the quantize pass forms the step sizes from the partial maxima where that pays.  The one launch
 * fills the chip: beside other work, with which it shares the CUs, it takes up to a fifth more than the separate ones.
 *   workspace  device scratch of at least qmm_scale_quantize_workspace_size() bytes, 16-byte aligned (0: may be NULL).
 * An empty tensor writes its groups' step sizes (1) and no codes.  Errors as for the two calls.
 */
size_t qmm_scale_quantize_workspace_size(const qmm_tensor* x, const qmm_granularity* g);
qmm_status qmm_scale_quantize(const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g, qmm_round mode,
                              uint64_t seed, uint64_t offset, float* delta_out, uint8_t* codes_out,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_scale_multi / qmm_quantize_multi -- steps 1 and 2 (Eq. 1) for `count` tensors in one call each, e.g. the
 * activations and the weights of one product: the results are those of `count` calls of qmm_scale / qmm_quantize.
 *   x, g        host arrays of `count` descriptors / granularities.
 *   delta_out, delta, codes_out   host arrays of `count` device pointers, each as the single-tensor call takes it.
 *   offsets     host array of `count` stream offsets for stochastic rounding, or NULL for zeros.
 *   workspace   device scratch, qmm_scale_multi_workspace_size() bytes (the tensors' own sizes, each rounded up to 16),
 *               16-byte aligned.
 * When all tensors (at most 8) are single dense bfloat16 matrices in 16-byte aligned whole vectors with one step size
 * each (and, for quantize: contract_axis 1, cols a multiple of 16, round to nearest even), each call is one launch
 * (for scale too: one of each tensor's workgroups folds the partial maxima) with the tensor index as a grid dimension, so that the
 * small tensors' latency-bound kernels run inside the large tensors' launches.  Otherwise the tensors are processed
 * one after the other by the single-tensor code, after every tensor's arguments have been checked (an argument
 * error in any of them is returned before anything is launched).  Errors as for the single-tensor calls; count = 0
 * is a no-op, count < 0 QMM_ERR_SHAPE.
 */
size_t qmm_scale_multi_workspace_size(int32_t count, const qmm_tensor* x, const qmm_granularity* g);
qmm_status qmm_scale_multi(int32_t count, const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g,
                           float* const* delta_out, void* workspace, size_t workspace_bytes, void* stream);
qmm_status qmm_quantize_multi(int32_t count, const qmm_tensor* x, qmm_format fmt, const qmm_granularity* g,
                              const float* const* delta, qmm_round mode, uint64_t seed, const uint64_t* offsets,
                              uint8_t* const* codes_out, void* stream);

/* One operand of qmm_gemm: a dense batch [batch][rows][K] with K contiguous. */
typedef struct {
    const void* data;        /* device; 8-bit codes, or bfloat16 values (see is_codes)          */
    int32_t format;          /* qmm_format the operand is multiplied in                          */
    int32_t is_codes;        /* 1: data holds 8-bit codes of `format`.
                                0: data holds bfloat16; with an 8-bit `format` the values are
                                   quantized with `delta` (RTNE) while they are staged for the
                                   multiply; with QMM_FMT_BF16 they are multiplied as they are. */
    const float* delta;      /* device step sizes (ignored for QMM_FMT_BF16)                     */
    qmm_granularity gran;    /* how delta is indexed; per_channel refers to the operand's rows   */
} qmm_operand;

/*
 * Steps 3 and 4 -- Y[b][i][j] = (acc * deltaA[i]) * deltaB[j],
 * acc = sum_k value(A[b][i][k]) * value(B[b][j][k])   (third Methodology bullet:
 * scaling before and after the multiply, result held in a wider accumulator).
 *   INT8 x INT8 accumulates exactly in int32 (|acc| must stay below 2^31);
 *   FP8 x FP8 (E4M3 and E5M2 may be mixed) accumulates in binary32; the
 *   summation order is unspecified;  BF16 x BF16 accumulates in binary32 and
 *   is not descaled (the high-precision reference product).
 *   Both operands must be 8-bit formats of the same family (both INT8 or both
 *   FP8) or both BF16.  INT8 code 0x80 (-128) is outside the format: undefined.
 *   y          device [batch][M][N], y_dtype F32 or BF16 (RNE).  May be NULL if
 *              acc_out is given.
 *   acc_out    device [batch][M][N] raw accumulators (int32 for INT8, else
 *              binary32) or NULL.
 *   K must be a multiple of 16 bytes' worth of elements (16 codes / 8 bf16)
 *   and all data pointers 16-byte aligned, else QMM_ERR_ALIGN.
 *   K in bytes (K codes, or 2 K for BF16) must not exceed 2^22, else
 *   QMM_ERR_UNSUPPORTED.
 *   workspace  device scratch of at least qmm_gemm_workspace_size() bytes,
 *              16-byte aligned (may be 0, then NULL is accepted).  It is non-zero
 *              for small outputs with a long K (weight-gradient shapes): K is
 *              then split into ranges whose partial accumulators are kept there
 *              and added in ascending order by a second kernel, so results do
 *              not depend on timing.  Too small: QMM_ERR_WORKSPACE.
 */
size_t qmm_gemm_workspace_size(const qmm_operand* a, const qmm_operand* b,
                               int64_t batch, int64_t M, int64_t N, int64_t K);
qmm_status qmm_gemm(const qmm_operand* a, const qmm_operand* b,
                    int64_t batch, int64_t M, int64_t N, int64_t K,
                    void* y, qmm_dtype y_dtype, void* acc_out,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_gemm_nsr -- qmm_gemm with the noise-to-signal sums taken in its epilogue (the error metric the path reduces
 * for every op, here without a second pass over Y; an extension: the paper measures, it does not say where).
 * Computes Y exactly as qmm_gemm does and, over the values it stores (rounded to y_dtype),
 *     out2[0] = sum (y - y_ref)^2      out2[1] = sum y_ref^2
 * in binary64, elements whose error is NaN left out of both sums -- fields 0 and 1 of qmm_metric(Y, y_ref).  The
 * order of additions is fixed by the shapes (per-wavefront sums folded by a second kernel), so results are
 * reproducible run to run; it differs from qmm_metric's order, so the sums agree with it to rounding only.
 *   a, b       8-bit operands given as codes (is_codes = 1); BF16 and quantize-on-load operands: QMM_ERR_UNSUPPORTED.
 *   y          device [batch][M][N], required.      y_ref  device [batch][M][N] binary32, 16-byte aligned.
 *   out2       device, 2 doubles, 8-byte aligned.
 *   workspace  device scratch of at least qmm_gemm_nsr_workspace_size() bytes, 16-byte aligned: QMM_ERR_WORKSPACE
 *              if missing or too small.  K is never split here.
 * Other argument rules and errors as for qmm_gemm.  An empty output writes two zeros.
 */
size_t qmm_gemm_nsr_workspace_size(int64_t batch, int64_t M, int64_t N);
qmm_status qmm_gemm_nsr(const qmm_operand* a, const qmm_operand* b,
                        int64_t batch, int64_t M, int64_t N, int64_t K,
                        void* y, qmm_dtype y_dtype, const float* y_ref, double* out2,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * Step 6 -- error metrics of y against the high-precision result y_ref, one
 * pass, binary64 accumulation, e = y - y_ref.  out16 (device, 16 doubles):
 *   [0] sum e^2          [1] sum ref^2        (noise-to-signal ratio = [0]/[1])
 *   [2] sum |e|          [3] sum |ref|
 *   [4] max |e|          [5] max |ref|
 *   [6] sum over ref != 0 of |e|/|ref|   [7] its max   [8] its term count   (Eq. 2)
 *   [9] sum over d > 0 of |e|/d          [10] its max  [11] its term count  (Eq. 3, element-wise;
 *        d = (|L|.|R|)_ij supplied by the caller in denom, or NULL: [9..11] = 0)
 *   [12] elements counted   [13] elements skipped because e is NaN   [14],[15] = 0
 * Elements whose error is NaN are left out of every sum and maximum.
 *   y          device, n elements of y_dtype;  y_ref, denom: device, n floats.
 *   workspace  device scratch, qmm_metric_workspace_size(n) bytes, 16-byte aligned.
 * n = 0 writes sixteen zeros.  Up to 2^22 elements one launch; beyond, and under stream capture, a second one folds the sums.
 */
size_t qmm_metric_workspace_size(int64_t n);
qmm_status qmm_metric(const void* y, qmm_dtype y_dtype, const float* y_ref, const float* denom,
                      int64_t n, double* out16, void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_dequantize -- the reduced-precision value of every quantized element (the v-tilde of Eq. 2), for looking at
 * the quantization error of a tensor itself rather than of a product:
 *     out[b][r][k] = fl32( value(codes[b][r][k]) * delta[group(b) * C + (per_channel ? r : 0)] )
 * with codes and delta exactly as qmm_quantize takes / writes them (C = rows if per_channel, else 1); the code's
 * value is exact in binary32, so this is one rounding; bfloat16 output rounds that once more (RNE).
 * An FP8 NaN code gives NaN, an E5M2 infinity code gives infinity, the INT8 code 0x80 gives -128 delta.
 *   codes  device [batch][rows][K] uint8;  out  device [batch][rows][K] of out_dtype; caller-owned.
 * Asynchronous on `stream`, uses no workspace.  Empty tensors return QMM_OK.
 * Errors: QMM_ERR_NULL, QMM_ERR_ENUM, QMM_ERR_SHAPE, QMM_ERR_ALIGN (out not aligned to its element), QMM_ERR_LAUNCH.
 */
qmm_status qmm_dequantize(const uint8_t* codes, int64_t batch, int64_t rows, int64_t K, qmm_format fmt,
                          const qmm_granularity* g, const float* delta, void* out, qmm_dtype out_dtype, void* stream);

/*
 * qmm_rmsnorm_quantize -- the root-mean-square norm in front of a quantized product, with the addition to the residual
 * stream before it and steps 1 and 2 (one step size per row, i.e. per token) behind it, in one pass over the row:
 *     h    = x + residual in binary32, then rounded to x's type (x itself without a residual)
 *     rstd = 1 / sqrt(mean_j h_j^2 + eps)          y_j = (h_j * weight_j) * rstd     (binary32, in this order)
 *     delta, codes = what qmm_scale and qmm_quantize give for the row y in binary32 (y is not rounded in between)
 *   x, residual   tensors of the same extent and type, contract_axis 1, cols up to 2^22; residual may be NULL.
 *   weight        device, cols values of weight_dtype, or NULL for ones.
 *   eps           finite and not negative.
 *   h_out         device, dense [batch][rows][cols] of x's type, required with a residual and not written without one; may be the memory
 *                 of x or of the residual where that is dense (QMM_ERR_SHAPE where it is not).
 *   y_out         device, dense, x's type: y rounded once, or NULL.  rstd_out  device, batch * rows floats, or NULL.
 *   delta_out     device, batch * rows floats;  codes_out  device [batch][rows][cols]: an operand with per_channel = 1 and
 *                 batch_groups = batch.  Random bits of stochastic rounding as in qmm_quantize.
 * A row whose squares overflow binary32 has rstd 0, so y 0 and delta 1, also where h_j * weight_j overflows; a row with an inf or NaN has delta NaN and,
 * in FP8, codes 0x7F.  A row of zeros has y 0, codes 0 and delta 1, also with eps = 0, where its rstd is infinite and it has no gradient
 * (qmm_rmsnorm_backward: NaN in its dx and in dw).  cols = 0: delta 1, rstd 1 / sqrt(eps).  Uses no workspace.
 * Other types, extents or axes: QMM_ERR_SHAPE / QMM_ERR_UNSUPPORTED / QMM_ERR_ENUM; a pointer off its element's boundary: QMM_ERR_ALIGN.
 */
qmm_status qmm_rmsnorm_quantize(const qmm_tensor* x, const qmm_tensor* residual, const void* weight, qmm_dtype weight_dtype, float eps,
                                qmm_format fmt, qmm_round mode, uint64_t seed, uint64_t offset, void* h_out, void* y_out,
                                float* rstd_out, float* delta_out, uint8_t* codes_out, void* stream);

/*
 * qmm_rmsnorm_backward -- the gradients of y = h rstd weight (the quantization behind it passes them on unchanged):
 *     a = weight * dy,  n = h * rstd,  dx = rstd * (a - n * mean_j(a n)) + dresidual,  dw = sum over all rows of dy n
 * dx is the gradient of x and of the residual alike.
 *   dy, h, dresidual   tensors of one extent and type, contract_axis 1; dresidual (the gradient that reaches h past the norm) or NULL.
 *   rstd               device, batch * rows floats, as qmm_rmsnorm_quantize wrote it.
 *   dx_out             device, dense, their type; may be the memory of one of them where that is dense.
 *   dw_out             device, cols floats, or NULL.  Sums in binary32 in an order fixed by the extents.
 *   workspace          qmm_rmsnorm_backward_workspace_size(dy) bytes, 16-byte aligned (0: may be NULL); not needed without dw_out.
 * Errors as above; without rows dw is zero.
 */
size_t qmm_rmsnorm_backward_workspace_size(const qmm_tensor* dy);
qmm_status qmm_rmsnorm_backward(const qmm_tensor* dy, const qmm_tensor* h, const float* rstd, const void* weight, qmm_dtype weight_dtype,
                                const qmm_tensor* dresidual, void* dx_out, float* dw_out, void* workspace, size_t workspace_bytes,
                                void* stream);

/* Activations of a gated feed-forward block: SiLU g / (1 + e^-g), GELU g Phi(g) with the normal distribution function Phi. */
typedef enum { QMM_ACT_SILU = 0, QMM_ACT_GELU = 1 } qmm_activation;

/*
 * qmm_gemm_gated -- both projections of a gated feed-forward block, the activation and the product in one kernel:
 *     g = A Bg^T,  u = A Bu^T  (each descaled as in qmm_gemm, binary32),   h = act(g) * u
 *   a          [batch][M][K].   b   [batch][2 F][K]: the F rows of the gate's weights, then the F rows of the other projection's; its
 *              step sizes are those of an operand of 2 F rows.  Both codes (of one family), or both BF16; operands
 *              to be quantized on load: QMM_ERR_UNSUPPORTED.
 *   h          device [batch][M][F] of out_dtype, rounded once.
 *   gu         device [batch][M][2 F] of out_dtype: g and u, rounded once (h is of the unrounded ones), for
 *              qmm_gated_backward; or NULL.
 *   workspace  qmm_gemm_gated_workspace_size() bytes, 16-byte aligned (0: may be NULL).  It is non-zero where M and F are small
 *              and K long: K is then split and the parts are added in a fixed order.
 * The activations are evaluated in binary32: act(g) is off by at most (1.3 |g| + 8) 2^-24 (SiLU, |g| <= 80) or (1.2 g^2 + 18) 2^-24 (GELU, |g| <= 12.5) of
 * itself, the loss of the power's argument; further out, where act(g) nears the smallest normal value, to that.
 * A gate of -infinity gives NaN.  F up to 2^22, else QMM_ERR_UNSUPPORTED.  Other rules and errors as for qmm_gemm.
 */
size_t qmm_gemm_gated_workspace_size(const qmm_operand* a, const qmm_operand* b, int64_t batch, int64_t M, int64_t F, int64_t K);
qmm_status qmm_gemm_gated(const qmm_operand* a, const qmm_operand* b, int64_t batch, int64_t M, int64_t F, int64_t K,
                          qmm_activation act, void* h, void* gu, qmm_dtype out_dtype, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * qmm_gated_backward -- the backward pass of h = act(g) * u up to the operand of the products behind it:
 *     dg = (dh * u) * act'(g),   du = dh * act(g)        a row's results are (dg | du), 2 F values (an infinite gate: NaN)
 * as values (for the weight gradient, whose operand is quantized along the other axis) and as codes with one step size per row
 * (the data gradient's operand [batch][rows][2 F], per_channel = 1, batch_groups = batch): what qmm_scale and qmm_quantize give for the
 * binary32 results.
 *   dh [..][F], gu [..][2 F]   tensors of one type, batch and rows, contract_axis 1, 2 F up to 2^22 (the K of the data gradient's product, as for
 *               qmm_gemm).
 *   dgu_out     device, dense [batch][rows][2 F], their type; or NULL.  May be gu's memory where that is dense.
 *   delta_out, codes_out   device; both or neither NULL.  At least one of codes_out and dgu_out.
 * Random bits of stochastic rounding as in qmm_quantize.  Errors as for qmm_rmsnorm_quantize.  Uses no workspace.
 */
qmm_status qmm_gated_backward(const qmm_tensor* dh, const qmm_tensor* gu, qmm_activation act, qmm_format fmt, qmm_round mode,
                              uint64_t seed, uint64_t offset, void* dgu_out, float* delta_out, uint8_t* codes_out, void* stream);

/*
 * ---- A step size for every block of 128.
 * An operand [batch][rows][K] has one for each 128 elements along K (the last block may be shorter) of one row (block_rows = 1) or of 128
 * neighbouring rows (block_rows = 128; the last ones may be fewer):
 *     delta[(b * ceil(K / 128) + k / 128) * ceil(rows / block_rows) + row / block_rows]
 * qmm_num_block_scales of them; -1 for arguments out of range.
 */
int64_t qmm_num_block_scales(int64_t batch, int64_t rows, int64_t K, int32_t block_rows);

/*
 * qmm_quantize_blocks -- steps 1 and 2 with such scale groups: delta and codes of a block are what qmm_scale and qmm_quantize give for the
 * block alone (zero and non-finite blocks included).
 *   x            any extent and strides; contract_axis as everywhere.   fmt  E4M3 or E5M2 (INT8: QMM_ERR_UNSUPPORTED).
 *   delta_out    device, floats as above for [batch][non-contracting][contracting];  codes_out  device, dense in that order.
 *   delta_t_out, codes_t_out   device, or both NULL: the same of the tensor contracted over its other axis, in the same pass over x (a gradient
 *                is an operand of the data gradient's product along one axis and of the weight gradient's along the other).
 * Random bits of stochastic rounding as in qmm_quantize, by the position in codes_out, in codes_t_out by the position there.  An empty tensor
 * writes nothing.  batch above 65535, an extent above 2^31 - 129: QMM_ERR_UNSUPPORTED.  Uses no workspace.
 */
qmm_status qmm_quantize_blocks(const qmm_tensor* x, qmm_format fmt, int32_t block_rows, qmm_round mode, uint64_t seed, uint64_t offset,
                               float* delta_out, uint8_t* codes_out, float* delta_t_out, uint8_t* codes_t_out, void* stream);

/* One operand of qmm_gemm_blocks: dense codes [batch][rows][K] and their step sizes. */
typedef struct {
    const void* data;        /* device, 16-byte aligned */
    int32_t format;          /* QMM_FMT_E4M3 or QMM_FMT_E5M2 */
    int32_t block_rows;      /* 1 or 128 */
    const float* delta;      /* device, as qmm_quantize_blocks writes it */
} qmm_block_operand;

/*
 * qmm_gemm_blocks -- Y[b][i][j] = sum over blocks t of (sum_{k in t} value(A[b][i][k]) value(B[b][j][k])) * deltaA[t][i] * deltaB[t][j].
 *   A block's sum is the matrix instruction's, as in qmm_gemm: of every eight neighbouring products all but the one with the largest exponents lose what
 *   lies below 2^-13 of that (1e-5 to 3e-5 of the result's 2-norm in all, below a bfloat16 rounding).  It is multiplied by the step sizes and added
 *   to the blocks before it in binary32; the order of blocks is fixed by the extents (ascending, in a fixed number of parts), so results do not depend
 *   on timing.
 *   a [batch][M][K], b [batch][N][K]: E4M3 and E5M2 may be mixed, each has its block_rows.  The usual pairs are rows by 128 x 128 blocks of weights, and in a
 *              weight gradient rows by rows; blocks of 128 rows in b are the faster ones.
 *   y          device [batch][M][N], y_dtype F32 or BF16 (RNE), 16-byte aligned.
 *   K a multiple of 16 and at most 2^22, M and N below 2^31, data 16-byte aligned.  Without a contraction (K = 0) y is zero.  2^31 tiles of 256 x 256 of y and more
 *              over the batch, or with K = 0 2^24 of 64 x 64: QMM_ERR_UNSUPPORTED.
 *   workspace  qmm_gemm_blocks_workspace_size() bytes, 16-byte aligned (0: may be NULL).  It is non-zero for small outputs with a long K: K is then split
 *              and the parts are added in ascending order.
 */
size_t qmm_gemm_blocks_workspace_size(int64_t batch, int64_t M, int64_t N, int64_t K);
qmm_status qmm_gemm_blocks(const qmm_block_operand* a, const qmm_block_operand* b, int64_t batch, int64_t M, int64_t N, int64_t K,
                           void* y, qmm_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_dropout -- out = x * 1 / (1 - p) where an element is kept, 0 (whatever x is there) where it is dropped.  The decisions are functions of (seed,
 * offset + the element's linear index in out) and are not stored: the gradient is the same call on the upstream gradient.
 *   Element number n = index + offset (modulo 2^64) has 16 random bits u: half n % 2 (0: the low one) of word (n % 8) / 2 of Philox4x32-10 with counter (n / 8 as two
 *   32-bit halves, 1, 0) and key = seed as two halves (the 1 keeps these bits apart from those of stochastic rounding).  It is dropped iff u < T,
 *   T = p * 65536 rounded to nearest; what is kept is multiplied by 65536 / (65536 - T) in binary32, the reciprocal of the probability that is used
 *   (p to within 2^-17), and rounded once to x's type.
 *   x      any extent and strides (contract_axis is not looked at further than its range).   p  0 to 1 (1: everything is dropped), else QMM_ERR_SHAPE.
 *   out    device, dense [batch][rows][cols] of x's type; may be x's memory where that is dense.
 * A tensor processed in pieces with matching offsets equals the whole.  Errors as for qmm_rmsnorm_quantize.
 */
qmm_status qmm_dropout(const qmm_tensor* x, float p, uint64_t seed, uint64_t offset, void* out, void* stream);

/*
 * qmm_layernorm_quantize -- behind a block of products: dropout of its result, the addition to the residual stream, layer norm, and the
 * quantization (Eq. 1) of what the next product reads, in one pass over the row:
 *     h    = dropout(x) + residual in binary32 (one rounding), then rounded to x's type (x itself without a residual and with dropout = 0)
 *     mean = mean_j h_j,  rstd = 1 / sqrt(mean_j (h_j - mean)^2 + eps),  y_j = ((h_j - mean) * rstd) * weight_j + bias_j     (binary32)
 *     delta, codes = what qmm_scale and qmm_quantize give for y in binary32 with one step size per row (block = 0, any 8-bit format), or
 *                    per row and 128 columns (block = 128, then those of qmm_quantize_blocks with block_rows = 1)
 *   x, residual   tensors of the same extent and type, contract_axis 1, cols up to 2^22; residual may be NULL.
 *   weight, bias  device, cols values of weight_dtype, or NULL for ones / zeros.      eps  finite and not negative.
 *   dropout       its p, decisions and factor as in qmm_dropout, by the element's index in the dense tensor + dropout_offset.
 *   h_out         device, dense, x's type: required with a residual or dropout > 0, else not written; may be x's or the residual's memory where that is
 *                 dense.
 *   y_out         device, dense, x's type: y rounded once, or NULL.   mean_out, rstd_out  device, batch * rows floats, or NULL.
 *   delta_out, codes_out  device, both NULL: no quantization (fmt, block, mode are then not looked at).
 * Random bits of stochastic rounding as in qmm_quantize.  The mean is subtracted before the squares are summed, and what its rounding left is taken out
 * again: a row's offset does not cost its variance's accuracy.  A row whose squares alone overflow binary32 has rstd 0 and y = bias; a row with an inf or
 * NaN, or of which a sum or a difference to the mean overflows, has y NaN, delta NaN and codes 0x7F (INT8 0).  Where all of a row's differences are zero and eps = 0, its rstd is infinite and y = bias.  cols = 0: delta 1
 * (block = 0), mean 0, rstd 1 / sqrt(eps).  Uses no workspace.  Errors as for qmm_rmsnorm_quantize; dropout outside 0 to 1: QMM_ERR_SHAPE; block: QMM_ERR_ENUM.
 */
qmm_status qmm_layernorm_quantize(const qmm_tensor* x, const qmm_tensor* residual, const void* weight, const void* bias, qmm_dtype weight_dtype,
                                  float eps, float dropout, uint64_t dropout_seed, uint64_t dropout_offset, qmm_format fmt, int32_t block,
                                  qmm_round mode, uint64_t seed, uint64_t offset, void* h_out, void* y_out, float* mean_out, float* rstd_out,
                                  float* delta_out, uint8_t* codes_out, void* stream);

/*
 * qmm_layernorm_backward -- the gradients of y (the quantization behind it passes them on unchanged):
 *     a = weight * dy,  n = (h - mean) * rstd,  dh = rstd * (a - mean_j(a) - n * mean_j(a n)) + dresidual
 *     dx = dh's dropout (that of the forward pass: same dropout, seed and offset),  dw = sum over all rows of dy n,  db = sum over all rows of dy
 * dh is the gradient of the residual, dx that of x (dropout = 0: dh is both, and dx_out is not written).
 * A row whose rstd is infinite (no spread, eps = 0) has n = 0 as in the forward pass: its dh is dresidual, or 0, it adds nothing to dw and dy to db.
 *   dy, h, dresidual   tensors of one extent and type, contract_axis 1; dresidual (the gradient that reaches h past the norm) or NULL.
 *   mean, rstd         device, batch * rows floats, as qmm_layernorm_quantize wrote them.
 *   dh_out, dx_out     device, dense, their type; each may be the memory of one of the inputs where that is dense.
 *   dw_out, db_out     device, cols floats, both or neither NULL.  Sums in binary32 in an order fixed by the extents.
 *   workspace          qmm_layernorm_backward_workspace_size(dy) bytes, 16-byte aligned (0: may be NULL); not needed without dw_out.
 * Errors as above; without rows dw and db are zero.
 */
size_t qmm_layernorm_backward_workspace_size(const qmm_tensor* dy);
qmm_status qmm_layernorm_backward(const qmm_tensor* dy, const qmm_tensor* h, const float* mean, const float* rstd, const void* weight,
                                  qmm_dtype weight_dtype, const qmm_tensor* dresidual, float dropout, uint64_t dropout_seed,
                                  uint64_t dropout_offset, void* dh_out, void* dx_out, float* dw_out, float* db_out, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * qmm_moments -- statistics of a tensor the method looks at before choosing a format (Results section, first
 * paragraph: mean, variance, skew and kurtosis of the matrix-multiply inputs).  Estimators (the paper names none):
 * population moments about the mean,  mean = sum x / n,  m_k = sum (x - mean)^k / n  for k = 2, 3, 4;
 * skew = m3 / m2^1.5 and kurtosis = m4 / m2^2 (3 for a normal distribution) are left to the caller.
 *   x        device, n contiguous elements (bfloat16 or binary32), 16-byte aligned; not modified
 *   center   finite value the power sums are taken about in the single pass over x (binary64).  0 is right for
 *            tensors whose mean lies within a few standard deviations of 0; otherwise pass an estimate of the
 *            mean: the relative error of m_k grows like (1 + ((mean - center) / sigma)^2)^(k/2) * 1e-15.
 *   out8     device, 8 doubles: n (non-NaN count), mean, m2, m3, m4, max |x|, NaN count, 0.
 *            NaN elements are counted and otherwise ignored; n = 0 gives zeros.  Infinite elements propagate.
 *   workspace  device scratch, qmm_moments_workspace_size(n) bytes, 16-byte aligned.
 * Asynchronous on `stream`; deterministic (fixed order of additions for a given n).
 * Errors: QMM_ERR_NULL, QMM_ERR_ENUM, QMM_ERR_SHAPE (n < 0 or center not finite), QMM_ERR_ALIGN,
 * QMM_ERR_WORKSPACE, QMM_ERR_LAUNCH.
 */
size_t qmm_moments_workspace_size(int64_t n);
qmm_status qmm_moments(const void* x, qmm_dtype dtype, int64_t n, double center, double* out8,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * qmm_mfma_rate -- measurement aid, not a step of the method: the rate the matrix units sustain on given operand
 * bytes with no memory traffic, against which the GEMM's rate is read (next to the datasheet peak, which is quoted
 * at the top clock; under matrix load the clock is set by power, and that depends on the operand bytes).
 *   operand_bytes device, 32-byte aligned, nbytes >= 32: 8-bit codes in the given formats (e.g. the codes
 *                 qmm_quantize wrote); every lane takes ten fragments from it.  Not modified.
 *   rounds        every wavefront issues rounds * 64 (FP8) or rounds * 16 (INT8) matrix instructions
 *   workgroups    number of workgroups of four wavefronts (one per CU fills the chip)
 *   sink          device, workgroups * 256 floats, written (keeps the work alive); caller-owned
 *   flops_out     host: operations the launch performs (2 per multiply-add)
 * Asynchronous on `stream`; the caller times it.  Formats: both INT8, or any pair of E4M3 / E5M2.
 * Errors: QMM_ERR_NULL, QMM_ERR_ENUM, QMM_ERR_UNSUPPORTED, QMM_ERR_SHAPE, QMM_ERR_ALIGN, QMM_ERR_LAUNCH.
 */
qmm_status qmm_mfma_rate(qmm_format a_format, qmm_format b_format, const void* operand_bytes, int64_t nbytes,
                         int64_t rounds, int32_t workgroups, float* sink, double* flops_out, void* stream);

/*
 * qmm_hbm_rate -- measurement aid, not a step of the method: a plain streaming kernel over `nbytes` of device memory,
 * the ceiling the memory-bound passes (steps 1, 2 and 6) are read against next to the datasheet bandwidth.
 *   src     device, nbytes (a multiple of 16), 16-byte aligned; read once with streaming loads
 *   dst     device, nbytes, 16-byte aligned: the bytes are copied there; or NULL: read only, folded into `sink`
 *   sink    device, workgroups * 256 words, written when dst is NULL (keeps the loads alive); caller-owned
 *   workgroups  grid size (1024 = four workgroups per CU, as the passes use)
 * Asynchronous on `stream`; the caller times it and rotates buffers larger than the caches.
 * Errors: QMM_ERR_NULL, QMM_ERR_SHAPE, QMM_ERR_ALIGN, QMM_ERR_LAUNCH.
 */
qmm_status qmm_hbm_rate(const void* src, void* dst, int64_t nbytes, int32_t workgroups, uint32_t* sink, void* stream);

const char* qmm_status_string(qmm_status s);
/* Version of this ABI (major*100 + minor). */
int qmm_version(void);

#ifdef __cplusplus
}
#endif
#endif /* QMM_H */
