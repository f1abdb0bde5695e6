/*
 * hif4.h -- C ABI of the HiF4 (HiFloat4) W4A4 linear-layer hot path for NVIDIA B200 (sm_100a).
 *
 * HiF4 is the 4-bit block floating-point format of "HiFloat4 Format for Language Model
 * Inference" (Section II).  One HiF4 *unit* stores 64 values in 288 bits: 32 bits of shared
 * three-level scaling metadata plus 64 four-bit sign-magnitude S1P2 elements (Section II-A,
 * Table I, Table II: 4.5 bits per value).
 *
 * ---------------------------------------------------------------------------------------------
 * Unit layout in memory (36 bytes, 4-byte aligned, units of a row consecutive, rows consecutive).
 * The paper's figure of the unit is not reproduced in its text, so this byte order is a
 * convention of this library:
 *
 *   bytes 0..3   little-endian uint32 `meta`
 *                  bits  7:0   E6M2 level-1 scale byte `eeeeee mm` (Table I): value
 *                              2^(e-48) * (1 + m/4); 0xFF is NaN, there is no zero or infinity
 *                  bits 15:8   E1_8  level-2 micro-exponents, bit 8+j  covers elements 8j..8j+7
 *                  bits 31:16  E1_16 level-3 micro-exponents, bit 16+k covers elements 4k..4k+3
 *   bytes 4..35  S1P2 codes, element i in byte 4 + i/2, low nibble for even i, high nibble for
 *                odd i; nibble = sign<<3 | magnitude, magnitude m in 0..7 meaning m/4.
 *
 * Value of element i (Eq. 2, 0-based indices):
 *   V_i = (-1)^sign * (m/4) * 2^(E1_8[i/8] + E1_16[i/4]) * E6M2,   all 64 are NaN if E6M2 is NaN.
 * ---------------------------------------------------------------------------------------------
 *
 * Conventions common to every call
 *   - All data pointers are DEVICE pointers unless a parameter says "host".  The caller owns every
 *     buffer; the library never allocates, frees or synchronises (hif4_last_device_status is the
 *     one documented exception and synchronises the stream it is given).
 *   - Every call is asynchronous on `stream` (a cudaStream_t passed as void* so that this header
 *     needs no CUDA header; NULL is the legacy default stream).
 *   - The return value is a status code.  Argument errors are found on the host before any launch.
 *     NaN and Inf in the data are not errors; they encode as the format defines.
 *   - Matrices are row-major.  Both GEMM operands are quantised along K (units contiguous in K),
 *     because Eq. 3 pairs unit k of a row of A with unit k of a row of B.  A weight W[K_in, N_out]
 *     is therefore handed over as its transpose [N, K].
 */
#ifndef HIF4_H_
#define HIF4_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HIF4_UNIT_ELEMS 64   /* elements per unit (Section II-A)                    */
#define HIF4_UNIT_BYTES 36   /* 4 metadata bytes + 32 code bytes = 288 bits         */

typedef enum {
  HIF4_OK = 0,
  HIF4_ERR_NULL = 1,           /* a required pointer is NULL                                   */
  HIF4_ERR_SHAPE = 2,          /* negative size, cols or K not a multiple of 64, ld too small  */
  HIF4_ERR_ALIGN = 3,          /* pointer or leading dimension breaks the stated alignment     */
  HIF4_ERR_DTYPE = 4,          /* unknown hif4_dtype / hif4_round value                        */
  HIF4_ERR_WORKSPACE = 5,      /* workspace smaller than hif4_*_workspace reports              */
  HIF4_ERR_CUDA = 6,           /* a CUDA call or launch failed; cudaGetLastError keeps the code*/
  HIF4_ERR_DEVICE_TIMEOUT = 7, /* a bounded wait inside a kernel ran out (see last_device_status) */
  HIF4_ERR_UNSUPPORTED = 8     /* valid request that this build does not implement             */
} hif4_status;

/* HIF4_FP16 is a source type only (hif4_quantize, hif4_linear): Section II-B extends the conversion to
 * further source types and names FP32 and FP16; FP16 arithmetic cannot hold the reciprocal of an
 * E6M2 scale (up to 2^48), so FP16 elements are widened exactly to FP32 and Algorithm 1 runs in FP32
 * arithmetic.  hif4_dequantize returns HIF4_ERR_DTYPE for it (HiF4's range exceeds FP16's).  */
typedef enum { HIF4_BF16 = 0, HIF4_FP32 = 1, HIF4_FP16 = 2 } hif4_dtype;

/* Rounding used where Algorithm 1 rounds to E6M2 and to S1P2 (Section II-B allows half-to-even or
 * half-away-from-zero).  Products inside the algorithm always round to
 * nearest-even.  */
typedef enum { HIF4_RNE = 0, HIF4_RHA = 1 } hif4_round;

/* Bytes of the packed form of a [rows, cols] matrix: rows * (cols/64) * 36 (Section II-A).
 * Returns 0 when cols is not a multiple of 64 or a size is negative.  Host-only, no GPU use.  */
size_t hif4_packed_bytes(int64_t rows, int64_t cols);

/* hif4_quantize -- Algorithm 1 (Section II-B) applied to every 64-element unit of a matrix.
 *   src        device, [rows, cols] of `dt`, row stride `ld_src` ELEMENTS (>= cols); base and row
 *              stride must keep every row 16-byte aligned.
 *   dst_units  device, rows*(cols/64) units of 36 bytes, row-major, 4-byte aligned (16-byte aligned
 *              storage gives the fastest stores).  Fully overwritten.
 *   mode       HIF4_RNE or HIF4_RHA.
 * The working precision of the algorithm is that of the source type (BF16 arithmetic for BF16
 * input, FP32 arithmetic for FP32 and FP16 input).  A unit holding a NaN becomes the canonical NaN unit
 * (meta 0x000000FF, codes 0).  rows == 0 or cols == 0 is a no-op returning HIF4_OK.  */
hif4_status hif4_quantize(const void* src, hif4_dtype dt, int64_t rows, int64_t cols,
                          int64_t ld_src, void* dst_units, hif4_round mode, void* stream);

/* hif4_quantize_transposed -- the same conversion with the units running down the columns: unit r of
 * column c holds src[64 r .. 64 r + 63][c], i.e. dst is hif4_quantize of the transposed matrix without the
 * transpose ever being written.  (Algorithm 1 converts 64 values at a time and does not say how those
 * 64 lie in memory; Eq. 3 needs both GEMM operands cut along the contraction dimension, so a matrix
 * that is contracted along its rows -- a weight kept as [K, N], or any operand of a transposed product --
 * is quantized this way.)
 *   src        device, [rows, cols] of `dt` (any source type of hif4_quantize, same working precision), row
 *              stride `ld_src` elements (>= cols), rows 16-byte aligned; rows must be a multiple of 64, cols
 *              a multiple of 8.
 *   dst_units  device, cols*(rows/64) units, column-major in the sense above ([cols, rows/64, 36 bytes]),
 *              4-byte aligned.  Fully overwritten.  */
hif4_status hif4_quantize_transposed(const void* src, hif4_dtype dt, int64_t rows, int64_t cols,
                                     int64_t ld_src, void* dst_units, hif4_round mode, void* stream);

/* hif4_dequantize -- Eq. 2 for every element; exact in BF16 and FP32.
 *   src_units  device, rows*(cols/64) units, 4-byte aligned.
 *   dst        device, [rows, cols] of `dt`, row stride `ld_dst` elements (>= cols), rows 16-byte
 *              aligned.  Fully overwritten inside [rows, cols]; padding beyond cols is untouched.  */
hif4_status hif4_dequantize(const void* src_units, int64_t rows, int64_t cols, void* dst,
                            hif4_dtype dt, int64_t ld_dst, void* stream);

/* Workspace (device scratch) that hif4_gemm needs for this shape on the current device; may be 0.
 * For M <= 32 it holds the decoded activation rows (2 * K * 8, 16 or 32 bytes); for larger M a few KB of
 * completion words when tiles are split along K.  The figure is the largest need over all kernels that
 * could serve the shape, so it stays valid whatever path is chosen at call time.  Host-only.  */
hif4_status hif4_gemm_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes);

/* hif4_gemm -- C = A * B^T with A, B in HiF4 and FP32 accumulation: C[i][j] is the sum over the
 * K/64 unit pairs of Eq. 3's dot product of unit k of row i of A with unit k of row j of B.
 *   A_units    device, [M, K/64] units.        B_units  device, [N, K/64] units.
 *   C          device, [M, N] FP32, row stride `ldc` elements (>= N), 4-byte aligned; 16-byte
 *              aligned rows (base % 16 == 0 and ldc % 4 == 0) allow vector stores.  Overwritten
 *              inside [M, N] (no alpha/beta); padding beyond N is untouched.
 *   workspace  device scratch of at least hif4_gemm_workspace bytes, 256-byte aligned, contents
 *              undefined on entry and exit; may be NULL when 0 bytes are needed.  Calls that may run
 *              at the same time (different streams) need workspaces of their own.
 * K must be a multiple of 64.  M == 0 or N == 0 is a no-op; K == 0 zero-fills C.
 * Units whose E6M2 byte is NaN make every C entry they touch NaN.  */
hif4_status hif4_gemm(const void* A_units, const void* B_units, float* C, int64_t M, int64_t N,
                      int64_t K, int64_t ldc, void* workspace, size_t workspace_bytes,
                      void* stream);

/* hif4_linear -- the W4A4 linear layer in one call (Section IV: every linear layer's activations
 * are converted to HiF4 before the matrix multiplication): Y = HiF4(X) * W^T, i.e. hif4_quantize of the
 * activations (Algorithm 1) followed by hif4_gemm with pre-quantized weights (Eq. 3), in stream order.
 *   X          device, [M, K] of `dt` (BF16 or FP32), row stride ld_x elements, rows 16-byte aligned.
 *   W_units    device, [N, K/64] units (the weight quantized along K beforehand).
 *   Y          device, [M, N] FP32, row stride ldy.
 *   workspace  device scratch of at least hif4_linear_workspace bytes, 256-byte aligned: holds the
 *              packed activations (and what hif4_gemm needs for this shape).
 * The result is bit-identical to calling hif4_quantize and hif4_gemm one after the other.  */
hif4_status hif4_linear_workspace(int64_t M, int64_t N, int64_t K, size_t* bytes);
hif4_status hif4_linear(const void* X, hif4_dtype dt, int64_t ld_x, const void* W_units, float* Y, int64_t M,
                        int64_t N, int64_t K, int64_t ldy, hif4_round mode, void* workspace,
                        size_t workspace_bytes, void* stream);

hif4_status hif4_grouped_gemm_workspace(int num_groups, int64_t total_rows, int64_t N, int64_t K,
                                        size_t* bytes);

/* hif4_grouped_gemm -- the same contraction per group g (an MoE expert, Section IV-B converts the
 * MoE linears):  C[off[g]:off[g+1], :] = A[off[g]:off[g+1], :] * B[g]^T.
 *   A_units            device, [total_rows, K/64] units, rows sorted by group.
 *   B_units            device, [num_groups, N, K/64] units.
 *   C                  device, [total_rows, N] FP32, row stride ldc.
 *   group_offsets_dev  device, num_groups+1 int64 prefix sums, off[0] = 0, off[num_groups] <=
 *                      total_rows, non-decreasing.  Read by the kernel only: routing results never
 *                      return to the host.  Empty groups are allowed.  Rows of C at and behind
 *                      off[num_groups] (assignments without a row here: padding, experts held elsewhere)
 *                      stay as they were.  Offsets are clamped to 0 .. total_rows.  */
hif4_status hif4_grouped_gemm(const void* A_units, const void* B_units, float* C,
                              const int64_t* group_offsets_dev, int num_groups, int64_t total_rows,
                              int64_t N, int64_t K, int64_t ldc, void* workspace,
                              size_t workspace_bytes, void* stream);

/* hif4_grouped_gemm_noalloc -- hif4_grouped_gemm without a workspace argument.  (The paper has no
 * counterpart: this is a packaging variant of the call above, not another operation.)
 *
 * For callers that cannot allocate device memory: code running under a fixed memory plan that was
 * sized at start-up, a plug-in that receives tensors but no allocator, or a section where the
 * device-wide synchronisation of a cudaMalloc is not acceptable.  The tile table that the
 * tensor-core kernel needs lives in a __device__ array of HIF4_NOALLOC_SCRATCH_BYTES bytes inside
 * the library; every GPU that loads the library holds it until the process exits.  The call itself
 * performs no cudaMalloc / cudaFree and uses no allocating library routine.
 *
 *   Arguments are those of hif4_grouped_gemm.  The result meets the same tolerance; it comes from the
 *   single-CTA tensor-core kernel (128-row tiles), whereas hif4_grouped_gemm normally runs the CTA-pair
 *   kernel, so the FP32 summation order and therefore the last bits of C may differ between the two.
 *   Limit     ceil(total_rows / 128) + num_groups table entries of 16 bytes, rounded up to 256,
 *             must fit in HIF4_NOALLOC_SCRATCH_BYTES (65536: e.g. 256 groups and 491520 rows);
 *             beyond that the call returns HIF4_ERR_WORKSPACE and launches nothing.
 *   Sharing   all calls on one GPU use the same array.  Calls ordered on one stream are safe (each
 *             call rewrites every entry it reads; nothing has to be zero beforehand).  Calls that
 *             may overlap on the GPU -- different streams or host threads without ordering -- race
 *             on the table and produce wrong results.
 *   Set-up    the first call on each GPU looks up the array's device address
 *             (cudaGetSymbolAddress, with that GPU current) and keeps it; make that first call
 *             outside any stream capture.
 * hif4_debug_set_gemm_path does not apply to this call.  */
#define HIF4_NOALLOC_SCRATCH_BYTES 65536
hif4_status hif4_grouped_gemm_noalloc(const void* A_units, const void* B_units, float* C,
                                      const int64_t* group_offsets_dev, int num_groups,
                                      int64_t total_rows, int64_t N, int64_t K, int64_t ldc,
                                      void* stream);

/* Size in bytes of the built-in scratch array (HIF4_NOALLOC_SCRATCH_BYTES).  Host-only.  */
size_t hif4_grouped_gemm_noalloc_capacity(void);

/* ---------------------------------------------------------------------------------------------
 * What stands between two HiF4 linears of a transformer block.  The paper converts the inputs of every linear layer
 * (Section IV); the calls below produce those inputs and consume the products without a round trip through FP32
 * matrices: the norms before and after a block, the linear with its epilogue, the gated feed-forward, each with its
 * backward pass.  Weights are codes and therefore constants here: the backward passes give the gradients of
 * activations, biases, norm weights and gates, and pass straight through the conversion of the activations.
 *
 * All arithmetic outside Algorithm 1 and Eq. 3 is FP32; a result is rounded once, to the type it is stored in.
 * Matrices that a call writes must not overlap what it reads, except where a parameter says so. */
typedef enum { HIF4_NORM_NONE = 0, HIF4_NORM_RMS = 1, HIF4_NORM_LAYER = 2 } hif4_norm_kind;
typedef enum {
  HIF4_ACT_NONE = 0,
  HIF4_ACT_RELU = 1,       /* max(z, 0)                                              */
  HIF4_ACT_SILU = 2,       /* z / (1 + e^-z)                                         */
  HIF4_ACT_GELU = 3,       /* z Phi(z), Phi the normal distribution function         */
  HIF4_ACT_GELU_TANH = 4   /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2        */
} hif4_activation;         /* within (8 + 2 |e|) 2^-22 of the value in FP32, e the formula's exponent: -z (SiLU), z^2 / 2 (GELU), twice
                              the argument of tanh; a sigmoid below 2^-126 is zero */

/* hif4_block_norm -- the norms around a block with its gate and residual, per row of `cols` elements:
 *     h = res_scale * residual + gate[row / rows_per_gate] * post(x)
 *     y = pre(h)
 *   RMS   v * w / sqrt(mean(v^2) + eps)              LAYER   (v - mean v) * w / sqrt(mean((v - mean v)^2) + eps) + b
 *   x is the output of the block that ends here, `post` the norm on it (NONE: x itself), `pre` the norm in front of
 *   the next block.  y is taken from h before h is rounded.  */
typedef struct {
  int64_t rows, cols;            /* cols <= 32768                                                              */
  hif4_dtype dt;                 /* type of x, residual, gate, h and y: BF16, FP16 or FP32                     */
  hif4_dtype dt_w;               /* type of the weights and of the bias                                        */
  const void* x;                 /* device, [rows, cols], row stride ld_x elements                             */
  int64_t ld_x;
  const void* residual;          /* device, [rows, cols], or NULL: no residual                                 */
  int64_t ld_residual;
  float res_scale;
  const void* gate;              /* device, [ceil(rows / rows_per_gate), cols], or NULL: 1                     */
  int64_t ld_gate;
  int64_t rows_per_gate;         /* rows that share a row of gates, >= 1 when there is a gate                  */
  hif4_norm_kind post;
  const void* post_weight;       /* device, [cols], or NULL: 1                                                 */
  hif4_norm_kind pre;            /* NONE: y must be NULL (only h is wanted)                                    */
  const void* pre_weight;        /* device, [cols], or NULL: 1                                                 */
  const void* pre_bias;          /* device, [cols], or NULL: 0 (LAYER only)                                    */
  float eps;                     /* >= 0                                                                       */
  void* h;                       /* device, [rows, cols], or NULL: not stored; may be x or residual itself     */
  int64_t ld_h;
  void* y;                       /* device, [rows, cols] of dt, or HiF4 units [rows, cols / 64] (4-byte aligned) */
  int64_t ld_y;                  /* (elements; not used for units)                                             */
  int y_units;                   /* 1: y is hif4_quantize of what y would be in dt; cols % 64 == 0             */
  hif4_round mode;               /* rounding of that conversion                                                */
} hif4_block_norm_args;
hif4_status hif4_block_norm(const hif4_block_norm_args* args, void* stream);

/* hif4_block_norm_backward -- gradients of hif4_block_norm from dy (of y), dh (of h, from the residual stream), the
 * stored h and x.  With n the normalised row of h, rstd its factor, and dn = dy * w:
 *     dt = dh + rstd * (dn - n mean(dn n) - [LAYER] mean(dn))
 *     dresidual = res_scale dt,  dweight = sum dy n,  dbias = sum dy,  dgate = sum over the gate's rows of dt post(x)
 *   and dx likewise through gate and post norm.  Statistics are taken again from h and x (nothing but them is kept
 *   from the forward pass).  Gradients of weights are FP32 and overwritten; their sums run in an order that depends
 *   only on the sizes.  Outputs that are NULL are not computed.  */
typedef struct {
  int64_t rows, cols;
  hif4_dtype dt, dt_w;
  const void* dy;                /* [rows, cols], or NULL: 0 (then pre does not matter)                        */
  int64_t ld_dy;
  const void* dh;                /* [rows, cols], or NULL: 0; at least one of dy and dh                        */
  int64_t ld_dh;
  const void* h;                 /* [rows, cols] as stored by the forward pass; not read when dy is NULL       */
  int64_t ld_h;
  const void* x;                 /* [rows, cols]; needed for post != NONE and for dgate                        */
  int64_t ld_x;
  float res_scale;
  const void* gate;
  int64_t ld_gate, rows_per_gate;
  hif4_norm_kind post;
  const void* post_weight;
  hif4_norm_kind pre;
  const void* pre_weight;
  float eps;
  void* dx;                      /* [rows, cols] of dt or NULL                                                 */
  int64_t ld_dx;
  void* dresidual;               /* [rows, cols] of dt or NULL; dx and dresidual may not be the same           */
  int64_t ld_dresidual;
  void* dgate;                   /* [ceil(rows / rows_per_gate), cols] of dt, contiguous, or NULL              */
  float* dpre_weight;            /* [cols] or NULL                                                             */
  float* dpre_bias;              /* [cols] or NULL (LAYER only)                                                */
  float* dpost_weight;
} hif4_block_norm_backward_args;
hif4_status hif4_block_norm_backward_workspace(int64_t rows, int64_t cols, size_t* bytes);
hif4_status hif4_block_norm_backward(const hif4_block_norm_backward_args* args, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* hif4_linear_act -- the linear layer with its epilogue:
 *     Y = act(HiF4(X) * W^T + bias) + res_scale * residual
 * hif4_gated_linear -- the gated feed-forward's first half, two projections of the same activations:
 *     Y = act(HiF4(X) * W^T + bias) * (HiF4(X) * W_up^T + bias_up) + res_scale * residual
 * The products are those of hif4_gemm; everything behind them is FP32 until Y is rounded to `dt`.  One token takes the
 * weight-streaming form, a prompt the tensor-core form, as in hif4_linear.  */
typedef struct {
  int64_t M, N, K;               /* K % 64 == 0                                                                */
  const void* X;                 /* device, [M, K] of dt_x, rows 16-byte aligned, or HiF4 units [M, K / 64]    */
  int64_t ld_x;                  /* (elements; not used for units)                                             */
  hif4_dtype dt_x;
  int x_units;                   /* 1: X holds units already                                                   */
  hif4_round mode;               /* rounding of the conversions to units                                       */
  const void* W_units;           /* device, [N, K / 64] units                                                  */
  const void* W_up_units;        /* the same; hif4_gated_linear only                                           */
  hif4_dtype dt;                 /* type of bias, residual and Y: BF16, FP16 or FP32                           */
  const void* bias;              /* device, [N], or NULL                                                       */
  const void* bias_up;           /* device, [N], or NULL; hif4_gated_linear only                               */
  hif4_activation act;
  const void* residual;          /* device, [M, N], or NULL                                                    */
  int64_t ld_residual;
  float res_scale;
  void* Y;                       /* device, [M, N] of dt (may be residual itself), or units [M, N / 64] (4-byte aligned) */
  int64_t ld_y;
  int y_units;                   /* 1: Y is hif4_quantize of what it would be in dt; N % 64 == 0               */
} hif4_linear_act_args;
/* Device scratch for these arguments (sizes, types and flags are read, no pointer is followed), 256-byte aligned.  */
hif4_status hif4_linear_act_workspace(const hif4_linear_act_args* args, size_t* bytes);
hif4_status hif4_linear_act(const hif4_linear_act_args* args, void* workspace, size_t workspace_bytes, void* stream);
hif4_status hif4_gated_linear_workspace(const hif4_linear_act_args* args, size_t* bytes);
hif4_status hif4_gated_linear(const hif4_linear_act_args* args, void* workspace, size_t workspace_bytes, void* stream);

/* hif4_linear_act_backward, hif4_gated_linear_backward -- gradients with respect to the activations and the biases from
 * dY, the weights being constants and the conversion of X passed straight through.  The products are taken again
 * from X (nothing else is kept from the forward pass):
 *     dZ = dY * act'(Z),  dX = dZ * W,  dbias = sum over the rows of dZ
 *     dG = dY * U * act'(G),  dU = dY * act(G),  dX = dG * W + dU * W_up,  dbias = sum dG,  dbias_up = sum dU
 * (the residual's gradient is res_scale * dY).  dZ, dG and dU enter the last product as sums of BF16 numbers: one for
 * BF16 gradients (two with `precise`), two for FP16 (which hold its 11 bits); sums of biases run over the unrounded values,
 * in an order that depends only on the sizes.  FP32 gradients are refused (HIF4_ERR_DTYPE).  */
typedef struct {
  int64_t M, N, K;
  const void* X;                 /* as in the forward pass; not read by hif4_linear_act_backward for act NONE   */
  int64_t ld_x;
  hif4_dtype dt_x;
  int x_units;
  hif4_round mode;
  const void* W_units;
  const void* W_up_units;
  hif4_dtype dt;                 /* type of the biases, dY and dX: BF16 or FP16                                 */
  const void* bias;
  const void* bias_up;
  hif4_activation act;
  const void* dY;                /* device, [M, N]                                                             */
  int64_t ld_dy;
  void* dX;                      /* device, [M, K], or NULL                                                    */
  int64_t ld_dx;
  float* dbias;                  /* device, [N], or NULL; overwritten                                          */
  float* dbias_up;
  int precise;                   /* 1: dZ, dG and dU as two BF16 numbers for BF16 gradients too                 */
} hif4_linear_act_backward_args;
hif4_status hif4_linear_act_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes);
hif4_status hif4_linear_act_backward(const hif4_linear_act_backward_args* args, void* workspace, size_t workspace_bytes,
                                     void* stream);
hif4_status hif4_gated_linear_backward_workspace(const hif4_linear_act_backward_args* args, size_t* bytes);
hif4_status hif4_gated_linear_backward(const hif4_linear_act_backward_args* args, void* workspace, size_t workspace_bytes,
                                       void* stream);

/* hif4_mse_roundtrip -- the quantization-error experiment of Section III-A for one tensor: convert a BF16 tensor
 * to a 4-bit block format and back, write the image as FP32 and sum the squared error against the source.
 *   HIF4_FMT_HIF4       Algorithm 1 (round-half-to-even), then Eq. 2
 *   HIF4_FMT_MXFP4      blocks of 32, power-of-two scale 2^(floor(log2 amax) - 2), E2M1 elements
 *   HIF4_FMT_NVFP4      blocks of 16, E4M3 scale = amax / 6, E2M1 elements ("direct cast")
 *   HIF4_FMT_NVFP4_PTS  NVFP4 after per-tensor scaling of the peak magnitude to 2688, undone afterwards
 * (E2M1 and E4M3 rounding to nearest, ties to even, saturating; every step one FP32 operation.)
 *   src_bf16    device, n BF16 elements, 16-byte aligned; n a multiple of 64.
 *   dst         device, n FP32 elements receiving the image, or NULL when only the error is wanted.
 *   sq_err_sum  device, one FP64: sum over the elements of (image - source)^2, accumulated in FP64 in an order
 *               that does not depend on scheduling.
 *   workspace   device scratch of at least hif4_mse_workspace bytes, 256-byte aligned.  */
typedef enum { HIF4_FMT_HIF4 = 0, HIF4_FMT_MXFP4 = 1, HIF4_FMT_NVFP4 = 2, HIF4_FMT_NVFP4_PTS = 3 } hif4_bfp4_format;
hif4_status hif4_mse_workspace(int64_t n, hif4_bfp4_format fmt, size_t* bytes);
hif4_status hif4_mse_roundtrip(const void* src_bf16, int64_t n, hif4_bfp4_format fmt, float* dst, double* sq_err_sum,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * What stands around the experts' products of a mixture-of-experts layer: which experts a token goes to, the experts' rows
 * in the order that hif4_grouped_gemm and hif4_bfp4_grouped_gemm read, and the weighted sum of what comes back.
 * Routing results stay on the device.  Matrices that a call writes must not overlap what it reads, except where a parameter
 * says so.  */
#define HIF4_ROUTE_MAX_EXPERTS 1024
#define HIF4_ROUTE_MAX_TOP_K 32
#define HIF4_ROUTE_MAX_GROUPS 32
typedef enum { HIF4_SCORE_SOFTMAX = 0, HIF4_SCORE_SIGMOID = 1 } hif4_score;

/* hif4_route -- per token: scores s of the logits, choice c = s + bias, the `top_k` experts of the largest choice in
 * descending order (equal ones: the lowest index first), and their weights w = scale * s, or scale * s / (sum of the chosen s).
 *   groups    the experts are `groups` equal runs; a run's value is the sum of its `group_best` (1 or 2) largest choices (-inf where
 *             fewer can be chosen), and only experts of the `top_groups` runs of the largest value are chosen.
 *   The order is that of the choices in 64 bits (of the logits themselves where there is no bias and no sum of two).
 *   Experts whose choice is -inf are not chosen: where none is left, the id is -1 and the weight 0.  A NaN counts as -inf in
 *   the choice, and every weight of its row is NaN (so too for an infinite logit under softmax).
 * Limits: experts <= 1024, top_k <= 32, groups <= 32 (HIF4_ERR_UNSUPPORTED); top_k <= top_groups * experts / groups.  */
typedef struct {
  int64_t tokens, experts, top_k;
  const void* logits;            /* device, [tokens, experts] of dt, row stride ld_logits elements              */
  hif4_dtype dt;                 /* BF16, FP16 or FP32                                                         */
  int64_t ld_logits;
  const float* bias;             /* device, [experts], or NULL: 0                                              */
  hif4_score score;
  int64_t groups, top_groups, group_best;
  int renormalize;               /* 1: weights of a token add up to scale                                      */
  float scale;
  int32_t* ids;                  /* device, [tokens, top_k]                                                    */
  float* weights;                /* device, [tokens, top_k]                                                    */
} hif4_route_args;
hif4_status hif4_route(const hif4_route_args* args, void* stream);

/* hif4_route_backward -- gradient of the weights with respect to the logits (the choice itself has none, nor has the
 * bias): dlogits [tokens, experts] of dt, every element written.  Ids outside 0 .. experts - 1 take no part.  */
typedef struct {
  int64_t tokens, experts, top_k;
  const void* logits;
  hif4_dtype dt;
  int64_t ld_logits;
  const int32_t* ids;            /* device, [tokens, top_k], as hif4_route wrote them                          */
  const float* dweights;         /* device, [tokens, top_k]                                                    */
  hif4_score score;
  int renormalize;
  float scale;
  void* dlogits;                 /* device, [tokens, experts] of dt                                            */
  int64_t ld_dlogits;
} hif4_route_backward_args;
hif4_status hif4_route_backward(const hif4_route_backward_args* args, void* stream);

/* hif4_expert_plan -- the order of the experts' rows: offsets[e] counts the assignments to experts below e
 * (experts + 1 of them, what the grouped products take), row_of[t][j] is the row of assignment j of token t: rows are sorted by
 * expert and within an expert by token and place.  Ids outside 0 .. experts - 1 (padding, experts held elsewhere) have no
 * row: -1.  tokens * top_k < 2^31; experts <= 1024.
 *   workspace  device scratch, 256-byte aligned, of hif4_expert_plan_workspace bytes (0 for few assignments).  */
hif4_status hif4_expert_plan_workspace(int64_t tokens, int64_t top_k, int64_t experts, size_t* bytes);
hif4_status hif4_expert_plan(const int32_t* ids, int64_t tokens, int64_t top_k, int64_t experts, int64_t* offsets, int32_t* row_of,
                             void* workspace, size_t workspace_bytes, void* stream);

/* What hif4_dispatch writes: rows of x as they are, or converted. */
typedef enum { HIF4_ROWS_PLAIN = 0, HIF4_ROWS_HIF4 = 1, HIF4_ROWS_MXFP4 = 2, HIF4_ROWS_NVFP4 = 3 } hif4_rows_kind;

/* hif4_dispatch -- the experts' rows: out[row_of[t][j]] = x[t] for every assignment that has a row; a token is read and
 * converted once.  Converted rows are bit for bit those of hif4_quantize and hif4_bfp4_quantize.  Rows that no assignment
 * has stay as they were; a row number outside 0 .. rows - 1 is no row.  Row numbers differ (hif4_expert_plan's do): where two assignments have
 * the same one, its row may be made of parts of both tokens.  (Its gradient is hif4_combine without weights.)  */
typedef struct {
  int64_t tokens, cols, top_k, rows;
  const void* x;                 /* device, [tokens, cols] of dt, row stride ld_x elements; 16-byte aligned rows unless PLAIN */
  hif4_dtype dt;
  int64_t ld_x;
  const int32_t* row_of;         /* device, [tokens, top_k]                                                    */
  hif4_rows_kind kind;           /* all but PLAIN: cols % 64 == 0                                              */
  hif4_round mode;               /* HIF4 only                                                                  */
  const float* gain;             /* MXFP4, NVFP4: as in hif4_bfp4_quantize, or NULL                            */
  void* out;                     /* device, [rows, cols] of dt; units [rows, cols / 64]; codes [rows, cols / 2] */
  int64_t ld_out;                /* PLAIN only                                                                 */
  void* out_scales;              /* MXFP4, NVFP4: scales of `rows` rows                                        */
} hif4_dispatch_args;
hif4_status hif4_dispatch(const hif4_dispatch_args* args, void* stream);

/* hif4_combine -- y[t] = res_scale * residual[t] + sum over j of weights[t][j] * in[row_of[t][j]], added in the order of j in
 * FP32; assignments without a row (outside 0 .. rows - 1) take no part.  */
typedef struct {
  int64_t tokens, cols, top_k, rows;
  const void* in;                /* device, [rows, cols] of dt_in, row stride ld_in elements                   */
  hif4_dtype dt_in;
  int64_t ld_in;
  const int32_t* row_of;         /* device, [tokens, top_k]                                                    */
  const float* weights;          /* device, [tokens, top_k], or NULL: 1                                        */
  hif4_dtype dt;                 /* type of residual and y                                                     */
  const void* residual;          /* device, [tokens, cols], or NULL: 0                                         */
  int64_t ld_residual;
  float res_scale;
  void* y;                       /* device, [tokens, cols]; may be residual itself                             */
  int64_t ld_y;
} hif4_combine_args;
hif4_status hif4_combine(const hif4_combine_args* args, void* stream);

/* hif4_combine_backward -- din[row_of[t][j]] = weights[t][j] * dy[t], dweights[t][j] = <dy[t], in[row_of[t][j]]> (0 without a
 * row); the residual's gradient is res_scale * dy.  Rows of din that no assignment has stay as they were; row numbers differ,
 * as for hif4_dispatch.  */
typedef struct {
  int64_t tokens, cols, top_k, rows;
  const void* dy;                /* device, [tokens, cols] of dt                                               */
  hif4_dtype dt;
  int64_t ld_dy;
  const int32_t* row_of;
  const float* weights;          /* or NULL: 1                                                                 */
  const void* in;                /* device, [rows, cols] of dt_in; needed for dweights                         */
  hif4_dtype dt_in;              /* type of in and din                                                         */
  int64_t ld_in;
  void* din;                     /* device, [rows, cols], or NULL                                              */
  int64_t ld_din;
  float* dweights;               /* device, [tokens, top_k], or NULL                                           */
} hif4_combine_backward_args;
hif4_status hif4_combine_backward(const hif4_combine_backward_args* args, void* stream);

/* ---------------------------------------------------------------------------------------------
 * The microscaled 4-bit formats that Section III-A compares HiF4 with, as packed operands and products on the tensor
 * core's own block-scaled instructions.  `fmt` is HIF4_FMT_MXFP4 (blocks of 32, scale a power of two: E8M0) or HIF4_FMT_NVFP4
 * (blocks of 16, scale E4M3); elements are E2M1.  The conversion is that of hif4_mse_roundtrip, step by step.
 *
 * A packed matrix [rows, cols], cols % 64 == 0, is two arrays:
 *   codes    [rows, cols / 2] bytes; element i in byte i / 2, low nibble for even i; sign in the nibble's top bit.
 *   scales   [ceil(cols / block / 16), rows, 16] bytes: the scales of sixteen consecutive blocks of a row are one 16-byte
 *            word, and the words of all rows lie side by side (any run of rows is one contiguous copy for the product).
 *            Bytes past the last block are written as 0 and never read.
 * A gain (device, one FP32) is multiplied in before the conversion, which then works on FP32 products: out of range
 * tensors are brought into range with it, and products undo it with alpha = 1 / (gain_a * gain_b).
 * A block that holds a NaN has a NaN scale and zero codes; infinities saturate.  */
size_t hif4_bfp4_scale_bytes(int64_t rows, int64_t cols, hif4_bfp4_format fmt);

/* Conversion along the rows.  src: device, [rows, cols] of dt (BF16, FP16, FP32), rows 16-byte aligned.  codes and scales:
 * 16-byte aligned, fully overwritten.  */
hif4_status hif4_bfp4_quantize(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld_src, hif4_bfp4_format fmt,
                               const float* gain, void* codes, void* scales, void* stream);
/* Conversion down the columns: codes and scales of the transposed matrix [cols, rows]; rows % 64 == 0, cols % 8 == 0.  With it the
 * products of a backward pass, which contract along other dimensions, take their operands: dX = dY W from dY's rows and W's columns,
 * dW = dY^T X from the columns of both.  */
hif4_status hif4_bfp4_quantize_transposed(const void* src, hif4_dtype dt, int64_t rows, int64_t cols, int64_t ld_src,
                                          hif4_bfp4_format fmt, const float* gain, void* codes, void* scales, void* stream);
/* Values in FP32 (6 * 2^126, which an infinity becomes in MXFP4, is one again), divided by the gain if there is one, rounded to dst:
 * BF16 or FP32, rows 16-byte aligned (exact without a gain; FP16 is refused as in hif4_dequantize).  */
hif4_status hif4_bfp4_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, hif4_bfp4_format fmt,
                                 const float* gain, void* dst, hif4_dtype dt, int64_t ld_dst, void* stream);

/* hif4_bfp4_gemm -- Y = alpha * A * B^T; hif4_bfp4_grouped_gemm -- the same per group g of rows, Y[off[g]:off[g+1]] =
 * alpha[g] * A[off[g]:off[g+1]] * B[g]^T.  FP32 accumulation, Y rounded once.  Rows of Y at and behind off[num_groups] stay as
 * they were; offsets are clamped to 0 .. M.  */
typedef struct {
  int64_t M, N, K;               /* K > 0, K % 64 == 0                                                         */
  hif4_bfp4_format fmt;          /* of both operands                                                           */
  const void* A_codes;           /* device, [M, K / 2], 16-byte aligned                                        */
  const void* A_scales;          /* device, scales of M rows                                                   */
  const void* B_codes;           /* device, [N, K / 2], or [num_groups, N, K / 2]                              */
  const void* B_scales;          /* device, scales of N rows, num_groups times                                 */
  const float* alpha;            /* device, one FP32, or [num_groups], or NULL: 1                              */
  hif4_dtype dt;                 /* of Y: BF16, FP16 or FP32                                                   */
  void* Y;                       /* device, [M, N], row stride ld_y elements                                   */
  int64_t ld_y;
  int num_groups;                /* grouped only                                                               */
  const int64_t* group_offsets;  /* grouped only: device, num_groups + 1                                       */
} hif4_bfp4_gemm_args;
hif4_status hif4_bfp4_gemm(const hif4_bfp4_gemm_args* args, void* stream);
hif4_status hif4_bfp4_grouped_gemm(const hif4_bfp4_gemm_args* args, void* stream);

/* Synchronises `stream` and returns HIF4_ERR_DEVICE_TIMEOUT if any kernel of this library gave up
 * a bounded wait since the last call (the flag is cleared), HIF4_ERR_CUDA if the stream reports
 * an error, else HIF4_OK.  For tests and debugging.  */
hif4_status hif4_last_device_status(void* stream);

/* Static, NUL-terminated description of a status code.  Host-only.  */
const char* hif4_status_string(hif4_status s);

/* ---------------------------------------------------------------------------------------------
 * Test and benchmark hooks (hif4_debug_*).  Not part of the product surface: nothing above depends on
 * them except that hif4_gemm honours the path override while it is set.
 *
 * hif4_debug_set_gemm_path: 0 = choose the GEMM kernel by shape (default), 1 = CUDA-core kernel only,
 * 2 = the single-CTA tensor-core (tcgen05) kernel whenever it is legal (K % 256 == 0, 16-byte aligned
 * operands), even for small M, 3 = the CTA-pair tensor-core kernel (256 x 256 tiles) whenever it is legal,
 * 4 = the weight-streaming kernel whenever it is legal (M <= 32), 5 = the variant of that kernel that follows
 * Eq. 3's factorisation (FP8 E4M3 tensor-core operands holding the elements with their micro-exponents, the two
 * level-1 scales applied to each unit pair's sum) whenever it is legal (M <= 32), 6 = hif4_linear converts BF16
 * activations inside the CTA-pair kernel whenever that is legal (M > 128).  Process-wide and not thread-safe.
 * hif4_gemm_workspace does not depend on it: it always reports the largest need over all paths.
 *
 * hif4_debug_launch_count: number of kernels this library has launched in this process (monotonic,
 * host-side counter).  */
hif4_status hif4_debug_set_gemm_path(int path);
uint64_t hif4_debug_launch_count(void);

/* hif4_debug_wait_timeout: launches a one-block kernel that waits on an mbarrier nobody arrives on, with the
 * same bounded-wait helper the GEMM kernels use but a budget of `budget_ns` (1 .. 100 000 000) instead of their
 * 2 s.  The wait runs out, the kernel raises the device error word and returns normally; the next
 * hif4_last_device_status on that stream returns HIF4_ERR_DEVICE_TIMEOUT, the one after it HIF4_OK.  Nothing
 * faults or hangs: no copy or MMA is in flight.  (The paper has no counterpart; this exercises the library's
 * failure reporting.)  */
hif4_status hif4_debug_wait_timeout(uint64_t budget_ns, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HIF4_H_ */
