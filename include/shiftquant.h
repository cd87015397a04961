/*
 * shiftquant.h -- C ABI of libshiftquant, the ShiftQuant backward path for
 * AMD Instinct MI355X (gfx950).
 *
 * ShiftQuant ("Towards Accurate and Efficient Sub-8-Bit Integer Training",
 * arXiv 2411.10948) quantizes the output gradient G_B = dY [M, C_out] of a
 * linear (or im2col'd conv) layer to b-bit integers whose channels fall into
 * N_G groups with power-of-two scales (Sec. 3.1), so that both backward GEMMs
 *     dX = dY . W      (loss propagation, inner dimension C_out)
 *     dW = dY^T . X    (weight gradient,  inner dimension M)
 * run as plain integer GEMMs with the group scales applied as bit shifts
 * (Sec. 3.2, "ShiftMM"; App. D).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every array argument is a DEVICE pointer owned by the caller.  The
 *    library never allocates device memory, never frees caller memory and
 *    never synchronizes the host: all work is enqueued on `stream` (a
 *    hipStream_t passed as void*, NULL = the default stream) and completes
 *    in stream order.  Scratch memory is passed in as `workspace`; its size
 *    comes from the matching *_workspace_size query.
 *  - Matrices are row-major with a leading dimension `ld` in elements;
 *    a buffer [rows, ld] must hold rows * ld elements.
 *  - int8 code matrices (q_fold, q_t, wq_t, xq_t) and the workspace must be
 *    16-byte aligned with ld a multiple of 16.  fp32/int32 arrays must be
 *    4-byte aligned.
 *  - Arguments are validated synchronously before anything is launched; on
 *    failure nothing is enqueued and a status other than SQ_OK is returned.
 *    sq_last_error() then describes the failure (thread-local).
 *  - Data-dependent anomalies cannot be seen on the host: they are reported
 *    in the `flags` word of the device-resident sq_scale and the codes are
 *    then all 0 (see SQ_FLAG_*).
 *  - Calls that share a workspace, layout or output buffer must not overlap
 *    in time (enqueue them on one stream, or synchronize between them).
 */
#ifndef SHIFTQUANT_H
#define SHIFTQUANT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SQ_OK = 0,
    SQ_ERR_INVALID_ARGUMENT = 1,   /* null pointer, bad size, stride or alignment  */
    SQ_ERR_OVERFLOW_RISK = 2,      /* the worst-case int32 accumulator would overflow */
    SQ_ERR_UNSUPPORTED = 3,        /* valid request outside what the library supports */
    SQ_ERR_WORKSPACE_TOO_SMALL = 4,
    SQ_ERR_HIP = 5                 /* a HIP runtime call or kernel launch failed     */
} sq_status;

/* Rounding of the gradient codes. */
enum {
    SQ_ROUND_NEAREST_EVEN = 0,     /* round(.) of App. D, ties to even                 */
    SQ_ROUND_STOCHASTIC = 1        /* SR of App. B, Eq. "sq", Philox4x32-10 uniforms   */
};

/* Bits of sq_scale.flags.  When either is set every code is 0, every channel
 * is in the last group and inv = step = 0. */
enum {
    SQ_FLAG_NONFINITE = 1u,        /* the tensor holds NaN or +-Inf                     */
    SQ_FLAG_ZERO = 2u              /* max |x| < 2^-96 (all-zero, tiny or empty tensor)  */
};

/* Layout of the int8 code matrices a call writes or reads (sq_quant_params.layout).
 *   SQ_LAYOUT_ROWS  row-major: element (r, k) at r * ld + k.
 *   SQ_LAYOUT_TILED tile-major: element (r, k) at
 *                     ((r / 16) * (ld / 64) + k / 64) * 1024 + (r % 16) * 64 + k % 64,
 *                   i.e. 16 x 64 tiles of 1 KB, the tiles of a 16-row group in
 *                   order of k.  ld must be a multiple of 64 and the buffer
 *                   must hold roundup(rows, 16) * ld bytes.  The GEMMs read
 *                   one K tile of 16 rows as one contiguous 1 KB block, which
 *                   keeps their operand streams sequential in HBM.  Writers fill
 *                   the K padding up to the next multiple of 64 with zeros
 *                   (q_fold columns [C_out, roundup(C_out, 64)), q_t and
 *                   transposed tensor columns [rows, roundup(rows, 64))).
 *                   Taken by sq_quantize_grad(_noalloc, _from_ranges),
 *                   sq_gemm_dgrad(_ranged), sq_gemm_wgrad and sq_quantize_tensor
 *                   (transpose = 2); the other calls that take sq_quant_params
 *                   return SQ_ERR_UNSUPPORTED for it. */
enum {
    SQ_LAYOUT_ROWS = 0,
    SQ_LAYOUT_TILED = 1
};

/* Quantizer parameters (host memory, read during the call only). */
typedef struct {
    int32_t bits;         /* b in [2, 8]: codes lie in [-Q, Q], Q = 2^(b-1) - 1            */
    int32_t num_groups;   /* N_G in [1, 8] (the paper's default is 4, Sec. 5.1)            */
    int32_t round_mode;   /* SQ_ROUND_*                                                    */
    int32_t layout;       /* SQ_LAYOUT_*: layout of the int8 code matrices of the call     */
    uint64_t seed;        /* stochastic rounding: Philox key                               */
    uint64_t offset;      /* stochastic rounding: stream offset (e.g. the training step)   */
} sq_quant_params;

/* Device-resident scale of a quantized tensor (written by the quantizers,
 * read by the GEMMs and sq_dequant).
 *   r_max : tau_0, the tensor's absolute maximum (Sec. 3.1)
 *   inv   : s = fl(Q / r_max), the scale of group 0 (App. B writes SR(X S) S^-1)
 *   step  : s^-1 = fl(r_max / Q), the quantization step of group 0
 *   flags : SQ_FLAG_* */
typedef struct {
    float r_max;
    float inv;
    float step;
    uint32_t flags;
} sq_scale;

/* ---------------------------------------------------------------------------
 * Size queries (host only, no device work).
 * ------------------------------------------------------------------------- */

/* Layout descriptor of the shift-folded dgrad operand produced by
 * sq_quantize_grad and consumed by sq_gemm_dgrad.
 *   *layout_bytes : size of the device buffer `layout`
 *   *min_ld_fold  : smallest admissible ld_fold for q_fold (a multiple of 16);
 *                   q_fold rows hold C_out main columns followed, from column
 *                   roundup(C_out, 64), by the appended columns of the fold:
 *                   none when N_G - 1 <= T (see sq_quantize_grad), else at
 *                   most roundup(C_out, 64) + 64 (N_G - 1). */
sq_status sq_grad_layout_size(int64_t C_out, const sq_quant_params* p,
                              size_t* layout_bytes, int64_t* min_ld_fold);

sq_status sq_quantize_grad_workspace_size(int64_t M, int64_t C_out, const sq_quant_params* p,
                                          size_t* bytes);
sq_status sq_quantize_tensor_workspace_size(int64_t rows, int64_t cols, size_t* bytes);
sq_status sq_gemm_dgrad_workspace_size(int64_t M, int64_t C_out, int64_t C_in,
                                       const sq_quant_params* p, size_t* bytes);
sq_status sq_gemm_wgrad_workspace_size(int64_t M, int64_t C_out, int64_t C_in,
                                       const sq_quant_params* p, size_t* bytes);

/* ---------------------------------------------------------------------------
 * sq_quantize_grad -- ShiftQuant of the output gradient.
 *
 * Follows Sec. 3.1 (channel ranges r_c, power-of-two thresholds
 * tau_g = r_max 2^-g), App. D (group g quantized with step
 * (r_max / Q) 2^-g) and App. B Eq. "sq" (stochastic rounding):
 *   r_c   = max_m |dY[m, c]|,  r_max = max_c r_c
 *   g_c   = the group whose interval (r_max 2^-(g+1), r_max 2^-g] holds r_c,
 *           the last group N_G - 1 also holding everything below
 *   v     = fl(dY[m, c] * fl(inv * 2^g_c)),  inv = fl(Q / r_max)
 *   code  = clamp(round(v), -Q, Q), round = ties-to-even or stochastic:
 *           floor(v) + [u16 < fl(v - floor(v)) * 2^16] with u16 the 16-bit
 *           half (i mod 2, low half first) of word (i / 2) mod 4 of
 *           Philox4x32-10(counter = (i / 8 as two 32-bit words, offset as two
 *           words), key = seed as two words), i = m * C_out + c.  One
 *           Philox block serves 8 elements; the rounding bias is below 2^-16
 *           of a step.
 *
 * Inputs : dY [M, ld_dY] fp32 (M >= 0, C_out >= 0, ld_dY >= C_out).
 * Outputs (any of q_fold / q_t may be NULL to skip it):
 *   q_fold [M, ld_fold] int8, the dgrad operand with the shifts of
 *          ShiftMM folded in.  The shifts sh_c = N_G - 1 - g_c are cut into
 *          windows [B, B + T] of T + 1 values, T the largest shift with
 *          Q 2^T <= 127, and each channel is stored once, as
 *          code << (sh_c - B) for its window's base B (this fits int8).  The
 *          window holding the most channels (lowest B on ties) uses the
 *          channel's own column c.  Every other non-empty window is a region
 *          of appended columns from column roundup(C_out, 64): its channels
 *          in ascending order, padded to a multiple of 64 columns; column c
 *          of such a channel holds 0.  When N_G - 1 <= T (b <= 5 at N_G = 4)
 *          there is one window and nothing is appended.  `layout` records
 *          the windows, and sq_gemm_dgrad applies their bases as left shifts
 *          of its accumulator.  Columns in [C_out, roundup(C_out, 64)) and
 *          the padding of appended regions are left unwritten (with
 *          SQ_LAYOUT_TILED the former are written as zeros).
 *   q_t    [C_out, ld_t] int8 (ld_t >= M), the codes themselves, transposed:
 *          q_t[c, m] = code(m, c); this is the wgrad operand.
 *   group  [C_out] uint8, g_c.
 *   scale  one sq_scale (r_max, inv, step, flags).
 *   layout [layout_bytes], the fold descriptor for sq_gemm_dgrad.
 * Workspace: sq_quantize_grad_workspace_size bytes.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_quantize_grad(const float* dY, int64_t M, int64_t C_out, int64_t ld_dY,
                           const sq_quant_params* p,
                           int8_t* q_fold, int64_t ld_fold,
                           int8_t* q_t, int64_t ld_t,
                           uint8_t* group, sq_scale* scale, int32_t* layout,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_quantize_grad_noalloc -- sq_quantize_grad without a workspace argument,
 * for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc).
 *
 * Same arguments, results and errors as sq_quantize_grad, minus workspace /
 * workspace_bytes.  Its scratch is a fixed 16 MiB device array inside the
 * library (one copy per GPU, held until the process ends); the call itself
 * allocates nothing.  A gradient whose quantizer scratch
 * (sq_quantize_grad_workspace_size) exceeds 1 MiB (about 65,000 channels) is rejected with
 * SQ_ERR_WORKSPACE_TOO_SMALL before any launch.  All calls on one GPU share
 * that array: calls that overlap in time on one GPU (other streams, other
 * host threads) race and must be serialized by the caller.  The first call
 * on a device looks up its scratch address (hipGetSymbolAddress) with that
 * device current.
 * ------------------------------------------------------------------------- */
sq_status sq_quantize_grad_noalloc(const float* dY, int64_t M, int64_t C_out, int64_t ld_dY,
                                   const sq_quant_params* p,
                                   int8_t* q_fold, int64_t ld_fold,
                                   int8_t* q_t, int64_t ld_t,
                                   uint8_t* group, sq_scale* scale, int32_t* layout, void* stream);

/* ---------------------------------------------------------------------------
 * sq_quantize_tensor -- per-tensor symmetric quantization of W or X.
 *
 * The paper's INT8 baseline quantizes weights, activations and gradients per
 * tensor (Sec. 5.1); it is ShiftQuant with a single group:
 *   a = max |T|,  inv = fl(Q / a),  step = fl(a / Q),
 *   code = clamp(round_half_even(fl(T * inv)), -Q, Q),  Q = 2^(bits-1) - 1.
 * Input : T [rows, ld] fp32 (ld >= cols).
 * Output: transpose == 0: q [rows, ld_q] int8 (ld_q >= cols)
 *         transpose == 1: q [cols, ld_q] int8 (ld_q >= rows), q[j, i] = code(i, j)
 *         transpose == 2: the same matrix tile-major (SQ_LAYOUT_TILED; ld_q a
 *         multiple of 64, >= roundup(rows, 64); columns [rows, roundup(rows,
 *         64)) written as zeros), the operand of the tile-major GEMMs
 *         (sq_gemm_dgrad takes W^T codes and sq_gemm_wgrad X^T codes, i.e.
 *         W [C_out, C_in] and X [M, C_in] quantized with transpose = 1).
 *         scale: one sq_scale.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_quantize_tensor(const float* T, int64_t rows, int64_t cols, int64_t ld, int32_t bits,
                             int32_t transpose, int8_t* q, int64_t ld_q, sq_scale* scale,
                             void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_quantize_channels -- per-channel symmetric quantization of a weight
 * matrix.
 *
 * Sec. 5.1 quantizes weights per output channel in the forward pass and per
 * input channel in loss propagation.  Each channel is quantized like a
 * tensor of its own (see sq_quantize_tensor): amax over the channel,
 * inv = fl(Q / amax), step = fl(amax / Q),
 * code = clamp(round_half_even(fl(T * inv)), -Q, Q); a channel whose amax is
 * NaN/Inf or below 2^-96 gets SQ_FLAG_NONFINITE / SQ_FLAG_ZERO in its scale
 * and all-zero codes.
 * Input : T [rows, ld] fp32; axis 0: one scale per row (W [C_out, C_in] per
 *         output channel), axis 1: one per column (per input channel).
 * Output: q as in sq_quantize_tensor (transpose 0: [rows, ld_q], 1:
 *         [cols, ld_q]); scales [rows] (axis 0) or [cols] (axis 1) sq_scale.
 * Workspace: sq_quantize_channels_workspace_size bytes (0 for axis 0).
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_quantize_channels_workspace_size(int64_t rows, int64_t cols, int32_t axis, size_t* bytes);
sq_status sq_quantize_channels(const float* T, int64_t rows, int64_t cols, int64_t ld, int32_t bits,
                               int32_t axis, int32_t transpose, int8_t* q, int64_t ld_q, sq_scale* scales,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_gemm_forward -- forward pass Y = X . W^T with ShiftQuant activations
 * and per-output-channel weights (Sec. 5.1; the first GEMM of Fig. "MMs").
 *
 * X is quantized by sq_quantize_grad (ShiftQuant groups over its channels,
 * which are this product's inner dimension), so the product is ShiftMM as in
 * sq_gemm_dgrad, with the weight scale taken per output column:
 *   acc[m, n] = sum_c (code_X(m, c) * wq[n, c]) << (N_G - 1 - g_c)     (int32)
 *   Y[m, n]   = fl(float(acc[m, n]) * gamma_n),
 *   gamma_n   = fl(fl(xscale.step * wscales[n].step) * 2^-(N_G - 1)).
 * The same call is loss propagation with per-input-channel weights: pass the
 * gradient's codes as X, W^T codes as wq and their per-column scales.
 * Inputs : xq_fold, ld_fold, layout, group, xscale from sq_quantize_grad of
 *          X [M, C_in] with the same p; wq [C_out, ld_w] int8 W codes
 *          (ld_w >= C_in) with wscales [C_out] from sq_quantize_channels
 *          (axis 0, transpose 0).
 * Outputs (either may be NULL, not both): acc [M, ld_acc] int32,
 *          Y [M, ld_Y] fp32.
 * Workspace: sq_gemm_dgrad_workspace_size(M, C_in, C_out, p) bytes.
 * Errors: SQ_ERR_INVALID_ARGUMENT; SQ_ERR_OVERFLOW_RISK when
 *         C_in * Q * 2^(N_G-1) * 128 >= 2^31; SQ_ERR_WORKSPACE_TOO_SMALL;
 *         SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_gemm_forward(const int8_t* xq_fold, int64_t ld_fold, const int32_t* layout,
                          const uint8_t* group, const sq_scale* xscale,
                          const int8_t* wq, int64_t ld_w, const sq_scale* wscales,
                          int64_t M, int64_t C_in, int64_t C_out, const sq_quant_params* p,
                          int32_t* acc, int64_t ld_acc, float* Y, int64_t ld_Y,
                          void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_gemm_dgrad -- loss propagation dX = dY . W as ShiftMM.
 *
 * Eq. "dq_mm_f" and App. D (left-shift form): with 0-indexed groups,
 *   acc[n, k] = sum_c (code(n, c) * wq[c, k]) << (N_G - 1 - g_c)      (int32)
 *   dX[n, k]  = fl(float(acc[n, k]) * alpha),
 *   alpha     = fl(fl(gscale.step * wscale.step) * 2^-(N_G - 1)).
 * Sec. 3.2 shifts every product before it is accumulated; here the shift of
 * each inner index c is folded into the int8 operand (q_fold) up to its
 * window's base B, and the bases are applied once per window to the int32
 * accumulator, which visits the windows in descending B (Horner's rule).
 * Inputs : q_fold, ld_fold, layout, group, gscale from sq_quantize_grad with
 *          the same M, C_out and p; wq_t [C_in, ld_w] int8 = W^T codes
 *          (ld_w >= C_out); wscale its sq_scale.
 * Outputs (either may be NULL, not both): acc [M, ld_acc] int32,
 *          dX [M, ld_dX] fp32.
 * Errors: SQ_ERR_INVALID_ARGUMENT; SQ_ERR_OVERFLOW_RISK when
 *         C_out * Q * 2^(N_G-1) * 128 >= 2^31; SQ_ERR_WORKSPACE_TOO_SMALL;
 *         SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_gemm_dgrad(const int8_t* q_fold, int64_t ld_fold, const int32_t* layout,
                        const uint8_t* group, const sq_scale* gscale,
                        const int8_t* wq_t, int64_t ld_w, const sq_scale* wscale,
                        int64_t M, int64_t C_out, int64_t C_in, const sq_quant_params* p,
                        int32_t* acc, int64_t ld_acc, float* dX, int64_t ld_dX,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_gemm_wgrad -- weight gradient dW = dY^T . X.
 *
 * The third training GEMM (Fig. "MMs"); its inner dimension is the token
 * index, so every output row c lies in one gradient group and the group
 * scale is a per-row factor (Eq. "dq_mm_f" applied to this product):
 *   acc[c, k] = sum_m code(m, c) * xq[m, k]                             (int32)
 *   dW[c, k]  = fl(float(acc[c, k]) * beta_c),
 *   beta_c    = fl(fl(gscale.step * xscale.step) * 2^-g_c).
 * Inputs : q_t [C_out, ld_t] int8 and group, gscale from sq_quantize_grad;
 *          xq_t [C_in, ld_x] int8 = X^T codes (ld_x >= M); xscale its scale.
 * Outputs (either may be NULL, not both): acc [C_out, ld_acc] int32,
 *          dW [C_out, ld_dW] fp32.
 * Errors: SQ_ERR_INVALID_ARGUMENT; SQ_ERR_OVERFLOW_RISK when
 *         M * Q * 128 >= 2^31; SQ_ERR_WORKSPACE_TOO_SMALL; SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_gemm_wgrad(const int8_t* q_t, int64_t ld_t, const uint8_t* group, const sq_scale* gscale,
                        const int8_t* xq_t, int64_t ld_x, const sq_scale* xscale,
                        int64_t M, int64_t C_out, int64_t C_in, const sq_quant_params* p,
                        int32_t* acc, int64_t ld_acc, float* dW, int64_t ld_dW,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_gemm_dgrad_grouped -- the GEMM-based implementation of the same loss
 * propagation, kept as a comparison for ShiftMM.
 *
 * Sec. 3.2 describes it in three steps: extract one pair of smaller matrices
 * per group (memory rearrangement: the group's code columns and weight rows
 * side by side), multiply each pair with a plain GEMM, then shift each
 * product by N_G - 1 - g and sum.  The result is the accumulator and dX of
 * sq_gemm_dgrad, bit for bit; only the cost differs.
 * Inputs, outputs and errors as sq_gemm_dgrad; the workspace
 * (sq_gemm_dgrad_grouped_workspace_size bytes, 256-byte aligned) holds the
 * rearranged operands [M + C_in, C_out + 63 N_G] and N_G int32 products
 * [M, C_in].  SQ_ERR_UNSUPPORTED when a rearranged operand spans 2^31 bytes.
 * ------------------------------------------------------------------------- */
sq_status sq_gemm_dgrad_grouped_workspace_size(int64_t M, int64_t C_out, int64_t C_in,
                                               const sq_quant_params* p, size_t* bytes);
sq_status sq_gemm_dgrad_grouped(const int8_t* q_fold, int64_t ld_fold, const int32_t* layout,
                                const uint8_t* group, const sq_scale* gscale,
                                const int8_t* wq_t, int64_t ld_w, const sq_scale* wscale,
                                int64_t M, int64_t C_out, int64_t C_in, const sq_quant_params* p,
                                int32_t* acc, int64_t ld_acc, float* dX, int64_t ld_dX,
                                void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_conv_dgrad -- input gradient of a stride-1 convolution, im2col and
 * col2im both implicit.
 *
 * The ResNet layers of Sec. 5 are convolutions that the GEMM of Eq. "dq_mm_f"
 * serves through im2col: X_col [N Ho Wo, KH KW C_in] with columns in
 * (r, s, ci) order, dX_col = dY . W, and dX = col2im(dX_col), col2im being
 * the adjoint of im2col.  This call computes dX directly, without writing
 * dX_col: with sh_c = N_G - 1 - g_c (0-indexed groups),
 *   acc[(n, ih, iw), ci] = sum_{r < KH, s < KW} sum_c
 *                          (code((n, ih + PH - r, iw + PW - s), c) * wq[c, (r, s, ci)]) << sh_c
 * over the window taps whose output pixel lies inside the Ho x Wo grid,
 * Ho = H + 2 PH - KH + 1, Wo = W + 2 PW - KW + 1, and
 *   dX = fl(float(acc) * alpha), alpha as in sq_gemm_dgrad.
 * The forward convolution this differentiates reads input pixel
 * (n, oh + r - PH, ow + s - PW) at tap (r, s) of output pixel (n, oh, ow).
 * Inputs : q_fold, ld_fold, layout, group, gscale from sq_quantize_grad of
 *          dY [N Ho Wo, C_out] (NHWC pixel order); wq_t [KH KW C_in, ld_w]
 *          int8 = W^T codes of W [C_out, KH KW C_in] (ld_w >= C_out);
 *          wscale its sq_scale.  1 <= KH, KW <= 15, 0 <= PH < KH,
 *          0 <= PW < KW, N H W < 2^31, N Ho Wo ld_fold < 2^31 bytes.
 * Outputs (either may be NULL, not both): acc [N H W, ld_acc] int32,
 *          dX [N H W, ld_dX] fp32 (NHWC).
 * Workspace: sq_conv_dgrad_workspace_size bytes (the weights regathered in
 *          the order of the implicit K sequence).
 * Errors: SQ_ERR_INVALID_ARGUMENT; SQ_ERR_OVERFLOW_RISK when
 *         KH KW C_out Q 2^(N_G-1) 128 >= 2^31; SQ_ERR_UNSUPPORTED beyond the
 *         size limits above; SQ_ERR_WORKSPACE_TOO_SMALL; SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_conv_dgrad_workspace_size(int64_t C_out, int64_t C_in, int32_t KH, int32_t KW,
                                       const sq_quant_params* p, size_t* bytes);
sq_status sq_conv_dgrad(const int8_t* q_fold, int64_t ld_fold, const int32_t* layout,
                        const uint8_t* group, const sq_scale* gscale,
                        const int8_t* wq_t, int64_t ld_w, const sq_scale* wscale,
                        int64_t N, int64_t H, int64_t W, int64_t C_out, int64_t C_in,
                        int32_t KH, int32_t KW, int32_t PH, int32_t PW, const sq_quant_params* p,
                        int32_t* acc, int64_t ld_acc, float* dX, int64_t ld_dX,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_dequant -- int32 accumulator to fp32 (Eq. "dq_mm_f": the inverse
 * scales multiply the integer sum once, outside the accumulation).
 *   kind 0 (dgrad): out = fl(float(acc) * alpha), alpha as in sq_gemm_dgrad
 *   kind 1 (wgrad): out[r, :] = fl(float(acc[r, :]) * beta_r), beta_r as in
 *                   sq_gemm_wgrad with g_r = group[r]
 *   kind 2 (per-column weight scales): out[:, c] = fl(float(acc[:, c]) * gamma_c),
 *                   gamma_c as in sq_gemm_forward, oscale an array [cols]
 * Inputs : acc [rows, ld_acc] int32; group [rows] (kind 1 only); gscale and
 *          oscale (the W scale for kind 0, the X scale for kind 1).
 * Output : out [rows, ld_out] fp32.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_dequant(const int32_t* acc, int64_t rows, int64_t cols, int64_t ld_acc, int32_t kind,
                     const uint8_t* group, const sq_scale* gscale, const sq_scale* oscale,
                     int32_t num_groups, float* out, int64_t ld_out, void* stream);

/* ---------------------------------------------------------------------------
 * sq_conv_dgrad_ranged -- sq_conv_dgrad that also writes the channel ranges
 * of dX for the quantizer of the layer below.
 *
 * Sec. 3.1's r_c = max_m |dY[m, c]| of the next layer's gradient, taken as
 * the conv input gradient dX [N H W, C_in] is stored:
 *   dX_ranges[s, c] = bits of max |dX[m, c]| over rows m in [s R, (s+1) R),
 * sign bit cleared, s < *range_slabs = ceil(N H W / R), R = *range_rows.
 * The streaming kernel (C_out <= 64 with one fold window, C_in <= 64 and a
 * multiple of 4, same-size window of at most 9 taps) takes them per block of
 * its own rows (R a multiple of 128, at most 512 slabs); the other conv
 * kernels store dX and one pass takes 32-row slab maxima (R = 32).
 * dX_ranges must hold sq_gemm_dgrad_range_slabs(N H W) x C_in words (the
 * most either path writes).  *range_slabs and *range_rows (host memory) are
 * set before the call returns, so the caller passes the slab count on to
 * sq_quantize_grad_from_ranges / sq_quantize_grad_conv_from_ranges without a
 * synchronization.  Arguments, outputs and errors as sq_conv_dgrad, with dX
 * required; SQ_ERR_UNSUPPORTED beyond 2^21 input pixels.
 * ------------------------------------------------------------------------- */
sq_status sq_conv_dgrad_ranged(const int8_t* q_fold, int64_t ld_fold, const int32_t* layout,
                               const uint8_t* group, const sq_scale* gscale,
                               const int8_t* wq_t, int64_t ld_w, const sq_scale* wscale,
                               int64_t N, int64_t H, int64_t W, int64_t C_out, int64_t C_in,
                               int32_t KH, int32_t KW, int32_t PH, int32_t PW, const sq_quant_params* p,
                               int32_t* acc, int64_t ld_acc, float* dX, int64_t ld_dX,
                               uint32_t* dX_ranges, int64_t* range_slabs, int64_t* range_rows,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_gemm_dgrad_ranged -- sq_gemm_dgrad that also writes the channel ranges
 * of dX for the quantizer of the layer below.
 *
 * In a chain of layers dX is the next dY to be quantized, and the quantizer's
 * first step is r_c = max_m |dY[m, c]| (Sec. 3.1).  Here the GEMM's epilogue
 * takes those maxima from the values it stores:
 *   dX_ranges[s, c] = bits of max |dX[m, c]| over rows m in [32 s, 32 s + 32),
 * sign bit cleared, s < sq_gemm_dgrad_range_slabs(M) = ceil(M / 32); they are
 * the `ranges` input of sq_quantize_grad_from_ranges.  The maxima come from
 * the GEMM's epilogue when C_out is a multiple of 64 (and every operand's byte
 * offsets fit in 31 bits); otherwise one extra pass over the stored dX takes
 * them.  Arguments, outputs and errors as sq_gemm_dgrad, with dX required;
 * SQ_ERR_UNSUPPORTED beyond 2^21 rows on the second path.
 * ------------------------------------------------------------------------- */
sq_status sq_gemm_dgrad_range_slabs(int64_t M, int64_t* slabs);
sq_status sq_gemm_dgrad_ranged(const int8_t* q_fold, int64_t ld_fold, const int32_t* layout,
                               const uint8_t* group, const sq_scale* gscale,
                               const int8_t* wq_t, int64_t ld_w, const sq_scale* wscale,
                               int64_t M, int64_t C_out, int64_t C_in, const sq_quant_params* p,
                               int32_t* acc, int64_t ld_acc, float* dX, int64_t ld_dX, uint32_t* dX_ranges,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Implicit-im2col weight gradient of a stride-1 convolution.
 *
 * The wgrad of the im2col'd conv layer (Fig. "MMs", third GEMM, on the conv
 * layers of Sec. 5), computed without the im2col:
 *   acc[co, (r KW + s) C_in + ci] = sum_{n, oh, ow} code(n, oh, ow, co)
 *                                   xq(n, oh + r - PH, ow + s - PW, ci)
 * (zero outside the input), with the epilogue of sq_gemm_wgrad
 * (dW[co, :] = fl(float(acc[co, :]) * beta_co)).  Columns follow the (r, s, ci)
 * order of W [C_out, KH KW C_in].  Stride 1, 0 <= PH < KH, 0 <= PW < KW,
 * KH, KW <= 16; Ho = H + 2 PH - KH + 1, Wo = W + 2 PW - KW + 1.
 *
 * Both operands live on a padded pixel grid of Hp = H + 2 PH rows and
 * Wp = roundup(W + 2 PW, 16) columns per image, on which tap (r, s) is the
 * constant shift r Wp + s of the pixel index:
 *   q_tp [C_out, ld_tp >= q_ld]: gradient code (n, oh, ow, c) at column
 *        n Hp Wp + oh Wp + ow of row c, every other column 0.
 *   xs   [C_in, ld_xs >= x_ld]: input pixel (n, ih, iw) of channel ci at
 *        column n Hp Wp + (ih + PH) Wp + iw + PW of row ci, 0 in the padding
 *        and in the x_ld - q_ld = (KH - 1) Wp + 64 columns past the grid, so
 *        that tap (r, s) of grid position P reads column P + r Wp + s.
 * sq_conv_wgrad_layout gives x_rows = C_in, x_ld and q_ld.
 * sq_conv_pack_input builds xs from the input codes xq_t [C_in, ld_xq >= N H W]
 *   (sq_quantize_tensor, transpose 1) and writes every byte of xs (x_ld
 *   columns); in training the input codes come from the forward pass, and
 *   the pack runs once per step.
 * sq_conv_pack_grad builds q_tp from transposed codes q_t [C_out, ld_t >= N Ho Wo]
 *   and writes every byte of q_tp.
 * sq_quantize_input_conv is the forward pass's quantizer of the layer input
 *   X [N H W, ld_X] (NHWC rows, fp32): the per-tensor b-bit codes of
 *   sq_quantize_tensor (Sec. 5.1: activations quantized per tensor) written
 *   straight onto the padded input grid xs, optionally also
 *   row-major into xq [N H W, ld_xq >= C_in] (the forward's layout; NULL to
 *   skip).  xs's padding is written with nothing but zeros, and not all of
 *   it, so the caller zero-fills that buffer once; then no pack is needed.
 *   Workspace:
 *   sq_quantize_tensor_workspace_size(N H W, C_in).  Errors as
 *   sq_quantize_tensor, plus SQ_ERR_UNSUPPORTED beyond 2^32 grid pixels.
 * sq_quantize_grad_conv is sq_quantize_grad for the conv's gradient
 *   dY [N Ho Wo, ld_dY] (same codes, groups, scale, layout, q_fold, workspace)
 *   that writes the transposed codes straight onto the padded grid: q_tp's
 *   padding is written with nothing but zeros, and not all of it, so the
 *   caller zero-fills that buffer once.
 * sq_quantize_grad_conv_from_ranges is the same with the channel ranges
 *   given as partial maxima (see sq_quantize_grad_from_ranges), e.g. the
 *   dX_ranges of sq_conv_dgrad_ranged of the layer above.
 * sq_conv_wgrad runs the int8 product over the padded grid (K = N Hp Wp
 *   rounded up to 64) with every tap read from the one copy of the input at
 *   its shift r Wp + s (1 x 1 windows: a plain int8 GEMM of the two grids),
 *   then, when K is split, the sum of the int32 partials.
 * Outputs: acc [C_out, ld_acc] int32 and/or dW [C_out, ld_dW] fp32, each row
 *          KH KW C_in wide.
 * Workspace: sq_conv_wgrad_workspace_size bytes (split-K partials, may be 0).
 * Errors: SQ_ERR_INVALID_ARGUMENT; SQ_ERR_OVERFLOW_RISK when
 *         N Ho Wo Q 128 >= 2^31; SQ_ERR_UNSUPPORTED when a padded grid
 *         exceeds 2^31 bytes; SQ_ERR_WORKSPACE_TOO_SMALL; SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_conv_wgrad_layout(int64_t N, int64_t H, int64_t W, int64_t C_in, int32_t KH, int32_t KW,
                               int32_t PH, int32_t PW, int64_t* x_rows, int64_t* x_ld, int64_t* q_ld);
sq_status sq_conv_pack_input(const int8_t* xq_t, int64_t ld_xq, int64_t N, int64_t H, int64_t W, int64_t C_in,
                             int32_t KH, int32_t KW, int32_t PH, int32_t PW, int8_t* xs, int64_t ld_xs,
                             void* stream);
sq_status sq_conv_pack_grad(const int8_t* q_t, int64_t ld_t, int64_t N, int64_t H, int64_t W, int64_t C_out,
                            int32_t KH, int32_t KW, int32_t PH, int32_t PW, int8_t* q_tp, int64_t ld_tp,
                            void* stream);
sq_status sq_quantize_input_conv(const float* X, int64_t N, int64_t H, int64_t W, int64_t C_in, int64_t ld_X,
                                 int32_t KH, int32_t KW, int32_t PH, int32_t PW, int32_t bits,
                                 int8_t* xq, int64_t ld_xq, int8_t* xs, int64_t ld_xs, sq_scale* scale,
                                 void* workspace, size_t workspace_bytes, void* stream);
sq_status sq_quantize_grad_conv(const float* dY, int64_t N, int64_t H, int64_t W, int64_t C_out, int64_t ld_dY,
                                int32_t KH, int32_t KW, int32_t PH, int32_t PW, const sq_quant_params* p,
                                int8_t* q_fold, int64_t ld_fold, int8_t* q_tp, int64_t ld_tp,
                                uint8_t* group, sq_scale* scale, int32_t* layout,
                                void* workspace, size_t workspace_bytes, void* stream);
sq_status sq_quantize_grad_conv_from_ranges(const float* dY, int64_t N, int64_t H, int64_t W, int64_t C_out,
                                            int64_t ld_dY, int32_t KH, int32_t KW, int32_t PH, int32_t PW,
                                            const sq_quant_params* p, const uint32_t* ranges, int64_t range_slabs,
                                            int8_t* q_fold, int64_t ld_fold, int8_t* q_tp, int64_t ld_tp,
                                            uint8_t* group, sq_scale* scale, int32_t* layout,
                                            void* workspace, size_t workspace_bytes, void* stream);
sq_status sq_conv_wgrad_workspace_size(int64_t N, int64_t H, int64_t W, int64_t C_out, int64_t C_in,
                                       int32_t KH, int32_t KW, int32_t PH, int32_t PW,
                                       const sq_quant_params* p, size_t* bytes);
sq_status sq_conv_wgrad(const int8_t* q_tp, int64_t ld_tp, const uint8_t* group, const sq_scale* gscale,
                        const int8_t* xs, int64_t ld_xs, const sq_scale* xscale,
                        int64_t N, int64_t H, int64_t W, int64_t C_out, int64_t C_in,
                        int32_t KH, int32_t KW, int32_t PH, int32_t PW, const sq_quant_params* p,
                        int32_t* acc, int64_t ld_acc, float* dW, int64_t ld_dW,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_quantize_grad_from_ranges -- sq_quantize_grad with the channel ranges
 * supplied by the producer of dY.
 *
 * The quantizer's first step (r_c = max_m |dY[m, c]|, Sec. 3.1) reads all of
 * dY once before the codes can be formed; a kernel that writes dY can take
 * those maxima on the fly instead.  `ranges` holds them as partial maxima:
 * ranges[s, c], s < range_slabs, is the bit pattern of max |dY[m, c]| over
 * some subset of the rows (sign bit cleared, so NaN and Inf compare above
 * every finite value), the subsets covering all M rows; r_c is the maximum
 * over s.  Everything else -- outputs, layout, workspace
 * (sq_quantize_grad_workspace_size), errors -- is as in sq_quantize_grad, and
 * the results are identical when the ranges are exact.
 * sq_l1bn_backward writes such ranges for its dx.
 * ------------------------------------------------------------------------- */
sq_status sq_quantize_grad_from_ranges(const float* dY, int64_t M, int64_t C_out, int64_t ld_dY,
                                       const sq_quant_params* p, const uint32_t* ranges, int64_t range_slabs,
                                       int8_t* q_fold, int64_t ld_fold,
                                       int8_t* q_t, int64_t ld_t,
                                       uint8_t* group, sq_scale* scale, int32_t* layout,
                                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Fully-quantized L1 batch normalization (L1BNQ), Sec. 4 (Fig. l1bnq) and
 * App. C.1 / C.2: input features, statistics and parameters are quantized,
 * and the normalization divides by the L1 deviation instead of the standard
 * deviation.
 *
 * Per-channel state written by sq_l1bn_forward and read by sq_l1bn_backward
 * (device memory, one entry per channel):
 *   mu       m_c = round_half_even(S_c / M), S_c = sum_m q[m, c]: the batch mean
 *            quantized onto the input's own 8-bit grid (mu^q = s_x m_c)
 *   sigma    k_c = max(1, round_half_even(127 A_c / A_max)): the L1 deviation
 *            sigma_c = s_x A_c / M quantized per tensor to 8 bits under the
 *            step max_c sigma_c / 127 (0 when the layer is flagged ZERO)
 *   sign_sum P_c = sum_m sgn(q[m, c] - m_c)
 *   gamma, beta  gamma^q_c, beta^q_c: the parameters quantized per tensor to
 *            8 bits (as sq_quantize_tensor), dequantized
 *   kappa    fl32(gamma^q_c 127 M / (A_max k_c)), evaluated in binary64
 *   dev_sum  A_c = sum_m |q[m, c] - m_c|
 * Layer state: rows M, dev_max A_max = max_c A_c, x_step s_x (the input's
 * step), flags (SQ_FLAG_ZERO when A_max = 0: every channel constant), and the
 * scales of gamma and beta.
 * ------------------------------------------------------------------------- */
typedef struct {
    int32_t mu;
    int32_t sigma;
    int32_t sign_sum;
    float gamma;
    float beta;
    float kappa;
    int64_t dev_sum;
} sq_l1bn_channel;      /* 32 bytes */

typedef struct {
    int64_t rows;
    int64_t dev_max;
    float x_step;
    uint32_t flags;
    sq_scale gamma_scale;
    sq_scale beta_scale;
} sq_l1bn_layer;        /* 56 bytes */

/* Partial-maximum slabs that sq_l1bn_backward writes to dx_ranges
 * ([slabs, C] uint32) for M rows and C channels. */
sq_status sq_l1bn_range_slabs(int64_t M, int64_t C, int64_t* slabs);
sq_status sq_l1bn_forward_workspace_size(int64_t M, int64_t C, size_t* bytes);
sq_status sq_l1bn_backward_workspace_size(int64_t M, int64_t C, const sq_quant_params* p, size_t* bytes);

/* ---------------------------------------------------------------------------
 * sq_l1bn_forward -- L1BNQ forward over a batch (training statistics).
 *   y[m, c] = fl(fl(kappa_c (q[m, c] - m_c)) + beta^q_c),
 * i.e. gamma^q (x^q - mu^q) / sigma^q + beta^q with x^q = s_x q (App. C.2's
 * normalization with quantized statistics); with A_max = 0, y = beta^q.
 * Inputs : xq [M, ld_x] int8, the 8-bit per-tensor codes of the layer input
 *          (sq_quantize_tensor, bits 8), 16-byte aligned, ld_x % 16 == 0;
 *          xscale its sq_scale (device); gamma, beta [C] fp32 (device).
 *          1 <= M <= 2^24.
 * Outputs: y [M, ld_y] fp32; chan [C] and layer (device) for the backward.
 * Workspace: sq_l1bn_forward_workspace_size bytes.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED (M > 2^24),
 *         SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_l1bn_forward(const int8_t* xq, int64_t M, int64_t C, int64_t ld_x, const sq_scale* xscale,
                          const float* gamma, const float* beta, float* y, int64_t ld_y,
                          sq_l1bn_channel* chan, sq_l1bn_layer* layer,
                          void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_l1bn_backward -- L1BNQ backward.
 * The incoming gradient dy is quantized with ShiftQuant (as sq_quantize_grad
 * with params p; codes qg, groups g_c, channel steps delta_c = step 2^-g_c);
 * the L1 normalization is differentiated exactly (App. C.1 with
 * sigma = mean |x - mu|, which brings in s = sgn(x - mu)), the quantizers of
 * mu and sigma passed straight through:
 *   dx = (gamma^q / sigma^q)(g - mean g - mean(g xhat)(s - mean s)).
 * With integer sums G1 = sum qg, G2 = sum qg (q - m), P = sign_sum,
 * rho = 127 M / (A_max k), lambda = gamma^q rho / s_x, in binary64:
 *   dbeta = delta G1,  dgamma = (delta G2) rho,  D = dgamma / M,
 *   a = lambda delta,  b = -(lambda D),  e = lambda (D P / M - delta G1 / M),
 * each rounded once to fp32, and dx = fl(fl(fl(a qg) + fl(b sgn(q - m))) + e).
 * With A_max = 0: dgamma = 0 and dx = 0.
 * Inputs : dy [M, ld_dy] fp32; p (b, N_G, rounding of the gradient codes);
 *          xq, ld_x, chan, layer: the forward's input codes and state.
 * Outputs: dx [M, ld_dx] fp32; dgamma, dbeta [C] fp32; group [C] and gscale:
 *          the gradient quantizer's groups and scale; dx_ranges (may be NULL):
 *          [sq_l1bn_range_slabs, C] partial maxima of |dx| per channel, the
 *          input of sq_quantize_grad_from_ranges for the layer below.
 * Workspace: sq_l1bn_backward_workspace_size bytes.
 * Errors: as sq_l1bn_forward.
 * ------------------------------------------------------------------------- */
sq_status sq_l1bn_backward(const float* dy, int64_t M, int64_t C, int64_t ld_dy, const sq_quant_params* p,
                           const int8_t* xq, int64_t ld_x, const sq_l1bn_channel* chan,
                           const sq_l1bn_layer* layer, float* dx, int64_t ld_dx,
                           float* dgamma, float* dbeta, uint8_t* group, sq_scale* gscale,
                           uint32_t* dx_ranges, void* workspace, size_t workspace_bytes, void* stream);

/* ===========================================================================
 * Microscaled 4-bit linear layers.
 *
 * The same three products as the integer path, Y = X W^T, dX = dY W and
 * dW = dY^T X, with operands in microscaled 4-bit floating point (E2M1
 * elements, one E8M0 scale for 32 consecutive elements of a product's inner
 * axis) and fp32 accumulation on the matrix cores, dense or by expert.
 *
 * A block of 32 with largest magnitude a:
 *   s    = the smallest byte with a / 2^(s - 127) <= 7 (at least 0)
 *   code = x / 2^(s - 127) rounded to the nearest of +-{0, 0.5, 1, 1.5, 2, 3,
 *          4, 6}, ties to the even code (so no element is off by more than half
 *          a step: 7 is halfway from 6 to the next power of two);
 *   a block that holds NaN or Inf: s = 255, which stands for NaN in all of it.
 * Every value that a code and scale stand for is exact in bf16 and fp32, but
 * 4 * 2^126 (of a block with a > 1.75 * 2^127), which is past their range: Inf.
 *
 * Layout of a matrix [rows, K] (sq_mx_size bytes): rows in groups of 16, K in
 * units of 512.  Element (r, k) is nibble k % 2 (0: low) of byte
 *   ((r / 16) * units + k / 512) * 4096 + (k / 128) % 4 * 1024
 *       + (k / 32) % 4 * 256 + (r % 16) * 16 + (k % 32) / 2,
 * its block's scale byte
 *   ((r / 16) * units + k / 512) * 256 + (k / 32) % 4 * 64 + (r % 16) * 4 + (k / 128) % 4.
 * This is the operand order of v_mfma_scale_f32_16x16x128_f8f6f4: a wave
 * loads a 16 x 128 tile as one contiguous 1 KB block.  Writers fill K up to the
 * next multiple of 128 with zeros; the rest of the padding is not written
 * and never used.  Matrices of a stack follow each other without a gap.
 * codes must be 16-byte aligned, scales 4-byte.
 *
 * Sizes, SQ_ERR_INVALID_ARGUMENT otherwise: rows < 2^31; columns of values (cols,
 * N, c_in, c_out, K of sq_mx_linear) < 2^20; experts < 2^16; batch < 2^16.  Inner
 * axes of products: see each call.
 *
 * By expert: `offsets` [experts + 1] (device memory) splits the rows; expert
 * e owns [offsets[e], offsets[e + 1]), possibly none.  Offsets ascend from
 * >= 0 to <= rows; rows outside of them are neither read nor written (of codes,
 * padded to whole groups of 16 rows, products read the groups that experts' rows
 * are in).
 * Offsets that break this never lead out of the buffers, but what is
 * computed is then unspecified.  The inner axis of the transposed form
 * starts anew at a multiple of 512 for each expert: expert e's rows are
 * columns P_e + (row - offsets[e]), P_e = sum over e' < e of
 * roundup(rows of e', 512), of a matrix with sq_mx_segment_cols columns.
 * ========================================================================= */

/* Element types of the arguments named `type`. */
enum {
    SQ_TYPE_F32 = 0,
    SQ_TYPE_BF16 = 1
};

sq_status sq_mx_size(int64_t rows, int64_t cols, size_t* code_bytes, size_t* scale_bytes);
sq_status sq_mx_segment_cols(int64_t rows, int64_t experts, int64_t* cols);

/* ---------------------------------------------------------------------------
 * sq_mx_quantize -- codes of X [batch, rows, cols] (row stride ld, matrix stride
 * `stride`, both in elements) in one read, along either axis or both:
 *   codes, scales      [batch] matrices [rows, cols], blocks along the columns
 *                      (the operand of a product over the columns)
 *   codes_t, scales_t  [batch] matrices [cols, rows], blocks along the rows (of a
 *                      product over the rows)
 * Either pair may be NULL, not both.  With offsets (batch == 1): codes_t is
 * [cols, sq_mx_segment_cols(rows, experts)], its blocks start anew at each
 * expert's first row.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED (with codes_t: rows >=
 * 2^23, or sq_mx_segment_cols >= 2^24), SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_mx_quantize(const void* X, int32_t type, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                         const int32_t* offsets, int64_t experts,
                         uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* stream);

/* sq_mx_dequantize -- the values [rows, cols] of a matrix, as fp32 or bf16 (exact in both). */
sq_status sq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols,
                           void* out, int32_t type, int64_t ld, void* stream);

/* ---------------------------------------------------------------------------
 * sq_mx_gemm -- C [M, N] = A B^T, A [M, K], B [N, K]; C fp32, or bf16 rounded
 * once to the nearest even.  K = 0 gives zeros.
 * Workspace: sq_mx_gemm_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED (K >= 2^23),
 * SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_mx_gemm_workspace_size(int64_t M, int64_t N, int64_t K, size_t* bytes);
sq_status sq_mx_gemm(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales,
                     int64_t M, int64_t N, int64_t K, void* C, int32_t type, int64_t ldc,
                     void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_mx_gemm_experts -- C[m] = A[m] B_e^T for the rows m of each expert e:
 * A [M, K], B a stack [experts] of [N, K], C [M, N].  The forward pass with W
 * stacks, the input gradient with W^T stacks.  Errors as sq_mx_gemm.
 * ------------------------------------------------------------------------- */
sq_status sq_mx_gemm_experts(const uint8_t* A, const uint8_t* A_scales, int64_t M, int64_t K,
                             const int32_t* offsets, int64_t experts,
                             const uint8_t* B, const uint8_t* B_scales, int64_t N,
                             void* C, int32_t type, int64_t ldc, void* stream);

/* ---------------------------------------------------------------------------
 * sq_mx_gemm_experts_wgrad -- C_e [M, N] = sum over the rows r of expert e of
 * A[:, r] B[:, r]^T: A [M, sq_mx_segment_cols(rows, experts)] and B [N, same]
 * are the transposed forms that sq_mx_quantize wrote with the same offsets;
 * C is a stack [experts] of [M, ldc].  An expert without rows gets zeros.
 * Workspace: sq_mx_gemm_experts_wgrad_workspace_size bytes (0: none; no size needs
 * one, the inner axis is not split).
 * Errors: as sq_mx_gemm; SQ_ERR_UNSUPPORTED for rows >= 2^23.
 * ------------------------------------------------------------------------- */
sq_status sq_mx_gemm_experts_wgrad_workspace_size(int64_t rows, int64_t experts, int64_t M, int64_t N, size_t* bytes);
sq_status sq_mx_gemm_experts_wgrad(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales,
                                   int64_t rows, const int32_t* offsets, int64_t experts, int64_t M, int64_t N,
                                   void* C, int32_t type, int64_t ldc,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_mx_linear -- Y [M, N] = X W^T with X [M, K] in fp32 or bf16, quantized on the
 * way: what sq_mx_quantize and sq_mx_gemm (offsets NULL, experts 0) or
 * sq_mx_gemm_experts give.  Few rows (at most 16, or 16 an expert on average;
 * more for small layers, fewer for wide ones of a short inner axis) take one
 * launch and no workspace, the serving form for single tokens.
 * Workspace: sq_mx_linear_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: as sq_mx_gemm.
 * ------------------------------------------------------------------------- */
sq_status sq_mx_linear_workspace_size(int64_t M, int64_t K, int64_t N, int64_t experts, size_t* bytes);
sq_status sq_mx_linear(const void* X, int32_t type, int64_t M, int64_t K, int64_t ld,
                       const int32_t* offsets, int64_t experts,
                       const uint8_t* W, const uint8_t* W_scales, int64_t N,
                       void* Y, int32_t out_type, int64_t ldy,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_mx_layer -- the buffers of a linear layer that is trained, allocated once by
 * the caller (host struct, read during the calls only), and its three steps:
 *   sq_mx_layer_weight    codes of W [c_out, c_in] (a stack [experts] of such)
 *                         along both axes, after each update of W
 *   sq_mx_layer_forward   codes of X [rows, c_in] along both axes, Y = X W^T; by
 *                         expert, a copy of the offsets in `offsets`
 *   sq_mx_layer_backward  codes of dY [rows, c_out] along both axes, then
 *                         dX = dY W [rows, c_in] and dW = dY^T X [c_out, c_in]
 *                         (a stack [experts] of such, ld_dw apart in its rows)
 * Each is what sq_mx_quantize and the sq_mx_gemm calls give, in fewer launches:
 * dX and dW share one.  Y and dX have the layer's type, dW is fp32.  offsets as
 * above, NULL when experts == 0.  The backward reads codes of X that are laid out
 * by the forward's offsets: with offsets NULL it takes the layer's copy of them,
 * which does not change when the caller's buffer does; others must be equal.
 * Sizes: w [c_out, c_in] and w_t [c_in, c_out], each experts times; x [rows, c_in],
 * x_t [c_in, inner], dy [rows, c_out], dy_t [c_out, inner] with inner = rows, or
 * sq_mx_segment_cols(rows, experts); every one of sq_mx_size bytes.  offsets
 * [experts + 1], or NULL: no copy is kept (nor read with experts == 0).
 * Workspace: sq_mx_layer_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: as sq_mx_quantize and sq_mx_gemm.
 * ------------------------------------------------------------------------- */
typedef struct {
    int64_t rows, c_in, c_out, experts;
    int32_t type;                          /* SQ_TYPE_* of X, Y, dY, dX and W */
    int32_t reserved;                      /* 0 */
    uint8_t *w, *w_scales, *w_t, *w_t_scales;
    uint8_t *x, *x_scales, *x_t, *x_t_scales;
    uint8_t *dy, *dy_scales, *dy_t, *dy_t_scales;
    void* workspace;
    size_t workspace_bytes;
    int32_t* offsets;                      /* the forward's, for the backward */
} sq_mx_layer;

sq_status sq_mx_layer_workspace_size(const sq_mx_layer* layer, size_t* bytes);
sq_status sq_mx_layer_weight(const sq_mx_layer* layer, const void* W, int64_t ld, int64_t stride, void* stream);
sq_status sq_mx_layer_forward(const sq_mx_layer* layer, const void* X, int64_t ld, const int32_t* offsets,
                              void* Y, int64_t ldy, void* stream);
sq_status sq_mx_layer_backward(const sq_mx_layer* layer, const void* dY, int64_t ld, const int32_t* offsets,
                               void* dX, int64_t ld_dx, float* dW, int64_t ld_dw, void* stream);

/* ---------------------------------------------------------------------------
 * sq_act_forward, sq_act_backward -- an activation between two layers, whose
 * backward pass reads a copy of its input in 8 bits.
 *   SQ_ACT_SILU  act(x) = x sigma(x)
 *   SQ_ACT_GELU  act(x) = x sigma(2 sqrt(2 / pi) (x + 0.044715 x^3)), the tanh form
 * gated == 0: X [M, F],   H = act(X),      dX = dH act'(x)
 * gated == 1: X [M, 2 F], the gate g first, H = act(g) u,
 *             dX = (dH u act'(g), dH act(g))
 * The forward is computed from X, the backward from the copy: x stands as
 * code 2^(s - 127), code an int8 in [-127, 127], s one byte for 32 consecutive
 * columns of g or of u, the smallest with max |x| / 2^(s - 127) < 127.5 (255, for
 * NaN in the whole block, where it holds NaN or Inf).  codes [M, n Fp] with
 * Fp = roundup(F, 32) and n = 1 or 2, g in columns [0, F), u in [Fp, Fp + F);
 * scales [M, n Fp / 32]; sizes from sq_act_size.  codes must be 16-byte
 * aligned.  X, H, dH and dX share one type; sums in fp32, rounded once.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
enum {
    SQ_ACT_SILU = 0,
    SQ_ACT_GELU = 1
};

sq_status sq_act_size(int64_t M, int64_t F, int32_t gated, size_t* code_bytes, size_t* scale_bytes);
sq_status sq_act_forward(const void* X, int32_t type, int32_t kind, int32_t gated, int64_t M, int64_t F, int64_t ld_x,
                         void* H, int64_t ld_h, int8_t* codes, uint8_t* scales, void* stream);
sq_status sq_act_backward(const void* dH, int32_t type, int32_t kind, int32_t gated, int64_t M, int64_t F, int64_t ld_h,
                          const int8_t* codes, const uint8_t* scales, void* dX, int64_t ld_x, void* stream);

/* =========================================================================
 * What stands around an expert layer's products: layer norm, the router, and the
 * exchange of rows between tokens and experts.  Rows are fp32 or bf16
 * (SQ_TYPE_*) with a row stride; sums, statistics and scores are fp32 or fp64,
 * results are rounded once to their type.  Results do not depend on how the work
 * is split over the GPU in another run: no sum is added up by atomics.
 * ========================================================================= */

/* ---------------------------------------------------------------------------
 * sq_norm_forward, sq_norm_backward -- layer norm of the rows of X [M, C], with the
 * residual sum before it.
 *   h = x, or x + residual rounded to the type (H [M, C]; both NULL or neither)
 *   mean, var of a row of h (var: divided by C);  r = 1 / sqrt(var + eps)
 *   y = (h - mean) r gamma + beta
 *   q = dy gamma, xh = (h - mean) r:
 *   dx = r (q - mean(q) - xh mean(q xh)) (+ dh);  dgamma = sum_rows dy xh;  dbeta = sum_rows dy
 * gamma and beta [C] of param_type, dgamma and dbeta [C] fp32.  The backward reads
 * h (X without a residual) and the forward's stats [M, 4] (fp32, 16-byte aligned;
 * the forward takes NULL where there is no backward); dH, the gradient that
 * reaches h past the norm, may be NULL; dX is the gradient of x and of the
 * residual.  M = 0 gives dgamma = dbeta = 0.  A row that holds NaN or Inf, or whose
 * sum of h passes fp32's range, gives NaN in all of its y and dx, and in all of
 * dgamma; squares that pass it, or vanish below it, do no harm.  H may be X or residual, dX
 * may be dH, in place; no other buffers overlap.  M < 2^31, C < 2^20.
 * Workspace: sq_norm_backward_workspace_size bytes, 16-byte aligned.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_WORKSPACE_TOO_SMALL, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_norm_forward(const void* X, const void* residual, int32_t type, int64_t M, int64_t C, int64_t ld_x, int64_t ld_r,
                          const void* gamma, const void* beta, int32_t param_type, float eps,
                          void* H, int64_t ld_h, void* Y, int64_t ld_y, float* stats, void* stream);
sq_status sq_norm_backward_workspace_size(int64_t M, int64_t C, size_t* bytes);
sq_status sq_norm_backward(const void* dY, const void* H, const void* dH, int32_t type, int64_t M, int64_t C,
                           int64_t ld_dy, int64_t ld_h, int64_t ld_dh, const void* gamma, int32_t param_type, const float* stats,
                           void* dX, int64_t ld_dx, float* dgamma, float* dbeta,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_route_forward -- the k best of E experts for each of T tokens, by their logits
 * [T, E], and where each token's rows go.
 *   SQ_SCORE_SOFTMAX  s = softmax(logits)       SQ_SCORE_SIGMOID  s_e = 1 / (1 + exp(-logit_e))
 * Experts are ordered by their logits, with a bias [E] (fp32, may be NULL) by
 * s + bias: the bias moves the choice, not the shares.  An expert whose logit (or
 * s + bias) is -Inf is never chosen.  groups > 1: the experts are `groups` runs of
 * E / groups; a group counts as the sum of its two highest s (+ bias), and experts
 * outside of the top_groups best groups are left out.  Equal ones: the lowest
 * index.  Comparisons of s are made in fp64.
 *   chosen [T, k]  the experts, best first; -1 where there are no more
 *   share  [T, k]  scale s_e, renormalize: scale s_e / sum of the chosen s (at least
 *                  1e-300); fp32; 0 where chosen is -1
 *   place  [T, k]  the position of (token, slot) in a stable sort of all of them by
 *                  expert: token t's row of expert e; -1 where chosen is -1
 *   offsets [E + 1] rows of expert e: [offsets[e], offsets[e + 1])
 * A token with NaN among its logits (or s + bias), or +Inf under softmax, has
 * chosen = place = -1 and share NaN.
 * Sizes: T <= 2^26 - 4, T k < 2^31, E <= 1024, k <= 64, groups <= 64 (SQ_ERR_UNSUPPORTED).
 * Workspace: sq_route_workspace_size bytes (0: none), 16-byte aligned.
 *
 * sq_route_backward -- the logits' gradient from dshare [T, k], the forward's
 * logits, share and chosen (the choice has no gradient); slots with chosen = -1
 * count for nothing, a token whose shares are NaN gets NaN.  A sigmoid's 1 - s is
 * formed in 64 bits from s, off by 2^-53 at most.  Every element of
 * dlogits [T, E] is written; it may be the logits, in place.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED, SQ_ERR_WORKSPACE_TOO_SMALL,
 * SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
enum {
    SQ_SCORE_SOFTMAX = 0,
    SQ_SCORE_SIGMOID = 1
};

sq_status sq_route_workspace_size(int64_t T, int64_t E, size_t* bytes);
sq_status sq_route_forward(const void* logits, int32_t type, int64_t T, int64_t E, int64_t ld, const float* bias,
                           int32_t score, int32_t k, int32_t groups, int32_t top_groups, int32_t renormalize, float scale,
                           float* share, int32_t* chosen, int32_t* place, int32_t* offsets,
                           void* workspace, size_t workspace_bytes, void* stream);
sq_status sq_route_backward(const float* dshare, const void* logits, int32_t type, int64_t T, int64_t E, int64_t ld,
                            int32_t score, int32_t k, int32_t renormalize, float scale,
                            const float* share, const int32_t* chosen, void* dlogits, int64_t ld_d, void* stream);

/* ---------------------------------------------------------------------------
 * sq_exchange_* -- rows [T, D] of tokens to rows [rows, D] sorted by expert and
 * back; place [T, k] and share [T, k] (fp32) as sq_route_forward writes them.
 *   dispatch          R[place[t, j]] = X[t]
 *   combine           out[t] = add[t] + sum_j share[t, j] R[place[t, j]]
 *                     (add NULL: 0; share NULL: 1, which is dispatch's gradient)
 *   combine_backward  dR[place[t, j]] = share[t, j] dout[t],
 *                     dshare[t, j] = sum_d dout[t, d] R[place[t, j], d]
 * A place outside [0, rows) is no row: it is neither read nor written, adds
 * nothing (whatever its share), and its dshare is 0.  No place comes twice.  Rows
 * that no place names stay as they were.  `add` may be out, in place; no other
 * buffers overlap.  T k < 2^31, k <= 64 (SQ_ERR_UNSUPPORTED), D < 2^20.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED, SQ_ERR_HIP.
 * ------------------------------------------------------------------------- */
sq_status sq_exchange_dispatch(const void* X, int32_t type, int64_t T, int64_t D, int64_t ld_x, const int32_t* place, int32_t k,
                               void* R, int64_t rows, int64_t ld_r, void* stream);
sq_status sq_exchange_combine(const void* R, int32_t type, int64_t rows, int64_t D, int64_t ld_r,
                              const int32_t* place, const float* share, int64_t T, int32_t k,
                              const void* add, int64_t ld_add, void* out, int64_t ld_out, void* stream);
sq_status sq_exchange_combine_backward(const void* dout, const void* R, int32_t type, int64_t rows, int64_t D,
                                       int64_t ld_dout, int64_t ld_r, const int32_t* place, const float* share, int64_t T, int32_t k,
                                       void* dR, int64_t ld_dr, float* dshare, void* stream);

/* =========================================================================
 * Dense linear layers Y = X W^T, trained (dX = dY W, dW = dY^T X) or served, with
 * operands in 8-bit floating point (E4M3 elements) and fp32 accumulation on the
 * matrix cores.  One E8M0 scale for 128 consecutive elements of a product's inner
 * axis (X and dY, along the axis of each product that they are in), or for 128 x 128
 * elements (square: W, so that W and W^T hold the same values).
 *
 * A block with largest magnitude a:
 *   s    = the smallest byte with a / 2^(s - 127) <= 464 (at least 0)
 *   code = x / 2^(s - 127) rounded to the nearest E4M3 value (bias 7, largest 448,
 *          below 2^-6 multiples of 2^-9), ties to the even code (464 is halfway
 *          from 448 to the next step, so nothing is off by more than half a step);
 *   a block that holds NaN or Inf: s = 255, which stands for NaN in all of it.
 * Values that a code and scale stand for are exact in bf16 and fp32, but those
 * past their range (of a block with a > 1.8125 * 2^127: Inf) and, of scales below
 * 2^-124 (bf16) or 2^-140 (fp32), those off their least step (2^-133, 2^-149).
 * Products with an fp32 result take the values in bf16, sums in fp32 (24 bits kept);
 * with a bf16 result sums of 16 products first, each cut 13 bits below the largest.
 *
 * Layout of a matrix [rows, K] (sq_f8_size bytes): rows in groups of 16, K in units
 * of 512.  Element (r, k) is byte
 *   ((r / 16) * units + k / 512) * 8192 + (k / 128) % 4 * 2048
 *       + (k / 16) % 8 * 256 + (r % 16) * 16 + k % 16,
 * its block's scale byte
 *   ((r / 16) * units + k / 512) * 64 + (r % 16) * 4 + (k / 128) % 4.
 * Writers fill K up to the next multiple of 128 with zeros; the rest of the padding
 * is not written and never used.  codes must be 16-byte aligned, scales 4-byte.
 *
 * Sizes, SQ_ERR_INVALID_ARGUMENT otherwise: rows < 2^31; columns of values < 2^20.
 * Inner axes of products < 2^22 (SQ_ERR_UNSUPPORTED).
 * ========================================================================= */
sq_status sq_f8_size(int64_t rows, int64_t cols, size_t* code_bytes, size_t* scale_bytes);

/* sq_f8_quantize -- codes of X [rows, cols] in one read: codes, scales of the matrix
 * [rows, cols] with blocks along the columns, codes_t, scales_t of the transpose
 * [cols, rows] with blocks along the rows (either pair may be NULL, not both);
 * square = 1: blocks of 128 x 128 in both.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED (with codes_t: rows >= 2^22),
 * SQ_ERR_HIP. */
sq_status sq_f8_quantize(const void* X, int32_t type, int64_t rows, int64_t cols, int64_t ld, int32_t square,
                         uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* stream);

/* sq_f8_dequantize -- the values [rows, cols] of a matrix, as fp32 or bf16. */
sq_status sq_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols,
                           void* out, int32_t type, int64_t ld, void* stream);

/* sq_f8_gemm -- C [M, N] = A B^T, A [M, K], B [N, K]; C fp32, or bf16 rounded once to
 * the nearest even.  K = 0 gives zeros.
 * Workspace: sq_f8_gemm_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: SQ_ERR_INVALID_ARGUMENT, SQ_ERR_UNSUPPORTED, SQ_ERR_WORKSPACE_TOO_SMALL,
 * SQ_ERR_HIP. */
sq_status sq_f8_gemm_workspace_size(int64_t M, int64_t N, int64_t K, size_t* bytes);
sq_status sq_f8_gemm(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales,
                     int64_t M, int64_t N, int64_t K, void* C, int32_t type, int64_t ldc,
                     void* workspace, size_t workspace_bytes, void* stream);

/* sq_f8_linear -- Y [M, N] = X W^T with X [M, K] in fp32 or bf16, quantized on the way:
 * what sq_f8_quantize and sq_f8_gemm give.  Few rows (at most 16, more for small
 * layers) take one launch and no workspace, the serving form for single tokens.
 * Workspace: sq_f8_linear_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: as sq_f8_gemm. */
sq_status sq_f8_linear_workspace_size(int64_t M, int64_t K, int64_t N, size_t* bytes);
sq_status sq_f8_linear(const void* X, int32_t type, int64_t M, int64_t K, int64_t ld,
                       const uint8_t* W, const uint8_t* W_scales, int64_t N, void* Y, int32_t out_type, int64_t ldy,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * sq_f8_layer -- the buffers of a linear layer that is trained, allocated once by the
 * caller (host struct, read during the calls only), and its three steps:
 *   sq_f8_layer_weight    codes of W [c_out, c_in] in square blocks, and of W^T, after
 *                         each update of W
 *   sq_f8_layer_forward   codes of X [rows, c_in] along both axes, Y = X W^T
 *   sq_f8_layer_backward  codes of dY [rows, c_out] along both axes, then
 *                         dX = dY W [rows, c_in] and dW = dY^T X [c_out, c_in]
 * Each is what sq_f8_quantize and sq_f8_gemm give; dX and dW share a launch where they
 * take the same tiles.  Y and dX have the layer's type, dW is fp32.
 * Sizes: w [c_out, c_in], w_t [c_in, c_out], x [rows, c_in], x_t [c_in, rows],
 * dy [rows, c_out], dy_t [c_out, rows]; every one of sq_f8_size bytes.
 * Workspace: sq_f8_layer_workspace_size bytes (0: none), 16-byte aligned.
 * Errors: as sq_f8_quantize and sq_f8_gemm.
 * ------------------------------------------------------------------------- */
typedef struct {
    int64_t rows, c_in, c_out;
    int32_t type;                          /* SQ_TYPE_* of X, Y, dY, dX and W */
    int32_t reserved;                      /* 0 */
    uint8_t *w, *w_scales, *w_t, *w_t_scales;
    uint8_t *x, *x_scales, *x_t, *x_t_scales;
    uint8_t *dy, *dy_scales, *dy_t, *dy_t_scales;
    void* workspace;
    size_t workspace_bytes;
} sq_f8_layer;

sq_status sq_f8_layer_workspace_size(const sq_f8_layer* layer, size_t* bytes);
sq_status sq_f8_layer_weight(const sq_f8_layer* layer, const void* W, int64_t ld, void* stream);
sq_status sq_f8_layer_forward(const sq_f8_layer* layer, const void* X, int64_t ld, void* Y, int64_t ldy, void* stream);
sq_status sq_f8_layer_backward(const sq_f8_layer* layer, const void* dY, int64_t ld, void* dX, int64_t ld_dx,
                               float* dW, int64_t ld_dw, void* stream);

/* Static description of a status code. */
const char* sq_status_string(sq_status s);

/* Message of the last failed call on this thread ("" if none);
 * sq_last_error_string is the same function under a second name. */
const char* sq_last_error(void);
const char* sq_last_error_string(void);

#ifdef __cplusplus
}
#endif

#endif /* SHIFTQUANT_H */
