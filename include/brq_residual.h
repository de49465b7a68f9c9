/*
 * brq_residual.h -- C ABI of the residual side of a block-rotated MXFP4 layer for MI355X (gfx950).
 *
 * What stands between the W4A4 products of two sublayers: a product's result joins the residual stream,
 * the stream's RMS norm is the next product's input.  So there are the norm with the residual's addition
 * in front of it, alone (with its gradients) and fused into the online step that makes the product's
 * operand, and the product with bias, activation and the residual's addition behind it.  The conventions
 * of brq.h hold (device pointers, caller-owned buffers, nothing allocated, work enqueued on `stream`,
 * argument errors found on the host before anything is launched, K % 32 == 0, 16-byte aligned pointers and
 * row pitches), and these besides:
 *   - Outputs may not overlap inputs or one another, except that an output may take the place of an input matrix
 *     where its function below says so: the same address, dtype and row pitch (anything else at that address is refused).
 *   - A workspace is one call's until that call's work is done: calls on one stream may share it, calls on two may not.
 *   - Infinities and NaN are not refused: they stay in their row (norms) or element (bias, residual).
 */
#ifndef BRQ_RESIDUAL_H
#define BRQ_RESIDUAL_H

#include "brq.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The residual's addition and the RMS norm of the sum, a row at a time:
 *     h[m][k] = x[m][k] + res[m][k]                         rounded once to rdt
 *     y[m][k] = h[m][k] / sqrt(mean_k h[m][k]^2 + eps) * w[k]     of the rounded h; rounded once to ydt
 * in fp32.  res NULL: h = x, and `h` must be NULL (rdt and ldr are not looked at).  h NULL: the sum is not
 * wanted.  w: [K] fp32, 16-byte aligned, or NULL (no weight).  eps >= 0 and not NaN; with eps = 0 a row of
 * zeros comes out as NaN, and one whose squares vanish in fp32 as infinities.  The sum of a row's squares has to be finite in fp32.
 * x [M][ldx] of xdt, res [M][ldr] and h [M][ldh] of rdt, y [M][ldy] of ydt.  K <= 32768.  h and y may each take the place of x or of res.
 */
brq_status brq_add_rms_norm(const void* x, brq_dtype xdt, int64_t ldx, const void* res, brq_dtype rdt,
                            int64_t ldr, int64_t M, int64_t K, const float* w, float eps, void* h, int64_t ldh,
                            void* y, brq_dtype ydt, int64_t ldy, void* stream);

/*
 * Its gradients.  From h (the sum as it was stored; x where there was no residual), the gradient gy of y and
 * the gradient gh that reaches h by the other way, through the residual stream (NULL: none):
 *     r = 1 / sqrt(mean h^2 + eps),   g = gy w,
 *     dh = r (g - h r^2 mean_k(g h)) + gh,      dw[k] = sum_m gy[m][k] h[m][k] r[m]
 * dh is the gradient of x and of res alike.  h, gh and dh are of hdt, gy of gdt; dh may take the place of h, gy
 * or gh.  dw: [K] fp32, set, not added to; NULL: not wanted (must be NULL where w is).
 * M = 0 sets it to zero.  Its sums are made in an order that depends on the sizes alone.
 * workspace: brq_add_rms_norm_backward_workspace bytes, 16-byte aligned; may be NULL where dw is.
 */
brq_status brq_add_rms_norm_backward(const void* h, brq_dtype hdt, int64_t ldh, const void* gy, brq_dtype gdt,
                                     int64_t ldgy, const void* gh, int64_t ldgh, int64_t M, int64_t K,
                                     const float* w, float eps, void* dh, int64_t lddh, float* dw,
                                     void* workspace, int64_t workspace_bytes, void* stream);
brq_status brq_add_rms_norm_backward_workspace(int64_t M, int64_t K, int64_t* bytes);

/*
 * The norm in front of the online step:
 *     brq_rotate_quantize_fused(y, B, signs)   with (h, y) = brq_add_rms_norm(x, res, w, eps) and y of ydt,
 * in one pass; y never visits memory.  Bit-identical to that two-call sequence of THIS library (ydt =
 * BRQ_BF16 rounds y to bf16 before the rotation; BRQ_F32 keeps the fp32 value).  h may take the place of x or of res.
 * B = 1 (no rotation; signs must then be NULL) or 8 ... 512: blocks that a wavefront holds.  Wider ones: the
 * two calls.  K <= 32768, as the norm alone.
 */
brq_status brq_add_rms_norm_rotate_quantize_fused(const void* x, brq_dtype xdt, int64_t ldx, const void* res,
                                                  brq_dtype rdt, int64_t ldr, int64_t M, int64_t K, const float* w,
                                                  float eps, void* h, int64_t ldh, brq_dtype ydt, int64_t B,
                                                  const int8_t* signs, uint8_t* codes, uint8_t* scales,
                                                  brq_layout layout, void* stream);

/*
 * The W4A4 product with what follows it:
 *     y[m][n] = act(p[m][n] + bias[n]) + residual[m][n],     p[m][n] = sum_k deq(a)[m][k] deq(w)[n][k] in fp32
 * evaluated in fp32 on the accumulators and rounded once to ydt.  p is not bit for bit brq_mxfp4_gemm's: up to 64 rows, and few
 * tiles with a long K, go to kernels that add its terms in another order (no less exact), so the last bits of a row may differ with M
 * too.  The same call gives the same bits.  With nothing behind the product (no bias, BRQ_ACT_NONE, no residual) the call is
 * brq_mxfp4_gemm, its kernels and its bits.
 * bias: [N] fp32, 4-byte aligned, or NULL.  residual: [M][ldr] of rdt or NULL (rdt and ldr are then not looked
 * at); its address is a multiple of its element's size, its pitch free, and y may take its place.  y's pitch is free (>= N) as in brq_mxfp4_gemm.
 * act of t:  BRQ_ACT_RELU  max(t, 0) (NaN stays NaN);   BRQ_ACT_SILU  t / (1 + exp(-t));
 *            BRQ_ACT_GELU  t/2 erfc(-t / sqrt 2)  (the exact one, not its tanh form)
 * workspace: brq_mxfp4_gemm_epilogue_workspace bytes (may be 0, then NULL; where nothing follows the product too),
 * 16-byte aligned: a product of few tiles and a long K is split along K, and the slices' fp32 sums are added in
 * their order.
 * Of the fp32 t the activations are within (8 + 2 |t|) 2^-24 |silu(t)| + 2^-119 |t| and (16 + 2 t^2) 2^-24 |gelu(t)|
 * + 2^-118.
 */
typedef enum {
    BRQ_ACT_NONE = 0,
    BRQ_ACT_RELU = 1,
    BRQ_ACT_SILU = 2,
    BRQ_ACT_GELU = 3,
    BRQ_ACT_INT_RANGE_ = 0x7fffffff
} brq_activation;      /* anything else: BRQ_ERR_ACTIVATION */

brq_status brq_mxfp4_gemm_epilogue(const uint8_t* aq, const uint8_t* as, brq_layout a_layout, const uint8_t* wq,
                                   const uint8_t* ws, brq_layout w_layout, int64_t M, int64_t N, int64_t K,
                                   const float* bias, brq_activation act, const void* residual, brq_dtype rdt,
                                   int64_t ldr, void* y, brq_dtype ydt, int64_t ldy, void* workspace,
                                   int64_t workspace_bytes, void* stream);
brq_status brq_mxfp4_gemm_epilogue_workspace(brq_layout a_layout, brq_layout w_layout, int64_t M, int64_t N, int64_t K,
                                             int64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* BRQ_RESIDUAL_H */
