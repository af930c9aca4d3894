/*
 * lmbp.h - C ABI of the low-memory backpropagation kernels for AMD MI355X (gfx950).
 *
 * Operations from "Reducing Fine-Tuning Memory Overhead by Approximate and
 * Memory-Sharing Backpropagation" (Yang et al., ICML 2024):
 *
 *   regelu2_fwd / regelu2_bwd   ReGELU2  (Sec. 4.2; constants Appendix E)
 *   resilu2_fwd / resilu2_bwd   ReSiLU2  (Sec. 4.2; constants Appendix E)
 *   msln_fwd    / msln_bwd      MS-LN    (Sec. 5.2 Alg. 1; Appendix G Alg. 2)
 *   msrms_fwd   / msrms_bwd     MS-RMSNorm (Appendix G Alg. 3)
 *   reswiglu2_fwd / reswiglu2_bwd  ReSiLU2 fused with the SwiGLU product (LLaMA MLP)
 *   stepact_fwd / stepact_bwd      k-bit family members with runtime tables (ReGELU2-d, ...)
 *   linear_act_fwd                 a linear layer whose output goes through ReGELU2 /
 *                                  ReSiLU2, fused (the pre-activation stays on chip)
 *   linear_swiglu_fwd              the LLaMA MLP's two projections + SwiGLU, fused
 *   msrms_linear_act_fwd           MS-RMSNorm, the merged linear layer and ReGELU2 /
 *                                  ReSiLU2 forward, fused (the norm in the GEMM)
 *   msrms_linear_swiglu_fwd        MS-RMSNorm and the LLaMA MLP's input side, fused
 *   q8_rows / q8_values            rows in 8 bits with one scale each, and back
 *   msrms_q8_fwd / msrms_q8_bwd    MS-RMSNorm with the residual's addition, output in 8 bits
 *   linear_q8_fwd / linear_q8_bwd  a frozen linear layer of 8-bit rows and 8-bit weights
 *   linear_bias_grad               the gradient of a linear layer's bias
 *   rope_fwd / rope_bwd            rotary positions of query and key heads, one or several axes
 *   msrms_rope_fwd / msrms_rope_bwd  MS-RMSNorm of each head and the rotation in one pass
 *   attention_fwd / attention_bwd  softmax(scale q k^T) v over packed, padded or equal sequences
 *
 * Conventions shared by every call
 * --------------------------------
 * - Pointers are device pointers (HBM) owned and allocated by the caller; the
 *   library never allocates, frees or synchronizes. Every call only enqueues
 *   kernels on `stream` (a hipStream_t; NULL means the null stream) and returns.
 * - Tensors are dense and row-major. Activation ops see a flat tensor of n
 *   elements; norm ops see `rows` rows of `cols` elements (cols = the normalized
 *   width p of the paper).
 * - dtype selects the storage of every floating-point tensor argument except the
 *   norm statistic `rstd`, which is always fp32. Arithmetic is fp32 in all cases.
 * - Pointers need only element alignment (2 bytes for bf16, 4 for fp32 and for
 *   codes / rstd); 16-byte aligned tensors whose rows are multiples of 16 bytes
 *   take the vectorized path, anything else a slower general path with the same
 *   results up to floating-point summation order.
 * - Aliasing: only the exact in-place pairs named for each call are allowed
 *   (same start address, same size). Any other overlap of two buffers of a call
 *   returns LMBP_EOVERLAP before anything is launched.
 * - Errors are checked on the host before any launch: LMBP_EINVAL for negative
 *   sizes, cols == 0 with rows > 0, a NULL pointer with a nonzero size, a
 *   misaligned pointer, or eps not finite and > 0; LMBP_EDTYPE for an unknown
 *   dtype. n == 0 or rows == 0 is a successful no-op. LMBP_EHIP means the kernel
 *   launch failed; lmbp_last_hip_error() then returns the hipError_t value for the
 *   calling thread. No C++ exception crosses this interface.
 * - Results are deterministic: no atomics, a reduction order fixed by the sizes, the
 *   alignment of the tensors and the device.
 */
#ifndef LMBP_H
#define LMBP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { LMBP_FP32 = 0, LMBP_BF16 = 1 } lmbp_dtype;

typedef enum {
  LMBP_OK = 0,
  LMBP_EINVAL = 1,
  LMBP_EDTYPE = 2,
  LMBP_EOVERLAP = 3,
  LMBP_EHIP = 4
} lmbp_status;

/* Bytes of the packed code buffer for n activation elements: 4 * ceil(n / 16).
 * The code of flat element i occupies bits [2(i mod 16), 2(i mod 16) + 1] of 32-bit
 * word i / 16 (least significant bits first); unused bits of the last word are 0.
 * Returns 0 for n <= 0. */
size_t lmbp_codes_bytes(int64_t n);

/* Static description of a status code. */
const char *lmbp_strerror(lmbp_status st);

/* hipError_t recorded by the last call on this thread that returned LMBP_EHIP. */
int lmbp_last_hip_error(void);

/* ------------------------------------------------------------------------
 * ReGELU2 / ReSiLU2 (Sec. 4.2, eq. relus_family with k = 2).
 *
 * Forward: y = GELU(x) = x/2 (1 + erf(x / sqrt 2))   (regelu2)
 *          y = SiLU(x) = x / (1 + e^-x)              (resilu2)
 * computed exactly (fp32 arithmetic), plus the 2-bit code of every element: the
 * number of the three biases c1 < c2 < c3 of Appendix E lying strictly below x.
 * Backward: dx = dy * s[code], where s = (0, a1, a1 + a2, 1) is the slope of the
 * three-ReLU combination on each of its four segments (Prop. 4.3).
 *
 *   x, y   : n elements of dtype. y == x (in place) is allowed.
 *   codes  : lmbp_codes_bytes(n) bytes, 4-byte aligned, written completely
 *            (including zero tail bits); must not overlap x or y.
 *   dy, dx : n elements of dtype. dx == dy is allowed.
 *   codes (bwd): as written by the matching forward; read only.
 * ------------------------------------------------------------------------ */
lmbp_status regelu2_fwd(lmbp_dtype dt, int64_t n, const void *x, void *y,
                        uint32_t *codes, void *stream);
lmbp_status regelu2_bwd(lmbp_dtype dt, int64_t n, const void *dy,
                        const uint32_t *codes, void *dx, void *stream);
lmbp_status resilu2_fwd(lmbp_dtype dt, int64_t n, const void *x, void *y,
                        uint32_t *codes, void *stream);
lmbp_status resilu2_bwd(lmbp_dtype dt, int64_t n, const void *dy,
                        const uint32_t *codes, void *dx, void *stream);

/* ------------------------------------------------------------------------
 * ReSiLU2 inside a SwiGLU product, h = SiLU(g) * u: the LLaMA MLP, where the paper
 * substitutes ReSiLU2 for SiLU (Sec. 6). The backward is the Approx-BP backward of
 * the product (Sec. 4.1): the exact product rule on the saved forward activation
 * s = SiLU(g), and the step derivative of the three-ReLU combination for SiLU.
 *
 * Forward:  s = SiLU(g), h = s * u, codes of g (as resilu2_fwd).
 * Backward: dg = dh * u * s[code],  du = dh * s.
 *
 *   g, u   : n elements of dtype (inputs). h: n elements (output; h == g or h == u
 *            allowed). s: n elements (output, saved for the backward; overlaps
 *            nothing). codes: lmbp_codes_bytes(n) bytes (output; overlaps nothing).
 *   dh, u, s, codes (bwd): inputs; dg, du: n elements (outputs; dg == dh and
 *            du == u allowed, no other overlap).
 * Saved state per element: the 2-bit code plus s (which the product keeps anyway);
 * g itself is not needed.
 * ------------------------------------------------------------------------ */
lmbp_status reswiglu2_fwd(lmbp_dtype dt, int64_t n, const void *g, const void *u,
                          void *h, void *s, uint32_t *codes, void *stream);
lmbp_status reswiglu2_bwd(lmbp_dtype dt, int64_t n, const void *dh, const void *u,
                          const void *s, const uint32_t *codes, void *dg, void *du,
                          void *stream);

/* ------------------------------------------------------------------------
 * General members of the ReLU-combination family (eq. relus_family with k bits;
 * Appendix I's ReGELU2-d is k = 2 with other constants), with runtime tables.
 *
 * Forward: y = GELU(x) or SiLU(x) exactly (act), and the k-bit code of every
 * element: the number of the 2^k - 1 thresholds strictly below x (the biases c of
 * the combination). Backward: dx = dy * levels[code] (2^k levels: the slopes of the
 * combination on its segments, cumulative sums of its weights).
 *
 *   bits       : k in {1, 2, 3, 4}; codes hold floor(32/k) elements per 32-bit word
 *                (32, 16, 10, 8), least significant first (code j of a word at bits
 *                k j .. k j + k - 1; for k = 3 the top two bits are 0), zero tail;
 *                lmbp_stepact_codes_bytes(k, n) bytes.
 *   thresholds : host array of 2^k - 1 finite, strictly increasing doubles (read
 *                during the call only). Each is applied as an exact real comparison.
 *   levels     : host array of 2^k finite doubles, used as fp32 values.
 *   x, y, dy, dx, codes: as for regelu2_fwd / regelu2_bwd (y == x, dx == dy allowed).
 * LMBP_EINVAL also for bad k, act, tables or a NULL table pointer.
 * ------------------------------------------------------------------------ */
typedef enum { LMBP_ACT_GELU = 0, LMBP_ACT_SILU = 1 } lmbp_act;

size_t lmbp_stepact_codes_bytes(int bits, int64_t n);
lmbp_status stepact_fwd(lmbp_act act, int bits, const double *thresholds, lmbp_dtype dt,
                        int64_t n, const void *x, void *y, uint32_t *codes, void *stream);
lmbp_status stepact_bwd(int bits, const double *levels, lmbp_dtype dt, int64_t n,
                        const void *dy, const uint32_t *codes, void *dx, void *stream);

/* ------------------------------------------------------------------------
 * MS-LN (Sec. 5.2 Alg. 1, Appendix G Alg. 2) and MS-RMSNorm (Alg. 3), for a
 * norm whose affine (alpha, beta) has been merged into the following linear
 * layer (W~ = W diag(alpha), b~ = W beta + b). Per row x of width p = cols:
 *
 * Forward:  sigma = sqrt(p^-1 |H x|^2 + eps),  z = H x / sigma,  rstd = 1 / sigma,
 *           with H x = x - mean(x) for MS-LN and H x = x for MS-RMSNorm.
 * Backward: dx = rstd * (H dz - z * mean(z * dz))   (= sigma^-1 (H - p^-1 z z^T) dz),
 *           computed from the saved output z and rstd only.
 *
 *   x, z    : rows x cols of dtype. z == x (in place) is allowed. z is the
 *             tensor the next (merged) linear layer keeps anyway.
 *   rstd    : rows fp32 values; must not overlap x, z, dz or dx.
 *   eps     : finite, > 0 (the paper uses 1e-6 or 1e-8; LLaMA-style RMSNorm 1e-5).
 *   dz, dx  : rows x cols of dtype. dx == dz is allowed; dx must not overlap z.
 * The sums are fp32 as they are: rows whose squares add up to 2^128 or more (values above 2^64)
 * are not handled (MS-RMSNorm gives rstd = 0 and z = 0; msrms_q8_fwd takes them).
 * ------------------------------------------------------------------------ */
lmbp_status msln_fwd(lmbp_dtype dt, int64_t rows, int64_t cols, float eps,
                     const void *x, void *z, float *rstd, void *stream);
lmbp_status msln_bwd(lmbp_dtype dt, int64_t rows, int64_t cols, const void *dz,
                     const void *z, const float *rstd, void *dx, void *stream);
lmbp_status msrms_fwd(lmbp_dtype dt, int64_t rows, int64_t cols, float eps,
                      const void *x, void *z, float *rstd, void *stream);
lmbp_status msrms_bwd(lmbp_dtype dt, int64_t rows, int64_t cols, const void *dz,
                      const void *z, const float *rstd, void *dx, void *stream);

/* ------------------------------------------------------------------------
 * Linear layer followed by ReGELU2 / ReSiLU2 (Sec. 4.2), forward, fused: the
 * activation runs in the epilogue of the matrix product, so the pre-activation z,
 * which the backward pass of ReGELU2 / ReSiLU2 does not need (it keeps only the
 * codes), never has to be written out.
 *
 *   z = bf16( x W^T + b )        products accumulated in fp32, bias added in fp32,
 *                                one rounding to bf16 (nearest even)
 *   y = act(z), codes = 2-bit codes of z, exactly as regelu2_fwd / resilu2_fwd
 *   compute them from a stored z (same bytes).
 *
 *   dt     : LMBP_BF16 only (LMBP_EDTYPE otherwise).
 *   act    : LMBP_ACT_GELU (ReGELU2) or LMBP_ACT_SILU (ReSiLU2).
 *   m,n,k  : x is m x k, w is n x k (the weight of a linear layer, row-major), y and
 *            z are m x n. n must be a multiple of 16 (each row of codes fills whole
 *            words) and k a multiple of 8 with k <= 2^21; m, n >= 0, k >= 0 (k == 0
 *            gives z = b).
 *   x, w, y, z : 16-byte aligned.
 *   bias   : n bf16 values, or NULL for none.
 *   codes  : lmbp_codes_bytes(m * n) bytes, codes of the flattened m x n output.
 *   z      : NULL (not stored) or m x n bf16.
 * y, codes and z must not overlap each other or any input. The backward pass is
 * regelu2_bwd / resilu2_bwd on the codes followed by the two products of a linear
 * layer's backward.
 * ------------------------------------------------------------------------ */
lmbp_status linear_act_fwd(lmbp_act act, lmbp_dtype dt, int64_t m, int64_t n, int64_t k,
                           const void *x, const void *w, const void *bias, void *y,
                           uint32_t *codes, void *z, void *stream);

/* ------------------------------------------------------------------------
 * The gated form of the same fusion, for the LLaMA MLP (Sec. 6; ReSiLU2 inside
 * SwiGLU as in reswiglu2_fwd): both projections of the MLP's input and the SwiGLU
 * product in one kernel, the gate pre-activation g never written out.
 *
 *   g = bf16( x Wg^T ),  u = bf16( x Wu^T )   (fp32 accumulation, one rounding each)
 *   h = SiLU(g) * u,  s = SiLU(g),  codes of g — exactly what reswiglu2_fwd computes
 *   from stored g and u (same bytes); u is written too, since the backward needs it.
 *
 *   dt : LMBP_BF16 only. m, n, k, alignment and limits as for linear_act_fwd.
 *   x [m x k]; w_gate, w_up [n x k]; h, s, u [m x n]; codes of the m x n output;
 *   g : NULL (not stored) or m x n.
 * Outputs must not overlap each other or any input. Backward: reswiglu2_bwd on
 * (dh, u, s, codes), then the two linear layers' products.
 * ------------------------------------------------------------------------ */
lmbp_status linear_swiglu_fwd(lmbp_dtype dt, int64_t m, int64_t n, int64_t k, const void *x,
                              const void *w_gate, const void *w_up, void *h, void *s, void *u,
                              uint32_t *codes, void *g, void *stream);

/* ------------------------------------------------------------------------
 * MS-RMSNorm in front of the fused linear layer (Sec. 5.2 eq. norm_linear, App. G
 * Alg. 3): the norm's affine merged into W (and b), the normalised row z consumed by
 * the linear layer and kept as the saved tensor of both.
 *
 *   rstd = 1 / sqrt(p^-1 |x|^2 + eps) per row of x (p = k), fp32;
 *   z    = bf16( x rstd )              the norm's output: the same bytes (and rstd the
 *                                      same bits) as msrms_fwd computes from x;
 *   y, codes as linear_act_fwd / linear_swiglu_fwd, with the pre-activation
 *        bf16( rstd (x W^T) + b )      i.e. the row scale is applied to the fp32 sums of
 *                                      the products of x, before the bias: the linear
 *                                      layer sees the normalised row before its storage
 *                                      rounding (equal to z W^T + b in exact arithmetic;
 *                                      not byte-equal to linear_act_fwd applied to z).
 *
 * The norm kernel writes z and rstd; then the GEMM runs on x and applies rstd to each
 * row's sums in its epilogue.
 *
 *   dt   : LMBP_BF16 only.
 *   m,n,k, x, w, bias, y, codes : as linear_act_fwd, with k >= 8 when m > 0.
 *   eps  : finite and > 0 (as msrms_fwd).
 *   pre  : NULL (not stored) or m x n bf16: the rounded pre-activation, from which y
 *          and codes are exactly what regelu2_fwd / resilu2_fwd compute (as
 *          linear_act_fwd's z).
 *   z    : m x k bf16, 16-byte aligned (required: the saved tensor).
 *   rstd : m fp32, 4-byte aligned.
 * n == 0 (no output features) still writes z and rstd, by the stand-alone norm kernel;
 * w, bias, y, codes and pre are then not used. m == 0 is a successful no-op.
 * No output may overlap another output or an input. The backward pass is the linear
 * layer's (or SwiGLU's) backward on the kept tensors, then msrms_bwd(dz, z, rstd).
 * ------------------------------------------------------------------------ */
lmbp_status msrms_linear_act_fwd(lmbp_act act, lmbp_dtype dt, int64_t m, int64_t n, int64_t k,
                                 float eps, const void *x, const void *w, const void *bias,
                                 void *y, uint32_t *codes, void *pre, void *z, float *rstd,
                                 void *stream);

/* The gated form: MS-RMSNorm, then linear_swiglu_fwd's two projections and SwiGLU
 * (g and u each bf16(rstd (x W^T))), z and rstd as above; h, s, u, codes and the
 * optional g (NULL: not stored) as linear_swiglu_fwd. */
lmbp_status msrms_linear_swiglu_fwd(lmbp_dtype dt, int64_t m, int64_t n, int64_t k, float eps,
                                    const void *x, const void *w_gate, const void *w_up, void *h,
                                    void *s, void *u, uint32_t *codes, void *g, void *z,
                                    float *rstd, void *stream);

/* ------------------------------------------------------------------------
 * Backward of the fused linear layers with respect to their parameters.
 *
 *   linear_weight_grad : dw = bf16( dz^T x ), sums over the m rows in fp32, one rounding.
 *   linear_act_bwd     : dz = dy * slope[code] (as regelu2_bwd / resilu2_bwd; db of the
 *                        column sums of the rounded dz, fp32 sums, one rounding) and dw.
 *
 *   dt  : LMBP_BF16 only. m, n, k >= 0; n a multiple of 16, k of 8; n, k <= 2^24.
 *   dz, dy [m x n], x [m x k], dw [n x k], db [n]. linear_act_bwd: codes as written by
 *         the forward; dw NULL: not computed (x is then not used); db NULL: not computed;
 *         dz overlaps no other buffer (not in place, as an activation backward may be).
 *   workspace : lmbp_linear_grad_bytes(m, n, k, bias) bytes on the calling thread's
 *         current device, 16-byte aligned (bias: nonzero if db is computed; k: 0 if dw is
 *         not). NULL if that is 0. Its contents do not matter before or after.
 * All tensors 16-byte aligned (db: 2, codes: 4); m == 0 gives zeros.
 * ------------------------------------------------------------------------ */
size_t lmbp_linear_grad_bytes(int64_t m, int64_t n, int64_t k, int bias);
lmbp_status linear_weight_grad(lmbp_dtype dt, int64_t m, int64_t n, int64_t k, const void *dz,
                               const void *x, void *dw, void *workspace, int64_t workspace_bytes,
                               void *stream);
lmbp_status linear_act_bwd(lmbp_act act, lmbp_dtype dt, int64_t m, int64_t n, int64_t k,
                           const void *dy, const uint32_t *codes, const void *x, void *dz,
                           void *dw, void *db, void *workspace, int64_t workspace_bytes,
                           void *stream);

/* ------------------------------------------------------------------------
 * Rows in 8 bits, one fp32 scale per row. Of a row t:
 *
 *   a = max(max |t|, 2^-100),  scale = a / 127,  q = t r rounded half to even
 *
 * with r = 127 / a rounded to fp32 and the product t r not rounded before q. The row stands
 * for q scale; q lies in -127 .. 127. A row that holds an infinity or a NaN gets scale NaN
 * and q = 0, so that what is formed from it is NaN.
 *
 *   q8_rows   : x [rows x cols] of dtype -> q [rows x cols], scale [rows].
 *   q8_values : v = q scale, one rounding to dtype. Any q (also -128) and scale.
 * Nothing overlaps. scale: 4-byte aligned.
 * ------------------------------------------------------------------------ */
lmbp_status q8_rows(lmbp_dtype dt, int64_t rows, int64_t cols, const void *x, int8_t *q,
                    float *scale, void *stream);
lmbp_status q8_values(lmbp_dtype dt, int64_t rows, int64_t cols, const int8_t *q,
                      const float *scale, void *v, void *stream);

/* ------------------------------------------------------------------------
 * MS-RMSNorm (Appendix G Alg. 3) with the residual's addition in front and its output in 8
 * bits: what the norm keeps takes one byte per element, and linear_q8_fwd takes it as it is
 * (a frozen layer keeps nothing of it). Per row:
 *
 * Forward:  s = x + res, rounded to dtype (s = x without res),
 *           rstd = 1 / sqrt(p^-1 |s|^2 + eps),  z = s rstd  as q scale:
 *           q the 8-bit row of s (as q8_rows), scale = a rstd / 127.
 *           Of finite rows of any size: squares that fp32 does not hold are formed again
 *           of smaller (larger) values.
 * Backward: with z = q scale,  dx = rstd (dz - z mean(z dz)) + ds.
 *           dx is the gradient of x and of res alike; ds is the gradient that reaches s
 *           past the norm.
 *           dz of any size, as long as dz - z mean(z dz) is one of fp32's numbers.
 *
 *   x, res, s : rows x cols of dtype. res and s both NULL or both given; s == x and
 *               s == res are allowed, x == res too.
 *   q         : rows x cols; scale, rstd: rows fp32 values.
 *   eps       : finite, > 0.
 *   dz, ds, dx: rows x cols, dz of dt_dz, ds (NULL for none) and dx of dtype: the same, or dz
 *               fp32 with dtype bf16 (a sum over several layers is worth keeping in fp32;
 *               LMBP_EDTYPE the other way round). dx == dz, if of one type, and dx == ds are
 *               allowed.
 * No other overlap. The rounding to 8 bits is passed over by the backward, which is the
 * gradient of the norm at the z that was kept.
 * ------------------------------------------------------------------------ */
lmbp_status msrms_q8_fwd(lmbp_dtype dt, int64_t rows, int64_t cols, float eps, const void *x,
                         const void *res, void *s, int8_t *q, float *scale, float *rstd,
                         void *stream);
lmbp_status msrms_q8_bwd(lmbp_dtype dt_dz, lmbp_dtype dt, int64_t rows, int64_t cols,
                         const void *dz, const int8_t *q, const float *scale, const float *rstd,
                         const void *ds, void *dx, void *stream);

/* ------------------------------------------------------------------------
 * A linear layer whose frozen weight is kept in 8 bits, one scale per output channel (as
 * q8_rows gives for w [n x k]), on rows in 8 bits:
 *
 *   y  = (sum_k q[m, k] w[n, k]) (scale[m] w_scale[n]) + bias[n]
 *   dx = (sum_n p[m, n] w[n, k]) p_scale[m] + add,   p, p_scale the 8-bit rows of dy w_scale
 *
 * The sums are exact (whole numbers in 32 bits), everything behind them is fp32 with one
 * rounding to dtype; scale[m] w_scale[n] is formed first.
 *
 *   dt     : type of y and bias, or of dy; dt_dx: type of add and dx.
 *   m,n,k  : any sizes >= 0 below 2^31; the length of the sums (k forward, n backward) at
 *            most 131071. k = 0 gives y = bias (0 without), n = 0 dx = add (0 without).
 *   q [m x k], w [n x k]: any values; scale [m], w_scale [n]; bias [n] or NULL; y, dy [m x n];
 *            add, dx [m x k], add NULL for none; dx == add is allowed (the sum of several
 *            layers' gradients).
 *   workspace : lmbp_linear_q8_fwd_bytes / lmbp_linear_q8_bwd_bytes(m, n, k) bytes on the
 *            calling thread's current device, 16-byte aligned, NULL if that is 0. Its contents
 *            do not matter before or after.
 * k a multiple of 16 and 16-byte aligned q and w are the fast case, anything else
 * slower with the same results. No other output overlaps another buffer.
 * ------------------------------------------------------------------------ */
lmbp_status linear_q8_fwd(lmbp_dtype dt, int64_t m, int64_t n, int64_t k, const int8_t *q,
                          const float *scale, const int8_t *w, const float *w_scale,
                          const void *bias, void *y, void *workspace, int64_t workspace_bytes,
                          void *stream);
size_t lmbp_linear_q8_fwd_bytes(int64_t m, int64_t n, int64_t k);
size_t lmbp_linear_q8_bwd_bytes(int64_t m, int64_t n, int64_t k);
lmbp_status linear_q8_bwd(lmbp_dtype dt, lmbp_dtype dt_dx, int64_t m, int64_t n, int64_t k,
                          const void *dy, const int8_t *w, const float *w_scale,
                          const void *add, void *dx, void *workspace, int64_t workspace_bytes,
                          void *stream);

/* ------------------------------------------------------------------------
 * Gradient of a linear layer's bias: db[n] = sum over the rows of dy [m x n], added up in fp32 in
 * an order fixed by m, n, the alignment of dy and the device, one rounding to dt_db.
 * (linear_act_bwd has it with the activation's backward.)
 *
 *   dt, dt_db : types of dy and db, any two.
 *   m, n      : any sizes >= 0, n below 2^31; m = 0 gives db = 0.
 *   workspace : lmbp_linear_bias_grad_bytes(m, n) bytes on the calling thread's current device,
 *               16-byte aligned, NULL if that is 0.
 * Nothing overlaps.
 * ------------------------------------------------------------------------ */
lmbp_status linear_bias_grad(lmbp_dtype dt, lmbp_dtype dt_db, int64_t m, int64_t n, const void *dy,
                             void *db, void *workspace, int64_t workspace_bytes, void *stream);
size_t lmbp_linear_bias_grad_bytes(int64_t m, int64_t n);

/* ------------------------------------------------------------------------
 * Tensors of heads: rows (tokens) of heads of `dim` columns. The columns of a head lie together; `row` and `head`
 * are the elements from one row, one head to the next (>= 0; 0 for inputs only). So queries, keys and values
 * may lie in the one output of a fused projection. Written tensors must not meet themselves: row at least
 * (heads - 1) head + dim, or head at least (rows - 1) row + dim. Two tensors of a call that are interleaved
 * without sharing an element (parts of the same rows, or of the heads of rows: [rows][heads][3][dim]) do not overlap.
 * ------------------------------------------------------------------------ */
typedef struct {
  void *data;
  int64_t row, head;
} lmbp_heads;

/* ------------------------------------------------------------------------
 * Rotary positions. Columns are taken in pairs; pair p of a token's head turns by the angle
 * t = freqs[p] * positions[axes[p]][token]:  (a, b) -> (a cos t - b sin t, a sin t + b cos t).
 *
 *   rope_fwd : y = x turned;  rope_bwd: dx = dy turned back. fp32 arithmetic, one rounding. A frequency (of less
 *              than 2^52 radians) is cut to a whole number of 2^-64 turns, within 1.5 of them, and nothing else is lost before
 *              sine and cosine: the angle is off by less than 1.5 |position| 2^-64 turns, 6e-7 radians at 2^40, 5e-3 at 2^53.
 *
 *   tokens, dim : tokens >= 0; 1 <= dim <= 512.
 *   q_heads, k_heads : heads of the two tensors; k_heads = 0: there is no second one (k, yk NULL).
 *   pairs   : 0 <= 2 pairs <= dim; pair p is columns p and p + pairs, or (interleaved) 2 p and 2 p + 1; columns from
 *             2 pairs on are left as they are.
 *   freqs   : pairs finite doubles in HOST memory, radians per position; axes: pairs numbers 0 .. n_axes - 1 in
 *             HOST memory, NULL for all 0. 1 <= n_axes <= 255. Both are read before the call returns.
 *   positions : n_axes x tokens whole numbers in device memory, int64 (wide != 0) or int32; any values.
 * Each y may be its x (same address, strides and heads); no other overlap.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t tokens, dim, q_heads, k_heads, pairs;
  const double *freqs;
  const int32_t *axes;
  const void *positions;
  int n_axes, wide, interleaved;
} lmbp_rope;

lmbp_status rope_fwd(lmbp_dtype dt, const lmbp_rope *r, const lmbp_heads *q, const lmbp_heads *k,
                     const lmbp_heads *yq, const lmbp_heads *yk, void *stream);
lmbp_status rope_bwd(lmbp_dtype dt, const lmbp_rope *r, const lmbp_heads *dq, const lmbp_heads *dk,
                     const lmbp_heads *dxq, const lmbp_heads *dxk, void *stream);

/* ------------------------------------------------------------------------
 * MS-RMSNorm (Appendix G Alg. 3) of each head and the rotation in one pass. Per head of D columns:
 *
 * Forward:  rstd = 1 / sqrt(D^-1 |x|^2 + eps), z = x rstd, y = turned (gain z).
 *           Heads of any size: squares that fp32 does not hold are formed again of smaller (larger) values.
 * Backward: without gain from the output y, which attention keeps anyway (turning keeps products):
 *           dx = turned back (rstd (dy - y D^-1 (y . dy))).
 *           With gain from x: g = dy turned back, dz = gain g, dx = rstd (dz - z D^-1 (z . dz)),
 *           dgain = sum of g z over tokens and heads, in fp32 in an order fixed by the sizes.
 *           The products y . dy (z . dz) have to be among fp32's numbers. A head that is not finite (rstd 0 or NaN) and whose dy
 *           is zeros gets zeros and adds nothing to dgain: rows of no sequence may hold anything.
 *
 *   eps     : finite, > 0. rstd_q, rstd_k: fp32 [tokens][heads].
 *   q_gain, k_gain : dim values of dt_gain (fp32 or bf16), both NULL or (k_gain only with k_heads) both given;
 *             dq_gain, dk_gain: dim values of dt_gain (outputs), NULL without gains.
 *   kept_q, kept_k : y of the forward without gains, x with.
 *   workspace : lmbp_msrms_rope_bwd_bytes(dim) bytes, 16-byte aligned, with gains; NULL without.
 * y may be its x, dx its dy; no other overlap.
 * ------------------------------------------------------------------------ */
lmbp_status msrms_rope_fwd(lmbp_dtype dt, lmbp_dtype dt_gain, const lmbp_rope *r, float eps,
                           const void *q_gain, const void *k_gain, const lmbp_heads *q,
                           const lmbp_heads *k, const lmbp_heads *yq, const lmbp_heads *yk,
                           float *rstd_q, float *rstd_k, void *stream);
lmbp_status msrms_rope_bwd(lmbp_dtype dt, lmbp_dtype dt_gain, const lmbp_rope *r,
                           const void *q_gain, const void *k_gain, const lmbp_heads *dq,
                           const lmbp_heads *dk, const lmbp_heads *kept_q,
                           const lmbp_heads *kept_k, const float *rstd_q, const float *rstd_k,
                           const lmbp_heads *dxq, const lmbp_heads *dxk, void *dq_gain,
                           void *dk_gain, void *workspace, int64_t workspace_bytes, void *stream);
size_t lmbp_msrms_rope_bwd_bytes(int64_t dim);

/* ------------------------------------------------------------------------
 * Attention (bf16). Of each query (a row of q, a head) over the keys that it sees:
 *
 * Forward:  S = scale q k^T, P = softmax(S), o = P v, lse = log sum exp S (natural).
 * Backward: D = sum of do o, dS = P (do v^T - D), dq = scale dS k, dk = scale dS^T q, dv = P^T do.
 *
 * Sums, maxima and lse are fp32; P and dS are rounded to bf16 as factors of the matrix products (the sum of P is
 * not), results once. heads / kv_heads query heads in a row share a key head; its gradients are summed over them.
 * Sequences: `batch` of them, one behind the other in the rows. Side by side, for queries and for keys:
 *   starts NULL : all of one length, rows / batch (a whole number);
 *   starts      : batch + 1 ascending row numbers in device memory, the first 0 (taken as 0), the last at most
 *                 the rows. Rows from the last on belong to no sequence.
 *   k_lens      : NULL, or batch numbers in device memory: only so many of a sequence's keys are in use (a
 *                 padded cache). What lies behind them is not read.
 * Of sequence lengths nq and nk (keys in use), query i sees keys j < nk and, if causal, j <= i + nk - nq: the
 * last query sees all. A query that sees none has o = 0 and lse = -inf, and gives and gets no gradient.
 * Keys that a query does not see may hold anything, infinities and NaN included.
 * An infinity in v of a key that is seen makes o infinite there, or NaN where the key's weight rounds to 0 on the way.
 * Starts or k_lens that break the rules above give wrong results, but no access outside the tensors.
 *
 *   dt          : LMBP_BF16 (LMBP_EDTYPE otherwise).
 *   heads, kv_heads : kv_heads divides heads. dim: a multiple of 8, 8 .. 128.
 *   q_rows heads / kv_heads and k_rows : below 2^31 - 1024. batch >= 1.
 *   scale       : > 0; scale log2(e) finite.
 *   fill        : 0 leaves o and lse, dq, dk, dv of rows of no sequence (and dk, dv of keys not in use) as they
 *                 were; otherwise they get zeros (lse -inf).
 *   q, k, v, o, d_o, dq, dk, dv : 16-byte aligned, strides multiples of 8; 128 row + heads head of each below 2^30.
 *   lse         : fp32 [q_rows][heads].
 *   workspace   : lmbp_attention_fwd_bytes / lmbp_attention_bwd_bytes on the calling thread's current device,
 *                 16-byte aligned, NULL if that is 0. Its contents do not matter before or after.
 * No output overlaps another buffer. Results do not depend on the order of blocks; how keys (forward) and rows
 * (dk, dv) are shared out goes by the sizes and the device.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t batch, heads, kv_heads, dim, q_rows, k_rows;
  const int32_t *q_starts, *k_starts, *k_lens;
  float scale;
  int causal, fill;
} lmbp_attention;

lmbp_status attention_fwd(lmbp_dtype dt, const lmbp_attention *a, const lmbp_heads *q,
                          const lmbp_heads *k, const lmbp_heads *v, const lmbp_heads *o, float *lse,
                          void *workspace, int64_t workspace_bytes, void *stream);
lmbp_status attention_bwd(lmbp_dtype dt, const lmbp_attention *a, const lmbp_heads *d_o,
                          const lmbp_heads *q, const lmbp_heads *k, const lmbp_heads *v,
                          const lmbp_heads *o, const float *lse, const lmbp_heads *dq,
                          const lmbp_heads *dk, const lmbp_heads *dv, void *workspace,
                          int64_t workspace_bytes, void *stream);
size_t lmbp_attention_fwd_bytes(const lmbp_attention *a);
size_t lmbp_attention_bwd_bytes(const lmbp_attention *a);

/* ------------------------------------------------------------------------
 * Test utilities (host only, no launch): the kernel form that a size takes on the calling
 * thread's current device, or on 256 CUs where there is none.
 *   lmbp_linear_form : 0, 1 split-K with 16, 32 rows to a block; 2 .. 5 tiles of 256 x 256,
 *                      128 x 256, 128 x 128, 64 x 128; *rounds (or NULL): the most tiles
 *                      that one block computes. -1 for sizes that run nothing.
 *   lmbp_linear_grad_form : 0 .. 2 tiles of 256 x 256, 128 x 256, 128 x 128; *splits (or
 *                      NULL): the shares of the rows; *rounds (or NULL): as above.
 *   lmbp_linear_q8_form : the 8-bit layers' forward, or (grad) input gradient, on 16-byte
 *                      aligned tensors: 0 dot products (forward), 1 .. 3 split-K with 16, 32,
 *                      64 rows to a block, 4 .. 7 tiles of 64 x 128, 128 x 128, 128 x 256,
 *                      256 x 256, 8 the general form; *shares (or NULL): the blocks that share
 *                      a sum; *copies (or NULL): 1 if rows are copied to aligned ones first.
 * ------------------------------------------------------------------------ */
int lmbp_linear_form(int64_t m, int64_t n, int64_t k, int gated, int64_t *rounds);
int lmbp_linear_grad_form(int64_t m, int64_t n, int64_t k, int64_t *splits, int64_t *rounds);
int lmbp_linear_q8_form(int64_t m, int64_t n, int64_t k, int grad, int64_t *shares, int64_t *copies);

/* ------------------------------------------------------------------------
 * Measurement utility (not part of the method): copies `bytes` bytes from src
 * to dst with 16-byte non-temporal vector loads and non-temporal device-scope vector
 * stores (written through the L2), the fastest plain copy measured on the GPU for
 * tensors of 32 MiB and more. src and dst must be 16-byte
 * aligned and must not overlap. Used as the plain-copy reference for bandwidth
 * and hardware-counter calibration.
 * ------------------------------------------------------------------------ */
lmbp_status lmbp_copy(const void *src, void *dst, int64_t bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LMBP_H */
