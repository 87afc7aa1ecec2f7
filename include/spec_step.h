/*
 * libspec, operators of a training step that the kernels of spec_train.h leave to the
 * caller (of use at decoding time too, as said at each): the gated half of a
 * feed-forward block (its down projection is a plain product, and not here), the
 * clipping of all gradients together, the embedding lookup with the gradient of its
 * table (for models that train their own: a draft layer as spec.h has it shares the
 * target's), and norms of the heads of q and k in the pass of their rotary embedding
 * (for models that have such norms: those of spec.h have none).  Same conventions as
 * spec_layer8.h: all data pointers are DEVICE pointers unless a comment says "host",
 * calls enqueue on `stream` (a hipStream_t, NULL = default stream, of the CURRENT
 * device) and return without waiting; no call
 * allocates device memory or keeps anything for the next; SPEC_OK, or SPEC_EINVAL
 * (nothing has been launched), or SPEC_EHIP.  dtype is SPEC_DTYPE_FP32 or
 * SPEC_DTYPE_BF16.  Buffers, scratch among them, are borrowed until the kernels have
 * run: two calls may run at once if neither writes what the other uses.  Calls may be
 * captured into a graph.  Results do not depend on timing: the same call gives the
 * same bits.  A value that is rounded to a smaller type is rounded once, to nearest,
 * ties to even, at the end, where nothing else is said.
 */
#ifndef SPEC_STEP_H_
#define SPEC_STEP_H_

#include <stdint.h>

#include "spec_layer8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- embedding ------------------------------------------------------------------
 * out[i] = scale * table[tok[i]] (the product in fp32), zeros where tok[i] is not in 0 .. vocab-1 (padding).
 * table [vocab, d] in dtype with row stride ldt >= d, out [rows, d] in out_dtype with
 * row stride ldo >= d (what lies between rows is left alone).  1 <= rows <= 2^24, 1 <=
 * d <= 2^20, 1 <= vocab <= 2^24; pointers aligned to their type (fastest where they, the
 * strides and d are multiples of 16 bytes); out overlaps neither table nor tok. */
int spec_k_embed(int32_t dtype, const void *table, int64_t ldt, int32_t vocab, int32_t d, const int32_t *tok, int32_t rows, float scale,
                 int32_t out_dtype, void *out, int64_t ldo, void *stream);

/* The gradient of the table: dtable[v] = scale * (sum of dy[i] over the i with tok[i] = v),
 * for every v (zeros where there is none).  accumulate != 0: dtable[v] += that, and rows
 * without a token are neither read nor written.  Rows whose tok is not in 0 .. vocab-1 have no part in it, whatever they hold.
 * dy [rows, d] in dtype, row stride ldy; dtable [vocab, d] in out_dtype, row stride ldt;
 * sums in fp32 in an order that depends on tok alone: up to 31 rows of a token in the order of their positions; more are added in groups that
 * depend on the other tokens too, so that such a row's last bits may change with them.  1 <= rows <= 2^20, the rest as
 * above.  scratch: spec_k_embed_grad_scratch_bytes (host only; 0 for bad sizes), 256-byte
 * aligned; dtable overlaps none of the others. */
uint64_t spec_k_embed_grad_scratch_bytes(int32_t rows, int32_t vocab, int32_t d);
int spec_k_embed_grad(int32_t dtype, const void *dy, int64_t ldy, const int32_t *tok, int32_t rows, int32_t d, int32_t vocab, float scale,
                      int32_t accumulate, int32_t out_dtype, void *dtable, int64_t ldt, void *scratch, uint64_t scratch_bytes, void *stream);

/* ---- norms of heads, with the rotary embedding ---------------------------------
 * For each head x [hd] of a part with a weight w [hd]:
 *     r = 1 / sqrt(sum x^2 / hd + eps),   z = x * r * (offset + w),
 * and out = z turned by spec_k_rotary's rule (plan, pos, part.turn; dims behind
 * plan.rot pass unturned).  w NULL: z = x, so that the call does what spec_k_rotary does.
 * Parts, strides, positions, sizes and aliasing as in spec_k_rotary; w in w_dtype,
 * aligned to it.  Squares, sums and products are fp32: heads with values
 * beyond 2^60 may come out as zeros.  eps >= 0 and finite; with eps = 0 a head of zeros gives NaN, one of values under 2^-60 may give
 * infinities or NaN too. */
typedef struct spec_headnorm_part {
  spec_rotary_part p;
  const void *w;
  int32_t w_dtype;
  float   offset;
} spec_headnorm_part;
int spec_k_headnorm_rotary(const spec_rotary_plan *plan /* host */, int32_t n_parts, const spec_headnorm_part *parts /* host */, int32_t hd, int32_t rows,
                           const int32_t *pos, int32_t pos0, float eps, void *stream);

/* Its gradients.  With dz = dy turned back (the adjoint of the turning), per head
 *     s = sum((offset + w) dz x) / hd,   dx = r ((offset + w) dz - x r^2 s),
 *     dw = sum over rows and heads of dz x r,
 * w NULL: dx = dz.  A part's p.x is dy in p.dtype, p.out is dx in p.out_dtype (p.x = p.out: in place, as
 * in spec_k_rotary); x, in x_dtype, is the call's input, head h of row r at r * ld + h * hs; it may
 * be NULL where w is.  dw: fp32 [hd], or NULL; summed in fp32 in an order that depends on the sizes alone.  No dx overlaps any x.  scratch:
 * spec_k_headnorm_rotary_grad_scratch_bytes (host only), 256-byte aligned; it
 * may be NULL if no part has a dw. */
typedef struct spec_headnorm_grad_part {
  spec_rotary_part p;
  const void *w;
  int32_t w_dtype;
  float   offset;
  const void *x;
  int64_t ld, hs;
  float  *dw;
  int32_t x_dtype;
  int32_t reserved;   /* 0 */
} spec_headnorm_grad_part;
uint64_t spec_k_headnorm_rotary_grad_scratch_bytes(int32_t n_parts, int32_t hd);
int spec_k_headnorm_rotary_grad(const spec_rotary_plan *plan /* host */, int32_t n_parts, const spec_headnorm_grad_part *parts /* host */, int32_t hd, int32_t rows,
                                const int32_t *pos, int32_t pos0, float eps, void *scratch, uint64_t scratch_bytes, void *stream);

/* ---- gated feed-forward block ------------------------------------------------------
 * h = act(x w_gate^T) * (x w_up^T): x [rows, d], w_gate and w_up [f, d], h [rows, f], all bf16 and row-major, as a
 * program trains them (spec_k_gemm_swiglu and spec_k_gemm8 take weights that are packed once).
 *   SPEC_ACT_SILU       g / (1 + e^-g)
 *   SPEC_ACT_GELU       g (1 + erf(g / sqrt 2)) / 2
 *   SPEC_ACT_GELU_TANH  g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2
 * Sums and activations in fp32.  Row strides ldx, ldw, .. in elements; d, f and the strides are multiples of 8,
 * pointers of 16 bytes.  1 <= rows <= 2^20, d, f <= 2^20, rows * d, rows * f and d * f <= 2^36, strides <=
 * 2^21.  What lies between rows is left alone.  h overlaps no input.  Up to 128 rows the call reads the weights once
 * and is bound by that (decoding with weights as they are trained); the order of a sum depends on the number of rows, so that a row's last bits may change
 * with it. */
#define SPEC_ACT_SILU 0
#define SPEC_ACT_GELU 1
#define SPEC_ACT_GELU_TANH 2
int spec_k_ffn_gated(const void *x, int64_t ldx, int32_t rows, int32_t d, const void *w_gate, const void *w_up, int64_t ldw, int32_t f, int32_t act,
                     void *h, int64_t ldh, void *stream);

/* Its gradients for dh [rows, f] (row stride lddh), from x and the weights: with g = x w_gate^T and u = x w_up^T formed again
 *     dg = dh u act'(g),  du = dh act(g),
 *     dx = dg w_gate + du w_up,   dw_gate = dg^T x,   dw_up = du^T x.
 * dx [rows, d] and dw_gate, dw_up [f, d] in bf16; dx may be NULL, and dw_gate and dw_up together.
 * dg and du are rounded to bf16 before the products that follow (one rounding more than the results', of the same size); sums in fp32.  No output
 * overlaps an input or another output.  scratch: spec_k_ffn_gated_grad_scratch_bytes (host only; 0 for bad sizes), 256-byte aligned. */
uint64_t spec_k_ffn_gated_grad_scratch_bytes(int32_t rows, int32_t d, int32_t f);
int spec_k_ffn_gated_grad(const void *x, int64_t ldx, int32_t rows, int32_t d, const void *w_gate, const void *w_up, int64_t ldw, int32_t f, int32_t act,
                          const void *dh, int64_t lddh, void *dx, int64_t lddx, void *dw_gate, void *dw_up, int64_t lddw, void *scratch,
                          uint64_t scratch_bytes, void *stream);

/* How calls of these sizes run (host only; for tests).  forward: 16, 64 or 65: the kernels of up to 16, 64 and 128 rows that read the weights once; 128 or 256: tiles of 128 x 128, or
 * of 256 x 256 and halves of it.  The gradients: again (g and u formed again), dx and dw (both weights' gradients, asked for alone): tiles of 128 or 256; dx_ranges and dw_ranges: into how
 * many ranges their k is cut; together != 0: a call for all of them forms dx and dw in one launch, of tiles of 128. */
int spec_k_ffn_gated_plan(int32_t rows, int32_t d, int32_t f, int32_t *forward, int32_t *again, int32_t *dx, int32_t *dx_ranges, int32_t *dw, int32_t *dw_ranges,
                          int32_t *together);

/* ---- gradient clipping ------------------------------------------------------------
 * The norm of n tensors' elements together, n = sqrt(sum g^2), and the tensors scaled by
 * min(1, max_norm / (norm + 1e-6)), without a wait in between:
 *   spec_k_grad_sums : g -> sums, SPEC_GRAD_SUMS doubles that add up to norm^2 (squares
 *                      and sums are 64-bit: no gradient in fp32 overflows them).  Processes that each hold a part of the
 *                      gradients add their sums up, element by element, before the next call.
 *   spec_k_grad_clip : out = g * factor (the product in fp32), the factor formed in 64 bits and held to 24; norm[0]: the norm in fp32
 *                      (infinite from 2^128 on, which the factor is not; NULL: not wanted).  out may be g (in place, same dtype; nothing is written if the factor is 1); else it
 *                      overlaps no g and no other out.  A norm that is not finite does as the formula says: an infinite one makes finite gradients 0 and infinite
 *                      ones NaN, NaN makes all NaN.
 * The sums and the norm overlap no g, no out and not each other.
 * The tensors are dense arrays of n elements, n >= 0 (0: skipped, pointers ignored), aligned to their type;
 * n_parts >= 0, any number; max_norm >= 0 and finite. */
#define SPEC_GRAD_SUMS 1024
typedef struct spec_grad_part {
  const void *g;
  void   *out;         /* spec_k_grad_sums: ignored */
  int64_t n;
  int32_t dtype, out_dtype;
} spec_grad_part;
int spec_k_grad_sums(int32_t n_parts, const spec_grad_part *parts /* host */, double *sums, void *stream);
int spec_k_grad_clip(int32_t n_parts, const spec_grad_part *parts /* host */, const double *sums, double max_norm, float *norm, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPEC_STEP_H_ */
