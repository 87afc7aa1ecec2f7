/*
 * libspec, operators of a decoder layer that holds its weights and its cache in
 * 8 bits: projections, attention over an 8-bit cache, and the rotary embedding
 * that stands between them (of use in training too).  Same conventions as
 * spec_kernels.h: all data pointers are DEVICE pointers unless a comment says
 * "host", calls enqueue on `stream` (a hipStream_t, NULL = default stream, of the
 * CURRENT device) and return without waiting; no call allocates device memory;
 * return SPEC_OK or SPEC_EINVAL / SPEC_EHIP (codes in spec.h; with SPEC_EINVAL
 * nothing has been launched).  dtype is SPEC_DTYPE_FP32 or SPEC_DTYPE_BF16.
 * Buffers are borrowed until the kernels have run.  Calls keep nothing between
 * them: two calls may run at once if neither writes what the other uses, their
 * scratch included.
 *
 * 8-bit values.  A block of values is held as e4m3 codes (4 exponent bits, 3
 * mantissa bits, largest 448, no infinities) and one exponent
 *     e = max(-100, the least e with amax <= 448 * 2^e),
 * amax the largest finite magnitude of the block (e = -100 if that is 0): the value x
 * is held as code(x / 2^e), rounded to nearest, ties to even, and stands for
 * code * 2^e.  The division is exact, so that a value is rounded once: by at most
 * 2^-4 of itself, or 2^(e - 10) if that is more.  Infinities and NaN are held as
 * NaN; magnitudes from 1.9375 * 2^127 on stand for 2^128, which is read as an infinity.  (A power of two as the scale: the matrix instructions and the conversions
 * apply it for nothing.)
 */
#ifndef SPEC_LAYER8_H_
#define SPEC_LAYER8_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- projections -------------------------------------------------------------
 * y[i][c] = sum over k of xq[i][k] * wq[c][k], xq and wq the 8-bit forms of x
 * [m, in] and w [rows, in] with blocks of 128 consecutive k of one row (the last
 * block of a row is what is left).  w is laid out once, at load time, by
 * spec_pack_weight8; x is put into 8 bits by the call.
 *   spec_packed8_bytes     : size of the packed form of w (host only; 0 if bad).
 *   spec_pack_weight8      : row-major src [rows, in] in dtype, any alignment of its
 *                            type -> dst, 256-byte aligned; no overlap.
 *   spec_k_gemm8_scratch_bytes : scratch of a call (host only; 0 if it needs none,
 *                            as calls of few tokens do, and for bad sizes).
 *   spec_k_gemm8           : x in dtype with row stride ldx >= in; y [m, rows] in
 *                            out_dtype with row stride ldy >= rows (strides in elements;
 *                            what lies between rows is left alone); scratch 256-byte aligned,
 *                            NULL if none is needed.
 * 1 <= m <= 2^20, 1 <= in <= 2^20, 1 <= rows <= 2^24.  y overlaps none of the inputs or the scratch.
 *
 * Sums: with out_dtype fp32 products are exact and added up in fp32.  With bf16 the 8-bit matrix instruction takes 128 k at a time
 * and lets go of what is under 2^-14 of its largest product (measured: 1.4e-5 of
 * a sum of normally distributed values, a hundredth of the result's rounding);
 * its results are added up in fp32.  A non-finite x makes its row of y NaN, a non-finite weight its
 * column.  The order of a sum may change with m, so that a row's last bits may
 * change with the rows beside it. */
uint64_t spec_packed8_bytes(int32_t rows, int32_t in);
int spec_pack_weight8(int32_t dtype, const void *src, int32_t rows, int32_t in, void *dst, void *stream);
uint64_t spec_k_gemm8_scratch_bytes(int32_t m, int32_t in, int32_t rows);
int spec_k_gemm8(int32_t dtype, const void *x, int32_t ldx, int32_t m, int32_t in, const void *w8, int32_t rows, int32_t out_dtype, void *y,
                 int32_t ldy, void *scratch, uint64_t scratch_bytes, void *stream);

/* ---- attention over an 8-bit cache -------------------------------------------
 * The cache of a layer is a row of blocks of SPEC_KV8_BLOCK tokens, each put into
 * 8 bits once, when it is whole, with one exponent per block, kv head and K or V;
 * the tokens behind the last whole block, and the rows that a forward adds (a
 * prompt's chunk, a draft tree), stay in a bf16 window.  So no value is rounded
 * twice, and rows of a tree that are not accepted never touch the blocks.
 *   spec_kv8_bytes   : size of n_blocks blocks (host only; 0 if bad).  Blocks do not depend on each
 *                      other: a cache may be copied, cut or joined at multiples of spec_kv8_bytes(1, ..).
 *   spec_k_kv8_store : rows k, v [n_blocks * SPEC_KV8_BLOCK, hkv*hd] bf16, row stride ld
 *                      -> blocks first_block .. of cache8 (256-byte aligned).
 *   spec_k_kv8_load  : the same back: what the codes stand for, which bf16 holds exactly (but 2^128).
 * hd 64 or 128, 1 <= hkv <= 128, ld >= hkv*hd.  The caller sees to it that cache8 holds
 * first_block + n_blocks blocks.  n_blocks = 0 does nothing. */
#define SPEC_KV8_BLOCK 64
uint64_t spec_kv8_bytes(int32_t n_blocks, int32_t hkv, int32_t hd);
int spec_k_kv8_store(const void *k, const void *v, int64_t ld, int32_t n_blocks, int32_t hkv, int32_t hd, void *cache8, int32_t first_block,
                     void *stream);
int spec_k_kv8_load(const void *cache8, int32_t first_block, int32_t n_blocks, int32_t hkv, int32_t hd, void *k, void *v, int64_t ld, void *stream);

/* Tree attention as spec_k_attention, with the positions p < n8 = n_blocks *
 * SPEC_KV8_BLOCK in cache8 (n_blocks 0: none, cache8 may be NULL).  Row i has its
 * query in q[i] ([hq*hd], fp32), sits at position base + depth[i] (base >= n8) and
 * attends to positions 0 .. base + depth[i]: n8 <= p < base is window row p - n8,
 * p >= base is window row base - n8 + anc[i*16 + p - base] (anc NULL: p - n8, a
 * causal chain).  A position whose window row is negative or not below win_rows is left out; a row that sees nothing, or only window rows with scores of -infinity, gets zeros.
 * A row of negative depth is padding: its output is left as it was.  What a row
 * does not see does not touch its result, whatever is stored there (NaN included).
 * kwin, vwin: [win_rows, hkv*hd] bf16, 1 <= win_rows <= 2^24, 16-byte aligned, as are q, out and cache8 (256).
 * out: [rows, hq*hd] bf16, overlaps no input.  depth[i] <= max_depth for every row (a row beyond is taken to be at max_depth); with anc, max_depth <= 15.
 * hd 64 or 128, hq/hkv one of 1, 2, 4, 8; hkv <= 128; rows <= 2^20.  Scratch: spec_k_attention8_scratch_bytes(..), 256-byte aligned
 * (host only; 0 if the call needs none, then scratch may be NULL, and for bad sizes).  Softmax statistics and sums are fp32.  In the 8-bit part queries are rounded to
 * fp16 relative to the row's largest value (2^-11) and weights cut to fp16: with its block's value exponent e a weight w counts as w 2^e, and down to 2^-26 of the largest
 * weight times the largest 2^e it is at most 2^-10 off, centred; smaller ones are cut to multiples of 2^-36 of that.  In
 * the window both go in two bf16 terms (2^-16).
 * Sums are weighted by up to 2^45 before the division: values beyond 2^80 may end as infinities.
 * The result of a row may change in its last bits with the rows beside it (another kernel, other ranges): unlike spec_k_attention's, a row verified in a tree need not
 * have the bits of the row decoded alone, and a greedy choice between logits that close may differ. */
uint64_t spec_k_attention8_scratch_bytes(int32_t rows, int32_t hq, int32_t hkv, int32_t hd, int32_t n_blocks, int32_t win_rows);
int spec_k_attention8(const float *q, const void *cache8, int32_t n_blocks, const void *kwin, const void *vwin, int32_t win_rows, int32_t rows,
                      int32_t hq, int32_t hkv, int32_t hd, int32_t base, const int32_t *depth, const int32_t *anc, int32_t max_depth,
                      void *scratch, uint64_t scratch_bytes, void *out, void *stream);

/* How a call of these sizes runs (host only; for tests).  waves: wavefronts of 32 queries in a workgroup, 0: up to 32 queries, whose keys the wavefronts of a workgroup
 * share; query_blocks: workgroups that the queries of a kv head take; block_parts: ranges of the cache's blocks; win_parts: ranges of the
 * window, 0: it belongs to the last range of blocks. */
int spec_k_attention8_plan(int32_t rows, int32_t hq, int32_t hkv, int32_t hd, int32_t n_blocks, int32_t win_rows, int32_t *waves, int32_t *query_blocks,
                           int32_t *block_parts, int32_t *win_parts);

/* ---- rotary embedding ----------------------------------------------------------
 * The plane j of a head, dims (j, j + rot/2) in the half layout or (2j, 2j + 1) in
 * the interleaved one, j < rot/2, turns by the angle t = pos * freq[j]:
 *     (a, b) -> mscale * (a cos t - b sin t,  b cos t + a sin t);
 * dims rot .. hd-1 pass unchanged.  adjoint != 0 turns by -t: the transpose, which
 * takes the gradient of the output to that of the input.  Angles, cosines and sines, mscale
 * in them, are formed in 64 bits, so that far positions keep their phase, and rounded once; the turning is fp32.
 *
 * The frequencies are theta^(-2j/rot), changed for contexts beyond the trained
 * length as the plan says (host only, once; a plan is plain data and may be copied):
 *   SPEC_ROPE_NONE, SPEC_ROPE_LINEAR (divided by factor),
 *   SPEC_ROPE_LLAMA3: by the turns that a plane makes over trained_len: kept from high_freq turns on, divided by factor below low_freq, in
 *     between a linear mix by the turns,
 *   SPEC_ROPE_YARN: planes that turn more than beta_fast times kept, less than
 *     beta_slow divided by factor, a linear ramp over j between (the two places rounded outward);
 *     mscale = 0.1 ln(factor) + 1.
 * scaling parameters that a kind does not use are ignored.  rot even, 0 <= rot <= SPEC_ROPE_MAX_DIM
 * (0: nothing turns), theta > 1, factor >= 1, trained_len >= 1, high_freq > low_freq > 0, beta_fast > beta_slow > 0. */
#define SPEC_ROPE_MAX_DIM 256
#define SPEC_ROPE_HALF 0
#define SPEC_ROPE_INTERLEAVED 1
#define SPEC_ROPE_NONE 0
#define SPEC_ROPE_LINEAR 1
#define SPEC_ROPE_LLAMA3 2
#define SPEC_ROPE_YARN 3
typedef struct spec_rope_scaling {
  int32_t kind;             /* SPEC_ROPE_NONE ..                                    */
  int32_t trained_len;      /* LLAMA3, YARN                                          */
  double  factor;           /* LINEAR, LLAMA3, YARN                                  */
  double  low, high;        /* LLAMA3: low_freq, high_freq; YARN: beta_slow, beta_fast */
} spec_rope_scaling;
typedef struct spec_rotary_plan {   /* filled by spec_rotary_init; a caller may set frequencies of its own */
  int32_t rot, layout;
  double  mscale;
  double  freq[SPEC_ROPE_MAX_DIM / 2];   /* radians per position */
} spec_rotary_plan;
int spec_rotary_init(int32_t rot, int32_t layout, double theta, const spec_rope_scaling *scaling /* host; NULL: none */, spec_rotary_plan *plan /* host */);

/* Up to three tensors of the same rows in one launch (a layer's q, k and v).  Head
 * h of row r of a part begins at element r * ldx + h * hsx of x and r * ldo + h *
 * hso of out.  turn = 0: copied (converted), not turned.  x and out may be the same
 * tensor (same pointer, strides and dtype); else no part's out overlaps any x or other out.
 * Heads of one tensor must not overlap each other.  pos: DEVICE int32 [rows], any value; NULL: row r is at pos0 + r.  1 <= rows <= 2^24, rot <= hd <=
 * SPEC_ROPE_MAX_DIM, 1 <= heads <= 1024, pointers aligned to their type.  (Fastest where pointers and strides are multiples of 16 bytes and hd, rot and, for
 * the half layout, rot/2 multiples of 8.) */
typedef struct spec_rotary_part {
  const void *x;
  void   *out;
  int64_t ldx, hsx, ldo, hso;
  int32_t heads, dtype, out_dtype, turn;
} spec_rotary_part;
int spec_k_rotary(const spec_rotary_plan *plan /* host */, int32_t n_parts, const spec_rotary_part *parts /* host */, int32_t hd, int32_t rows,
                  const int32_t *pos, int32_t pos0, int32_t adjoint, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPEC_LAYER8_H_ */
