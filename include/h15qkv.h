/*
 * h15qkv: what lies between a layer's projections and the attention of h15attn
 * (h15attn.h), on AMD Instinct MI355X (gfx950):
 *
 *   attn_rope           norms of queries and keys for each head and their
 *                       position rotation, from the projections' layout into
 *                       the attention's;
 *   attn_rope_bwd       its gradient;
 *   attn_cache_append   writes new keys and values into a cache of 8-bit codes
 *                       with a scale for each block of tokens and head;
 *   attn_decode_blocks  attention over such a cache.
 *
 * A layer that serves runs attn_rope on its projections, attn_cache_append on
 * the keys and values and attn_decode_blocks on the queries (or attn_fwd on all
 * three, for a prompt without a cache); one that trains runs attn_rope, any
 * attention with a gradient, and attn_rope_bwd.
 *
 * As in h15attn.h: every pointer is a device pointer (attn_rope_spec,
 * attn_strides and attn_opts are read on the host, within the call), calls are
 * asynchronous on opts->stream (NULL: the default stream; it must belong to the
 * current device, as must the pointers), nothing is allocated, freed or
 * synchronised, arguments are validated before anything is launched, and every
 * entry point returns ATTN_OK or a negative attn_status.  Tensors are row-major
 * and contiguous unless strides are given.  All calls can be captured into a
 * HIP graph.  opts may be NULL where no descale is needed.
 */
#ifndef H15QKV_H
#define H15QKV_H

#include "h15attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of norm weights, next to ATTN_BF16. */
#define ATTN_FP32 2

/* Distances in elements between batches, positions and heads of a tensor
 * [B][S][H][d]; the d channels of a row are contiguous.  Multiples of 8. */
typedef struct attn_strides {
  int64_t batch, position, head;
} attn_strides;

/* The rotation of the first rot channels of each row (rot a multiple of 16, 0
 * for none) and the norms.
 *
 * Position of row i of sequence b: positions[b][i] if each_position, else
 * positions[b] + i (int32, any value; positions NULL: i).  Pair j < rot / 2 is
 * turned by position * freqs[j] radians (freqs: fp64 [rot / 2] on the device);
 * its channels are (2 j, 2 j + 1) if interleaved, else (j, j + rot / 2).
 * Angles are reduced to a turn in 64 bits: at position 10^6 they are as exact
 * as at 0.  The rotated channels are multiplied by amplitude, which contexts
 * stretched by interpolated frequencies take different from 1. */
typedef struct attn_rope_spec {
  const int32_t* positions;
  int each_position;
  const double* freqs;
  int rot;
  int interleaved;
  float amplitude;
  const void* q_weight; /* [d] of weight_dtype, or NULL: queries have no norm */
  const void* k_weight; /* likewise, for the keys */
  int weight_dtype;     /* ATTN_BF16 or ATTN_FP32 */
  float eps;
} attn_rope_spec;

/* ---- Norms and position rotation ----------------------------------------
 *
 * For each row x of q and k (d channels of one head at one position)
 *
 *   y = x / sqrt(mean(x^2) + eps) * weight       (y = x without a weight)
 *   (z_a, z_b) = amplitude * (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
 *
 * for the channels a, b of each pair and its angle t, z = y elsewhere; rows of
 * v are taken as they are.  The output is z, rounded once to BF16, or, for
 * dtype ATTN_FP8_E4M3, z * (1 / descale) rounded to e4m3 after it is held to
 * +-448 (descales from opts: what attn_fwd_ex and attn_decode then take).
 * Everything before is in FP32; the squares of a row's values may leave it.  A
 * NaN stays one, and a NaN or an infinity in a row with a norm makes the row NaN.
 *
 * Layouts: q: [B][S][Hq][d], k, v: [B][S][Hkv][d] bf16, strides of each in
 * strides[0..2] (NULL: contiguous), so that all three may be views of one
 * projection's output; q_out: [B][Hq][S][d], k_out, v_out: [B][Hkv][S][d] of
 * dtype.  Any of q, k, v may be NULL, with its output, not all of them.
 *
 * Errors: ATTN_EINVAL for a null spec or pointer (freqs if rot > 0), one of an
 * input and its output, a size that is not positive (Hq without q and Hkv
 * without k and v may be; such a count still enters the limits below and the
 * launch's shape, below 0 as 0), rot < 0 or > d, an amplitude or descale that is
 * not positive and finite, an eps below 2^-126 or not finite with a weight, or
 * an output that overlaps an input or another output; ATTN_EUNSUPPORTED for d
 * not in {64, 128}, rot not a multiple of 16, an unknown dtype or
 * weight_dtype, a stride that is negative or no multiple of 8, a pointer that
 * is not 16-byte aligned (positions: 4, freqs: 8), more than 2^31 - 1 rows (of
 * one head and position) in one output, more than 2^24 - 1 times 4096 / d
 * positions in all, or Hq + 2 Hkv > 65535. */
int attn_rope(const void* q, const void* k, const void* v, const attn_strides* strides, const attn_rope_spec* spec,
              void* q_out, void* k_out, void* v_out, int B, int S, int Hq, int Hkv, int d, int dtype,
              const attn_opts* opts);

/* ---- Their gradient -------------------------------------------------------
 *
 * From the gradients gq, gk, gv of attn_rope's outputs (bf16, laid out as
 * those) to those of its inputs and weights:
 *
 *   (h_a, h_b) = amplitude * (g_a cos t + g_b sin t, g_b cos t - g_a sin t)
 *   without a weight:  dx = h
 *   with one:  u = x r, r = 1 / sqrt(mean(x^2) + eps);
 *              dweight = sum over rows of h u;  e = h weight;
 *              dx = r (e - u mean(e u))
 *
 * dx is rounded once to BF16; dweight is FP32, each sum in a fixed order, so
 * that results are deterministic.  A NaN or an infinity in a row of q or k with a
 * norm makes its dx and the weight's gradient NaN.  (FP8 outputs have this same
 * gradient, their rounding and limits left out.)
 *
 * q, k: attn_rope's inputs, read only where there is a weight (else NULL may
 * be given), with strides[0..1]; dq, dk, dv: laid out as q, k, v, with
 * grad_strides[0..2] (NULL: contiguous): they may be views of one tensor.  Any
 * of gq, gk, gv may be NULL, with its output, not all of them.  dq_weight,
 * dk_weight: fp32 [d], written where there is a weight and its gradient gq, gk
 * (required then).
 *
 * workspace: attn_rope_bwd_workspace_bytes() bytes of the same sizes (an absent
 * tensor's heads included, 0 for those below 0), 16-byte aligned, where a
 * weight's gradient is written; it needs no initialising; two calls in flight at
 * once must not share it.
 *
 * Errors: as attn_rope; a missing or short workspace: ATTN_EINVAL.  Rows of a
 * gradient that lie over each other by their strides, or in each other's
 * tensors, are the caller's to avoid; tensors whose whole ranges overlap an
 * input's are refused. */
int attn_rope_bwd(const void* gq, const void* gk, const void* gv, const void* q, const void* k,
                  const attn_strides* strides, const attn_rope_spec* spec, void* dq, void* dk, void* dv,
                  const attn_strides* grad_strides, float* dq_weight, float* dk_weight, int B, int S, int Hq, int Hkv,
                  int d, void* workspace, size_t workspace_bytes, const attn_opts* opts);

/* Bytes of workspace attn_rope_bwd needs for weights' gradients (0 for invalid
 * sizes, heads below 0 among them). */
size_t attn_rope_bwd_workspace_bytes(int B, int S, int Hq, int Hkv, int d);

/* ---- A cache of 8-bit blocks ----------------------------------------------
 *
 * k_cache, v_cache: e4m3 codes [B][Hkv][cap][d]; scales: one byte
 * [B][Hkv][ceil(cap / block)][2], those of K and of V.  Slot j of a head
 * stands for code * 2^(e - 127), e the byte of its block j / block, 1 to 254
 * (the E8M0 format of the OCP microscaling formats; 0 counts as 1, 255 as
 * 254).  Scales of two lose nothing in an 8-bit float's relative precision,
 * and a block's scale can grow without rounding its codes again, but for those
 * that become subnormal.
 *
 * attn_cache_append writes the first c = counts[b] (NULL: n) of n new rows of
 * k and v at the slots lens[b] .. lens[b] + c - 1 of each head.  In each block
 * that gets one, for K and V each,
 *
 *   e   = the least byte with max |x| <= 448 * 2^(e - 127) over the new finite
 *         values x, and no less than the block's byte so far if it held a row
 *         already;
 *   new rows are rounded to e4m3 (nearest, ties to even) of x / 2^(e - 127),
 *   rows that it held to that of code * 2^(e_before - e).
 *
 * Infinities become +-448, NaN stays NaN; neither moves a scale.  Everything
 * else is left as it was.  lens: int32 [B]; lens_out[b] = lens[b] + c, and may
 * be lens itself.  A length below 0 counts as 0, one above cap as cap, a count
 * below 0 as 0, one above n as n; rows that would lie beyond cap are dropped,
 * and lens_out is cap.  So a padded batch has a sequence's rows first, its padding
 * last; attn_decode_blocks, whose Sq rows end with a sequence's last key, takes
 * them the other way round (see there).
 *
 * Layouts: k, v: [B][Hkv][n][d] bf16.  block: 16, 32, 64 or 128.
 *
 * Errors: ATTN_EINVAL for a null pointer (counts may be), a size that is not
 * positive, or an output (the caches, scales and lens_out) that overlaps an
 * input or another output (lens_out may be lens); ATTN_EUNSUPPORTED for d not
 * in {64, 128}, another block, k, v, k_cache or v_cache not 16-byte aligned
 * (lens, counts, lens_out: 4), one head's cache beyond 2^31 - 1 codes, one
 * head's new rows beyond 2^31 - 1 bytes, or more than 2^24 - 1 workgroups (one
 * for each block, head and tensor). */
int attn_cache_append(const void* k, const void* v, void* k_cache, void* v_cache, uint8_t* scales,
                      const int32_t* lens, const int32_t* counts, int32_t* lens_out, int B, int Hkv, int n, int cap,
                      int d, int block, const attn_opts* opts);

/* ---- Attention over it ------------------------------------------------------
 *
 * attn_decode (h15attn.h) for BF16 queries over such a cache, with a length
 * for each sequence: Sq query rows per head and sequence attend to the first
 * n = lens[b] (NULL: Sk) slots.  Position i (0 <= i < Sq) sees the keys j <=
 * n - Sq + i when causal (none if that is negative), every key otherwise: a
 * sequence with c new rows, fewer than Sq, has them last, after its padding.  The
 * queries of a batch that attn_cache_append took with counts have them first:
 * handed on as they are, each row's mask would be off by Sq - c keys, which no
 * check can see.  They are moved behind the padding before the call, or each
 * sequence has a call of its own, with Sq = c.
 *
 * A row that sees no key has O = 0 and LSE = -inf.  Sq may be anything from 1
 * up: a decoded token, a few drafted ones, a chunk of a prompt that has been
 * appended before.  A length below 0 counts as 0, one above Sk as Sk; slots
 * from lens[b] on, and scales of blocks without a slot below it, are never
 * read.  The kernel's form, attn_decode_blocks_split_keys' cut and the workspace
 * go by Sk, as lens is not on the host: the least bound of lens that is known
 * there serves best.
 *
 * Parts of split_keys keys, their weights by exp_mode (ATTN_EXP_EXACT, H15, SQ4
 * or SQ8; for the lattice weights the cut is part of the result) and their
 * merge are those of attn_decode.  Logits are FP32 sums of products of BF16
 * queries and keys, which hold every code times its scale (values below
 * 2^-126 count as 0); P is rounded to BF16 for the exact weights
 * (the lattice ones are exact in it), sums are FP32.  The operands are finite;
 * NaN in a sequence's rows stays within that sequence's heads.
 *
 * Layouts: q: [B][Hq][Sq][d] bf16; o: the same; lse: [B][Hq][Sq] fp32 (may be
 * NULL); k, v, scales: as above, cap = Sk_cap.  opts: its descales and its
 * rescale threshold are not used (the threshold must be 0).
 *
 * workspace: attn_decode_blocks_workspace_bytes() bytes, 16-byte aligned, for
 * more than one part; it needs no initialising; two calls in flight at once
 * must not share it.
 *
 * Errors: ATTN_EINVAL for a null pointer (lens and lse may be), a size that is
 * not positive, Sk > Sk_cap, Hq % Hkv != 0, a scale that is not positive and
 * finite, a cut that is negative or no multiple of attn_tile_bc(), a missing or
 * short workspace, or an output or workspace that overlaps an input or another
 * output; ATTN_EUNSUPPORTED for d not in {64, 128}, another block, another
 * exp_mode, q, k, v or o not 16-byte aligned (lse, lens: 4, scales: 2), a
 * rescale threshold other than 0, B * Hq * Sq > 2^30 (2^26 - 4 with more than
 * one part), one head's cache beyond 2^31 - 1 bytes, or more workgroups than
 * have 2^32 - 256 threads. */
int attn_decode_blocks(const void* q, const void* k, const void* v, const uint8_t* scales, const int32_t* lens,
                       void* o, float* lse, int B, int Hq, int Hkv, int Sq, int Sk, int Sk_cap, int d, int block,
                       int causal, float scale, int exp_mode, int split_keys, void* workspace,
                       size_t workspace_bytes, const attn_opts* opts);

/* Bytes of workspace attn_decode_blocks needs (0 for a single part, or for
 * invalid sizes). */
size_t attn_decode_blocks_workspace_bytes(int B, int Hq, int Sq, int Sk, int d, int split_keys);

/* A cut for attn_decode_blocks that fills the GPU (0: one part): a function of
 * the arguments only; 0 for invalid sizes. */
int attn_decode_blocks_split_keys(int B, int Hq, int Hkv, int Sq, int Sk, int d);

#ifdef __cplusplus
}
#endif

#endif /* H15QKV_H */
