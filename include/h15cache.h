/*
 * h15cache: the operators of h15attn (h15attn.h) for serving with key/value
 * caches that are shared and kept small, on AMD Instinct MI355X (gfx950):
 *
 *   attn_decode_prefix  decode for a batch whose sequences share a prefix,
 *                       whose keys are held and read once for all of them,
 *                       and have own caches of different lengths;
 *   attn_key_weights    the attention weight that each cached key received;
 *   attn_evict          which keys of a cache stay, by that weight, gathered
 *                       into a compact cache.
 *
 * A serving loop runs them in this order: decode, add the weights that its
 * query rows gave, and, when the caches have outgrown their budget, evict.
 *
 * As in h15attn.h: every pointer is a device pointer, tensors are row-major
 * and contiguous, calls are asynchronous on opts->stream (NULL: the default
 * stream; it must belong to the current device, as must the pointers), nothing
 * is allocated, freed or synchronised, arguments are validated before
 * anything is launched, and every entry point returns ATTN_OK or a negative
 * attn_status.  All calls can be captured into a HIP graph.
 *
 * lens: keys in each sequence's own cache, int32 [B] on the device (NULL: Sk
 * in every one).  The values are read by the kernels: one below 0 counts as 0,
 * one above Sk as Sk.  Rows of a cache from lens[b] on are never read.
 *
 * Operands are finite, as in attn_decode.  Infinities and NaN in a sequence's
 * rows of q, k and v reach no other sequence (those of the prefix reach all),
 * but within it: in v, also the rows that do not see that key, with the
 * weight 0; the lattice weights give a logit of NaN the least weight there is.
 */
#ifndef H15CACHE_H
#define H15CACHE_H

#include "h15attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Decode over a shared prefix ---------------------------------------
 *
 * Sq query rows per query head and sequence attend to the first P keys of a
 * prefix that all sequences share and to the first n = lens[b] keys of their
 * own cache.  Query position i (0 <= i < Sq) sees every key of the prefix and,
 * of its own cache, the keys j <= n - Sq + i when causal (bottom-right
 * alignment, none if that is negative), every key otherwise.  A row that sees
 * no key at all has O = 0 and LSE = -inf.
 *
 * Prefix and own caches are cut into parts of prefix_split_keys and split_keys
 * keys (multiples of attn_tile_bc(); 0, or any value >= the number of keys,
 * gives one part), each starting at key 0 of its cache.  Weights, parts and
 * their exact merge are as in attn_decode: within a part the weights follow
 * the recurrence over tiles, so for the lattice weights the cuts are part of
 * the result.  P = 0 (no prefix) and Sk = 0 (no own caches) are allowed, not
 * both; the pointers of what is absent may be NULL.
 *
 * FP8: the operands are taken as stored and the logits are sums in FP32; P is
 * rounded to BF16 (attn_decode: to e4m3), so results are closer to the
 * definition than attn_decode's on the same operands.  One set of descales
 * serves the prefix and the own caches.  BF16 results equal attn_decode's for
 * the same parts up to the order of sums.
 *
 * Layouts: q: [B][Hq][Sq][d]; kp, vp: [Hkv][P_cap][d]; k, v:
 * [B][Hkv][Sk_cap][d]; o: [B][Hq][Sq][d] bf16; lse: [B][Hq][Sq] fp32 (may be
 * NULL).  exp_mode: ATTN_EXP_EXACT, H15, SQ4 or SQ8; the rescale threshold
 * must be 0.
 *
 * workspace: attn_decode_prefix_workspace_bytes() bytes, 16-byte aligned, for
 * more than one part (also where a short prefix is taken together with the own
 * caches, and nothing is written to it); it needs no initialising; two calls
 * in flight at once must not share it.
 *
 * Errors: ATTN_EINVAL for a null pointer, a size that is not positive
 * (P, Sk: negative, or both 0), P > P_cap, Sk > Sk_cap, Hq % Hkv != 0, a scale
 * or descale that is not positive and finite, a cut that is negative or no
 * multiple of attn_tile_bc(), or a missing or short workspace;
 * ATTN_EUNSUPPORTED for d not in {64, 128}, an unknown dtype or exp_mode, a
 * pointer that is not 16-byte aligned (lse, lens: 4), a rescale threshold
 * other than 0, B * Hq * Sq > 2^30 (2^26 - 1 with more than one part), one
 * head's cache or prefix beyond 2^31 - 1 bytes, or more than 2^24 - 1
 * workgroups. */
int attn_decode_prefix(const void* q, const void* kp, const void* vp, const void* k, const void* v,
                       const int32_t* lens, void* o, float* lse, int B, int Hq, int Hkv, int Sq, int P, int P_cap,
                       int Sk, int Sk_cap, int d, int causal, float scale, int dtype, int exp_mode,
                       int prefix_split_keys, int split_keys, void* workspace, size_t workspace_bytes,
                       const attn_opts* opts);

/* Bytes of workspace attn_decode_prefix needs (0 for a single part, or for
 * invalid sizes). */
size_t attn_decode_prefix_workspace_bytes(int B, int Hq, int Sq, int P, int Sk, int d, int prefix_split_keys,
                                          int split_keys);

/* Cuts for attn_decode_prefix that fill the GPU: a function of the arguments
 * only.  ATTN_EINVAL (and cuts of 0) for invalid sizes. */
int attn_decode_prefix_split_keys(int B, int Hq, int Hkv, int Sq, int P, int Sk, int d, int dtype,
                                  int* prefix_split_keys, int* split_keys);

/* ---- The attention weight that each cached key received -----------------
 *
 *   acc[b][hkv][j] = decay * acc[b][hkv][j] + sum over the query heads h of
 *       KV head hkv and the positions i that see key j of
 *       exp(scale * q_descale * k_descale * (q . k_j) - lse[b][h][i])
 *
 * for j < n = lens[b]; acc beyond is left as it was.  Position i sees the keys
 * j <= n - Sq + i when causal, every key otherwise.  lse is what an attention
 * call returned for these rows (any entry point; with a prefix the weights are
 * shares of the whole, own keys only being counted); a row with lse = -inf
 * gives nothing, whatever its q holds.
 *
 * The exponential is the exact one: with lse of ATTN_EXP_EXACT these are the
 * weights of that call, and a row's add up to 1.  With lse of a lattice mode
 * they are not the lattice weights, which differ from them by the map's own
 * error (a factor of 0.84 to 1.26 for H15, 0.92 to 1.16 for SQ4, 0.96 to 1.11
 * for SQ8), and a row adds up to the ratio of the two normalisers.
 *
 * decay = 1 accumulates; with decay = 0 the old values are not read.  decay
 * must be finite and >= 0.
 *
 * Sums are in FP32 (of FP32 logits), in a fixed order: results are
 * deterministic.
 *
 * Layouts: q: [B][Hq][Sq][d]; k: [B][Hkv][Sk_cap][d]; lse: [B][Hq][Sq] fp32;
 * acc: [B][Hkv][Sk_cap] fp32.  Sq may be anything from 1 up, more than Sk
 * included.
 *
 * workspace: attn_key_weights_workspace_bytes() bytes, 16-byte aligned, for
 * calls with many query rows (may be NULL where that is 0); it needs no
 * initialising; two calls in flight at once must not share it.
 *
 * Errors: as attn_decode_prefix (lse, acc: 4-byte aligned); ATTN_EINVAL for
 * a decay that is negative or not finite; ATTN_EUNSUPPORTED for one KV head's
 * query rows (G Sq) beyond 2^31 - 1 bytes. */
int attn_key_weights(const void* q, const void* k, const float* lse, const int32_t* lens, float* acc, int B, int Hq,
                     int Hkv, int Sq, int Sk, int Sk_cap, int d, int causal, float scale, float decay, int dtype,
                     void* workspace, size_t workspace_bytes, const attn_opts* opts);

size_t attn_key_weights_workspace_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int d);

/* ---- Eviction ------------------------------------------------------------
 *
 * Of the n = lens[b] keys of each (b, hkv), min(n, keep) stay: all of them if
 * n <= keep, else the last min(recent, keep) and, of the keys before those,
 * the ones with the largest acc (equal ones: the lowest index first; NaN
 * counts as the largest, -0 as 0).  They keep their order:
 *
 *   index[b][hkv][r]  = source index of the r-th key that stays, ascending
 *                       (-1 for r >= min(n, keep))
 *   k_out, v_out, acc_out[b][hkv][r] = k, v, acc[b][hkv][index[b][hkv][r]]
 *   lens_out[b]       = min(n, keep)
 *
 * Rows of the outputs from lens_out[b] on are left as they were.
 *
 * Layouts: k, v: [B][Hkv][Sk_cap][d]; acc: [B][Hkv][Sk_cap] fp32; k_out,
 * v_out: [B][Hkv][out_cap][d]; acc_out: [B][Hkv][out_cap] fp32; index:
 * [B][Hkv][keep] int32; lens_out: [B] int32.  opts may be NULL; only its
 * stream is used.
 *
 * workspace: attn_evict_workspace_bytes() bytes, 16-byte aligned, for long
 * caches (may be NULL where that is 0); it needs no initialising; two calls in
 * flight at once must not share it.
 *
 * Errors: ATTN_EINVAL for a null pointer (lens may be), a size that is not
 * positive, Sk > Sk_cap, keep < 1 or > out_cap, recent < 0, a missing or short
 * workspace, or an output or workspace that overlaps an input or another
 * output; ATTN_EUNSUPPORTED for d not in {64, 128}, an unknown dtype, k, v,
 * k_out or v_out not 16-byte aligned (the others: 4), Sk beyond 2^31 - 8193,
 * B * Hkv beyond 2^22 - 1, or more than 2^32 - 256 chunks of 16 bytes in the
 * rows of K that may stay. */
int attn_evict(const void* k, const void* v, const float* acc, const int32_t* lens, void* k_out, void* v_out,
               float* acc_out, int32_t* index, int32_t* lens_out, int B, int Hkv, int Sk, int Sk_cap, int out_cap,
               int d, int keep, int recent, int dtype, void* workspace, size_t workspace_bytes,
               const attn_opts* opts);

size_t attn_evict_workspace_bytes(int B, int Hkv, int Sk);

#ifdef __cplusplus
}
#endif

#endif /* H15CACHE_H */
