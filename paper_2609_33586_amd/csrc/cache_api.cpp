// The C entry points declared in h15cache.h: argument checks, cuts and
// workspaces, then the launchers of h15prefix.hip, h15weights.hip and
// h15evict.hip.  Plain C++: no HIP types or calls here, so the same checks
// build with a host compiler alone under the sanitizers.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "cache_params.h"
#include "h15cache.h"

using namespace h15;

namespace {

bool finite_pos(float x) { return x > 0.0f && x < INFINITY; }

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Work-items of a launch are counted in 32 bits: workgroups of 256 threads, and
// rows of a merge, which have 64 each.
constexpr long long MAX_GROUPS = (1LL << 24) - 1, MAX_MERGE_ROWS = (1LL << 26) - 1;

// Input-rounding order of an exp_mode that the caches' decode offers, 0 for
// the hardware exponential, -1 for others.
int exp_order(int exp_mode) {
  switch (exp_mode) {
    case ATTN_EXP_EXACT: return 0;
    case ATTN_EXP_H15: return 1;
    case ATTN_EXP_SQ4: return 2;
    case ATTN_EXP_SQ8: return 3;
    default: return -1;
  }
}

int elem_bytes(int dtype) { return dtype == ATTN_BF16 ? 2 : 1; }

bool misaligned(const void* x, uintptr_t to) { return ((uintptr_t)x & (to - 1)) != 0; }

// Parts of `keys` keys cut at `split` (0 or >= keys: one part; no keys: none).
int part_count(int keys, int split) {
  if (keys <= 0) return 0;
  return split <= 0 || split >= keys ? 1 : (int)ceil_div(keys, split);
}

// Type, head dimension, scale and descales; c1: the base-two logit scale.
int check_kind(int d, float scale, int dtype, const attn_opts* opts, float* c1, float* vd) {
  if (!finite_pos(scale)) return ATTN_EINVAL;
  if (dtype != ATTN_BF16 && dtype != ATTN_FP8_E4M3) return ATTN_EUNSUPPORTED;
  if (d != 64 && d != 128) return ATTN_EUNSUPPORTED;
  if (opts && opts->rescale_threshold != 0.0f)
    return opts->rescale_threshold > 0.0f && opts->rescale_threshold <= 64.0f ? ATTN_EUNSUPPORTED : ATTN_EINVAL;
  float qd = 1.0f, kd = 1.0f;
  *vd = 1.0f;
  if (dtype == ATTN_FP8_E4M3) {
    if (!opts) return ATTN_EINVAL;
    qd = opts->q_descale;
    kd = opts->k_descale;
    *vd = opts->v_descale;
    if (!finite_pos(qd) || !finite_pos(kd) || !finite_pos(*vd)) return ATTN_EINVAL;
  }
  *c1 = (float)((double)scale * (double)qd * (double)kd * 1.4426950408889634);
  return ATTN_OK;
}

// Query rows of a prefix workgroup.  Up to four blocks of WROWS rows of a KV head
// over the batch, each takes its own workgroup, whose four waves share out the
// keys (the others' reads come from L2): fewer rows would leave waves of the
// rows form idle, and a part takes half as long.  Beyond, PREFIX_ROWS rows share
// each tile.  Times of a call with blocks of 32 / of 128 rows: 84 rows, 5003 keys
// FP8 18 / 29 us; 128 rows, 8K keys BF16 33 / 35; 256 rows, 32K keys FP8 87 / 72.
int prefix_rows(long long rows) { return rows > 4 * WROWS ? PREFIX_ROWS : WROWS; }

// A short prefix in one part before own caches in one: each own cache's
// workgroup takes the prefix's keys too, at most two rounds of them, and there is
// nothing to merge.  Not where many caches of a few rows would each take them.
// Times of a call so / by two launches: 4 caches, 500 + 60 keys BF16 d = 64
// 11.0 / 13.6 us; 64 caches of 8 heads, 256 + 3000 keys d = 128 138 / 143; a
// prompt of 512 positions, 256 + 512 keys 20.9 / 34.6; 128 caches of 8 heads, 500 +
// 512 keys FP8 37 / 31.
bool chained(int P, int row_bytes, const PrefixParams& p) {
  const int round = row_bytes >= 256 ? BC : 2 * BC;  // keys
  return p.p_parts == 1 && p.o_parts == 1 && P <= 2 * round && (p.R >= WROWS || p.o_groups <= 512);
}

// Whether ragged own caches are taken longest first: where they are more than
// one for each slot (two workgroups a compute unit, one of them the prefix's), so
// that no long one starts last (32 heads over 8; in their own order / so: 128 caches of
// up to 2K keys after 8K BF16 156 / 150 us, 64 92 / 87; up to 8K after 32K FP8 180 / 170,
// 2K level).  With a slot each there is nothing to order; more than 256 caches, whose
// lengths a workgroup does not rank with a thread each, keep their own order.
bool by_length(const PrefixParams& p) {
  const int slots = 512 - (p.p_groups < 256 ? p.p_groups : 256);
  return p.lens && p.B > 1 && p.B <= 256 && p.o_groups > slots;
}

size_t prefix_workspace(long long rows, int parts, int d) {
  return parts <= 1 ? 0 : (size_t)rows * (size_t)parts * ((size_t)d + 2) * sizeof(float);
}

// The runs of query rows that the tiles of a key-weights call stay within: a
// head's rows, or all rows of a KV head where a head has fewer than half a tile.
void weights_runs(int G, int Sq, int& heads, int& hrows) {
  heads = Sq >= KW_ROWS / 2 ? G : 1;
  hrows = Sq >= KW_ROWS / 2 ? Sq : G * Sq;
}

// Tiles of each run in a row part of a key-weights call: 32 tiles in all.
int weights_span(int heads) { return heads >= 32 ? 1 : 32 / heads; }

int weights_parts(int G, int Sq) {
  if ((long long)G * Sq <= KW_FEW_ROWS) return 1;
  int heads, hrows;
  weights_runs(G, Sq, heads, hrows);
  return (int)ceil_div(ceil_div(hrows, KW_ROWS), weights_span(heads));
}

// Units of keys in a wave's run: about two workgroups per compute unit, three
// units at most (B16 8K BF16, ragged: runs of 1, 2, 3 and 4 units 48, 41, 40 and
// 49 us; B5 5K FP8 d = 64, whose 800 workgroups have runs of one: 5.0, of three
// 6.6; 64 query rows B2 16K FP8, runs of 1, 2, 3 and 4: 30, 27, 32 and 34).
int weights_run(long long heads, long long units) {
  const long long run = heads * units / (512 * 4);
  return run < 1 ? 1 : run > 3 ? 3 : (int)run;
}

// Chunks of 16 bytes of a head's kept rows of K that the selecting workgroup
// copies itself (times of a call so / with a second launch: 2 heads, 100 rows of 128
// bytes 9.5 / 12.0 us; 256 rows of 256 bytes, 2 heads 9.7 / 12.0, 256 heads 18 / 20;
// 512 rows, 2 heads 12.3 / 12.1, 320 heads 48 / 42).
constexpr int EVICT_GATHER = 4096;

// Keys of a workgroup's part in the selection for a head: all of them, unless few heads
// have long caches (of which one workgroup holds eight parts of EVICT_PART in LDS).  Times of a
// call with one workgroup a head for spread / for equal weights, and in parts for
// either, 256 FP8 rows of d = 64 staying: 8 heads, 25K keys 20 / 27 and 25 us, 33K 24 / 33
// and 24, 128K 132 / 163 and 27, 1M 1197 / 1385 and 59; 32 heads, 33K 24 / 33 and 31, 64K
// 62 / 79 and 33; 64 heads, 33K 24 / 33 and 40, 50K 48 / 61 and 41, 1M 1655 / 1904 and 348.
// A head has 32 parts at most, all heads 640 (beyond, each takes more keys, as far as
// its counts can): every workgroup adds up the counts of its head's parts (8 heads of 256K
// keys in 32 / 64 parts 36 / 55 us, of 1M 58 / 79).
int evict_part_keys(long long heads, int Sk) {
  if (Sk <= 5 * EVICT_PART || heads > (Sk > 8 * EVICT_PART ? 64 : 32)) return Sk;
  const long long most = heads > 20 ? 640 / heads : 32;
  const long long keys = ceil_div(ceil_div(Sk, EVICT_PART), most) * EVICT_PART;
  return (int)(keys < EVICT_PART_MOST ? keys : EVICT_PART_MOST);
}

size_t evict_workspace(long long heads, int Sk) {
  const size_t keys = (size_t)evict_part_keys(heads, Sk), parts = (size_t)ceil_div(Sk, (long long)keys);
  return parts == 1 ? 0 : (size_t)heads * parts * EVICT_PART_BYTES;
}

struct Range {
  uintptr_t from, to;
};
Range range(const void* p, size_t bytes) { return {(uintptr_t)p, (uintptr_t)p + bytes}; }
bool overlap(const Range& a, const Range& b) { return a.from < b.to && b.from < a.to; }
}  // namespace

extern "C" {

int attn_decode_prefix_split_keys(int B, int Hq, int Hkv, int Sq, int P, int Sk, int d, int dtype,
                                  int* prefix_split_keys, int* split_keys) {
  // (parts are counted in tiles, whatever a tile's bytes are: a cut of one type is
  // one of all, and lattice weights, which depend on it, compare across them)
  (void)d;
  (void)dtype;
  if (!prefix_split_keys || !split_keys) return ATTN_EINVAL;
  *prefix_split_keys = *split_keys = 0;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || P < 0 || Sk < 0 || Hq % Hkv != 0) return ATTN_EINVAL;
  const long long rows = (long long)(Hq / Hkv) * Sq;
  auto cut = [](int keys, long long groups, long long want, long long least) {
    const long long tiles = ceil_div(keys, BC);
    long long parts = ceil_div(want, groups);
    if (parts > tiles / least) parts = tiles / least;
    return parts <= 1 ? 0 : (int)(ceil_div(tiles, parts) * BC);
  };
  // two workgroups a compute unit, half of them for each of the two kinds
  const long long blocks = Hkv * ceil_div(B * rows, prefix_rows(B * rows));
  const long long own = (long long)B * Hkv * ceil_div(rows, WROWS);
  if (P > 0) *prefix_split_keys = cut(P, blocks, Sk > 0 ? 256 : 512, 4);
  if (Sk > 0 && *prefix_split_keys > 0) {
    // the parts are merged in any case: own caches in as many as are left, no more
    // (own keys in one part / in these: 7 caches of 777 after 5003 FP8 18.9 / 16.6 us,
    // 16 of 1K and Sq = 4 after 8K 27.3 / 24.3; 24 of 1K, which are not cut, in two
    // 19.9 / 23.8)
    *split_keys = cut(Sk, own, (512 - blocks * part_count(P, *prefix_split_keys)) / own * own, 2);
  } else if (Sk > 0) {
    *split_keys = cut(Sk, own, P > 0 ? 256 : 512, 8);
  }
  return ATTN_OK;
}

size_t attn_decode_prefix_workspace_bytes(int B, int Hq, int Sq, int P, int Sk, int d, int prefix_split_keys,
                                          int split_keys) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || P < 0 || Sk < 0 || d <= 0 || prefix_split_keys < 0 || split_keys < 0) return 0;
  return prefix_workspace((long long)B * Hq * Sq, part_count(P, prefix_split_keys) + part_count(Sk, split_keys), d);
}

int attn_decode_prefix(const void* q, const void* kp, const void* vp, const void* k, const void* v,
                       const int32_t* lens, void* o, float* lse, int B, int Hq, int Hkv, int Sq, int P, int P_cap,
                       int Sk, int Sk_cap, int d, int causal, float scale, int dtype, int exp_mode,
                       int prefix_split_keys, int split_keys, void* workspace, size_t workspace_bytes,
                       const attn_opts* opts) {
  if (!q || !o || (P > 0 && (!kp || !vp)) || (Sk > 0 && (!k || !v))) return ATTN_EINVAL;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || d <= 0 || P < 0 || Sk < 0 || P + (long long)Sk <= 0)
    return ATTN_EINVAL;
  if (Hq % Hkv != 0 || P > P_cap || Sk > Sk_cap) return ATTN_EINVAL;
  if (prefix_split_keys < 0 || prefix_split_keys % BC != 0 || split_keys < 0 || split_keys % BC != 0)
    return ATTN_EINVAL;
  PrefixParams p = {};
  const int rc = check_kind(d, scale, dtype, opts, &p.c1, &p.vd);
  if (rc != ATTN_OK) return rc;
  const int order = exp_order(exp_mode);
  if (order < 0) return ATTN_EUNSUPPORTED;
  if (misaligned(q, 16) || misaligned(o, 16) || misaligned(lse, 4) || misaligned(lens, 4)) return ATTN_EUNSUPPORTED;
  if (P > 0 && (misaligned(kp, 16) || misaligned(vp, 16))) return ATTN_EUNSUPPORTED;
  if (Sk > 0 && (misaligned(k, 16) || misaligned(v, 16))) return ATTN_EUNSUPPORTED;
  const long long row = (long long)d * elem_bytes(dtype), rows = (long long)B * Hq * Sq;
  if (rows > (1LL << 30)) return ATTN_EUNSUPPORTED;
  if ((P > 0 && P_cap * row > INT32_MAX) || (Sk > 0 && Sk_cap * row > INT32_MAX)) return ATTN_EUNSUPPORTED;
  p.q = (const uint8_t*)q;
  p.kp = (const uint8_t*)kp;
  p.vp = (const uint8_t*)vp;
  p.k = (const uint8_t*)k;
  p.v = (const uint8_t*)v;
  p.lens = lens;
  p.o = (uint16_t*)o;
  p.lse = lse;
  p.B = B;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.Sq = Sq;
  p.G = Hq / Hkv;
  p.R = p.G * Sq;
  p.P = P;
  p.P_cap = P_cap;
  p.Sk = Sk;
  p.Sk_cap = Sk_cap;
  p.causal = causal && Sq > 1;  // a single row sees its whole cache either way
  p.p_parts = part_count(P, prefix_split_keys);
  p.o_parts = part_count(Sk, split_keys);
  p.parts = p.p_parts + p.o_parts;
  // (one part of whole tiles: the cut at its end)
  p.p_split = p.p_parts == 1 ? (int)(ceil_div(P, BC) * BC) : prefix_split_keys;
  p.o_split = p.o_parts == 1 ? (int)(ceil_div(Sk, BC) * BC) : split_keys;
  // a single part writes O itself, which only workgroups of WROWS rows do
  p.p_rows = p.parts == 1 ? WROWS : prefix_rows((long long)B * p.R);
  p.p_blocks = (int)ceil_div((long long)B * p.R, p.p_rows);
  p.o_blocks = (int)ceil_div(p.R, WROWS);
  const long long pg = (long long)Hkv * p.p_parts * p.p_blocks, og = (long long)B * Hkv * p.o_parts * p.o_blocks;
  if (pg + og > MAX_GROUPS || (p.parts > 1 && rows > MAX_MERGE_ROWS)) return ATTN_EUNSUPPORTED;
  p.p_groups = (int)pg;
  p.o_groups = (int)og;
  p.ck = ldexpf(p.c1, order);
  const size_t need = prefix_workspace(rows, p.parts, d);
  if (chained(P, (int)row, p)) {
    p.chain = p.parts = 1;
    p.p_groups = 0;
  }
  p.longest = by_length(p);
  if (need) {
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < need) return ATTN_EINVAL;
    p.part_o = (float*)workspace;
    p.part_ml = p.part_o + (size_t)rows * p.parts * d;
  }
  const int mode = order == 0 ? (int)MODE_EXACT : 2 * order - 1;
  return launch_prefix(p, dtype, d, mode, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

size_t attn_key_weights_workspace_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int d) {
  (void)d;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv != 0) return 0;
  if ((long long)(Hq / Hkv) * Sq > INT32_MAX) return 0;
  const int parts = weights_parts(Hq / Hkv, Sq);
  return parts <= 1 ? 0 : (size_t)parts * B * Hkv * Sk * sizeof(float);
}

int attn_key_weights(const void* q, const void* k, const float* lse, const int32_t* lens, float* acc, int B, int Hq,
                     int Hkv, int Sq, int Sk, int Sk_cap, int d, int causal, float scale, float decay, int dtype,
                     void* workspace, size_t workspace_bytes, const attn_opts* opts) {
  if (!q || !k || !lse || !acc) return ATTN_EINVAL;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || d <= 0) return ATTN_EINVAL;
  if (Hq % Hkv != 0 || Sk > Sk_cap) return ATTN_EINVAL;
  if (!(decay >= 0.0f && decay < INFINITY)) return ATTN_EINVAL;
  WeightsParams p = {};
  float vd;
  const int rc = check_kind(d, scale, dtype, opts, &p.c1, &vd);
  if (rc != ATTN_OK) return rc;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(lse, 4) || misaligned(lens, 4) || misaligned(acc, 4))
    return ATTN_EUNSUPPORTED;
  const long long row = (long long)d * elem_bytes(dtype);
  if ((long long)B * Hq * Sq > (1LL << 30)) return ATTN_EUNSUPPORTED;
  if (Sk_cap * row > INT32_MAX || (long long)(Hq / Hkv) * Sq * row > INT32_MAX) return ATTN_EUNSUPPORTED;
  p.q = (const uint8_t*)q;
  p.k = (const uint8_t*)k;
  p.lse = lse;
  p.lens = lens;
  p.acc = acc;
  p.B = B;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.Sq = Sq;
  p.G = Hq / Hkv;
  p.Sk = Sk;
  p.Sk_cap = Sk_cap;
  p.causal = causal && Sq > 1;
  weights_runs(p.G, Sq, p.heads, p.hrows);
  p.parts = weights_parts(p.G, Sq);
  p.span = weights_span(p.heads);
  p.blocks = (int)ceil_div(Sk, KW_KEYS);
  if ((long long)p.G * Sq <= KW_FEW_ROWS) {
    const long long units = ceil_div(Sk, KW_FEW_KEYS);
    p.span = weights_run((long long)B * Hkv, units);
    p.blocks = (int)ceil_div(units, 4 * p.span);
  }
  p.decay = decay;
  // (the sum of the parts takes blocks of 256 keys)
  const long long heads = (long long)B * Hkv;
  if (heads * p.parts * p.blocks > MAX_GROUPS || heads * ceil_div(Sk, 256) > MAX_GROUPS) return ATTN_EUNSUPPORTED;
  if (p.parts > 1) {
    const size_t need = (size_t)p.parts * B * Hkv * Sk * sizeof(float);
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < need) return ATTN_EINVAL;
    p.part = (float*)workspace;
  }
  return launch_weights(p, dtype, d, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

size_t attn_evict_workspace_bytes(int B, int Hkv, int Sk) {
  if (B <= 0 || Hkv <= 0 || Sk <= 0) return 0;
  return evict_workspace((long long)B * Hkv, Sk);
}

int attn_evict(const void* k, const void* v, const float* acc, const int32_t* lens, void* k_out, void* v_out,
               float* acc_out, int32_t* index, int32_t* lens_out, int B, int Hkv, int Sk, int Sk_cap, int out_cap,
               int d, int keep, int recent, int dtype, void* workspace, size_t workspace_bytes,
               const attn_opts* opts) {
  if (!k || !v || !acc || !k_out || !v_out || !acc_out || !index || !lens_out) return ATTN_EINVAL;
  if (B <= 0 || Hkv <= 0 || Sk <= 0 || Sk_cap <= 0 || out_cap <= 0 || d <= 0 || keep <= 0) return ATTN_EINVAL;
  if (Sk > Sk_cap || keep > out_cap || recent < 0) return ATTN_EINVAL;
  if (dtype != ATTN_BF16 && dtype != ATTN_FP8_E4M3) return ATTN_EUNSUPPORTED;
  if ((d != 64 && d != 128) || Sk > INT32_MAX - 2 * EVICT_PART) return ATTN_EUNSUPPORTED;
  if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_out, 16) || misaligned(v_out, 16))
    return ATTN_EUNSUPPORTED;
  if (misaligned(acc, 4) || misaligned(lens, 4) || misaligned(acc_out, 4) || misaligned(index, 4) ||
      misaligned(lens_out, 4))
    return ATTN_EUNSUPPORTED;
  EvictParams p = {};
  p.row_bytes = d * elem_bytes(dtype);
  const size_t heads = (size_t)B * Hkv;
  // a selection has 1024 threads; the gather 4 to 16 a row
  if (heads > MAX_GROUPS / 4 || (long long)heads * keep * (p.row_bytes / 16) > MAX_GROUPS * 256)
    return ATTN_EUNSUPPORTED;
  const Range in[] = {range(k, heads * Sk_cap * p.row_bytes), range(v, heads * Sk_cap * p.row_bytes),
                      range(acc, heads * Sk_cap * 4), range(lens, lens ? (size_t)B * 4 : 0)};
  const Range out[] = {range(k_out, heads * out_cap * p.row_bytes), range(v_out, heads * out_cap * p.row_bytes),
                       range(acc_out, heads * out_cap * 4), range(index, heads * keep * 4),
                       range(lens_out, (size_t)B * 4)};
  for (const Range& x : out) {
    for (const Range& y : in)
      if (overlap(x, y)) return ATTN_EINVAL;
    for (const Range& y : out)
      if (&x != &y && overlap(x, y)) return ATTN_EINVAL;
  }
  p.k = (const uint8_t*)k;
  p.v = (const uint8_t*)v;
  p.acc = acc;
  p.lens = lens;
  p.k_out = (uint8_t*)k_out;
  p.v_out = (uint8_t*)v_out;
  p.acc_out = acc_out;
  p.index = index;
  p.lens_out = lens_out;
  p.B = B;
  p.Hkv = Hkv;
  p.Sk = Sk;
  p.Sk_cap = Sk_cap;
  p.keep = keep;
  p.recent = recent;
  p.out_cap = out_cap;
  p.part_keys = evict_part_keys((long long)heads, Sk);
  p.parts = (int)ceil_div(Sk, p.part_keys);
  p.gather = p.parts == 1 && (long long)keep * (p.row_bytes / 16) <= EVICT_GATHER;
  if (p.parts > 1) {
    const size_t need = evict_workspace((long long)heads, Sk);
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < need) return ATTN_EINVAL;
    p.scratch = (uint8_t*)workspace;
    const Range ws = range(workspace, need);
    for (const Range& x : in)
      if (overlap(ws, x)) return ATTN_EINVAL;
    for (const Range& x : out)
      if (overlap(ws, x)) return ATTN_EINVAL;
  }
  return launch_evict(p, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

}  // extern "C"
