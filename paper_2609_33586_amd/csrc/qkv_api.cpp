// The C entry points declared in h15qkv.h: argument checks, launch shapes and
// workspaces, then the launchers of h15rope.hip, h15append.hip and h15blocks.hip.
// Plain C++: no HIP types or calls here, so the same checks build with a host
// compiler alone under the sanitizers.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "h15qkv.h"
#include "qkv_params.h"

using namespace h15;

namespace {

bool finite_pos(float x) { return x > 0.0f && x < INFINITY; }

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

bool misaligned(const void* x, uintptr_t to) { return ((uintptr_t)x & (to - 1)) != 0; }

// Work-items of a launch are counted in 32 bits: workgroups of 256 threads, and
// rows of a merge, four to a workgroup.
constexpr long long MAX_GROUPS = (1LL << 24) - 1, MAX_MERGE_ROWS = 4 * MAX_GROUPS;

struct Range {
  uintptr_t from, to;
};
Range range(const void* p, size_t bytes) { return {(uintptr_t)p, (uintptr_t)p + (p ? bytes : 0)}; }
bool overlap(const Range& a, const Range& b) { return a.from < b.to && b.from < a.to; }

template <size_t N, size_t M>
bool any_overlap(const Range (&out)[N], const Range (&in)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = 0; j < M; ++j)
      if (overlap(out[i], in[j])) return true;
    for (size_t j = i + 1; j < N; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

// Strides of [B][S][H][d], the given ones or the contiguous ones; false if they
// are not usable.
bool strides_of(const attn_strides* given, int B, int S, int H, int d, attn_strides* s) {
  *s = given ? *given : attn_strides{(int64_t)S * H * d, (int64_t)H * d, d};
  const int64_t most = INT64_MAX >> 4;  // (three of them in bytes)
  const int64_t all[] = {s->batch, s->position, s->head}, n[] = {B, S, H};
  for (int i = 0; i < 3; ++i)
    if (all[i] < 0 || all[i] > most / n[i] || all[i] % 8 != 0) return false;
  return true;
}

// The bytes that a tensor of these strides reaches over.
Range reach(const void* p, const attn_strides& s, int B, int S, int H, int d) {
  return range(p, 2 * (size_t)((B - 1) * s.batch + (S - 1) * s.position + (H - 1) * s.head + d));
}

// Heads that a thread takes one after the other at most: its sines and cosines serve
// all of them, as long as there are workgroups enough.
int rope_run(long long tiles, int Hq, int Hkv, int least) {
  int run = 8;
  while (run > 1 && tiles * (ceil_div(Hq, run) + 2 * ceil_div(Hkv, run)) < least) run /= 2;
  return run;
}

// Workgroups of the backward pass for a run of heads: each takes several tiles of
// positions where there are many, so that its sums of the weights' gradient are
// few.
int rope_groups(long long tiles, long long runs) {
  const long long most = ceil_div(4096, runs);
  return (int)(tiles < most ? tiles : most);
}

struct RopeShape {
  long long tiles;
  int groups, runs[3];
};
RopeShape rope_shape(int B, int S, int Hq, int Hkv, int d, bool backward) {
  RopeShape r;
  r.tiles = ceil_div((long long)B * S, rope_tokens(d));
  // (times with 1024 workgroups or more / so many: 3 x 1510 positions of 32 heads over 8, d = 128,
  // norms 26.5 / 23.4 us, their gradient 37.9 / 36.0; that of 700 positions 13.6 / 11.7)
  const int run = rope_run(r.tiles, Hq, Hkv, backward ? 512 : 768);
  r.runs[0] = (int)ceil_div(Hq, run);
  r.runs[1] = r.runs[2] = (int)ceil_div(Hkv, run);
  r.groups = rope_groups(r.tiles, (long long)r.runs[0] + 2 * r.runs[1]);
  return r;
}

// What both directions check and set; heads[i]: 0 where tensor i is absent.  (The
// launch's shape goes by the heads that the call names, absent or not, so that the
// workspace's size does too.)
int check_rope(const attn_rope_spec* spec, int B, int S, int Hq, int Hkv, const int (&heads)[3], int d, bool backward,
               RopeParams* p) {
  if (!spec || B <= 0 || S <= 0 || d <= 0) return ATTN_EINVAL;
  if (spec->rot < 0 || spec->rot > d || (spec->rot > 0 && !spec->freqs) || !finite_pos(spec->amplitude))
    return ATTN_EINVAL;
  const bool norm = (heads[0] && spec->q_weight) || (heads[1] && spec->k_weight);
  if (norm && !(spec->eps >= 0x1p-126f && spec->eps < INFINITY)) return ATTN_EINVAL;
  if ((d != 64 && d != 128) || spec->rot % 16 != 0) return ATTN_EUNSUPPORTED;
  if (norm && spec->weight_dtype != ATTN_BF16 && spec->weight_dtype != ATTN_FP32) return ATTN_EUNSUPPORTED;
  if (misaligned(spec->positions, 4) || misaligned(spec->freqs, 8) || misaligned(spec->q_weight, 16) ||
      misaligned(spec->k_weight, 16))
    return ATTN_EUNSUPPORTED;
  const long long tokens = (long long)B * S;
  if (tokens > INT32_MAX) return ATTN_EUNSUPPORTED;
  if (Hq < 0) Hq = 0;
  if (Hkv < 0) Hkv = 0;
  if (tokens * Hq > INT32_MAX || tokens * Hkv > INT32_MAX) return ATTN_EUNSUPPORTED;
  p->positions = spec->positions;
  p->each_position = spec->each_position;
  p->freqs = spec->freqs;
  p->rot = spec->rot;
  p->interleaved = spec->interleaved != 0;
  p->weight_bf16 = spec->weight_dtype == ATTN_BF16;
  p->amplitude = spec->amplitude;
  p->eps = spec->eps;
  p->B = B;
  p->S = S;
  p->d = d;
  const RopeShape r = rope_shape(B, S, Hq, Hkv, d, backward);
  if (r.tiles > MAX_GROUPS || Hq + 2LL * Hkv > 65535) return ATTN_EUNSUPPORTED;
  p->tiles = (int)r.tiles;
  p->groups = r.groups;
  const void* weight[3] = {spec->q_weight, spec->k_weight, nullptr};
  int rows = 0;
  for (int i = 0; i < 3; ++i) {
    RopeTensor& t = p->t[i];
    t.heads = heads[i];
    t.runs = heads[i] ? r.runs[i] : 0;
    t.run = heads[i] ? (int)ceil_div(heads[i], t.runs) : 0;
    t.turned = i < 2 && spec->rot > 0;
    t.weight = heads[i] ? weight[i] : nullptr;
    t.partials = rows;
    if (t.weight) rows += t.runs * r.groups;
  }
  return ATTN_OK;
}

// Input-rounding order of an exp_mode that decode over a cache offers, 0 for the
// hardware exponential, -1 for others.
int exp_order(int exp_mode) {
  switch (exp_mode) {
    case ATTN_EXP_EXACT: return 0;
    case ATTN_EXP_H15: return 1;
    case ATTN_EXP_SQ4: return 2;
    case ATTN_EXP_SQ8: return 3;
    default: return -1;
  }
}

int log2_block(int block) {
  switch (block) {
    case 16: return 4;
    case 32: return 5;
    case 64: return 6;
    case 128: return 7;
    default: return -1;
  }
}

// Parts of `keys` keys cut at `split` (0 or >= keys: one part).
int part_count(int keys, int split) { return split <= 0 || split >= keys ? 1 : (int)ceil_div(keys, split); }

// What a form of attn_decode_blocks takes for `tiles` tiles of keys cut into `parts`, as
// fitted to its times: the workgroups that one of 256 compute units gets, times the tiles
// of a part and what starting costs, in tiles of a workgroup of 128 rows that has its
// compute unit alone (2.4 us at d = 128).  Two of these share one at 0.85 of their time
// one after the other; of several sequences, whose lengths differ, many fill up as others
// end.  Of 512 rows one has a compute unit, and takes a tile in 2.35 times the time.
double blocks_cost(int rows, long long heads, long long R, double tiles, long long parts, bool ragged) {
  const double n = (double)ceil_div(heads * ceil_div(R, rows) * parts, 256), part = tiles / (double)parts;
  if (rows == BLOCKS_WIDE) return n * 2.35 * (part + 6);
  return n * (n == 1 ? 1 : !ragged ? 0.85 : n < 4 ? 0.82 : 0.72) * (part + 1);
}

// The same of 32 rows (tiles of 0.7 us at d = 128, 0.4 at 64), the merge included.  Two on
// a compute unit gain little at d = 128, where a whole cache each ends with the longest,
// more at 64; more than two wait for each other, and fill up as others end.
double blocks_cost_keys(long long groups, double tiles, long long parts, int d) {
  const long long all = groups * parts;
  const double turns = all > 512 ? 1.15 / 256 * (double)all : all > 256 ? 2.0 : d == 64 ? 1.25 : parts == 1 ? 1.2 : 1.0;
  return turns * (tiles / (double)parts + 1) + (parts == 1 ? 0 : d == 64 ? 6 : 4);
}

// Query rows of a workgroup, for R rows of a sequence and KV head.  The wide form
// (exact weights) takes a third less time for its rows' keys, once it runs and if it has them:
// for long caches, whose causal ends weigh little, by the cost above.  Times of a call in
// 128 / 512 rows, each with its best cut, 8 KV heads, d = 128, R rows: 8192 after 32K keys
// 1059 / 931 us, 2048 after 16K 152 / 150, 1200 of 26K 154 / 161, 4 sequences of 528 rows of
// up to 26K 241 / 324, of 1000 379 / 344; 8192 of 4K 136 / 144, 2048 after 4K 54 / 66, 4
// sequences of 2048 of 2K 71 / 94.
int blocks_rows(int B, long long heads, long long R, int Sk, long long parts, bool exact) {
  if (R <= 4 * WROWS) return WROWS;
  const double tiles = (double)ceil_div(Sk, BC);
  const bool wide = exact && Sk >= 8192 && R >= BLOCKS_WIDE &&
                    blocks_cost(BLOCKS_WIDE, heads, R, tiles, parts, B > 1) <
                        blocks_cost(BLOCKS_ROWS, heads, R, tiles, parts, B > 1);
  return wide ? BLOCKS_WIDE : BLOCKS_ROWS;
}

// Workgroups that run at once.
int blocks_slots(int rows) { return rows == BLOCKS_WIDE ? 256 : 512; }

// Whether keys are read with a streaming hint: where one workgroup reads each, and
// they are more than the last-level cache keeps from one step to the next (256 MB, of
// which other data have a part).  Times of a call without / with it: 64 ragged caches of
// up to 32K keys 504 / 455 us (5.5 / 6.1 TB/s), 16 of 8K 41.6 / 36.9; 7 of 5K, 57 MB
// that it finds there again, 17.6 / 17.9.
bool blocks_stream(long long heads, int row_blocks, int Sk, int d) {
  return row_blocks == 1 && heads * Sk * 2 * d >= (128LL << 20);
}

size_t blocks_workspace(long long rows, int parts, int d) {
  return parts <= 1 ? 0 : (size_t)rows * (size_t)parts * ((size_t)d + 2) * sizeof(float);
}
}  // namespace

extern "C" {

int attn_rope(const void* q, const void* k, const void* v, const attn_strides* strides, const attn_rope_spec* spec,
              void* q_out, void* k_out, void* v_out, int B, int S, int Hq, int Hkv, int d, int dtype,
              const attn_opts* opts) {
  const void* in[3] = {q, k, v};
  void* out[3] = {q_out, k_out, v_out};
  int heads[3] = {Hq, Hkv, Hkv};
  if (!q && !k && !v) return ATTN_EINVAL;
  for (int i = 0; i < 3; ++i) {
    if (!in[i] != !out[i] || (in[i] && heads[i] <= 0)) return ATTN_EINVAL;
    if (!in[i]) heads[i] = 0;
  }
  RopeParams p = {};
  const int rc = check_rope(spec, B, S, Hq, Hkv, heads, d, false, &p);
  if (rc != ATTN_OK) return rc;
  if (dtype != ATTN_BF16 && dtype != ATTN_FP8_E4M3) return ATTN_EUNSUPPORTED;
  const bool fp8 = dtype == ATTN_FP8_E4M3;
  if (fp8 && !opts) return ATTN_EINVAL;
  const float descale[3] = {fp8 ? opts->q_descale : 1.0f, fp8 ? opts->k_descale : 1.0f, fp8 ? opts->v_descale : 1.0f};
  Range ins[7], outs[3];
  for (int i = 0; i < 3; ++i) {
    RopeTensor& t = p.t[i];
    attn_strides s = {};
    if (in[i]) {
      if (!finite_pos(descale[i])) return ATTN_EINVAL;
      if (misaligned(in[i], 16) || misaligned(out[i], 16) ||
          !strides_of(strides ? strides + i : nullptr, B, S, heads[i], d, &s))
        return ATTN_EUNSUPPORTED;
      ins[i] = reach(in[i], s, B, S, heads[i], d);
    } else {
      ins[i] = range(nullptr, 0);
    }
    outs[i] = range(out[i], (size_t)B * S * heads[i] * d * (fp8 ? 1 : 2));
    t.in = (const uint16_t*)in[i];
    t.out = out[i];
    t.sb = s.batch;
    t.ss = s.position;
    t.sh = s.head;
    t.inv = 1.0f / descale[i];
    if (in[i] && !finite_pos(t.inv)) return ATTN_EINVAL;
  }
  ins[3] = range(spec->positions, (size_t)B * (spec->each_position ? S : 1) * 4);
  ins[4] = range(spec->freqs, (size_t)spec->rot * 4);
  ins[5] = range(spec->q_weight, (size_t)d * (p.weight_bf16 ? 2 : 4));
  ins[6] = range(spec->k_weight, (size_t)d * (p.weight_bf16 ? 2 : 4));
  if (any_overlap(outs, ins)) return ATTN_EINVAL;
  return launch_rope(p, dtype, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

size_t attn_rope_bwd_workspace_bytes(int B, int S, int Hq, int Hkv, int d) {
  if (B <= 0 || S <= 0 || Hq < 0 || Hkv < 0 || Hq + (long long)Hkv <= 0 || (d != 64 && d != 128)) return 0;
  if ((long long)B * S * Hq > INT32_MAX || (long long)B * S * Hkv > INT32_MAX) return 0;
  const RopeShape r = rope_shape(B, S, Hq, Hkv, d, true);
  return (size_t)(r.runs[0] + r.runs[1]) * r.groups * d * sizeof(float);
}

int attn_rope_bwd(const void* gq, const void* gk, const void* gv, const void* q, const void* k,
                  const attn_strides* strides, const attn_rope_spec* spec, void* dq, void* dk, void* dv,
                  const attn_strides* grad_strides, float* dq_weight, float* dk_weight, int B, int S, int Hq, int Hkv,
                  int d, void* workspace, size_t workspace_bytes, const attn_opts* opts) {
  const void* g[3] = {gq, gk, gv};
  const void* in[3] = {q, k, nullptr};
  void* out[3] = {dq, dk, dv};
  float* dweight[3] = {dq_weight, dk_weight, nullptr};
  int heads[3] = {Hq, Hkv, Hkv};
  if (!gq && !gk && !gv) return ATTN_EINVAL;
  for (int i = 0; i < 3; ++i) {
    if (!g[i] != !out[i] || (g[i] && heads[i] <= 0)) return ATTN_EINVAL;
    if (!g[i]) heads[i] = 0;
  }
  RopeParams p = {};
  const int rc = check_rope(spec, B, S, Hq, Hkv, heads, d, true, &p);
  if (rc != ATTN_OK) return rc;
  Range ins[9], grads[3], sums[3];
  int rows = 0;
  for (int i = 0; i < 3; ++i) {
    RopeTensor& t = p.t[i];
    attn_strides s = {}, gs = {};
    const bool norm = t.weight != nullptr;
    if (norm && (!in[i] || !dweight[i])) return ATTN_EINVAL;
    if (g[i] && (misaligned(g[i], 16) || misaligned(out[i], 16) ||
                 !strides_of(grad_strides ? grad_strides + i : nullptr, B, S, heads[i], d, &gs)))
      return ATTN_EUNSUPPORTED;
    if (norm && (misaligned(in[i], 16) || misaligned(dweight[i], 4) ||
                 !strides_of(strides ? strides + i : nullptr, B, S, heads[i], d, &s)))
      return ATTN_EUNSUPPORTED;
    ins[i] = range(g[i], (size_t)B * S * heads[i] * d * 2);
    ins[3 + i] = norm ? reach(in[i], s, B, S, heads[i], d) : range(nullptr, 0);
    grads[i] = g[i] ? reach(out[i], gs, B, S, heads[i], d) : range(nullptr, 0);
    sums[i] = range(norm ? dweight[i] : nullptr, (size_t)d * 4);
    t.in = (const uint16_t*)in[i];
    t.out = (void*)g[i];
    t.grad = (uint16_t*)out[i];
    t.dweight = norm ? dweight[i] : nullptr;
    t.sb = s.batch;
    t.ss = s.position;
    t.sh = s.head;
    t.gb = gs.batch;
    t.gs = gs.position;
    t.gh = gs.head;
    if (norm) rows += t.runs * p.groups;
  }
  ins[6] = range(spec->positions, (size_t)B * (spec->each_position ? S : 1) * 4);
  ins[7] = range(spec->freqs, (size_t)spec->rot * 4);
  ins[8] = range(nullptr, 0);
  const size_t need = (size_t)rows * d * sizeof(float);
  if (need && (!workspace || misaligned(workspace, 16) || workspace_bytes < need)) return ATTN_EINVAL;
  const size_t weight_bytes = (size_t)d * (p.weight_bf16 ? 2 : 4);
  const Range weights[2] = {range(p.t[0].weight, weight_bytes), range(p.t[1].weight, weight_bytes)};
  // (the gradients may be views of one tensor, whose ranges overlap by their strides)
  for (const Range& x : grads) {
    for (const Range& y : ins)
      if (overlap(x, y)) return ATTN_EINVAL;
    for (const Range& y : weights)
      if (overlap(x, y)) return ATTN_EINVAL;
    for (const Range& y : sums)
      if (overlap(x, y)) return ATTN_EINVAL;
  }
  const Range more[4] = {sums[0], sums[1], range(workspace, need), range(nullptr, 0)};
  if (any_overlap(more, ins) || any_overlap(more, weights)) return ATTN_EINVAL;
  for (const Range& x : grads)
    if (overlap(x, more[2])) return ATTN_EINVAL;
  p.part = (float*)workspace;
  return launch_rope_bwd(p, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

int attn_cache_append(const void* k, const void* v, void* k_cache, void* v_cache, uint8_t* scales,
                      const int32_t* lens, const int32_t* counts, int32_t* lens_out, int B, int Hkv, int n, int cap,
                      int d, int block, const attn_opts* opts) {
  if (!k || !v || !k_cache || !v_cache || !scales || !lens || !lens_out) return ATTN_EINVAL;
  if (B <= 0 || Hkv <= 0 || n <= 0 || cap <= 0 || d <= 0) return ATTN_EINVAL;
  const int shift = log2_block(block);
  if ((d != 64 && d != 128) || shift < 0) return ATTN_EUNSUPPORTED;
  if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16))
    return ATTN_EUNSUPPORTED;
  if (misaligned(lens, 4) || misaligned(counts, 4) || misaligned(lens_out, 4)) return ATTN_EUNSUPPORTED;
  if ((long long)cap * d > INT32_MAX || (long long)n * d * 2 > INT32_MAX) return ATTN_EUNSUPPORTED;
  AppendParams p = {};
  p.blocks = (int)ceil_div(cap, block);
  const long long reach = ((long long)n + block - 2) / block + 1;
  p.reach = (int)(reach < p.blocks ? reach : p.blocks);
  const long long heads = (long long)B * Hkv;
  if (heads > MAX_GROUPS || heads * 2 * p.reach > MAX_GROUPS) return ATTN_EUNSUPPORTED;
  const size_t fresh = (size_t)heads * n * d * 2, codes = (size_t)heads * cap * d;
  const Range in[] = {range(k, fresh), range(v, fresh), range(lens, lens_out == lens ? 0 : (size_t)B * 4),
                      range(counts, (size_t)B * 4)};
  const Range out[] = {range(k_cache, codes), range(v_cache, codes), range(scales, (size_t)heads * p.blocks * 2),
                       range(lens_out, (size_t)B * 4)};
  if (any_overlap(out, in)) return ATTN_EINVAL;
  p.x[0] = (const uint16_t*)k;
  p.x[1] = (const uint16_t*)v;
  p.cache[0] = (uint8_t*)k_cache;
  p.cache[1] = (uint8_t*)v_cache;
  p.scales = scales;
  p.lens = lens;
  p.counts = counts;
  p.lens_out = lens_out;
  p.B = B;
  p.Hkv = Hkv;
  p.n = n;
  p.cap = cap;
  return launch_append(p, d, block, lens_out == lens, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

size_t attn_decode_blocks_workspace_bytes(int B, int Hq, int Sq, int Sk, int d, int split_keys) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || Sk <= 0 || d <= 0 || split_keys < 0) return 0;
  return blocks_workspace((long long)B * Hq * Sq, part_count(Sk, split_keys), d);
}

int attn_decode_blocks_split_keys(int B, int Hq, int Hkv, int Sq, int Sk, int d) {
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv != 0) return 0;
  const long long R = (long long)(Hq / Hkv) * Sq, heads = (long long)B * Hkv, tiles = ceil_div(Sk, BC);
  long long parts = 1;
  const long long groups = heads * ceil_div(R, R > 4 * WROWS ? BLOCKS_ROWS : WROWS);
  if (R <= 4 * WROWS && groups > 256) {
    // bound by HBM, whatever the cut: only so many that ragged caches end together (one part /
    // three / five, d = 128, 8 KV heads: 64 sequences of up to 32K keys 461 / 453 / 442 us, of
    // 16K 233 / 210 / 206; 45 of 8K 105 / 88 / 86, of 4K 58 / 55 / 56, of 2.2K 34 / 34 / 44; where
    // others follow the ones that run, few do: 100 of 9K 191 / 201 / 203)
    parts = tiles >= 128 ? 5 : tiles >= 48 && groups < 512 ? 3 : 1;
  } else {
    // the cheapest of all, whose parts have eight tiles or more (four of sixteen and more,
    // where each workgroup has its compute unit), and the merge (8 KV heads, d = 128, one row: 20 sequences of up to
    // 8K keys in 3 parts, 480 workgroups, 42 us, in 4, 640, 46; 3 of 4K in 4 / 8 parts 12.0 /
    // 10.3; 16 of 8K in 2 / 4 33.3 / 34.1, of d = 64 22.0 / 20.0)
    const long long most = tiles / 4 < 2048 / groups ? tiles / 4 : 2048 / groups;
    double best = INFINITY;
    for (long long n = 1; n <= most || n == 1; ++n) {
      if (n > 1 && n > tiles / 8 && (R > 4 * WROWS || groups * n > 256 || tiles < 16)) break;
      const double cost = R <= 4 * WROWS ? blocks_cost_keys(groups, (double)tiles, n, d)
                                         : blocks_cost(blocks_rows(B, heads, R, Sk, n, true), heads, R, (double)tiles, n, B > 1) +
                                               (n > 1 ? 5e-5 * (double)(heads * R * n) : 0);
      if (cost < best) best = cost, parts = n;
    }
  }
  return parts <= 1 ? 0 : (int)(ceil_div(tiles, parts) * BC);
}

int attn_decode_blocks(const void* q, const void* k, const void* v, const uint8_t* scales, const int32_t* lens,
                       void* o, float* lse, int B, int Hq, int Hkv, int Sq, int Sk, int Sk_cap, int d, int block,
                       int causal, float scale, int exp_mode, int split_keys, void* workspace,
                       size_t workspace_bytes, const attn_opts* opts) {
  if (!q || !k || !v || !scales || !o) return ATTN_EINVAL;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || d <= 0) return ATTN_EINVAL;
  if (Hq % Hkv != 0 || Sk > Sk_cap || !finite_pos(scale)) return ATTN_EINVAL;
  if (split_keys < 0 || split_keys % BC != 0) return ATTN_EINVAL;
  const int order = exp_order(exp_mode), shift = log2_block(block);
  if ((d != 64 && d != 128) || shift < 0 || order < 0) return ATTN_EUNSUPPORTED;
  if (opts && opts->rescale_threshold != 0.0f)
    return opts->rescale_threshold > 0.0f && opts->rescale_threshold <= 64.0f ? ATTN_EUNSUPPORTED : ATTN_EINVAL;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(o, 16) || misaligned(lse, 4) ||
      misaligned(lens, 4) || misaligned(scales, 2))
    return ATTN_EUNSUPPORTED;
  const long long rows = (long long)B * Hq * Sq;
  if (rows > (1LL << 30) || (long long)Sk_cap * d > INT32_MAX) return ATTN_EUNSUPPORTED;
  BlocksParams p = {};
  p.c1 = (float)((double)scale * 1.4426950408889634);
  p.ck = ldexpf(p.c1, order);
  p.q = (const uint8_t*)q;
  p.k = (const uint8_t*)k;
  p.v = (const uint8_t*)v;
  p.scales = scales;
  p.lens = lens;
  p.o = (uint16_t*)o;
  p.lse = lse;
  p.B = B;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.Sq = Sq;
  p.G = Hq / Hkv;
  p.R = p.G * Sq;
  p.Sk = Sk;
  p.Sk_cap = Sk_cap;
  p.causal = causal && Sq > 1;  // a single row sees its whole cache either way
  p.shift = shift;
  p.blocks = (int)ceil_div(Sk_cap, block);
  p.parts = part_count(Sk, split_keys);
  // (one part of whole tiles: the cut at its end)
  p.split = p.parts == 1 ? (int)(ceil_div(Sk, BC) * BC) : split_keys;
  p.turn = p.parts % 8 == 0 ? 0 : p.parts % 4 == 0 ? 1 : p.parts % 2 == 0 ? 2 : 3;
  p.rows = blocks_rows(B, (long long)B * Hkv, p.R, Sk, p.parts, order == 0);
  p.row_blocks = (int)ceil_div(p.R, p.rows);
  const long long groups = (long long)B * Hkv * p.parts * p.row_blocks;
  if (groups > MAX_GROUPS / (p.rows == BLOCKS_WIDE ? 2 : 1) || (p.parts > 1 && rows > MAX_MERGE_ROWS))
    return ATTN_EUNSUPPORTED;
  p.groups = (int)groups;
  // ragged caches that are more than one for each slot are taken longest first, so
  // that no long one starts last
  p.longest = lens && B > 1 && B <= 256 && groups > blocks_slots(p.rows);
  p.stream = blocks_stream((long long)B * Hkv, p.row_blocks, Sk, d);
  const size_t need = blocks_workspace(rows, p.parts, d);
  if (need) {
    if (!workspace || misaligned(workspace, 16) || workspace_bytes < need) return ATTN_EINVAL;
    p.part_o = (float*)workspace;
    p.part_ml = p.part_o + (size_t)rows * p.parts * d;
  }
  const size_t heads = (size_t)B * Hkv, codes = heads * Sk_cap * d;
  const Range in[] = {range(q, (size_t)rows * d * 2), range(k, codes), range(v, codes),
                      range(scales, heads * p.blocks * 2), range(lens, (size_t)B * 4)};
  const Range out[] = {range(o, (size_t)rows * d * 2), range(lse, (size_t)rows * 4), range(need ? workspace : nullptr, need)};
  if (any_overlap(out, in)) return ATTN_EINVAL;
  const int mode = order == 0 ? (int)MODE_EXACT : 2 * order - 1;
  return launch_blocks(p, d, mode, opts ? opts->stream : nullptr) == 0 ? ATTN_OK : ATTN_ELAUNCH;
}

}  // extern "C"
