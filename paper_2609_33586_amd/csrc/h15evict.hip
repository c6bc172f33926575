// Which keys of a cache stay (attn_evict): of the n keys of each (batch, KV
// head) the last `recent` and, of the others, those with the largest
// accumulated weight, `keep` in all (equal weights: the lowest index first),
// in their order.  One workgroup a (batch, KV head) finds them and writes their
// indexes; then their rows of K, V and acc are gathered into the compact caches,
// 16 bytes a thread, by that workgroup if they are few, else by a launch of their
// own.  Where few heads have long caches, parts of the keys have a workgroup each,
// in four launches.  (The rules: cache_api.cpp.)
//
// The selection is a radix search for the weight of rank keep - recent in three
// rounds over 11, 11 and 10 bits, each a histogram in LDS of the keys that agree
// with the digits found so far; then a count of the keys that stay, stretch by
// stretch, and a second pass that writes their indexes in order.  The weights
// are read once, as ordered numbers into LDS (of a cache of more than 32K keys
// every pass reads the rest again).  (In registers, 32 a thread, the passes had
// to be unrolled, and a workgroup spent its time fetching code that it runs once:
// 41 us for 32K keys; re-read from memory in every pass 53 us.)
//
// What bounds it: the gather (read and written once: 32 caches of 8 heads, 4096 of
// 5000 FP8 rows, 75 us at 5.4 TB/s after 9 of the selection); with few caches the
// passes' latency.  A selection of 300 keys takes 7.5 us, the copy of 100 rows
// included; of 32K keys by one workgroup 25 us: 6 for the first digits, whose
// counts in LDS follow each other where weights are equal, 4 and 1.3 for the others,
// 5 for the indexes, each instruction a key taking 0.25 us of a compute unit; in
// parts 4 + 5 + 5 + 6 us, whatever the weights are, and 5 for the gather.
#include "cache_params.h"

#include <hip/hip_runtime.h>
#include <math.h>

namespace {

using namespace h15;

constexpr int SEL = 1024;  // threads of a selection
constexpr int SW = SEL / 64;
constexpr int BINS = 2048;
// Weights in LDS.  Few: two workgroups share a compute unit (a call on 320 heads,
// 1000 keys of which 512 rows stay: 42 -> 38 us).
constexpr int HELD_FEW = 8192, HELD_MANY = 32768;
constexpr int STEP = 256;    // keys of a wave and step: four a lane

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Weights as unsigned numbers in their order: +0 and -0 alike, NaN above all.
__device__ __forceinline__ uint32_t rank_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Adds one to the bin of every lane that has one (bin >= 0), in two histograms,
// of odd and of even lanes.  LDS adds to one
// address follow each other: lanes that all have the same bin, as with equal
// weights, are counted together.
__device__ __forceinline__ void count(uint32_t* hist, int bin, int lane) {
  const int one = __builtin_amdgcn_readfirstlane(bin);
  if (!__ballot(bin != one)) {
    if (lane == 0 && one >= 0) atomicAdd(&hist[one], 64u);
  } else if (bin >= 0) {
    atomicAdd(&hist[bin], 1u);
  }
}

// Inclusive sum over the lanes of a wave: within rows of 16 by shifts, then from
// row to row.
__device__ __forceinline__ uint32_t scan(uint32_t x) {
  int v = (int)x;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);   // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);   // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);   // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
  return (uint32_t)v;
}

// Sum of the waves' numbers below this wave's
__device__ __forceinline__ uint32_t sum_below(const uint32_t* waves, int wave) {
  uint32_t sum = 0;
#pragma unroll
  for (int i = 0; i < SW; i += 4) {
    const u32x4 x = *(const u32x4*)&waves[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += i + e < wave ? x[e] : 0;
  }
  return sum;
}

// The bin from the top in which a count passes `left`: c[j] is the count of this
// thread's bin BINS - 1 - (PER tid + j).  Makes it the next digits, and `left`
// what is still wanted of it.
constexpr int PER = BINS / SEL;
struct Search {
  uint32_t waves[SW];
  uint32_t found[2];  // digits so far, keys still wanted among those that agree
};
__device__ __forceinline__ void next_digits(Search& sh, const uint32_t (&c)[PER], int width, uint32_t& digits,
                                            uint32_t& left, int tid, int lane, int wave) {
  static_assert(PER == 2, "two bins a thread");
  const uint32_t own = c[0] + c[1];
  const uint32_t upto = scan(own);
  if (lane == 63) sh.waves[wave] = upto;
  __syncthreads();
  const uint32_t before = upto - own + sum_below(sh.waves, wave);
  if (before < left && before + own >= left) {
    const bool second = before + c[0] < left;
    sh.found[0] = (digits << width) | (uint32_t)(BINS - 1 - (PER * tid + (second ? 1 : 0)));
    sh.found[1] = left - before - (second ? c[0] : 0);
  }
  __syncthreads();
  digits = sh.found[0];
  left = sh.found[1];
}

// The indexes of the keys of one (batch, KV head) that stay.  HELD: weights in LDS.
template <int HELD>
__device__ __forceinline__ void select_keys(const EvictParams& p, int bh, int n, int32_t* index) {
  __shared__ __attribute__((aligned(16))) uint32_t ranks[HELD];
  __shared__ uint32_t hist[2][BINS];  // odd and even lanes' counts
  __shared__ __attribute__((aligned(16))) Search search;
  __shared__ __attribute__((aligned(16))) uint32_t above[SW], equal[SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* const acc = p.acc + (size_t)bh * p.Sk_cap;
  if (n <= p.keep) {
    for (int i = tid; i < p.keep; i += SEL) index[i] = i < n ? i : -1;
    return;
  }
  const int late = n - min(p.recent, p.keep);  // the keys from here on stay
  const uint32_t want = (uint32_t)(p.keep - (n - late));
  auto put_late = [&] {
    for (int i = late + tid; i < n; i += SEL) index[want + (uint32_t)(i - late)] = i;
  };
  if (want == 0) return put_late();

#pragma unroll
  for (int i = 0; i < 2 * PER; ++i) hist[0][i * SEL + tid] = 0;
  __syncthreads();
  // The first digits are counted as the weights come in.  (Rank 0, which no
  // weight has, up to a whole step.)
  const int held = min((late + STEP - 1) / STEP * STEP, HELD);
  constexpr int BATCH = HELD / SEL;  // loads of a thread at a time
  for (int i0 = tid; i0 < held; i0 += BATCH * SEL) {
    float x[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) x[j] = acc[min(i0 + j * SEL, late - 1)];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int i = i0 + j * SEL;
      if (i - lane >= held) break;
      const uint32_t u = i < late ? rank_of(x[j]) : 0;
      ranks[i] = u;
      count(hist[lane & 1], u != 0 ? (int)(u >> 21) : -1, lane);
    }
  }
  for (int i0 = HELD + tid; i0 - lane < late; i0 += SEL)
    count(hist[lane & 1], i0 < late ? (int)(rank_of(acc[i0]) >> 21) : -1, lane);
  __syncthreads();
  // the ranks of this lane's four keys of the step from i (of the whole wave) on
  auto four = [&](int i) {
    if (i < HELD) return *(const u32x4*)&ranks[i + 4 * lane];
    i += 4 * lane;
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = i + e < late ? rank_of(acc[i + e]) : 0;
    return u;
  };
  uint32_t digits = 0, left = want;
#pragma unroll 1
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, width = round < 2 ? 11 : 10;
    if (round > 0) {
      // (whole waves: the lanes beyond the last key have no bin)
      for (int i = wave * STEP; i < late; i += SW * STEP) {
        const u32x4 u = four(i);
        bool in[4], any = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= in[e] = (u[e] >> (shift + width)) == digits;
        const unsigned long long who = __ballot(any);
        if (!who) continue;
        const bool few = __popcll(who) <= 16;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (few) {
            if (in[e]) atomicAdd(&hist[lane & 1][(u[e] >> shift) & ((1u << width) - 1)], 1u);
          } else if (__ballot(in[e])) {
            count(hist[lane & 1], in[e] ? (int)((u[e] >> shift) & ((1u << width) - 1)) : -1, lane);
          }
      }
      __syncthreads();
    }
    uint32_t c[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int bin = BINS - 1 - (PER * tid + j);
      c[j] = hist[0][bin] + hist[1][bin];
      hist[0][bin] = hist[1][bin] = 0;  // for the next round
    }
    next_digits(search, c, width, digits, left, tid, lane, wave);
  }
  // now: all keys above `digits` stay, and the first `left` of those equal to it.
  // Each wave has a stretch of the keys before `late`, in order.
  const int stretch = (late + SW * STEP - 1) / (SW * STEP) * STEP;
  const int i0 = min(wave * stretch, late), i1 = min(i0 + stretch, late);
  uint32_t na = 0, ne = 0;
  for (int i = i0; i < i1; i += STEP) {
    const u32x4 u = four(i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      na += u[e] > digits ? 1 : 0;
      ne += u[e] == digits ? 1 : 0;
    }
  }
  na = scan(na);
  ne = scan(ne);
  if (lane == 63) above[wave] = na, equal[wave] = ne;
  __syncthreads();
  put_late();
  // Above and equal ones before a key: of the equal ones the first `left` stay.
  uint32_t ab = sum_below(above, wave), eq = sum_below(equal, wave);
  for (int i = i0; i < i1; i += STEP) {
    const u32x4 u = four(i);
    uint32_t own = 0;  // equal ones, above ones: at most 256 each in a step
#pragma unroll
    for (int e = 0; e < 4; ++e) own += u[e] > digits ? 1 : u[e] == digits ? 1u << 16 : 0;
    const uint32_t upto = scan(own), all = __builtin_amdgcn_readlane(upto, 63);
    const uint32_t before = upto - own;
    uint32_t e0 = eq + (before >> 16), to = ab + (before & 0xFFFF) + min(e0, left);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool same = u[e] == digits;
      if (u[e] > digits || (same && e0 < left)) index[to++] = i + 4 * lane + e;
      e0 += same ? 1 : 0;
    }
    ab += all & 0xFFFF;
    eq += all >> 16;
  }
}

// The same by a workgroup for each part of a head's keys, in four launches: three
// count the digits of a part's weights, each after the digits before them have been
// found from the counts of all the head's parts; the last finds the lowest digits and
// places the part's keys.  What a workgroup reads depends on the number of keys and
// parts alone: all of them equal or all different take the same time.  (Three launches, the
// last of which passed over the keys of the whole head that agree with the first digits,
// took 21 us for 8 heads of 33000 spread weights, where these take 23, but 72 for
// equal ones, and grew with the square of the keys: 64 heads of one million equal ones
// 36 ms, now 0.34.)  What the launches hand on, for each part:
struct Part {
  uint32_t counts[2][BINS / 2];  // of two bins of the first and second digits, the even one's low
  uint32_t low[BINS / 4];        // of the third
  uint32_t digits, left;         // the digits so far, what is wanted of the keys with them
  uint32_t above;                // keys of the parts before this one with higher digits so far
  uint32_t unused;
};
static_assert(sizeof(Part) == EVICT_PART_BYTES, "the workspace is sized by it");
static_assert(EVICT_PART_MOST < 1 << 16, "a count has 16 bits");

struct Place {  // of a workgroup
  int bh, part, n, late;
  int from, to;  // the part's keys before `late`
  int used;      // parts with such keys
  uint32_t want;
  Part* parts;   // of its head
};

// False where nothing is to be sought: all keys stay, or only the late ones.
__device__ __forceinline__ bool place(const EvictParams& p, Place& w) {
  // the parts of a head run on one XCD (workgroup ids go round the eight), whose L2 then
  // serves their counts: 8 heads of 33000 keys 25 -> 23 us
  const int unit = blockIdx.x, even = p.B * p.Hkv / 8 * 8 * p.parts;
  if (unit < even) {
    const int k = (unit >> 3) / p.parts;
    w.bh = 8 * k + (unit & 7);
    w.part = (unit >> 3) - k * p.parts;
  } else {
    w.bh = unit / p.parts;
    w.part = unit - w.bh * p.parts;
  }
  w.n = p.lens ? min(max(p.lens[w.bh / p.Hkv], 0), p.Sk) : p.Sk;
  w.late = max(w.n - min(p.recent, p.keep), 0);
  w.want = (uint32_t)(p.keep - (w.n - w.late));
  w.from = w.part * p.part_keys;
  w.to = w.late - w.from > p.part_keys ? w.from + p.part_keys : w.late;
  w.used = w.late > 0 ? (w.late - 1) / p.part_keys + 1 : 0;
  w.parts = (Part*)p.scratch + (size_t)w.bh * p.parts;
  return w.n > p.keep && w.want > 0;
}

// The weights of four keys from i on, and their ranks, 0 from `to` on.  (Two steps:
// weights are asked for early, and waited for where the ranks are taken.)
__device__ __forceinline__ f32x4 weights_of(const float* acc, int i, int to) {
  f32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = acc[min(i + e, to - 1)];
  return x;
}
__device__ __forceinline__ u32x4 ranks_of(f32x4 x, int i, int to) {
  u32x4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = i + e < to ? rank_of(x[e]) : 0;
  return u;
}

// What is known of the rank sought: its digits so far, what is wanted of the keys with
// them, and of the parts before this one the keys above them and with them.
struct Found {
  uint32_t digits, left, above, equal;
};
struct Sums {
  uint32_t all[SW], before[SW];  // of each wave's bins: over all parts, over those before this one
  Found found;
};

// The next digits: c[j] is the count of bin BINS - 1 - (PER tid + j) over all parts, b[j]
// that over the parts before this one.
__device__ __forceinline__ void find_digits(Sums& sh, const uint32_t (&c)[PER], const uint32_t (&b)[PER], int width,
                                            Found& f, int tid, int lane, int wave) {
  static_assert(PER == 2, "two bins a thread");
  const uint32_t own = c[0] + c[1], upto = scan(own), upto_b = scan(b[0] + b[1]);
  if (lane == 63) sh.all[wave] = upto, sh.before[wave] = upto_b;
  __syncthreads();
  const uint32_t higher = upto - own + sum_below(sh.all, wave);
  if (higher < f.left && higher + own >= f.left) {
    const bool second = higher + c[0] < f.left;
    sh.found = {f.digits << width | (uint32_t)(BINS - 1 - (PER * tid + (second ? 1 : 0))),
                f.left - higher - (second ? c[0] : 0),
                f.above + sum_below(sh.before, wave) + upto_b - (second ? b[1] : b[0] + b[1]), second ? b[1] : b[0]};
  }
  __syncthreads();
  f = sh.found;
}

// The next digits from the counts of a level.
template <int LEVEL>
__device__ __forceinline__ void next_level(Sums& sh, const Place& w, Found& f, int tid, int lane, int wave) {
  uint32_t c[PER] = {0, 0}, b[PER] = {0, 0};
  const int at = SEL - 1 - tid;  // this thread's two bins
  if (LEVEL < 2 || at < BINS / 4) {
#pragma unroll 8
    for (int i = 0; i < w.used; ++i) {
      const uint32_t x = LEVEL < 2 ? w.parts[i].counts[LEVEL][at] : w.parts[i].low[at];
      c[0] += x >> 16;
      c[1] += x & 0xFFFF;
      if (i < w.part) {
        b[0] += x >> 16;
        b[1] += x & 0xFFFF;
      }
    }
  }
  find_digits(sh, c, b, LEVEL < 2 ? 11 : 10, f, tid, lane, wave);
}

template <int LEVEL>
__global__ __launch_bounds__(SEL) void attn_evict_count(EvictParams p) {
  __shared__ uint32_t hist[2][BINS];
  __shared__ __attribute__((aligned(16))) Sums sums;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place w;
  if (!place(p, w) || w.from >= w.late) return;
  Part& own = w.parts[w.part];
  const float* const acc = p.acc + (size_t)w.bh * p.Sk_cap;
  f32x4 x = weights_of(acc, w.from + 4 * tid, w.to);
#pragma unroll
  for (int i = 0; i < 2 * PER; ++i) hist[0][i * SEL + tid] = 0;
  Found f = {0, w.want, 0, 0};
  if constexpr (LEVEL == 2) f = {own.digits, own.left, own.above, 0};
  __syncthreads();
  if constexpr (LEVEL > 0) {
    next_level<LEVEL - 1>(sums, w, f, tid, lane, wave);
    if (tid == 0) {
      own.digits = f.digits;
      own.left = f.left;
      own.above = f.above;
    }
  }
  constexpr int SHIFT = LEVEL == 0 ? 21 : LEVEL == 1 ? 10 : 0, WIDTH = LEVEL < 2 ? 11 : 10;
  for (int i = w.from; i < w.to; i += 4 * SEL) {
    const u32x4 u = ranks_of(x, i + 4 * tid, w.to);
    if (i + 4 * SEL < w.to) x = weights_of(acc, i + 4 * (SEL + tid), w.to);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // (rank 0, behind the last key, has no weight's digits)
      const bool in = LEVEL == 0 ? u[e] != 0 : u[e] >> (SHIFT + WIDTH) == f.digits;
      if (__ballot(in)) count(hist[lane & 1], in ? (int)((u[e] >> SHIFT) & ((1u << WIDTH) - 1)) : -1, lane);
    }
  }
  __syncthreads();
  uint32_t* const counts = LEVEL < 2 ? own.counts[LEVEL] : own.low;
  if (LEVEL < 2 || tid < BINS / 4)
    counts[tid] = (hist[0][PER * tid] + hist[1][PER * tid]) | (hist[0][PER * tid + 1] + hist[1][PER * tid + 1]) << 16;
}

__global__ __launch_bounds__(SEL) void attn_evict_place(EvictParams p) {
  __shared__ __attribute__((aligned(16))) Sums sums;
  __shared__ __attribute__((aligned(16))) uint32_t waves[2][SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place w;
  const bool seek = place(p, w);
  int32_t* const index = p.index + (size_t)w.bh * p.keep;
  if (w.bh % p.Hkv == 0 && w.part == 0 && tid == 0) p.lens_out[w.bh / p.Hkv] = min(w.n, p.keep);
  // what needs no search is shared out over the head's workgroups
  const int first = w.part * SEL + tid, step = p.parts * SEL;
  if (w.n <= p.keep) {
    for (long long i = first; i < p.keep; i += step) index[i] = i < w.n ? (int)i : -1;
    return;
  }
  for (long long i = w.late + (long long)first; i < w.n; i += step) index[w.want + (uint32_t)(i - w.late)] = (int)i;
  if (!seek || w.from >= w.late) return;
  const float* const acc = p.acc + (size_t)w.bh * p.Sk_cap;
  const Part& own = w.parts[w.part];
  f32x4 x = weights_of(acc, w.from + 4 * tid, w.to);
  Found f = {own.digits, own.left, own.above, 0};
  next_level<2>(sums, w, f, tid, lane, wave);
  // now: all keys above f.digits stay, and the first f.left of those equal to it.
  // Above and equal ones before a key: of the equal ones the first `left` stay.
  uint32_t ab = f.above, eq = f.equal;
  int turn = 0;
  for (int i = w.from; i < w.to; i += 4 * SEL, turn ^= 1) {
    const u32x4 u = ranks_of(x, i + 4 * tid, w.to);
    if (i + 4 * SEL < w.to) x = weights_of(acc, i + 4 * (SEL + tid), w.to);
    uint32_t mine = 0;  // equal ones, above ones: at most 4096 each
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += u[e] > f.digits ? 1 : u[e] == f.digits ? 1u << 16 : 0;
    const uint32_t upto = scan(mine);
    // (two of them in turn: a wave that runs ahead writes the other)
    if (lane == 63) waves[turn][wave] = upto;
    __syncthreads();
    const uint32_t before = upto - mine + sum_below(waves[turn], wave), all = sum_below(waves[turn], SW);
    uint32_t e0 = eq + (before >> 16), to = ab + (before & 0xFFFF) + min(e0, f.left);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool same = u[e] == f.digits;
      if (u[e] > f.digits || (same && e0 < f.left)) index[to++] = i + 4 * tid + e;
      e0 += same ? 1 : 0;
    }
    ab += all & 0xFFFF;
    eq += all >> 16;
  }
}

// GATHER: the workgroup copies the rows itself.
template <bool GATHER, int HELD>
__global__ __launch_bounds__(SEL) void attn_evict_select(EvictParams p) {
  const int bh = blockIdx.x, b = bh / p.Hkv, tid = threadIdx.x;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  int32_t* const index = p.index + (size_t)bh * p.keep;
  if (bh % p.Hkv == 0 && tid == 0) p.lens_out[b] = min(n, p.keep);
  select_keys<HELD>(p, bh, n, index);
  if constexpr (GATHER) {
    __syncthreads();
    constexpr int U = 4;
    const int chunks = p.row_bytes / 16, shift = __builtin_ctz(chunks);
    const int items = min(n, p.keep) * chunks;
    const size_t from = (size_t)bh * p.Sk_cap, to = (size_t)bh * p.out_cap;
    const uint8_t* const k = p.k + from * p.row_bytes;
    const uint8_t* const v = p.v + from * p.row_bytes;
    for (int i0 = tid; i0 < items; i0 += U * SEL) {
      int src[U];
      u32x4 x[U], y[U];
#pragma unroll
      for (int j = 0; j < U; ++j) src[j] = index[min(i0 + j * SEL, items - 1) >> shift];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int c = (i0 + j * SEL) & (chunks - 1);
        x[j] = *(const u32x4*)(k + (size_t)src[j] * p.row_bytes + 16 * c);
        y[j] = *(const u32x4*)(v + (size_t)src[j] * p.row_bytes + 16 * c);
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int i = i0 + j * SEL;
        if (i >= items) break;
        *(u32x4*)(p.k_out + to * p.row_bytes + 16 * (size_t)i) = x[j];
        *(u32x4*)(p.v_out + to * p.row_bytes + 16 * (size_t)i) = y[j];
        if ((i & (chunks - 1)) == 0) p.acc_out[to + (i >> shift)] = p.acc[from + src[j]];
      }
    }
  }
}

// Rows of K, V and acc at the indexes.  A thread: 16 bytes of a row of K and of V.
__global__ __launch_bounds__(256) void attn_evict_gather(EvictParams p) {
  const int chunks = p.row_bytes / 16;
  const long long x = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = x / chunks;  // over [B Hkv][keep]
  if (row >= (long long)p.B * p.Hkv * p.keep) return;
  const int src = p.index[row];
  if (src < 0) return;
  const int c = (int)(x - row * chunks);
  const long long bh = row / p.keep, to = bh * p.out_cap + (row - bh * p.keep), from = bh * p.Sk_cap + src;
  const uint4 k = *(const uint4*)(p.k + (size_t)from * p.row_bytes + 16 * c);
  const uint4 v = *(const uint4*)(p.v + (size_t)from * p.row_bytes + 16 * c);
  *(uint4*)(p.k_out + (size_t)to * p.row_bytes + 16 * c) = k;
  *(uint4*)(p.v_out + (size_t)to * p.row_bytes + 16 * c) = v;
  if (c == 0) p.acc_out[to] = p.acc[from];
}
}  // namespace

namespace h15 {

int launch_evict(const EvictParams& p, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const dim3 heads((unsigned)(p.B * p.Hkv)), block(SEL);
  // (two workgroups a compute unit where their weights fit)
  if (p.parts > 1) {
    const dim3 all((unsigned)(p.B * p.Hkv * p.parts));
    hipLaunchKernelGGL(attn_evict_count<0>, all, block, 0, st, p);
    hipLaunchKernelGGL(attn_evict_count<1>, all, block, 0, st, p);
    hipLaunchKernelGGL(attn_evict_count<2>, all, block, 0, st, p);
    hipLaunchKernelGGL(attn_evict_place, all, block, 0, st, p);
  } else if (p.Sk <= HELD_FEW) {
    if (p.gather) hipLaunchKernelGGL((attn_evict_select<true, HELD_FEW>), heads, block, 0, st, p);
    else hipLaunchKernelGGL((attn_evict_select<false, HELD_FEW>), heads, block, 0, st, p);
  } else {
    if (p.gather) hipLaunchKernelGGL((attn_evict_select<true, HELD_MANY>), heads, block, 0, st, p);
    else hipLaunchKernelGGL((attn_evict_select<false, HELD_MANY>), heads, block, 0, st, p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && !p.gather) {
    const long long threads = (long long)p.B * p.Hkv * p.keep * (p.row_bytes / 16);
    hipLaunchKernelGGL(attn_evict_gather, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
