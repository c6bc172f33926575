// Which keys of a cache stay (attn_evict): of the n keys of each (batch, KV
// head) the last `recent` and, of the others, those with the largest
// accumulated weight, `keep` in all (equal weights: the lowest index first),
// in their order.  One workgroup a (batch, KV head) finds them and writes their
// indexes; then their rows of K, V and acc are gathered into the compact caches,
// 16 bytes a thread, by that workgroup if they are few, else by a launch of their
// own.  Where few heads have long caches, parts of the keys have a workgroup each,
// in three launches.  (The rules: cache_api.cpp.)
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
// parts 5 + 5 + 7 us, and 4 for the gather.
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

// The same by EVICT_PART keys a workgroup, in three launches: the first digits of
// every part's weights are counted; every workgroup adds up its head's counts and
// writes down its part's candidates, the keys with the digits found; every
// workgroup finds the remaining digits from its head's candidates, and places its
// own part's keys, those of the parts before it being counted from their
// candidates.  What the launches hand on, for each part:
struct Part {
  uint32_t counts[BINS / 2];     // of two bins, the even one's low
  uint32_t above, candidates;    // keys with higher first digits, and with these
  uint32_t rest[EVICT_PART];     // the candidates' remaining digits, in order of the keys
  uint32_t digits, left;         // the first digits, what is wanted of the head's candidates
};
static_assert(sizeof(Part) == EVICT_PART_BYTES, "the workspace is sized by it");

struct Place {  // of a workgroup
  int bh, part, n, late;
  uint32_t want;
  Part* parts;  // of its head
};

// False where nothing is to be sought: all keys stay, or only the late ones.
__device__ __forceinline__ bool place(const EvictParams& p, Place& w) {
  w.bh = blockIdx.x / p.parts;
  w.part = blockIdx.x - w.bh * p.parts;
  w.n = p.lens ? min(max(p.lens[w.bh / p.Hkv], 0), p.Sk) : p.Sk;
  w.late = w.n - min(p.recent, p.keep);
  w.want = (uint32_t)(p.keep - (w.n - w.late));
  w.parts = (Part*)p.scratch + (size_t)w.bh * p.parts;
  return w.n > p.keep && w.want > 0;
}

// The ranks of four keys from i on, 0 from `late` on
__device__ __forceinline__ u32x4 ranks_of(const float* acc, int i, int late) {
  float x[4];
  u32x4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = acc[min(i + e, late - 1)];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = i + e < late ? rank_of(x[e]) : 0;
  return u;
}

__global__ __launch_bounds__(SEL) void attn_evict_count(EvictParams p) {
  __shared__ uint32_t hist[2][BINS];
  const int tid = threadIdx.x, lane = tid & 63;
  Place w;
  if (!place(p, w) || w.part * EVICT_PART >= w.late) return;
  const u32x4 u = ranks_of(p.acc + (size_t)w.bh * p.Sk_cap, w.part * EVICT_PART + 4 * tid, w.late);
#pragma unroll
  for (int i = 0; i < 2 * PER; ++i) hist[0][i * SEL + tid] = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 4; ++e) count(hist[lane & 1], u[e] != 0 ? (int)(u[e] >> 21) : -1, lane);
  __syncthreads();
  w.parts[w.part].counts[tid] =
      (hist[0][2 * tid] + hist[1][2 * tid]) | (hist[0][2 * tid + 1] + hist[1][2 * tid + 1]) << 16;
}

__global__ __launch_bounds__(SEL) void attn_evict_narrow(EvictParams p) {
  __shared__ __attribute__((aligned(16))) Search search;
  __shared__ __attribute__((aligned(16))) uint32_t waves[SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place w;
  if (!place(p, w) || w.part * EVICT_PART >= w.late) return;
  const u32x4 u = ranks_of(p.acc + (size_t)w.bh * p.Sk_cap, w.part * EVICT_PART + 4 * tid, w.late);
  // the head's counts
  const int used = (w.late + EVICT_PART - 1) / EVICT_PART;
  uint32_t c[PER] = {0, 0};
#pragma unroll 8
  for (int i = 0; i < used; ++i) {
    const uint32_t x = w.parts[i].counts[SEL - 1 - tid];
    c[0] += x >> 16;
    c[1] += x & 0xFFFF;
  }
  uint32_t digits = 0, left = w.want;
  next_digits(search, c, 11, digits, left, tid, lane, wave);
  uint32_t own = 0;  // candidates, above ones: EVICT_PART each at most
#pragma unroll
  for (int e = 0; e < 4; ++e) own += (u[e] >> 21) > digits ? 1 : (u[e] >> 21) == digits ? 1u << 16 : 0;
  const uint32_t upto = scan(own);
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  const uint32_t before = upto - own + sum_below(waves, wave);
  Part& part = w.parts[w.part];
  uint32_t at = before >> 16;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if ((u[e] >> 21) == digits) part.rest[at++] = u[e] & ((1u << 21) - 1);
  if (tid == SEL - 1) {
    part.above = (before + own) & 0xFFFF;
    part.candidates = (before + own) >> 16;
    part.digits = digits;
    part.left = left;
  }
}

__global__ __launch_bounds__(SEL) void attn_evict_place(EvictParams p) {
  __shared__ uint32_t hist[2][BINS];
  __shared__ __attribute__((aligned(16))) Search search;
  __shared__ __attribute__((aligned(16))) uint32_t above[SW], equal[SW], waves[SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Place w;
  const bool seek = place(p, w);
  int32_t* const index = p.index + (size_t)w.bh * p.keep;
  if (w.bh % p.Hkv == 0 && w.part == 0 && tid == 0) p.lens_out[w.bh / p.Hkv] = min(w.n, p.keep);
  const int first = w.part * SEL + tid, step = p.parts * SEL;
  if (w.n <= p.keep) {
    for (int i = first; i < p.keep; i += step) index[i] = i < w.n ? i : -1;
    return;
  }
  for (int i = w.late + first; i < w.n; i += step) index[w.want + (uint32_t)(i - w.late)] = i;
  if (!seek || w.part * EVICT_PART >= w.late) return;
  const int k0 = w.part * EVICT_PART + 4 * tid;
  const u32x4 u = ranks_of(p.acc + (size_t)w.bh * p.Sk_cap, k0, w.late);
#pragma unroll
  for (int i = 0; i < 2 * PER; ++i) hist[0][i * SEL + tid] = 0;
  __syncthreads();
  const uint32_t top = w.parts[w.part].digits;
  uint32_t digits = 0, left = w.parts[w.part].left;
  // (a wave: the candidates of every SW-th part)
  const int used = (w.late + EVICT_PART - 1) / EVICT_PART;
#pragma unroll 1
  for (int round = 1; round < 3; ++round) {
    const int shift = round == 1 ? 10 : 0, width = round == 1 ? 11 : 10;
    for (int i = wave; i < used; i += SW) {
      const Part& part = w.parts[i];
      const int m = (int)part.candidates;
      for (int j = lane; j - lane < m; j += 64) {
        const uint32_t r = j < m ? part.rest[j] : ~0u;  // (no digits are that high)
        const bool in = j < m && (round == 1 || r >> width == digits);
        if (__ballot(in)) count(hist[lane & 1], in ? (int)((r >> shift) & ((1u << width) - 1)) : -1, lane);
      }
    }
    __syncthreads();
    uint32_t c[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int bin = BINS - 1 - (PER * tid + j);
      c[j] = hist[0][bin] + hist[1][bin];
      hist[0][bin] = hist[1][bin] = 0;
    }
    next_digits(search, c, width, digits, left, tid, lane, wave);
  }
  // above and equal ones in the parts before this one
  uint32_t na = 0, ne = 0;
  for (int i = wave; i < w.part; i += SW) {
    const Part& part = w.parts[i];
    const int m = (int)part.candidates;
    if (lane == 0) na += part.above;
    for (int j = lane; j < m; j += 64) {
      const uint32_t r = part.rest[j];
      na += r > digits ? 1 : 0;
      ne += r == digits ? 1 : 0;
    }
  }
  na = scan(na);
  ne = scan(ne);
  digits |= top << 21;
  uint32_t own = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) own += u[e] > digits ? 1 : u[e] == digits ? 1u << 16 : 0;
  const uint32_t upto = scan(own);
  if (lane == 63) above[wave] = na, equal[wave] = ne, waves[wave] = upto;
  __syncthreads();
  const uint32_t before = upto - own + sum_below(waves, wave);
  uint32_t e0 = sum_below(equal, SW) + (before >> 16);
  uint32_t to = sum_below(above, SW) + (before & 0xFFFF) + min(e0, left);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool same = u[e] == digits;
    if (u[e] > digits || (same && e0 < left)) index[to++] = k0 + e;
    e0 += same ? 1 : 0;
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
    hipLaunchKernelGGL(attn_evict_count, all, block, 0, st, p);
    hipLaunchKernelGGL(attn_evict_narrow, all, block, 0, st, p);
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
