// Which keys of a cache stay (attn_evict): of the n keys of each (batch, KV
// head) the last `recent` and, of the others, those with the largest
// accumulated weight, `keep` in all (equal weights: the lowest index first),
// in their order.  Two launches: one workgroup a (batch, KV head) finds them
// and writes their indexes; then their rows of K, V and acc are gathered into
// the compact caches, 16 bytes a thread.
//
// The selection is a radix search for the weight of rank keep - recent in three
// rounds over 11, 11 and 10 bits, each a histogram in LDS of the keys that agree
// with the digits found so far; then a count of the keys that stay, stretch by
// stretch, and a second pass that writes their indexes in order.  The weights
// are read once, as ordered numbers into LDS (of a cache of more than 32K keys
// every pass reads the rest again).  (In registers, 32 a thread, the passes had
// to be unrolled, and a workgroup spent its time fetching code that it runs once:
// 41 us for 32K keys; re-read from memory in every pass 53 us.)  What bounds the
// call is the gather (read and written once) and, with few caches, the passes'
// latency.
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

// The indexes of the keys of one (batch, KV head) that stay.  HELD: weights in LDS.
template <int HELD>
__device__ __forceinline__ void select_keys(const EvictParams& p, int bh, int n, int32_t* index) {
  __shared__ __attribute__((aligned(16))) uint32_t ranks[HELD];
  __shared__ uint32_t hist[2][BINS];  // odd and even lanes' counts
  __shared__ uint32_t found[2];  // digits so far, keys still wanted among those that agree
  __shared__ __attribute__((aligned(16))) uint32_t above[SW], equal[SW], waves[SW];
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

  constexpr int PER = BINS / SEL;
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
          } else if (__ballot(in[e])) count(hist[lane & 1], in[e] ? (int)((u[e] >> shift) & ((1u << width) - 1)) : -1, lane);
      }
      __syncthreads();
    }
    // a thread: two bins, from the top; the bin in which the count passes `left`
    uint32_t c[PER], own = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int bin = BINS - 1 - (PER * tid + j);
      c[j] = hist[0][bin] + hist[1][bin];
      hist[0][bin] = hist[1][bin] = 0;  // for the next round
      own += c[j];
    }
    const uint32_t upto = scan(own);
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    const uint32_t before = upto - own + sum_below(waves, wave);
    if (before < left && before + own >= left) {
      const bool second = before + c[0] < left;
      found[0] = (digits << width) | (uint32_t)(BINS - 1 - (PER * tid + (second ? 1 : 0)));
      found[1] = left - before - (second ? c[0] : 0);
    }
    __syncthreads();
    digits = found[0];
    left = found[1];
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
  if (p.Sk <= HELD_FEW) {
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
