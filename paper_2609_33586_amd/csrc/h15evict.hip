// Which keys of a cache stay (attn_evict): of the n keys of each (batch, KV
// head) the last `recent` and, of the others, those with the largest
// accumulated weight, `keep` in all (equal weights: the lowest index first),
// in their order.  Two launches: one workgroup a (batch, KV head) finds them
// and writes their indexes; then their rows of K, V and acc are gathered into
// the compact caches, 16 bytes a thread.
//
// The selection is a radix search for the weight of rank keep - recent: four
// rounds over 8 bits, each a histogram in LDS of the keys that agree with the
// digits found so far.  A first pass over the keys in order then counts, and a
// second writes.  What bounds the call is the gather (read and written once)
// and, with few caches, the rounds' latency.
#include "cache_params.h"

#include <hip/hip_runtime.h>
#include <math.h>

namespace {

using namespace h15;

constexpr int SEL = 1024;  // threads of a selection
constexpr int SW = SEL / 64;
constexpr int BINS = 256;

// Weights as unsigned numbers in their order: +0 and -0 alike, NaN above all.
__device__ __forceinline__ uint32_t rank_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(SEL) void attn_evict_select(EvictParams p) {
  __shared__ uint32_t hist[BINS];
  __shared__ uint32_t found[2];  // digits so far, keys still wanted among those that agree
  __shared__ uint32_t above[SW], equal[SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x, b = bh / p.Hkv;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  int32_t* const index = p.index + (size_t)bh * p.keep;
  const float* const acc = p.acc + (size_t)bh * p.Sk_cap;
  if (bh % p.Hkv == 0 && tid == 0) p.lens_out[b] = min(n, p.keep);
  if (n <= p.keep) {
    for (int i = tid; i < p.keep; i += SEL) index[i] = i < n ? i : -1;
    return;
  }
  const int late = n - min(p.recent, p.keep);  // the keys from here on stay
  const uint32_t want = (uint32_t)(p.keep - (n - late));
  uint32_t digits = 0, left = want;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < BINS) hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < late; i += SEL) {
        const uint32_t u = rank_of(acc[i]);
        if (shift == 24 || (u >> (shift + 8)) == digits) atomicAdd(&hist[(u >> shift) & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {
        // lane: four bins, from the top; the bin in which the count passes `left`
        uint32_t c[4], own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) own += c[j] = hist[255 - (4 * lane + j)];
        uint32_t upto = own;
        for (int x = 1; x < 64; x <<= 1) {
          const uint32_t y = __shfl_up(upto, x, 64);
          if (lane >= x) upto += y;
        }
        uint32_t before = upto - own;
        if (before < left && upto >= left) {
          int j = 0;
          while (before + c[j] < left) before += c[j++];
          found[0] = (digits << 8) | (uint32_t)(255 - (4 * lane + j));
          found[1] = left - before;
        }
      }
      __syncthreads();
      digits = found[0];
      left = found[1];
    }
  }
  // now: all keys above `digits` stay, and the first `left` of those equal to it.
  // Each wave has a stretch of the keys before `late`, in order.
  const int stretch = (late + SEL - 1) / SEL * 64;
  const int i0 = min(wave * stretch, late), i1 = min(i0 + stretch, late);
  uint32_t na = 0, ne = 0;
  for (int i = i0; i < i1; i += 64) {
    const bool in = i + lane < i1;
    const uint32_t u = in && want > 0 ? rank_of(acc[i + lane]) : 0;
    na += __popcll(__ballot(in && want > 0 && u > digits));
    ne += __popcll(__ballot(in && want > 0 && u == digits));
  }
  if (lane == 0) above[wave] = na, equal[wave] = ne;
  __syncthreads();
  uint32_t at = 0, eq = 0;  // kept, and equal, in the stretches before
  for (int w = 0; w < wave; ++w) at += above[w], eq += equal[w];
  at += min(eq, left);
  const unsigned long long below = (1ull << lane) - 1;
  for (int i = i0; i < i1; i += 64) {
    const bool in = i + lane < i1;
    const uint32_t u = in && want > 0 ? rank_of(acc[i + lane]) : 0;
    const unsigned long long es = __ballot(in && want > 0 && u == digits);
    const bool stays = in && want > 0 && (u > digits || (u == digits && eq + (uint32_t)__popcll(es & below) < left));
    const unsigned long long ss = __ballot(stays);
    if (stays) index[at + (uint32_t)__popcll(ss & below)] = i + lane;
    at += (uint32_t)__popcll(ss);
    eq += (uint32_t)__popcll(es);
  }
  for (int i = late + tid; i < n; i += SEL) index[want + (uint32_t)(i - late)] = i;
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
  hipLaunchKernelGGL(attn_evict_select, dim3((unsigned)(p.B * p.Hkv)), dim3(SEL), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    const long long threads = (long long)p.B * p.Hkv * p.keep * (p.row_bytes / 16);
    hipLaunchKernelGGL(attn_evict_gather, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
