// Writing new rows of K and V into a cache of 8-bit codes with a scale of two for
// each block of tokens and head (attn_cache_append).
//
// A workgroup for each block that n rows can lie in, each head, and K or V, of one, two or
// four waves, so that a thread has two to eight chunks of 16 bytes: it reads the new rows
// once, into registers, finds their largest finite value, takes the larger of the
// scale that this needs and the one that the block has (if it held rows before), and
// writes the codes.  Only where the scale grows are the rows that were there read,
// shrunk by a power of two and written back.  Division by a scale of two is exact,
// so a code is rounded once.
//
// What bounds it: HBM for many rows (4 sequences of 8 heads, 4096 rows each, d = 128: 101 MB in
// 19.3 to 20 us for every block; blocks of 16 with four waves 24.4), and for few the launch and a
// chain of loads, each of which needs the one before: the arguments, a count and a length, K's
// or V's pointers, the scale of a block that held rows, the rows (one row of each of 16
// sequences of 8 heads 4.3 us).  Up to 4096 ragged rows, 40 MB: blocks of 16, 32 and 64 in 10.9,
// 11.0 and 11.0 us; with workgroups of four waves for several blocks, whose indexes differ from
// wave to wave and whose waves stay where a block gets no row, in 14.3, 14.3 and 11.6.
//
// The largest value is found on the bits of the BF16 values: without the sign
// they order as the values do, and the scale's exponent byte follows from them
// in integers, 448 being 1.75 * 2^8.
#include "qkv_params.h"
#include "attn_device.h"

namespace {

// Waves that share a block of T rows of D channels.
constexpr int block_waves(int D, int T) { return T * D <= 2048 ? 1 : T * D <= 4096 ? 2 : 4; }

__device__ __forceinline__ float held(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f); }

// The larger of the finite magnitudes in both halves of each word (0 for others)
__device__ __forceinline__ uint32_t finite_max(uint32_t top, uint32_t x) {
  const uint32_t lo = x & 0x7FFFu, hi = (x >> 16) & 0x7FFFu;
  const uint32_t a = lo < 0x7F80u ? lo : 0u, b = hi < 0x7F80u ? hi : 0u;
  return max(top, max(a, b));
}

template <int D, int T>
__global__ __launch_bounds__(64 * block_waves(D, T)) void attn_append_kernel(AppendParams p, bool write_lens) {
  constexpr int CH = D / 8;               // chunks of 8 channels in a row
  constexpr int W = block_waves(D, T), N = 64 * W, EACH = T * CH / N;  // waves, threads, a thread's chunks
  static_assert(T * CH % N == 0, "whole chunks");
  __shared__ uint32_t tops[W];
  const int tid = threadIdx.x;
  const int unit = blockIdx.x / p.reach, j = blockIdx.x - unit * p.reach;  // unit: (b, h, K or V)
  const int which = unit & 1, bh = unit >> 1, b = bh / p.Hkv;
  const int held_rows = min(max(p.lens[b], 0), p.cap);
  const int fresh = min(p.counts ? min(max(p.counts[b], 0), p.n) : p.n, p.cap - held_rows);
  const int end = held_rows + fresh;
  if (write_lens && j == 0 && unit - b * 2 * p.Hkv == 0 && tid == 0) p.lens_out[b] = end;
  const int block = held_rows / T + j;
  const long long first = (long long)block * T;
  const int lo = (int)max(first, (long long)held_rows), hi = (int)min(first + T, (long long)end);
  if (lo >= hi) return;
  const uint16_t* x = p.x[which] + ((size_t)bh * p.n + (lo - held_rows)) * D;
  uint8_t* const cache = p.cache[which] + ((size_t)bh * p.cap + (size_t)first) * D;
  uint8_t* const scale = p.scales + ((size_t)bh * p.blocks + block) * 2 + which;
  const int chunks = (hi - lo) * CH, old_rows = lo - (int)first;
  int e_old = 1;
  if (old_rows > 0) e_old = min(max((int)*scale, 1), 254);
  u32x4 v[EACH];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int c = i * N + tid;
    v[i] = c < chunks ? *(const u32x4*)(x + (size_t)c * 8) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) top = finite_max(top, v[i][w]);
#pragma unroll
  for (int y = 32; y >= 1; y >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, y, 64));
  if constexpr (W > 1) {
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) top = max(top, tops[i]);
  }
  // the exponent of top / 448, one up where top's fraction lies above 448's
  const int need = (int)((top + (0x7Fu - 0x60u)) >> 7) - 8;
  const int e = max(need, e_old);
  if (tid == 0) *scale = (uint8_t)e;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int c = i * N + tid;
    if (c >= chunks) break;
    u32x2 r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float f[4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f[2 * m] = held(__builtin_ldexpf(__uint_as_float(v[i][2 * k + m] << 16), 127 - e));
        f[2 * m + 1] = held(__builtin_ldexpf(__uint_as_float(v[i][2 * k + m] & 0xFFFF0000u), 127 - e));
      }
      const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      r[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    }
    *(u32x2*)(cache + (size_t)old_rows * D + (size_t)c * 8) = r;
  }
  if (old_rows == 0 || e == e_old) return;
  // (codes are at most 448: 32 steps of two and more leave nothing of them)
  const int shrink = max(e_old - e, -32);
  for (int c = tid; c < old_rows * CH; c += N) {
    u32x2 r = *(const u32x2*)(cache + (size_t)c * 8);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[k], false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[k], true);
      const int w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(a[0], shrink), __builtin_ldexpf(a[1], shrink), 0, false);
      r[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(d[0], shrink), __builtin_ldexpf(d[1], shrink), w, true);
    }
    *(u32x2*)(cache + (size_t)c * 8) = r;
  }
}

// lens_out over lens itself, once every workgroup has read it
__global__ __launch_bounds__(256) void attn_append_lens(AppendParams p) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= p.B) return;
  const int held_rows = min(max(p.lens[b], 0), p.cap);
  p.lens_out[b] = held_rows + min(p.counts ? min(max(p.counts[b], 0), p.n) : p.n, p.cap - held_rows);
}

template <int D>
void launch_one(const AppendParams& p, int block, bool write_lens, hipStream_t st) {
  const dim3 threads(64 * block_waves(D, block));
  const dim3 grid((unsigned)((long long)p.B * p.Hkv * 2 * p.reach));
  switch (block) {
    case 16: hipLaunchKernelGGL((attn_append_kernel<D, 16>), grid, threads, 0, st, p, write_lens); break;
    case 32: hipLaunchKernelGGL((attn_append_kernel<D, 32>), grid, threads, 0, st, p, write_lens); break;
    case 64: hipLaunchKernelGGL((attn_append_kernel<D, 64>), grid, threads, 0, st, p, write_lens); break;
    default: hipLaunchKernelGGL((attn_append_kernel<D, 128>), grid, threads, 0, st, p, write_lens); break;
  }
}
}  // namespace

namespace h15 {

int launch_append(const AppendParams& p, int d, int block, bool in_place, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  d == 128 ? launch_one<128>(p, block, !in_place, st) : launch_one<64>(p, block, !in_place, st);
  if (in_place) hipLaunchKernelGGL(attn_append_lens, dim3((unsigned)((p.B + 255) / 256)), dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace h15
