// Device code of attention in parts over a key/value cache, shared by
// h15prefix.hip and h15blocks.hip: copies into LDS, a unit's weights, V's
// addresses in LDS, the order of workgroups, and the merge of a row's parts.
// Everything has internal linkage; each file includes it once.
#ifndef H15ATTN_PART_DEVICE_H
#define H15ATTN_PART_DEVICE_H

#include "unit_device.h"

namespace {

// One 1 KB copy into LDS: 64 chunks of 16 bytes, chunk i of the destination
// holding row i / NCH, chunk (i % NCH) ^ swizzle(row).
template <int NCH>
__device__ __forceinline__ int copy_row(int i, int lane) {
  return (i * 64 + lane) / NCH;
}

// The weights of NB blocks of 32 keys (in place for the exponential, else
// packed in w), their sum added to l; masked keys get weight 0.
template <int MODE, int NB>
__device__ __forceinline__ void weigh(f32x16 (&sv)[NB], uint32_t (&w)[NB][8], float m_use, float c1, float ck,
                                      bool need_mask, int lim, float& l) {
  if constexpr (mode_lattice(MODE)) {
    const float nbk = -m_use * ck;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int j = 0; j < 16; ++j) sv[kb][j] = __uint_as_float(sq_pre<MODE>(sv[kb][j], ck, nbk));
    if (need_mask) mask_unit(sv, lim, __uint_as_float(sq_masked<MODE>()));
    float a[4] = {l, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        w[kb][q] = sq_pack<MODE>(__float_as_uint(sv[kb][2 * q]), __float_as_uint(sv[kb][2 * q + 1]));
        a[q & 3] = dot2_ones(w[kb][q], a[q & 3]);
      }
    l = (a[0] + a[1]) + (a[2] + a[3]);
  } else {
    const float nb1 = -m_use * c1;
    float a[4] = {l, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        sv[kb][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[kb][j], c1, nb1));
        a[j & 3] += sv[kb][j];
      }
    l = (a[0] + a[1]) + (a[2] + a[3]);
  }
}

// P of 16 keys (half hf of a block) as the BF16 operand
template <int MODE>
__device__ __forceinline__ bf16x8 p_operand(const f32x16& s, const uint32_t (&w)[8], int hf) {
  if constexpr (mode_lattice(MODE)) {
    return __builtin_bit_cast(bf16x8, u32x4{w[4 * hf], w[4 * hf + 1], w[4 * hf + 2], w[4 * hf + 3]});
  } else {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)s[8 * hf + i];
    return r;
  }
}

// Lane's address in V's LDS area for the transposing reads of column block db
template <int DT, int D>
__device__ __forceinline__ uint32_t v_address(uint32_t base, int db, int lane) {
  using C = Cfg<DT, D>;
  const int G4 = lane >> 4, L16 = lane & 15;
  int row, cb;
  if constexpr (DT == DT_BF16) {
    row = 4 * (G4 >> 1) + (L16 >> 2);
    cb = 64 * db + (16 * (G4 & 1) + 4 * (L16 & 3)) * 2;
  } else {
    row = 4 * (G4 >> 1) + 8 * (L16 >> 3) + ((L16 >> 1) & 3);
    cb = 32 * db + 16 * (G4 & 1) + 8 * (L16 & 1);
  }
  return base + row * C::RB + (((cb >> 4) ^ v_swz<DT, D>(row)) << 4) + (cb & 15);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, BUF_DWORD3);
}

__device__ __forceinline__ void store_row4(uint16_t* to, f32x4 a, float inv) {
  uint32_t w[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    w[e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)(a[2 * e] * inv)) |
           ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)(a[2 * e + 1] * inv)) << 16);
  *(u32x2*)to = u32x2{w[0], w[1]};
}

// A row that has seen no key (l = 0) has O = 0 and LSE = -inf.
__device__ __forceinline__ float inverse(float l, float vd) { return l == 0.0f ? 0.0f : vd / l; }
__device__ __forceinline__ float row_lse(float m, float l, float c1) {
  return l == 0.0f ? -INFINITY : 0.69314718055994531f * (m * c1 + log2f(l));
}

// Row block and unit (KV head, batch, part) of workgroup L of `units` x
// `blocks`: the row blocks that read the same keys run on one XCD (workgroup
// ids go round-robin over the 8 XCDs), so that its L2 serves all but the first.
__device__ __forceinline__ void place(int L, int units, int blocks, int& unit, int& rb) {
  const int n8 = units / 8 * 8 * blocks;
  if (L < n8) {
    rb = (L >> 3) % blocks;
    unit = (L >> 3) / blocks * 8 + (L & 7);
  } else {
    rb = (L - n8) % blocks;
    unit = n8 / blocks + (L - n8) / blocks;
  }
}

// The sequence of rank `at` by the length of its cache, the longest first (B <= 256
// lengths, 256 threads or more, an int of lens for each).
__device__ __forceinline__ int longest(const int32_t* of, int B, int Sk, int at, int* lens) {
  const int tid = threadIdx.x;
  const int n = tid < B ? min(max(of[tid], 0), Sk) : -1;
  lens[tid] = n;
  __syncthreads();
  int rank = 0;
  for (int j = 0; j < B; j += 4) {
    const i32x4 x = *(const i32x4*)&lens[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) rank += x[e] > n || (x[e] == n && j + e < tid) ? 1 : 0;
  }
  __syncthreads();
  if (tid < B && rank == at) lens[0] = tid;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(lens[0]);
  __syncthreads();
  return b;
}

// O and LSE of a row from its parts: m = max m_p, f_p = 2^(c1 (m_p - m)),
// l = sum f_p l_p, O = sum f_p O_p / l * v_descale, LSE = ln2 (m c1 + log2 l),
// over the parts with l_p != 0 (the O of others was never written).  One wave
// a row; a lane holds four columns and every (64 / (D / 4))th part.  32 parts'
// (m, l), one a lane, and then their rows are asked for at once: read one after
// the other, 17 parts of 1024 rows took 8 us.
template <int D, typename P>
__device__ __forceinline__ void merge_parts(const P& p, float vd) {
  constexpr int LPP = D / 4, PG = 64 / LPP, MOST = 32, EACH = MOST / PG;
  const int lane = threadIdx.x & 63, pg = lane / LPP, col = 4 * (lane % LPP);
  const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= (long long)p.B * p.Hq * p.Sq) return;
  const float* const ml = p.part_ml + (size_t)row * p.parts * 2;
  const float* const po = p.part_o + (size_t)row * p.parts * D;
  float m = -INFINITY, l = 0.0f;  // of the parts so far
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < p.parts; s0 += MOST) {
    const int here = min(p.parts - s0, MOST);
    const f32x2 x = *(const f32x2*)(ml + 2 * (s0 + min(lane, here - 1)));
    const bool some = lane < here && x[1] != 0.0f;
    // (rows beyond the last part read as zero and touch no memory)
    const __amdgpu_buffer_rsrc_t rsrc = rows_rsrc((const uint8_t*)(po + (size_t)s0 * D), here * D * 4);
    f32x4 v[EACH];
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      if (u > 0 && u * PG >= here) break;
      v[u] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, ((u * PG + pg) * D + col) * 4, 0, 0));
    }
    float top = some ? x[0] : -INFINITY;
#pragma unroll
    for (int y = 32; y >= 1; y >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, y, 64));
    const float m_new = __builtin_fmaxf(m, top);
    if (m_new == -INFINITY && !__ballot(some)) continue;  // nothing yet
    const float base = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - base) * p.c1);
    const float f = some ? __builtin_amdgcn_exp2f((x[0] - base) * p.c1) : 0.0f;
    float sum = some ? f * x[1] : 0.0f;
#pragma unroll
    for (int y = 32; y >= 1; y >>= 1) sum += __shfl_xor(sum, y, 64);
    l = l * alpha + sum;
    m = m_new;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      if (u > 0 && u * PG >= here) break;
      const float fs = __shfl(f, u * PG + pg, 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += fs != 0.0f ? fs * v[u][e] : 0.0f;
    }
  }
#pragma unroll
  for (int x = LPP; x < 64; x <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x, 64);
  if (pg == 0) {
    store_row4(p.o + (size_t)row * D + col, acc, inverse(l, vd));
    if (p.lse && col == 0) p.lse[row] = row_lse(m, l, p.c1);
  }
}

}  // namespace

#endif  // H15ATTN_PART_DEVICE_H
