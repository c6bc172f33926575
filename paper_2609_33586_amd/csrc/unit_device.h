// Device code of a wave's unit of keys (32 or 64 keys against 32 query rows),
// shared by the kernels over a key/value cache (h15decode.hip, h15prefix.hip):
// the hold between the matrix core and inline asm, masking, the maximum, and
// the transposing LDS reads of V.  Everything has internal linkage; each file
// includes it once.
#ifndef H15ATTN_UNIT_DEVICE_H
#define H15ATTN_UNIT_DEVICE_H

#include "attn_device.h"

namespace {

// The scores are next read by inline asm (v_max3_f32, the masking's compare
// and select), and the compiler inserts no wait states between a matrix-core
// write and an inline-asm read: this holds the wave for 24, more than the 20
// that gfx950 requires after a 16-pass write.
template <int NB>
__device__ __forceinline__ void settle_unit(f32x16 (&v)[NB]) {
  if constexpr (NB == 2) asm("s_nop 15\n\ts_nop 7" : "+v"(v[0]), "+v"(v[1]));
  else asm("s_nop 15\n\ts_nop 7" : "+v"(v[0]));
}

// y over the scores of a unit (32 or 64 keys) whose key offset lies beyond lim
template <int NB, int E = 0>
__device__ __forceinline__ void mask_unit(f32x16 (&v)[NB], int lim, float y) {
  if constexpr (E < 16 * NB) {
    constexpr int kb = E / 16, j = E % 16;
    v[kb][j] = select_beyond<kb * 32 + 8 * (j >> 2) + (j & 3)>(lim, v[kb][j], y);
    mask_unit<NB, E + 1>(v, lim, y);
  }
}

template <int NB>
__device__ __forceinline__ float unit_max(const f32x16 (&v)[NB]) {
  // 32 -> 11 -> 4 -> 2 -> 1, or 16 -> 6 -> 2 -> 1
  if constexpr (NB == 2) {
    float a[11], b[4];
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const int e0 = 3 * i, e1 = 3 * i + 1, e2 = 3 * i + 2;
      a[i] = max3(v[e0 >> 4][e0 & 15], v[e1 >> 4][e1 & 15], v[e2 >> 4][e2 & 15]);
    }
    a[10] = max3(v[1][14], v[1][15], v[1][15]);
    b[0] = max3(a[0], a[1], a[2]);
    b[1] = max3(a[3], a[4], a[5]);
    b[2] = max3(a[6], a[7], a[8]);
    b[3] = max3(a[9], a[10], a[10]);
    const float c = max3(b[0], b[1], b[2]);
    return max3(c, b[3], b[3]);
  } else {
    float a[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) a[i] = max3(v[0][3 * i], v[0][3 * i + 1], v[0][3 * i + 2]);
    const float b0 = max3(a[0], a[1], a[2]), b1 = max3(a[3], a[4], v[0][15]);
    return max3(b0, b1, b1);
  }
}

// The transposing LDS reads of V operands, with their wait in the same
// statement: the builtin forms make the compiler wait for every copy into LDS
// that is in flight, also those of the next round's K.
// bf16: two blocks of 32 columns (a0, a1), the eight 8-row steps of 64 keys
template <int RB>
__device__ __forceinline__ void read_v16(i32x2v (&r)[16], uint32_t a0, uint32_t a1) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:%18\n\t"
      "ds_read_b64_tr_b16 %2, %16 offset:%19\n\tds_read_b64_tr_b16 %3, %16 offset:%20\n\t"
      "ds_read_b64_tr_b16 %4, %16 offset:%21\n\tds_read_b64_tr_b16 %5, %16 offset:%22\n\t"
      "ds_read_b64_tr_b16 %6, %16 offset:%23\n\tds_read_b64_tr_b16 %7, %16 offset:%24\n\t"
      "ds_read_b64_tr_b16 %8, %17\n\tds_read_b64_tr_b16 %9, %17 offset:%18\n\t"
      "ds_read_b64_tr_b16 %10, %17 offset:%19\n\tds_read_b64_tr_b16 %11, %17 offset:%20\n\t"
      "ds_read_b64_tr_b16 %12, %17 offset:%21\n\tds_read_b64_tr_b16 %13, %17 offset:%22\n\t"
      "ds_read_b64_tr_b16 %14, %17 offset:%23\n\tds_read_b64_tr_b16 %15, %17 offset:%24\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]),
        "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(a0), "v"(a1), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB), "n"(32 * RB), "n"(40 * RB), "n"(48 * RB),
        "n"(56 * RB)
      : "memory");
}
// the four 8-row steps of 32 keys
template <int RB>
__device__ __forceinline__ void read_v16(i32x2v (&r)[8], uint32_t a0, uint32_t a1) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %2, %8 offset:%11\n\tds_read_b64_tr_b16 %3, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %9\n\tds_read_b64_tr_b16 %5, %9 offset:%10\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:%11\n\tds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(a0), "v"(a1), "n"(8 * RB), "n"(16 * RB), "n"(24 * RB)
      : "memory");
}
// fp8: two blocks of 32 columns, the four 16-row steps of 64 keys
template <int RB>
__device__ __forceinline__ void read_v8(i32x2v (&r)[8], uint32_t a0, uint32_t a1) {
  asm volatile(
      "ds_read_b64_tr_b8 %0, %8\n\tds_read_b64_tr_b8 %1, %8 offset:%10\n\t"
      "ds_read_b64_tr_b8 %2, %8 offset:%11\n\tds_read_b64_tr_b8 %3, %8 offset:%12\n\t"
      "ds_read_b64_tr_b8 %4, %9\n\tds_read_b64_tr_b8 %5, %9 offset:%10\n\t"
      "ds_read_b64_tr_b8 %6, %9 offset:%11\n\tds_read_b64_tr_b8 %7, %9 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(a0), "v"(a1), "n"(16 * RB), "n"(32 * RB), "n"(48 * RB)
      : "memory");
}

// the two 16-row steps of 32 keys
template <int RB>
__device__ __forceinline__ void read_v8(i32x2v (&r)[4], uint32_t a0, uint32_t a1) {
  asm volatile(
      "ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %4 offset:%6\n\t"
      "ds_read_b64_tr_b8 %2, %5\n\tds_read_b64_tr_b8 %3, %5 offset:%6\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(a0), "v"(a1), "n"(16 * RB)
      : "memory");
}

// Eight e4m3 values as BF16 (exact: BF16 holds every one), times a scale of two
// (2^-126 and more; products below that become 0).
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale = 1.0f) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Rows as BF16 matrix operands.  A lane holds a row's 16-byte chunks 2 t + g
// (g: the lane's half of the wave): of a BF16 row one operand of 8 channels
// each, of an FP8 row two, widened.  (A product may take the channels in any
// order, as long as both of its operands take the same.)
template <int DT, int D>
struct RowOperand {
  static constexpr int CHUNKS = Cfg<DT, D>::NCH / 2;  // a lane's
  static constexpr int PER = DT == DT_BF16 ? 1 : 2;   // operands of a chunk
  bf16x8 x[CHUNKS * PER];
  __device__ __forceinline__ void set(int t, i32x4 c) {
    if constexpr (DT == DT_BF16) {
      x[t] = __builtin_bit_cast(bf16x8, c);
    } else {
      x[2 * t] = widen(c[0], c[1]);
      x[2 * t + 1] = widen(c[2], c[3]);
    }
  }
};

// 16 bytes, chunk c of consecutive rows, into their BF16 rows in LDS, which are
// then read as operands with K's swizzle.  An
// FP8 chunk becomes two, in the operand order of RowOperand: chunk 2 t + g of a
// row holds the operands 2 t and 2 t + 1 of half g, which lie at 2 (2 t) + g and
// 2 (2 t + 1) + g.
template <int DT, int D>
__device__ __forceinline__ void store_row_chunk(uint8_t* rows, int c, i32x4 x) {
  constexpr int NCH = Cfg<DT, D>::NCH;
  const int r = c / NCH, i = c % NCH, swz = k_swz<DT_BF16, D>(r);
  uint8_t* const row = rows + r * Cfg<DT_BF16, D>::RB;
  if constexpr (DT == DT_BF16) {
    *(i32x4*)(row + ((i ^ swz) << 4)) = x;
  } else {
    const int t = i >> 1, g = i & 1;
    *(bf16x8*)(row + (((4 * t + g) ^ swz) << 4)) = widen(x[0], x[1]);
    *(bf16x8*)(row + (((4 * t + 2 + g) ^ swz) << 4)) = widen(x[2], x[3]);
  }
}

}  // namespace

#endif  // H15ATTN_UNIT_DEVICE_H
