// Attention over a cache of 8-bit codes with a scale of two for each block of
// tokens and head (attn_decode_blocks): Sq BF16 query rows per head and sequence
// against the first lens[b] slots of its cache, cut into parts that a second
// launch merges.
//
// Codes become BF16 operands by the conversion that also multiplies by a scale
// of two, so that the scales cost a read of two bytes a block and nothing in the
// inner loops.  K's rows meet them one scale a lane, V's transposed operands one
// for each 16 keys, which never straddle a block.
//
// The exact weights go to the matrix core as BF16, its operand type beside V's BF16 (their
// sum stays FP32): O is off by 1.9e-3 to 2.3e-3 of its norm, where its own rounding
// alone gives 1.7e-3, which the lattice weights, exact in BF16, have.  Two BF16 terms of a weight
// would double the products of P V.
//
// Three forms of a workgroup (their rules: qkv_api.cpp), the first two, of 4 waves,
// those of attn_decode_prefix:
//   keys  32 query rows; each wave takes its own 64 keys of a round, copies them
//         into its own LDS slots and, for the lattice weights, exchanges the maxima of
//         its units with the others (one barrier a round), as a weight is rounded
//         relative to the running maximum at its own tile, the prefix maximum of the
//         round's units; the exact weights' anchors are each wave's own (20 sequences
//         of 2.2K keys, one part 20.2 -> 16.4 us, 16 of 8K in 4 parts 36.8 -> 35.8);
//   rows  128 query rows, 32 a wave; the waves share each tile of 128 keys (exact
//         weights: anchors that stay as in the others, 528 .. 1200 rows 5 to 8% less);
//   wide  512 query rows, 64 a wave: many rows of long caches.
#include "qkv_params.h"
#include "part_device.h"

namespace {

constexpr int NW = 4;  // waves per workgroup
constexpr int AUX_NT = 2;  // non-temporal, among a buffer load's cache bits

template <int D>
struct BCfg {
  static constexpr int RB = D, NCH = D / 16;  // bytes and chunks of a row of codes
  static constexpr int UNIT = 64, NB = 2;     // keys of a wave and round (keys form), blocks of 32
  static constexpr int TPR = NW * UNIT / BC;  // tiles in a round
  static constexpr int SLOT = UNIT * RB;      // one wave's K (or V) of a round
  static constexpr int TILE = BC * RB;
  // K (and V) area of LDS: the slots of a round (a tile is half of it), or half
  // of the waves' O rows in the keys form's final reduction
  static constexpr int RED = NW * 16 * D * 4;
  static constexpr int AREA = NW * SLOT > RED ? NW * SLOT : RED;
};

// Query rows as operands in the order of the codes' 16-byte chunks.
template <int D>
__device__ __forceinline__ void load_q(RowOperand<DT_FP8, D>& q, const uint8_t* row, int g) {
#pragma unroll
  for (int t = 0; t < q.CHUNKS; ++t) {
    const uint8_t* at = row + 64 * t + 32 * g;
    q.x[2 * t] = __builtin_bit_cast(bf16x8, *(const i32x4*)at);
    q.x[2 * t + 1] = __builtin_bit_cast(bf16x8, *(const i32x4*)(at + 16));
  }
}

// acc + chunk t of the keys (16 bytes a lane), times their scale, times the rows q
template <int D>
__device__ __forceinline__ f32x16 product(i32x4 k, float scale, const RowOperand<DT_FP8, D>& q, int t, f32x16 acc) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(k[0], k[1], scale), q.x[2 * t], acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(k[2], k[3], scale), q.x[2 * t + 1], acc, 0, 0, 0);
}

// O^T += V^T P^T over 64 keys, two column blocks at once
template <int D>
__device__ __forceinline__ void add_pv(f32x16& o0, f32x16& o1, uint32_t a0, uint32_t a1, const bf16x8 (&pb)[4],
                                       const float (&scale)[4]) {
  i32x2v r[8];
  read_v8<D>(r, a0, a1);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    o0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(r[ks][0], r[ks][1], scale[ks]), pb[ks], o0, 0, 0, 0);
    o1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(r[4 + ks][0], r[4 + ks][1], scale[ks]), pb[ks], o1, 0, 0, 0);
  }
}

// An exact weight's anchor stays until a unit's weights add up to more than this (FP32
// and BF16 hold them with the same relative steps; with 2^40 no less time, but values
// beyond 2^80 could overflow): a row's maximum is looked for only then, as its first unit
// does, whose anchor of -inf gives inf or NaN.
constexpr float ANCHOR_HOLDS = 0x1p10f;

// 2^(c1 s + nb) of 32 scores, and their sum
__device__ __forceinline__ float weights(const f32x16 (&s)[2], float (&e)[32], float nb, float c1) {
  float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 4][j & 15], c1, nb));
    a[j & 3] = j < 4 ? e[j] : a[j & 3] + e[j];
  }
  return (a[0] + a[1]) + (a[2] + a[3]);
}

// The same as the operands of 64 keys, and their sum
__device__ __forceinline__ float packed_weights(const f32x16 (&s)[2], bf16x8 (&w)[4], float nb, float c1) {
  float e[32];
  const float sum = weights(s, e, nb, c1);
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) w[k][j] = (__bf16)e[8 * k + j];
  return sum;
}

// A workgroup's share: query rows of one sequence and KV head against one part
// of its keys.
struct Work {
  const uint8_t* k;  // the part's first key row, and its value row
  const uint8_t* v;
  const uint8_t* scales;  // of the head
  int used;   // bytes of them that belong to slots that are filled
  int j0;     // the part's first key
  int nk;     // its keys that some row sees
  int part, b, h;
  int row0, nrows;  // its rows of the sequence's R
  int open;   // the keys from here on (in the part) are not seen by every row
  int last0;  // last key (in the part) that position 0 sees, or nk - 1
};

// The scales of a lane's keys (low byte: K's, high: V's) at key `key` of the head;
// blocks without a filled slot read as 0.
__device__ __forceinline__ int scale_pair(const BlocksParams& p, const __amdgpu_buffer_rsrc_t rsrc, int key) {
  return __builtin_amdgcn_raw_buffer_load_b16(rsrc, (key >> p.shift) * 2, 0, 0);
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)min(max(byte, 1), 254) << 23); }

// V's scale of 16 keys from the lane that holds their first
__device__ __forceinline__ float v_scale(int pair, int lane) {
  return scale_of((__builtin_amdgcn_readlane(pair, lane) >> 8) & 255);
}

__device__ __forceinline__ size_t out_row(const BlocksParams& p, const Work& w, int r) {
  return ((size_t)w.b * p.Hq + (size_t)w.h * p.G) * (size_t)p.Sq + w.row0 + r;
}

// Last key of the part that row r of the workgroup sees
__device__ __forceinline__ int row_limit(const BlocksParams& p, const Work& w, int r) {
  return p.causal ? min(w.last0 + (w.row0 + r) % p.Sq, w.nk - 1) : w.nk - 1;
}

// STREAM: the keys are read once and fill more than the caches hold (p.stream).
template <int D, int MODE, bool STREAM>
__device__ __forceinline__ void keys_form(const BlocksParams& p, const Work& w, uint8_t* ksm, uint8_t* vsm,
                                          float (*mx_lds)[32][NW], float (*m_lds)[NW], float (*l_lds)[NW]) {
  using C = BCfg<D>;
  constexpr int NB = C::NB, UNIT = C::UNIT, TPR = C::TPR, SLOT = C::SLOT, RB = C::RB;
  constexpr int NDB = D / 32, LOADS = SLOT / 1024, RHALF = 16;
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rowc = min(i32, w.nrows - 1);
  RowOperand<DT_FP8, D> q;
  load_q<D>(q, p.q + out_row(p, w, rowc) * (2 * D), g);
  const int limit = row_limit(p, w, rowc);
  // rows beyond the part read as zero without touching memory; scalar offsets
  // stop at the resource's size, where every lane is out of range
  const uint32_t part_bytes = (uint32_t)w.nk * RB;
  const auto krsrc = rows_rsrc(w.k, part_bytes), vrsrc = rows_rsrc(w.v, part_bytes);
  const auto srsrc = rows_rsrc(w.scales, w.used);
  uint8_t* const kslot = ksm + wave * SLOT;
  uint8_t* const vslot = vsm + wave * SLOT;
  // the chunk swizzles repeat after every fourth copy at the latest
  uint32_t koff[4], voff[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = copy_row<C::NCH>(i, lane);
    koff[i] = (r - i * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ k_swz<DT_FP8, D>(r)) << 4);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = copy_row<C::NCH>(i, lane);
    voff[i] = (r - i * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ v_swz<DT_FP8, D>(r)) << 4);
  }
  auto first_key = [&](int c) { return c * (TPR * BC) + wave * UNIT; };
  auto stage = [&](const __amdgpu_buffer_rsrc_t rsrc, uint8_t* slot, const uint32_t* off, int mask,
                   int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t soff = min((uint32_t)first_key(c) * RB + i * 1024, part_bytes);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, LDS_PTR(void, slot + i * 1024), 16, off[i & mask], soff, 0,
                                               STREAM ? AUX_NT : 0);
    }
  };
  int pair[NB];
  auto load_scales = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) pair[kb] = scale_pair(p, srsrc, w.j0 + first_key(c) + 32 * kb + i32);
  };
  uint32_t vaddr[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
    vaddr[db] = v_address<DT_FP8, D>((uint32_t)(size_t)LDS_PTR(const uint8_t, vslot), db, lane);

  f32x16 oacc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) oacc[db] = f32x16{0.0f};
  float m_seen = -INFINITY, m_wave = -INFINITY, l_part = 0.0f;
  const int kswz = k_swz<DT_FP8, D>(i32);
  const int wt = wave >> 1;  // tile of the round

  __builtin_amdgcn_sched_barrier(0);
  load_scales(0);
  __builtin_amdgcn_sched_barrier(0);
  stage(krsrc, kslot, koff, 3, 0);
  __builtin_amdgcn_sched_barrier(0);
  stage(vrsrc, vslot, voff, 1, 0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < q.CHUNKS * q.PER; ++t) asm volatile("" : "+v"(q.x[t]));
  const int nrounds = (w.nk + TPR * BC - 1) / (TPR * BC);
#pragma unroll 1
  for (int c = 0; c < nrounds; ++c) {
    const int kw0 = first_key(c);
    const bool need_mask = kw0 + UNIT > w.open || kw0 + UNIT > w.nk;
    const int lim = limit - kw0 - 4 * g;
    // this round's scales and K have landed once at most the V copies behind them
    // are outstanding
    wait_vmcnt<LOADS>();
    float ks[NB], vs[2 * NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      ks[kb] = scale_of(pair[kb] & 255);
      vs[2 * kb] = v_scale(pair[kb], 0);
      vs[2 * kb + 1] = v_scale(pair[kb], 16);
    }
    f32x16 sv[NB];
#pragma unroll
    for (int t = 0; t < q.CHUNKS; ++t)
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const i32x4 kk = *(const i32x4*)(kslot + (32 * kb + i32) * RB + (((2 * t + g) ^ kswz) << 4));
        sv[kb] = product<D>(kk, ks[kb], q, t, t == 0 ? f32x16{0.0f} : sv[kb]);
      }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load_scales(c + 1);
    __builtin_amdgcn_sched_barrier(0);
    stage(krsrc, kslot, koff, 3, c + 1);
    settle_unit(sv);
    if (need_mask) mask_unit(sv, lim, -INFINITY);
    bf16x8 pb[2 * NB];
    float alpha = 1.0f;
    if constexpr (mode_lattice(MODE)) {
      float ma, mb;
      with_partner(unit_max(sv), ma, mb);
      if (g == 0) mx_lds[c & 1][i32][wave] = __builtin_fmaxf(ma, mb);
      // (the two copies of mx_lds alternate: a wave that runs ahead writes the other)
      lds_barrier();
      const f32x4 x = *(const f32x4*)&mx_lds[c & 1][i32][0];
      const float t0 = __builtin_fmaxf(x[0], x[1]), t1 = __builtin_fmaxf(x[2], x[3]);
      float anchor = __builtin_fmaxf(m_seen, t0);
      m_seen = max3(m_seen, t0, t1);
      if (wt != 0) anchor = m_seen;
      // a row that has seen no key yet keeps m = -inf, l = 0, O = 0
      if (anchor != -INFINITY) alpha = __builtin_amdgcn_exp2f((m_wave - anchor) * p.c1);
      m_wave = anchor;
      l_part *= alpha;
      uint32_t wpk[NB][8];
      weigh<MODE, NB>(sv, wpk, anchor == -INFINITY ? 0.0f : anchor, p.c1, p.ck, need_mask, lim, l_part);
#pragma unroll
      for (int k = 0; k < 2 * NB; ++k) pb[k] = p_operand<MODE>(sv[k >> 1], wpk[k >> 1], k & 1);
    } else {
      float e[32], sum = weights(sv, e, -m_wave * p.c1, p.c1);
      if (__builtin_amdgcn_ballot_w64(!(sum <= ANCHOR_HOLDS)) != 0) {
        float ma, mb;
        with_partner(unit_max(sv), ma, mb);
        const float top = max3(m_wave, ma, mb);
        if (top != -INFINITY) alpha = __builtin_amdgcn_exp2f((m_wave - top) * p.c1);
        m_wave = top;
        l_part *= alpha;
        sum = weights(sv, e, top == -INFINITY ? 0.0f : -top * p.c1, p.c1);
      }
      l_part += sum;
#pragma unroll
      for (int k = 0; k < 2 * NB; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) pb[k][j] = (__bf16)e[8 * k + j];
    }
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) oacc[db][j] *= alpha;
    }
    wait_vmcnt<LOADS + NB>();  // V has landed, the next round's scales and K may be outstanding
#pragma unroll
    for (int db = 0; db < NDB; db += 2) add_pv<D>(oacc[db], oacc[db + 1], vaddr[db], vaddr[db + 1], pb, vs);
    stage(vrsrc, vslot, voff, 1, c + 1);
  }
  // every copy has landed (the last round's went to no key) and every wave is
  // done with its slots before they are reused
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();

  // ---- the waves' sums, each relative to its own anchor, added up: rows 0..15
  // of every wave's O in vsm, rows 16..31 in ksm
  {
    float la, lb;
    with_partner(l_part, la, lb);
    if (g == 0) {
      m_lds[i32][wave] = m_wave;
      l_lds[i32][wave] = la + lb;
    }
  }
  if (i32 < w.nrows) {
    const int ri = i32 & (RHALF - 1);
    float* red = (float*)(i32 < RHALF ? vsm : ksm) + (wave * RHALF + ri) * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int jq = 0; jq < 4; ++jq)
        *(f32x4*)(red + 4 * ((8 * db + 2 * jq + g) ^ ri)) =
            f32x4{oacc[db][4 * jq], oacc[db][4 * jq + 1], oacc[db][4 * jq + 2], oacc[db][4 * jq + 3]};
  }
  lds_barrier();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r0 = half * RHALF;
    if (r0 >= w.nrows) break;
    const float* red = (const float*)(half == 0 ? vsm : ksm);
#pragma unroll
    for (int i = 0; i < RHALF * (D / 4) / (NW * 64); ++i) {
      const int idx = i * NW * 64 + tid, rr = idx / (D / 4), ch = idx % (D / 4), r = r0 + rr;
      if (r >= w.nrows) continue;
      const f32x4 mw = *(const f32x4*)m_lds[r], lw = *(const f32x4*)l_lds[r];
      const float m = __builtin_fmaxf(__builtin_fmaxf(mw[0], mw[1]), __builtin_fmaxf(mw[2], mw[3]));
      float l = 0.0f;
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        const float f = mw[x] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mw[x] - m) * p.c1);
        l += f * lw[x];
        const f32x4 o = *(const f32x4*)(red + (x * RHALF + rr) * D + 4 * (ch ^ rr));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += f * o[e];
      }
      const size_t orow = out_row(p, w, r);
      if (p.parts == 1) {
        store_row4(p.o + orow * D + 4 * ch, acc, inverse(l, 1.0f));
        if (p.lse && ch == 0) p.lse[orow] = row_lse(m, l, p.c1);
      } else {
        const size_t at = orow * (size_t)p.parts + w.part;
        *(f32x4*)(p.part_o + at * D + 4 * ch) = acc;
        if (ch == 0) *(f32x2*)(p.part_ml + at * 2) = f32x2{m, l};
      }
    }
  }
}

template <int D, int MODE>
__device__ __forceinline__ void rows_form(const BlocksParams& p, const Work& w, uint8_t* ksm, uint8_t* vsm) {
  using C = BCfg<D>;
  constexpr int RB = C::RB, NDB = D / 32, LOADS = C::TILE / (NW * 1024), NSC = BC / 32;
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool active = wave * WROWS < w.nrows;
  const int rowc = min(wave * WROWS + i32, w.nrows - 1);
  const size_t orow = out_row(p, w, rowc);
  RowOperand<DT_FP8, D> q;
  load_q<D>(q, p.q + orow * (2 * D), g);
  const int limit = row_limit(p, w, rowc);
  const uint32_t part_bytes = (uint32_t)w.nk * RB;
  const auto krsrc = rows_rsrc(w.k, part_bytes), vrsrc = rows_rsrc(w.v, part_bytes);
  const auto srsrc = rows_rsrc(w.scales, w.used);
  // a wave copies a quarter of each tile: LOADS consecutive KB
  // (d = 128: eight rows on, both swizzles differ in their third bit)
  constexpr uint32_t NEXT = D == 128 ? 64 : 0;
  static_assert(LOADS % 2 == 0, "a wave's first copy is an even one");
  uint32_t koff, voff;
  {
    const int r = copy_row<C::NCH>(wave * LOADS, lane), first = wave * LOADS * (64 / C::NCH);
    koff = (r - first) * RB + (((lane % C::NCH) ^ k_swz<DT_FP8, D>(r)) << 4);
    voff = (r - first) * RB + (((lane % C::NCH) ^ v_swz<DT_FP8, D>(r)) << 4);
  }
  auto stage = [&](const __amdgpu_buffer_rsrc_t rsrc, uint8_t* area, uint32_t off, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t at = (wave * LOADS + i) * 1024;
      const uint32_t soff = min((uint32_t)t * C::TILE + at, part_bytes);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, LDS_PTR(void, area + at), 16, off ^ (NEXT * (i & 1)), soff, 0, 0);
    }
  };
  int pair[NSC];
  auto load_scales = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < NSC; ++kb) pair[kb] = scale_pair(p, srsrc, w.j0 + t * BC + 32 * kb + i32);
  };
  uint32_t vaddr[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
    vaddr[db] = v_address<DT_FP8, D>((uint32_t)(size_t)LDS_PTR(const uint8_t, vsm), db, lane);
  f32x16 oacc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) oacc[db] = f32x16{0.0f};
  float m = -INFINITY, l = 0.0f;
  const int kswz = k_swz<DT_FP8, D>(i32);

  load_scales(0);
  stage(krsrc, ksm, koff, 0);
#pragma unroll
  for (int t = 0; t < q.CHUNKS * q.PER; ++t) asm volatile("" : "+v"(q.x[t]));
  const int ntiles = (w.nk + BC - 1) / BC;
#pragma unroll 1
  for (int t = 0; t < ntiles; ++t) {
    // this wave's part of K has landed; past the barrier everyone's has, and
    // everyone is done with the last tile's V
    wait_vmcnt<0>();
    lds_barrier();
    stage(vrsrc, vsm, voff, t);
    const int kw0 = t * BC;
    const bool need_mask = kw0 + BC > w.open || kw0 + BC > w.nk;
    const int lim = limit - kw0 - 4 * g;
    f32x16 lo[2], hi[2];  // keys 0..63 and 64..127
    float ks[NSC], vlo[4], vhi[4];
#pragma unroll
    for (int kb = 0; kb < NSC; ++kb) {
      ks[kb] = scale_of(pair[kb] & 255);
      float* const vs = kb < 2 ? vlo + 2 * kb : vhi + 2 * (kb - 2);
      vs[0] = v_scale(pair[kb], 0);
      vs[1] = v_scale(pair[kb], 16);
    }
    if (active) {
#pragma unroll
      for (int kt = 0; kt < q.CHUNKS; ++kt)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const i32x4 kk = *(const i32x4*)(ksm + (32 * kb + i32) * RB + (((2 * kt + g) ^ kswz) << 4));
          f32x16& s = kb < 2 ? lo[kb & 1] : hi[kb & 1];
          s = product<D>(kk, ks[kb], q, kt, kt == 0 ? f32x16{0.0f} : s);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();  // everyone has read K
    load_scales(t + 1);
    __builtin_amdgcn_sched_barrier(0);
    stage(krsrc, ksm, koff, t + 1);
    bf16x8 pb[4], pc[4];
    if (active) {
      settle_unit(lo);
      settle_unit(hi);
      if (need_mask) {
        mask_unit(lo, lim, -INFINITY);
        mask_unit(hi, lim - 64, -INFINITY);
      }
      float alpha = 1.0f;
      // the row's maximum, a row that has seen no key yet keeping m = -inf, l = 0, O = 0
      auto move = [&]() __attribute__((always_inline)) {
        float ma, mb;
        with_partner(__builtin_fmaxf(unit_max(lo), unit_max(hi)), ma, mb);
        const float anchor = max3(m, ma, mb);
        if (anchor != -INFINITY) alpha = __builtin_amdgcn_exp2f((m - anchor) * p.c1);
        m = anchor;
        l *= alpha;
      };
      if constexpr (mode_lattice(MODE)) {
        move();
        const float m_use = m == -INFINITY ? 0.0f : m;
        uint32_t wlo[2][8], whi[2][8];
        weigh<MODE, 2>(lo, wlo, m_use, p.c1, p.ck, need_mask, lim, l);
        weigh<MODE, 2>(hi, whi, m_use, p.c1, p.ck, need_mask, lim - 64, l);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          pb[k] = p_operand<MODE>(lo[k >> 1], wlo[k >> 1], k & 1);
          pc[k] = p_operand<MODE>(hi[k >> 1], whi[k >> 1], k & 1);
        }
      } else {
        auto all = [&](float nb) __attribute__((always_inline)) {
          return packed_weights(lo, pb, nb, p.c1) + packed_weights(hi, pc, nb, p.c1);
        };
        float sum = all(-m * p.c1);
        if (__builtin_amdgcn_ballot_w64(!(sum <= ANCHOR_HOLDS)) != 0) {
          move();
          sum = all(m == -INFINITY ? 0.0f : -m * p.c1);
        }
        l += sum;
      }
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) oacc[db][j] *= alpha;
      }
    }
    wait_vmcnt<LOADS + NSC>();  // V has landed, the next tile's scales and K may be outstanding
    lds_barrier();
    if (active) {
#pragma unroll
      for (int db = 0; db < NDB; db += 2) {
        add_pv<D>(oacc[db], oacc[db + 1], vaddr[db], vaddr[db + 1], pb, vlo);
        add_pv<D>(oacc[db], oacc[db + 1], vaddr[db] + 64 * RB, vaddr[db + 1] + 64 * RB, pc, vhi);
      }
    }
  }
  wait_vmcnt<0>();
  float la, lb;
  with_partner(l, la, lb);
  l = la + lb;
  if (wave * WROWS + i32 >= w.nrows) return;
  const float inv = inverse(l, 1.0f);
  const size_t at = orow * (size_t)p.parts + w.part;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int jq = 0; jq < 4; ++jq) {
      const f32x4 x = {oacc[db][4 * jq], oacc[db][4 * jq + 1], oacc[db][4 * jq + 2], oacc[db][4 * jq + 3]};
      const int col = 32 * db + 8 * jq + 4 * g;
      if (p.parts == 1) store_row4(p.o + orow * D + col, x, inv);
      else *(f32x4*)(p.part_o + at * D + col) = x;
    }
  if (g == 0) {
    if (p.parts > 1) *(f32x2*)(p.part_ml + at * 2) = f32x2{m, l};
    else if (p.lse) p.lse[orow] = row_lse(m, l, p.c1);
  }
}

// ---- the wide form: 512 query rows, 64 a wave, the hardware exponential.
// Eight waves, two on a SIMD: while the four of one group are at the matrix core
// (P V of the last step, Q K^T of this one), those of the other make weights, and
// a barrier after each such half step keeps it so.  A step has 64 keys, so that the
// query rows, which no registers are left for, are read from LDS once for all of them.
//
// What bounds it (8192 rows of 8 KV heads after 32K keys, d = 128: 905 us + 26 of the
// merge, 1.14 PFLOP/s; the rows form 1059): the clock that the board's power allows
// (1.94 GHz, with the matrix core busy 56% of the cycles and the VALU 58%): each of
// the steps to here took more off the cycles than off the time.  Widening a step's
// codes once for all waves into BF16 rows saved a third of the VALU's work and lost
// as much to LDS (steps of 32 keys, whose rows LDS has room for: 1033 us; the same
// with codes in LDS 1004).  Two workgroups of 256 rows in place of the two groups: 1030.
// At d = 128 all 256 registers are taken and 4 spilled; one of them is loaded again, in
// steps with masked keys.
template <int D>
struct WCfg {
  static constexpr int NW = BLOCKS_WIDE / 64;
  static constexpr int RB = D, NCH = D / 16;      // bytes and chunks of a row of codes
  static constexpr int STEP = 64, HALF = STEP * RB;  // keys of a step, bytes of its K (or V)
  static constexpr int LOADS = HALF / 4096;       // copies of 1 KB of a wave
  static constexpr int QRB = 2 * D;               // bytes of a query row
  static constexpr int QAREA = BLOCKS_WIDE * QRB;
};

template <int D>
__device__ __forceinline__ void wide_form(const BlocksParams& p, const Work& w, uint8_t* qsm, uint8_t* k0, uint8_t* k1,
                                          uint8_t* v0, uint8_t* v1) {
  using C = WCfg<D>;
  constexpr int RB = C::RB, NCH = C::NCH, NDB = D / 32, STEP = C::STEP, QCH = C::QRB / 16;
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t part_bytes = (uint32_t)w.nk * RB;
  // the first group copies K, the second V, a quarter of a step a wave
  const bool second = wave >= C::NW / 2;
  const int mine = wave & (C::NW / 2 - 1);
  const auto rsrc = rows_rsrc(second ? w.v : w.k, part_bytes);
  const auto srsrc = rows_rsrc(w.scales, w.used);
  uint32_t off;
  {
    const int kb = mine * C::LOADS, r = copy_row<NCH>(kb, lane), first = kb * (64 / NCH);
    off = (r - first) * RB + (((lane % NCH) ^ (second ? v_swz<DT_FP8, D>(r) : k_swz<DT_FP8, D>(r))) << 4);
  }
  auto stage = [&](int c, uint8_t* buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      const int at = (mine * C::LOADS + i) * 1024;
      const uint32_t soff = min((uint32_t)c * C::HALF + at, part_bytes);
      // (d = 128: eight rows on, both swizzles differ in their third bit)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, LDS_PTR(void, buf + at), 16, off ^ (64 * i), soff, 0, 0);
    }
  };
  int pair[2];
  auto load_scales = [&](int c) __attribute__((always_inline)) {
    pair[0] = scale_pair(p, srsrc, w.j0 + c * STEP + i32);
    pair[1] = scale_pair(p, srsrc, w.j0 + c * STEP + 32 + i32);
  };
  // the query rows, chunk 4 t + 2 g + j of a row at 4 t + 2 j + g: operand 2 t + j of half g
#pragma unroll 4
  for (int i = tid; i < BLOCKS_WIDE * QCH; i += C::NW * 64) {
    const int r = i / QCH, c = i % QCH;
    const i32x4 x = *(const i32x4*)(p.q + out_row(p, w, min(r, w.nrows - 1)) * C::QRB + 16 * c);
    *(i32x4*)(qsm + r * C::QRB + ((((c & ~3) | ((c & 1) << 1) | ((c >> 1) & 1)) ^ k_swz<DT_BF16, D>(r)) << 4)) = x;
  }
  // addresses of the first chunks of K, V and the query rows: the swizzles are
  // exclusive ors, so that the others follow from these
  uint32_t kat = i32 * RB + ((g ^ k_swz<DT_FP8, D>(i32)) << 4), vat = v_address<DT_FP8, D>(0, 0, lane);
  uint32_t qat = (wave * 64 + i32) * C::QRB + ((g ^ k_swz<DT_BF16, D>(i32)) << 4);
  f32x16 oacc[2][NDB];
  float m[2], l[2];
  bf16x8 pb[2][4];  // the last step's weights (none before the first), and its values' scales
  float vs[4] = {1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    m[s] = -INFINITY;
    l[s] = 0.0f;
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[s][db] = f32x16{0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k) pb[s][k] = bf16x8{};
  }
  const int nsteps = (w.nk + STEP - 1) / STEP;

  // P V of the last step, its V in vbuf
  auto add_values = [&](const uint8_t* vbuf) __attribute__((always_inline)) {
    i32x2v r[2][4];
    auto read_v = [&](int db) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        r[db & 1][k] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(i32x2v, vbuf + (vat ^ (db << 5)) + 16 * RB * k));
    };
    read_v(0);
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      if (db + 1 < NDB) read_v(db + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bf16x8 x = widen(r[db & 1][k][0], r[db & 1][k][1], vs[k]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
          oacc[s][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pb[s][k], oacc[s][db], 0, 0, 0);
      }
    }
  };
  // One step: its K is in kbuf, the last one's V in vbuf, which takes the next one's
  // once it is done with; the next one's K goes to knext.  (The buffers are arrays
  // of their own: the compiler waits for a copy into an array that it reads.)
  auto step = [&](int c, const uint8_t* kbuf, uint8_t* knext, uint8_t* vbuf) __attribute__((always_inline)) {
    // (made anew in each step: kept, the addresses of all buffers spill)
    asm volatile("" : "+v"(kat), "+v"(vat), "+v"(qat));
    float ks[2], vnext[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      ks[kb] = scale_of(pair[kb] & 255);
      vnext[2 * kb] = v_scale(pair[kb], 0);
      vnext[2 * kb + 1] = v_scale(pair[kb], 16);
    }
    load_scales(c + 1);
    if (!second) stage(c + 1, knext);
    __builtin_amdgcn_sched_barrier(0);
    i32x4 kk[2][2];
    bf16x8 q[2][2];
    auto read_k = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) kk[t & 1][kb] = *(const i32x4*)(kbuf + (kat ^ (t << 5)) + 32 * RB * kb);
    };
    auto read_q = [&](int u) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s) q[u & 1][s] = *(const bf16x8*)(qsm + (qat ^ (u << 5)) + 32 * s * C::QRB);
    };
    add_values(vbuf);
    read_k(0);
    read_q(0);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 sv[2][2];
#pragma unroll
    for (int u = 0; u < NCH; ++u) {
      if (u % 2 == 0 && u + 2 < NCH) read_k(u / 2 + 1);
      if (u + 1 < NCH) read_q(u + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const i32x4& x4 = kk[(u / 2) & 1][kb];
        const bf16x8 x = widen(x4[2 * (u & 1)], x4[2 * (u & 1) + 1], ks[kb]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
          sv[s][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[u & 1][s], u == 0 ? f32x16{0.0f} : sv[s][kb], 0, 0, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) vs[k] = vnext[k];
    __builtin_amdgcn_sched_barrier(0);
    if (second) wait_vmcnt<2>();  // V of this step has landed; the next one's scales may be outstanding
    lds_barrier();
    if (second) stage(c + 1, vbuf);
    const int kw0 = c * STEP;
    const bool need_mask = kw0 + STEP > w.open || kw0 + STEP > w.nk;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (need_mask) {
        settle_unit(sv[s]);
        mask_unit(sv[s], row_limit(p, w, min(wave * 64 + 32 * s + i32, w.nrows - 1)) - 4 * g - kw0, -INFINITY);
      }
      float e[32], sum = weights(sv[s], e, -m[s] * p.c1, p.c1);
      if (__builtin_amdgcn_ballot_w64(!(sum <= ANCHOR_HOLDS)) != 0) {
        float ma, mb;
        settle_unit(sv[s]);
        with_partner(unit_max(sv[s]), ma, mb);
        const float top = max3(m[s], ma, mb);
        const float alpha = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m[s] - top) * p.c1);
        m[s] = top;
        l[s] *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) oacc[s][db][j] *= alpha;
        sum = weights(sv[s], e, top == -INFINITY ? 0.0f : -top * p.c1, p.c1);
      }
      l[s] += sum;
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) pb[s][k][j] = (__bf16)e[8 * k + j];
    }
    if (!second) wait_vmcnt<0>();  // the next step's K has landed
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
  };
  load_scales(0);
  if (second) stage(0, v0);
  else stage(0, k0);
  // (the values before the first step have the weight 0, but must not be NaN)
  for (int i = tid; i < C::HALF / 16; i += C::NW * 64) *(i32x4*)(v1 + 16 * i) = i32x4{0, 0, 0, 0};
  if (!second) wait_vmcnt<0>();
  lds_barrier();
  if (second) lds_barrier();  // the second group is half a step behind
#pragma unroll 1
  for (int c = 0; c < nsteps; c += 2) {
    step(c, k0, k1, v1);
    step(c + 1, k1, k0, v0);  // (a step beyond the last key is masked whole)
  }
  if (!second) lds_barrier();
  wait_vmcnt<0>();
  add_values(v1);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float la, lb;
    with_partner(l[s], la, lb);
    const float sum = la + lb, inv = inverse(sum, 1.0f);
    const int r = wave * 64 + 32 * s + i32;
    if (r >= w.nrows) continue;
    const size_t orow = out_row(p, w, r), at = orow * (size_t)p.parts + w.part;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int jq = 0; jq < 4; ++jq) {
        const f32x4 x = {oacc[s][db][4 * jq], oacc[s][db][4 * jq + 1], oacc[s][db][4 * jq + 2], oacc[s][db][4 * jq + 3]};
        const int col = 32 * db + 8 * jq + 4 * g;
        if (p.parts == 1) store_row4(p.o + orow * D + col, x, inv);
        else *(f32x4*)(p.part_o + at * D + col) = x;
      }
    if (g == 0) {
      if (p.parts > 1) *(f32x2*)(p.part_ml + at * 2) = f32x2{m[s], sum};
      else if (p.lse) p.lse[orow] = row_lse(m[s], sum, p.c1);
    }
  }
}

// A workgroup's sequence, head, part and rows; false if there is nothing to read
// (several parts: said so to the merge, which skips a part with l = 0).
template <int D>
__device__ __forceinline__ bool find_work(const BlocksParams& p, int* scratch, Work& w) {
  int unit, rb;
  place(blockIdx.x, p.B * p.Hkv * p.parts, p.row_blocks, unit, rb);
  int bh = unit / p.parts;
  // (parts in turn, begun at another one for each cache of an XCD, which gets every
  // (8 / gcd(8, parts))-th: the last ones, empty for short caches, would else be all of
  // one XCD where there are eight, or of four where there are two)
  w.part = (unit - bh * p.parts + (bh >> p.turn)) % p.parts;
  w.b = bh / p.Hkv;
  w.h = bh - w.b * p.Hkv;
  if (p.longest) {
    w.b = longest(p.lens, p.B, p.Sk, w.b, scratch);
    bh = w.b * p.Hkv + w.h;
  }
  const int n = p.lens ? min(max(p.lens[w.b], 0), p.Sk) : p.Sk;
  w.row0 = rb * p.rows;
  w.nrows = min(p.rows, p.R - w.row0);
  w.j0 = w.part * p.split;
  w.nk = max(min(p.split, n - w.j0), 0);
  w.open = w.nk;
  w.last0 = w.nk - 1;
  if (p.causal) {
    // positions of its rows: from i0 on, or all of them where they pass a head's last
    const int i0 = w.row0 % p.Sq, i1 = i0 + w.nrows - 1;
    w.last0 = n - p.Sq - w.j0;
    w.nk = max(min(w.nk, w.last0 + min(i1, p.Sq - 1) + 1), 0);
    w.open = w.last0 + (i1 < p.Sq ? i0 : 0) + 1;
  }
  if (w.nk == 0 && p.parts > 1) {
    if ((int)threadIdx.x < w.nrows)
      *(f32x2*)(p.part_ml + (out_row(p, w, threadIdx.x) * (size_t)p.parts + w.part) * 2) = f32x2{-INFINITY, 0.0f};
    return false;
  }
  const size_t at = ((size_t)bh * (size_t)p.Sk_cap + (size_t)(w.nk ? w.j0 : 0)) * D;
  w.k = p.k + at;
  w.v = p.v + at;
  w.scales = p.scales + (size_t)bh * (size_t)p.blocks * 2;
  w.used = 2 * ((n + (1 << p.shift) - 1) >> p.shift);
  return true;
}

enum { FORM_KEYS = 0, FORM_KEYS_STREAM = 1, FORM_ROWS = 2 };

template <int D, int MODE, int FORM>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_blocks_kernel(
    BlocksParams p) {
  using C = BCfg<D>;
  // (arrays of their own, so that the compiler tells the copies apart)
  __shared__ __attribute__((aligned(16))) uint8_t ksm[C::AREA];
  __shared__ __attribute__((aligned(16))) uint8_t vsm[C::AREA];
  __shared__ __attribute__((aligned(16))) float mx_lds[2][32][NW];
  __shared__ __attribute__((aligned(16))) float m_lds[32][NW], l_lds[32][NW];
  Work w;
  if (!find_work<D>(p, (int*)mx_lds, w)) return;
  if constexpr (FORM == FORM_ROWS) rows_form<D, MODE>(p, w, ksm, vsm);
  else keys_form<D, MODE, FORM == FORM_KEYS_STREAM>(p, w, ksm, vsm, mx_lds, m_lds, l_lds);
}

template <int D>
__global__ __launch_bounds__(BLOCKS_WIDE) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_blocks_wide_kernel(
    BlocksParams p) {
  using C = WCfg<D>;
  // (aligned further, the buffers lie first, where an instruction's offset tells
  // them apart)
  __shared__ __attribute__((aligned(1024))) uint8_t k0[C::HALF];
  __shared__ __attribute__((aligned(1024))) uint8_t k1[C::HALF];
  __shared__ __attribute__((aligned(1024))) uint8_t v0[C::HALF];
  __shared__ __attribute__((aligned(1024))) uint8_t v1[C::HALF];
  __shared__ __attribute__((aligned(16))) uint8_t qsm[C::QAREA];
  Work w;
  if (!find_work<D>(p, (int*)qsm, w)) return;
  wide_form<D>(p, w, qsm, k0, k1, v0, v1);
}

template <int D>
__global__ __launch_bounds__(256) void attn_blocks_merge(BlocksParams p) {
  merge_parts<D>(p, 1.0f);
}

template <int D, int MODE>
hipError_t launch_one(const BlocksParams& p, hipStream_t st) {
  const dim3 grid((unsigned)p.groups), block(NW * 64);
  if (p.rows == BLOCKS_WIDE && MODE == MODE_EXACT) hipLaunchKernelGGL((attn_blocks_wide_kernel<D>), grid, dim3(BLOCKS_WIDE), 0, st, p);
  else if (p.rows != WROWS) hipLaunchKernelGGL((attn_blocks_kernel<D, MODE, FORM_ROWS>), grid, block, 0, st, p);
  else if (p.stream) hipLaunchKernelGGL((attn_blocks_kernel<D, MODE, FORM_KEYS_STREAM>), grid, block, 0, st, p);
  else hipLaunchKernelGGL((attn_blocks_kernel<D, MODE, FORM_KEYS>), grid, block, 0, st, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_mode(const BlocksParams& p, int mode, hipStream_t st) {
  hipError_t e;
  switch (mode) {
    case MODE_EXACT: e = launch_one<D, MODE_EXACT>(p, st); break;
    case 1: e = launch_one<D, 1>(p, st); break;
    case 3: e = launch_one<D, 3>(p, st); break;
    case 5: e = launch_one<D, 5>(p, st); break;
    default: return hipErrorInvalidValue;
  }
  if (e != hipSuccess || p.parts == 1) return e;
  const dim3 grid((unsigned)(((long long)p.B * p.Hq * p.Sq + 3) / 4));
  hipLaunchKernelGGL(attn_blocks_merge<D>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}
}  // namespace

namespace h15 {

int launch_blocks(const BlocksParams& p, int d, int mode, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const hipError_t e = d == 128 ? launch_mode<128>(p, mode, st) : launch_mode<64>(p, mode, st);
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
