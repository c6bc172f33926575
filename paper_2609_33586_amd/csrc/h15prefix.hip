// Decode for a batch that shares a prefix (attn_decode_prefix): Sq query rows
// per head and sequence against a prefix's keys, which all sequences have in
// common, and then against each sequence's own cache of lens[b] keys.
//
// The prefix is read once for all sequences: its rows are the B G Sq query
// rows of a KV head over the whole batch (row rr: sequence rr / R, row rr % R
// of it, R = G Sq), in blocks that a workgroup holds against one part of the
// prefix's keys.  The own caches are cut into parts as in attn_decode.  Both
// kinds of workgroups are one launch, so that the prefix's, which the matrix
// core and the VALU bound, share the compute units with those of the own
// caches, which HBM bounds.  A second launch merges the parts of each row.
//
// Two forms of a workgroup (4 waves):
//   keys  32 query rows; each wave takes its own keys of a round (UNIT of
//         them), copies them into its own LDS slots and exchanges only the
//         maxima of its units with the others (one barrier a round); a weight
//         is rounded relative to the running maximum at its own tile, the
//         prefix maximum of the round's units.  All own caches, and prefixes
//         of up to four blocks of rows;
//   rows  128 query rows, 32 a wave; the waves share each tile of 128 keys, so
//         that more rows do not read the prefix again.
// A workgroup of an own cache may take a short prefix first, in the keys form:
// one launch and nothing to merge.  (The rules between these: cache_api.cpp.)
//
// What bounds it: HBM where there is enough to read (BF16, 64 sequences of 32 heads
// over 8 KV heads, 32K prefix and 2K own keys: 143 us for 671 MB, 4.7 TB/s).  With
// fewer keys the rounds of a workgroup, one after the other (32 such sequences, 8K
// prefix, up to 1K own keys: 29 us + 4 of the merge for 115 MB): its 512 workgroups
// start within 0.2 us, two on a compute unit, and ask for 33 MB at once; those of the
// prefix have their first keys after 2.4 us, the own ones after 5 on average and 10
// at most; a round of 128 keys then takes 2 us (3900 cycles, of which 750 wait for K),
// the last of 8 ends after 18 and 20..26 us, the reduction takes 1 to 2.  FP8 with many rows: a rows tile takes 5900 cycles, 1500 for Q K^T, 1900
// for the weights and 1800 for P V (1024 of the matrix core each) in turn, next
// to one workgroup of own caches (64 sequences, 32K prefix, 2K own keys: 66 us +
// 6 for 230 MB).  Widening each FP8 tile once for the four waves, through
// registers into BF16 tiles, was level for the exponential (LDS reads double)
// and slower for the lattice weights, whose registers spilled (5K keys, 84 rows:
// 25 -> 36 us).  Two FP8 tiles in LDS at a time, with a tile's time for their copies
// and one barrier, V's reads in half as many waits, and a higher wave priority of one
// kind of workgroup were level (66 -> 66..72 us): the waits are filled by the other
// workgroup.  Short caches wait: 4 chats of 500 + 60 keys BF16 d = 64 take 8.9 us
// in one launch (10.5 with the call), three rounds in series on 8 workgroups.
//
// Arithmetic: that of attn_decode for BF16.  FP8 operands are widened to BF16,
// which holds every e4m3 value, and meet in the BF16 matrix core: the FP8
// products sum to about 2^-13 of sum |q k| (64 deep, attn_decode's) or 2^-16
// (16 deep), and P, rounded to BF16 here (half a step of 2^-8 of it at most),
// would be off by up to 2^-4 in e4m3, 2.6% rms a weight.  The matrix core takes
// no wider P; the weights' sum takes them unrounded.  With the hardware exponential O
// is off by 2.1e-3 of its norm (500 keys; 32K 2.3e-3), of which rounding O itself
// to BF16 is 1.7e-3.  Lattice weights are exact in BF16.
#include "cache_params.h"
#include "unit_device.h"

namespace {

constexpr int NW = 4;  // waves per workgroup

template <int DT, int D>
struct PCfg {
  using C = Cfg<DT, D>;
  static constexpr int RB = C::RB, NCH = C::NCH;
  // keys of a wave and round (keys form): at most 32 KB of K, and of V, in LDS,
  // so that two workgroups share a compute unit
  static constexpr int UNIT = NW * 64 * RB <= 32 * 1024 ? 64 : 32;
  static constexpr int NB = UNIT / 32;        // blocks of 32 keys in a unit
  static constexpr int TPR = NW * UNIT / BC;  // tiles in a round
  static constexpr int SLOT = UNIT * RB;      // one wave's K (or V) of a round
  static constexpr int TILE = BC * RB;
  // K (and V) area of LDS: the slots of a round, a tile, or half of the waves'
  // O rows in the keys form's final reduction
  static constexpr int RED = NW * 16 * D * 4;
  static constexpr int A0 = NW * SLOT > TILE ? NW * SLOT : TILE;
  static constexpr int AREA = A0 > RED ? A0 : RED;
  static constexpr int NKQ = D / 16;  // products of 16 channels
};

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

// acc + chunk t of the keys (16 bytes a lane) times the rows q
template <int DT, int D>
__device__ __forceinline__ f32x16 product(i32x4 k, const RowOperand<DT, D>& q, int t, f32x16 acc) {
  if constexpr (DT == DT_BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), q.x[t], acc, 0, 0, 0);
  } else {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(k[0], k[1]), q.x[2 * t], acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(k[2], k[3]), q.x[2 * t + 1], acc, 0, 0, 0);
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

// O^T += V^T P^T over NB blocks of 32 keys (NB 1 or 2), two column blocks at once
template <int DT, int D, int NB>
__device__ __forceinline__ void add_pv(f32x16& o0, f32x16& o1, uint32_t a0, uint32_t a1, const bf16x8 (&pb)[2 * NB]) {
  using C = Cfg<DT, D>;
  if constexpr (DT == DT_BF16) {
    i32x2v r[8 * NB];
    read_v16<C::RB>(r, a0, a1);
#pragma unroll
    for (int ks = 0; ks < 2 * NB; ++ks) {
      o0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[2 * ks], r[2 * ks + 1], 0, 1, 2, 3)), pb[ks], o0, 0, 0,
          0);
      o1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8,
                             __builtin_shufflevector(r[4 * NB + 2 * ks], r[4 * NB + 2 * ks + 1], 0, 1, 2, 3)),
          pb[ks], o1, 0, 0, 0);
    }
  } else {
    i32x2v r[4 * NB];
    read_v8<C::RB>(r, a0, a1);
#pragma unroll
    for (int ks = 0; ks < 2 * NB; ++ks) {
      o0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(r[ks][0], r[ks][1]), pb[ks], o0, 0, 0, 0);
      o1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(r[2 * NB + ks][0], r[2 * NB + ks][1]), pb[ks], o1, 0, 0, 0);
    }
  }
}

// A workgroup's share: query rows against one part of keys.
struct Work {
  const uint8_t* k;  // the part's first key row, and its value row
  const uint8_t* v;
  int nk;     // keys of the part
  int part;   // its index among all parts
  int b, h;   // sequence (own caches) and KV head
  int row0;   // first of its rows: of the sequence's R, or of the prefix's B R
  int nrows;
  int open;   // the keys from here on (in the part) are not seen by every row
  bool prefix;  // the rows are the prefix's
  bool whole;   // every row sees every key
};

// Output row (over [B][Hq][Sq]) of row r of a workgroup
__device__ __forceinline__ size_t out_row(const PrefixParams& p, const Work& w, int r) {
  const int rr = w.row0 + r;
  const int b = w.prefix ? rr / p.R : w.b;
  const int in = w.prefix ? rr - b * p.R : rr;
  return ((size_t)b * p.Hq + (size_t)w.h * p.G) * (size_t)p.Sq + in;
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

// CHAIN: the same rows meet `before` first, a part of its own with a running
// maximum of its own, whose sums wait in registers and are merged in at the end.
template <int DT, int D, int MODE, bool CHAIN>
__device__ __forceinline__ void keys_form(const PrefixParams& p, const Work& before, const Work& own, uint8_t* ksm,
                                          uint8_t* vsm, float (*mx_lds)[32][NW], float (*m_lds)[NW],
                                          float (*l_lds)[NW]) {
  using C = PCfg<DT, D>;
  constexpr int NB = C::NB, UNIT = C::UNIT, TPR = C::TPR, SLOT = C::SLOT, RB = C::RB;
  constexpr int NDB = D / 32, LOADS = SLOT / 1024, RHALF = 16;
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rowc = min(i32, own.nrows - 1);
  RowOperand<DT, D> q;
  {
    const uint8_t* qp = p.q + out_row(p, own, rowc) * RB;
#pragma unroll
    for (int t = 0; t < q.CHUNKS; ++t) q.set(t, *(const i32x4*)(qp + 32 * t + 16 * g));
  }
  // the chained part's sums: rows idx / (D / 4) of each half, four columns
  constexpr int ITEMS = RHALF * (D / 4) / (NW * 64);
  f32x4 held[2][ITEMS];
  float held_m[2][ITEMS], held_l[2][ITEMS];
#pragma unroll 1
  for (int turn = CHAIN ? 0 : 1; turn < 2; ++turn) {
    const Work& w = CHAIN && turn == 0 ? before : own;
    // last key of the part that this lane's row sees
    int limit = w.nk - 1;
    if (!w.whole) limit = w.open + (w.row0 + rowc) % p.Sq - 1;
    // rows beyond the part read as zero without touching memory; scalar offsets
    // stop at the resource's size, where every lane is out of range
    const uint32_t part_bytes = (uint32_t)w.nk * RB;
    const auto krsrc = rows_rsrc(w.k, part_bytes), vrsrc = rows_rsrc(w.v, part_bytes);
    uint8_t* const kslot = ksm + wave * SLOT;
    uint8_t* const vslot = vsm + wave * SLOT;
    // the chunk swizzles repeat after every fourth copy at the latest
    uint32_t koff[4], voff[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = copy_row<C::NCH>(i, lane);
      koff[i] = (r - i * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ k_swz<DT, D>(r)) << 4);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = copy_row<C::NCH>(i, lane);
      voff[i] = (r - i * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ v_swz<DT, D>(r)) << 4);
    }
    auto first_key = [&](int c) { return c * (TPR * BC) + wave * UNIT; };
    auto stage = [&](const __amdgpu_buffer_rsrc_t rsrc, uint8_t* slot, const uint32_t* off, int mask,
                     int c) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const uint32_t soff = min((uint32_t)first_key(c) * RB + i * 1024, part_bytes);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, LDS_PTR(void, slot + i * 1024), 16, off[i & mask], soff, 0, 0);
      }
    };
    uint32_t vaddr[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      vaddr[db] = v_address<DT, D>((uint32_t)(size_t)LDS_PTR(const uint8_t, vslot), db, lane);

    f32x16 oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = f32x16{0.0f};
    float m_seen = -INFINITY, m_wave = -INFINITY, l_part = 0.0f;
    const int kswz = k_swz<DT, D>(i32);
    const int wt = TPR == 1 ? 0 : wave >> 1;  // tile of the round

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
      const int lim = min(limit, w.nk - 1) - kw0 - 4 * g;
      // this round's K has landed once at most the V copies behind it are outstanding
      wait_vmcnt<LOADS>();
      f32x16 sv[NB];
#pragma unroll
      for (int t = 0; t < q.CHUNKS; ++t)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
          const i32x4 kk = *(const i32x4*)(kslot + (32 * kb + i32) * RB + (((2 * t + g) ^ kswz) << 4));
          sv[kb] = product(kk, q, t, t == 0 ? f32x16{0.0f} : sv[kb]);
        }
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      stage(krsrc, kslot, koff, 3, c + 1);
      settle_unit(sv);
      if (need_mask) mask_unit(sv, lim, -INFINITY);
      float ma, mb;
      with_partner(unit_max(sv), ma, mb);
      if (g == 0) mx_lds[c & 1][i32][wave] = __builtin_fmaxf(ma, mb);
      // (the two copies of mx_lds alternate: a wave that runs ahead writes the other)
      lds_barrier();
      float anchor = m_seen;
      {
        const f32x4 x = *(const f32x4*)&mx_lds[c & 1][i32][0];
        const float t0 = __builtin_fmaxf(x[0], x[1]), t1 = __builtin_fmaxf(x[2], x[3]);
        m_seen = max3(m_seen, t0, t1);
        anchor = TPR == 2 && wt == 0 ? __builtin_fmaxf(anchor, t0) : m_seen;
      }
      // a row that has seen no key yet keeps m = -inf, l = 0, O = 0
      const float alpha = anchor == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m_wave - anchor) * p.c1);
      m_wave = anchor;
      l_part *= alpha;
      uint32_t wpk[NB][8];
      weigh<MODE, NB>(sv, wpk, anchor == -INFINITY ? 0.0f : anchor, p.c1, p.ck, need_mask, lim, l_part);
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) oacc[db][j] *= alpha;
      }
      bf16x8 pb[2 * NB];
#pragma unroll
      for (int ks = 0; ks < 2 * NB; ++ks) pb[ks] = p_operand<MODE>(sv[ks >> 1], wpk[ks >> 1], ks & 1);
      wait_vmcnt<LOADS>();  // V has landed, the next round's K may be outstanding
#pragma unroll
      for (int db = 0; db < NDB; db += 2) add_pv<DT, D, NB>(oacc[db], oacc[db + 1], vaddr[db], vaddr[db + 1], pb);
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
      for (int i = 0; i < ITEMS; ++i) {
        const int idx = i * NW * 64 + tid, rr = idx / (D / 4), ch = idx % (D / 4), r = r0 + rr;
        if (r >= w.nrows) continue;
        const f32x4 mw = *(const f32x4*)m_lds[r], lw = *(const f32x4*)l_lds[r];
        float m = __builtin_fmaxf(__builtin_fmaxf(mw[0], mw[1]), __builtin_fmaxf(mw[2], mw[3]));
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
        if constexpr (CHAIN) {
          if (turn == 0) {
            held[half][i] = acc;
            held_m[half][i] = m;
            held_l[half][i] = l;
            continue;
          }
          // (as the merge: a part with l = 0 takes no part)
          const float l0 = held_l[half][i], m0 = l0 == 0.0f ? -INFINITY : held_m[half][i];
          const float m1 = l == 0.0f ? -INFINITY : m;
          const float top = __builtin_fmaxf(m0, m1);
          const float f0 = l0 == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((m0 - top) * p.c1);
          const float f1 = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((m1 - top) * p.c1);
          l = f0 * l0 + f1 * l;
          m = top;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = f0 * held[half][i][e] + f1 * acc[e];
        }
        const size_t orow = out_row(p, w, r);
        if (p.parts == 1) {
          store_row4(p.o + orow * D + 4 * ch, acc, inverse(l, p.vd));
          if (p.lse && ch == 0) p.lse[orow] = row_lse(m, l, p.c1);
        } else {
          const size_t at = orow * (size_t)p.parts + w.part;
          *(f32x4*)(p.part_o + at * D + 4 * ch) = acc;
          if (ch == 0) *(f32x2*)(p.part_ml + at * 2) = f32x2{m, l};
        }
      }
    }
    if (CHAIN && turn == 0) __syncthreads();  // the next part's copies go over the sums
  }
}

template <int DT, int D, int MODE>
__device__ __forceinline__ void rows_form(const PrefixParams& p, const Work& w, uint8_t* ksm, uint8_t* vsm) {
  using C = PCfg<DT, D>;
  constexpr int RB = C::RB, NDB = D / 32, LOADS = C::TILE / (NW * 1024);
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool active = wave * WROWS < w.nrows;
  const int rowc = min(wave * WROWS + i32, w.nrows - 1);
  const size_t orow = out_row(p, w, rowc);

  RowOperand<DT, D> q;
  {
    const uint8_t* qp = p.q + orow * RB;
#pragma unroll
    for (int t = 0; t < q.CHUNKS; ++t) q.set(t, *(const i32x4*)(qp + 32 * t + 16 * g));
  }
  const uint32_t part_bytes = (uint32_t)w.nk * RB;
  const auto krsrc = rows_rsrc(w.k, part_bytes), vrsrc = rows_rsrc(w.v, part_bytes);
  // a wave copies a quarter of each tile: LOADS consecutive KB
  uint32_t koff[4], voff[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = copy_row<C::NCH>(wave * LOADS + i, lane);
    koff[i] = (r - (wave * LOADS + i) * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ k_swz<DT, D>(r)) << 4);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = copy_row<C::NCH>(wave * LOADS + i, lane);
    voff[i] = (r - (wave * LOADS + i) * (64 / C::NCH)) * RB + (((lane % C::NCH) ^ v_swz<DT, D>(r)) << 4);
  }
  auto stage = [&](const __amdgpu_buffer_rsrc_t rsrc, uint8_t* area, const uint32_t* off, int mask,
                   int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t at = (wave * LOADS + i) * 1024;
      const uint32_t soff = min((uint32_t)t * C::TILE + at, part_bytes);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, LDS_PTR(void, area + at), 16, off[i & mask], soff, 0, 0);
    }
  };
  uint32_t vaddr[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
    vaddr[db] = v_address<DT, D>((uint32_t)(size_t)LDS_PTR(const uint8_t, vsm), db, lane);
  f32x16 oacc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) oacc[db] = f32x16{0.0f};
  float m = -INFINITY, l = 0.0f;
  const int kswz = k_swz<DT, D>(i32);

  stage(krsrc, ksm, koff, 3, 0);
#pragma unroll
  for (int t = 0; t < q.CHUNKS * q.PER; ++t) asm volatile("" : "+v"(q.x[t]));
  const int ntiles = (w.nk + BC - 1) / BC;
#pragma unroll 1
  for (int t = 0; t < ntiles; ++t) {
    // this wave's part of K has landed; past the barrier everyone's has, and
    // everyone is done with the last tile's V
    wait_vmcnt<0>();
    lds_barrier();
    stage(vrsrc, vsm, voff, 1, t);
    const int kw0 = t * BC;
    const bool need_mask = kw0 + BC > w.nk;
    const int lim = w.nk - 1 - kw0 - 4 * g;
    f32x16 lo[2], hi[2];  // keys 0..63 and 64..127
    if (active) {
#pragma unroll
      for (int kt = 0; kt < q.CHUNKS; ++kt)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const i32x4 kk = *(const i32x4*)(ksm + (32 * kb + i32) * RB + (((2 * kt + g) ^ kswz) << 4));
          f32x16& s = kb < 2 ? lo[kb & 1] : hi[kb & 1];
          s = product(kk, q, kt, kt == 0 ? f32x16{0.0f} : s);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();  // everyone has read K
    stage(krsrc, ksm, koff, 3, t + 1);
    uint32_t wlo[2][8], whi[2][8];
    if (active) {
      settle_unit(lo);
      settle_unit(hi);
      if (need_mask) {
        mask_unit(lo, lim, -INFINITY);
        mask_unit(hi, lim - 64, -INFINITY);
      }
      float ma, mb;
      with_partner(__builtin_fmaxf(unit_max(lo), unit_max(hi)), ma, mb);
      // (a tile of the prefix has a key for every row: the maximum is finite
      // unless every logit is -inf)
      const float anchor = max3(m, ma, mb);
      const float alpha = anchor == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - anchor) * p.c1);
      const float m_use = anchor == -INFINITY ? 0.0f : anchor;
      m = anchor;
      l *= alpha;
      weigh<MODE, 2>(lo, wlo, m_use, p.c1, p.ck, need_mask, lim, l);
      weigh<MODE, 2>(hi, whi, m_use, p.c1, p.ck, need_mask, lim - 64, l);
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) oacc[db][j] *= alpha;
      }
    }
    wait_vmcnt<LOADS>();  // V has landed, the next tile's K may be outstanding
    lds_barrier();
    if (active) {
      bf16x8 pb[4], pc[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        pb[ks] = p_operand<MODE>(lo[ks >> 1], wlo[ks >> 1], ks & 1);
        pc[ks] = p_operand<MODE>(hi[ks >> 1], whi[ks >> 1], ks & 1);
      }
#pragma unroll
      for (int db = 0; db < NDB; db += 2) {
        add_pv<DT, D, 2>(oacc[db], oacc[db + 1], vaddr[db], vaddr[db + 1], pb);
        add_pv<DT, D, 2>(oacc[db], oacc[db + 1], vaddr[db] + 64 * RB, vaddr[db + 1] + 64 * RB, pc);
      }
    }
  }
  wait_vmcnt<0>();
  if (wave * WROWS + i32 < w.nrows) {
    float la, lb;
    with_partner(l, la, lb);
    const size_t at = orow * (size_t)p.parts + w.part;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int jq = 0; jq < 4; ++jq)
        *(f32x4*)(p.part_o + at * D + 32 * db + 8 * jq + 4 * g) =
            f32x4{oacc[db][4 * jq], oacc[db][4 * jq + 1], oacc[db][4 * jq + 2], oacc[db][4 * jq + 3]};
    if (g == 0) *(f32x2*)(p.part_ml + at * 2) = f32x2{m, la + lb};
  }
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

// The sequence of rank `at` by the length of its cache, the longest first.
__device__ __forceinline__ int longest(const PrefixParams& p, int at, int* lens) {
  const int tid = threadIdx.x;
  const int n = tid < p.B ? min(max(p.lens[tid], 0), p.Sk) : -1;
  lens[tid] = n;
  __syncthreads();
  int rank = 0;
  for (int j = 0; j < p.B; j += 4) {
    const i32x4 x = *(const i32x4*)&lens[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) rank += x[e] > n || (x[e] == n && j + e < tid) ? 1 : 0;
  }
  __syncthreads();
  if (tid < p.B && rank == at) lens[0] = tid;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(lens[0]);
  __syncthreads();
  return b;
}

// FORM: how the prefix's rows are taken.
enum { FORM_KEYS = 0, FORM_ROWS = 1, FORM_CHAIN = 2 };

template <int DT, int D, int MODE, int FORM>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_prefix_kernel(
    PrefixParams p) {
  using C = PCfg<DT, D>;
  // (arrays of their own, so that the compiler tells the copies apart)
  __shared__ __attribute__((aligned(16))) uint8_t ksm[C::AREA];
  __shared__ __attribute__((aligned(16))) uint8_t vsm[C::AREA];
  __shared__ __attribute__((aligned(16))) float mx_lds[2][32][NW];
  __shared__ __attribute__((aligned(16))) float m_lds[32][NW], l_lds[32][NW];
  Work w;
  int unit, rb;
  if (FORM != FORM_CHAIN && (int)blockIdx.x < p.p_groups) {
    place(blockIdx.x, p.Hkv * p.p_parts, p.p_blocks, unit, rb);
    w.h = unit / p.p_parts;
    w.part = unit - w.h * p.p_parts;
    w.b = 0;
    w.prefix = w.whole = true;
    const int j0 = w.part * p.p_split;
    w.nk = min(p.p_split, p.P - j0);
    w.open = w.nk;
    w.row0 = rb * p.p_rows;
    w.nrows = min(p.p_rows, p.B * p.R - w.row0);
    const size_t at = ((size_t)w.h * (size_t)p.P_cap + (size_t)j0) * C::RB;
    w.k = p.kp + at;
    w.v = p.vp + at;
    if constexpr (FORM == FORM_ROWS) {
      rows_form<DT, D, MODE>(p, w, ksm, vsm);
      return;
    }
  } else {
    place(blockIdx.x - p.p_groups, p.B * p.Hkv * p.o_parts, p.o_blocks, unit, rb);
    int bh = unit / p.o_parts;
    const int split = unit - bh * p.o_parts;
    w.b = bh / p.Hkv;
    w.h = bh - w.b * p.Hkv;
    if (p.longest) {
      w.b = longest(p, w.b, (int*)mx_lds);
      bh = w.b * p.Hkv + w.h;
    }
    w.part = p.p_parts + split;
    w.prefix = false;
    w.whole = !p.causal;
    const int n = p.lens ? min(max(p.lens[w.b], 0), p.Sk) : p.Sk;
    const int j0 = split * p.o_split;
    // keys of this part that some row sees (the last row sees all n)
    w.nk = max(min(p.o_split, n - j0), 0);
    w.row0 = rb * WROWS;
    w.nrows = min(WROWS, p.R - w.row0);
    // position 0 sees the first n - Sq + 1 keys
    w.open = p.causal ? n - p.Sq + 1 - j0 : w.nk;
    const size_t at = ((size_t)bh * (size_t)p.Sk_cap + (size_t)(w.nk ? j0 : 0)) * C::RB;
    w.k = p.k + at;
    w.v = p.v + at;
  }
  if constexpr (FORM == FORM_CHAIN) {
    Work pre = w;
    pre.whole = true;
    pre.nk = pre.open = p.P;
    pre.k = p.kp + (size_t)w.h * (size_t)p.P_cap * C::RB;
    pre.v = p.vp + (size_t)w.h * (size_t)p.P_cap * C::RB;
    keys_form<DT, D, MODE, true>(p, pre, w, ksm, vsm, mx_lds, m_lds, l_lds);
  } else {
    if (w.nk == 0 && p.parts > 1) {
      // nothing to read: the merge skips a part with l = 0
      if ((int)threadIdx.x < w.nrows) {
        const size_t at = out_row(p, w, threadIdx.x) * (size_t)p.parts + w.part;
        *(f32x2*)(p.part_ml + at * 2) = f32x2{-INFINITY, 0.0f};
      }
      return;
    }
    keys_form<DT, D, MODE, false>(p, w, w, ksm, vsm, mx_lds, m_lds, l_lds);
  }
}

// O and LSE of a row from its parts: m = max m_p, f_p = 2^(c1 (m_p - m)),
// l = sum f_p l_p, O = sum f_p O_p / l * v_descale, LSE = ln2 (m c1 + log2 l),
// over the parts with l_p != 0 (the O of others was never written).  One wave
// a row; a lane holds four columns and every (64 / (D / 4))th part.  32 parts'
// (m, l), one a lane, and then their rows are asked for at once: read one after
// the other, 17 parts of 1024 rows took 8 us.
template <int D>
__global__ __launch_bounds__(256) void attn_prefix_merge(PrefixParams p) {
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
    store_row4(p.o + (size_t)row * D + col, acc, inverse(l, p.vd));
    if (p.lse && col == 0) p.lse[row] = row_lse(m, l, p.c1);
  }
}

template <int DT, int D, int MODE>
hipError_t launch_one(const PrefixParams& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.p_groups + p.o_groups));
  const dim3 block(NW * 64);
  if (p.chain)
    hipLaunchKernelGGL((attn_prefix_kernel<DT, D, MODE, FORM_CHAIN>), grid, block, 0, st, p);
  else if (p.p_rows == PREFIX_ROWS)
    hipLaunchKernelGGL((attn_prefix_kernel<DT, D, MODE, FORM_ROWS>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((attn_prefix_kernel<DT, D, MODE, FORM_KEYS>), grid, block, 0, st, p);
  return hipGetLastError();
}

template <int DT, int D>
hipError_t launch_mode(const PrefixParams& p, int mode, hipStream_t st) {
  switch (mode) {
    case MODE_EXACT: return launch_one<DT, D, MODE_EXACT>(p, st);
    case 1: return launch_one<DT, D, 1>(p, st);
    case 3: return launch_one<DT, D, 3>(p, st);
    case 5: return launch_one<DT, D, 5>(p, st);
    default: return hipErrorInvalidValue;
  }
}
}  // namespace

namespace h15 {

int launch_prefix(const PrefixParams& p, int dtype, int d, int mode, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (dtype == ATTN_BF16) e = d == 128 ? launch_mode<DT_BF16, 128>(p, mode, st) : launch_mode<DT_BF16, 64>(p, mode, st);
  else e = d == 128 ? launch_mode<DT_FP8, 128>(p, mode, st) : launch_mode<DT_FP8, 64>(p, mode, st);
  if (e == hipSuccess && p.parts > 1) {
    const dim3 grid((unsigned)(((long long)p.B * p.Hq * p.Sq + 3) / 4));
    if (d == 128) hipLaunchKernelGGL(attn_prefix_merge<128>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(attn_prefix_merge<64>, grid, dim3(256), 0, st, p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
