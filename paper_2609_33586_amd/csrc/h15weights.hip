// The attention weight that each cached key receives (attn_key_weights):
//   acc[b][hkv][j] = decay acc[b][hkv][j]
//                    + sum over the G query heads and their rows i that see j
//                      of exp(scale q_i . k_j - lse_i).
//
// S = Q K^T with the query rows as the matrix rows, so that a lane's 16 scores
// belong to one key and to 16 rows: their sum is 15 additions in the lane, and
// the two halves of a wave meet once at the end.
//
// Two forms.  Up to KW_FEW_ROWS query rows of a KV head (a decode step, the last
// tokens of a prompt) keep the rows and stream the keys: attn_key_weights_few,
// below.  Beyond:
//
// One workgroup = 4 waves for 256 keys of one (batch, KV head), 64 keys a wave,
// which stay in registers, against a run of tiles of 64 query rows.  A tile
// passes through LDS, where all four waves read it: two copies, the next tile
// being written while one is read, a third on its way in registers, one barrier
// a tile.  A wave takes a tile in two halves of 32 rows and issues, between the
// products of one half, the exponentials, fmas and additions of the half
// before: one instruction stream keeps the matrix core and the VALU busy at
// once (32 x 64 scores take 275 ns of the one or 234 ns of the other alone, and
// 293 ns together).
//
// FP8 operands are widened to BF16 (exact) on their way to LDS and registers:
// the FP8 products sum less exactly than the FP32 sums promised.  A key's weights
// are summed in FP32, 16 rows at a time in the lane and then one sum a half tile: with
// 32 heads of 8K rows acc is off by 1.5e-7 of its norm.
//
// Measured: a decode step of 16 ragged 8K caches (BF16, 8 KV heads) reads 180 MB
// in 39 us; a prompt of 8K rows of 32 heads takes 314 us (875 TFLOP/s; FP8 297, 925),
// 1.8 times its matrix operations at a large product's rate: a turn of 64 rows takes 3200
// cycles at two waves a SIMD, at 1.75 GHz, against 2048 of the matrix core and
// about 2500 of the VALU, and the last workgroups end 40 us apart.  (One pass
// without the interleaving, three waves a SIMD: 384 us; row parts of 16 and of 64
// tiles 332.)
//
// Long runs of query rows are cut into parts, which write their sums to a
// workspace; a second launch adds them up in their order, so results do not
// depend on timing.
#include "cache_params.h"
#include "unit_device.h"

namespace {

constexpr int NW = 4;
constexpr int HALF = 32;  // rows of a product

template <int DT, int D>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_key_weights_kernel(
    WeightsParams p) {
  using C = Cfg<DT, D>;
  using B16 = Cfg<DT_BF16, D>;  // rows in LDS
  constexpr int RB = C::RB, NB = KW_KEYS / (NW * 32), KEYS = 32 * NB, NQ = D / 16;
  constexpr int STEPS = KW_ROWS * C::NCH / (NW * 64);  // 16-byte chunks a thread copies
  static_assert(STEPS * NW * 64 == KW_ROWS * C::NCH && KW_ROWS == 2 * HALF, "tiles");
  __shared__ __attribute__((aligned(16))) uint8_t tile[2][KW_ROWS * B16::RB];
  __shared__ __attribute__((aligned(16))) float top[4][KW_ROWS];  // lse log2(e) of the row, +inf for none
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // (batch, KV head) innermost, so that the blocks of one run on one XCD where
  // their number is a multiple of 8 (workgroup ids go round-robin over the
  // XCDs), then key blocks: those that run at once read the same query rows,
  // from their XCD's L2.  The last rows first: with a causal mask the first ones
  // are seen by few blocks.
  int u = blockIdx.x;
  const int bh = u % (p.B * p.Hkv);
  u /= p.B * p.Hkv;
  const int block = u % p.blocks, part = p.parts - 1 - u / p.blocks;
  const int b = bh / p.Hkv, h = bh - b * p.Hkv;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  const int k0 = block * KW_KEYS;
  if (k0 >= n) return;
  const int shift = p.causal ? n - p.Sq : n;  // position i sees the keys up to shift + i

  // ---- tiles of this workgroup: of each run of rows (run innermost) those of
  // its part, from the first that sees key k0 on (runs of one head: in a packed
  // run positions repeat)
  const bool by_head = p.hrows == p.Sq;
  const int first = max(part * p.span, p.causal && by_head && k0 > shift ? (k0 - shift) / KW_ROWS : 0);
  const int end = min((part + 1) * p.span, (p.hrows + KW_ROWS - 1) / KW_ROWS);
  const int turns = max(end - first, 0) * p.heads;
  if (turns == 0 && p.parts > 1) {
    if (k0 + tid < n) p.part[((size_t)part * p.B * p.Hkv + bh) * (size_t)p.Sk + k0 + tid] = 0.0f;
    return;
  }

  // ---- keys: lane holds key 32 kb + i32
  const __amdgpu_buffer_rsrc_t krsrc = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(p.k + ((size_t)bh * (size_t)p.Sk_cap + (size_t)k0) * RB), (short)0, min(n - k0, KW_KEYS) * RB, BUF_DWORD3);
  RowOperand<DT, D> keys[NB];
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int t = 0; t < keys[kb].CHUNKS; ++t)
      keys[kb].set(t, __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                    krsrc, (wave * KEYS + 32 * kb + i32) * RB + 32 * t + 16 * g, 0, 0)));

  // ---- query rows of this (batch, KV head): heads * hrows consecutive ones.
  // Tile in flight: chunk `step * 256 + tid` of its rows, and each lane's row's
  // log-sum.  The loads have no branch, so that the waits can count
  // them: rows beyond the last read as zero and touch no memory.  (Rows beyond
  // the end of a run are the next run's; the masks leave them out.)
  const size_t row0 = ((size_t)b * p.Hq + (size_t)h * p.G) * (size_t)p.Sq;
  const int nrows = p.G * p.Sq;
  const __amdgpu_buffer_rsrc_t qrsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.q + row0 * RB), (short)0, nrows * RB, BUF_DWORD3);
  const __amdgpu_buffer_rsrc_t lrsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.lse + row0), (short)0, nrows * 4, BUF_DWORD3);
  i32x4 chunk[STEPS];
  float lse;
  int head = 0, pos = first * KW_ROWS;  // the next tile to load: run and first row there
  auto load = [&]() __attribute__((always_inline)) {
    const int row = min(head * p.hrows + pos, nrows);
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      chunk[i] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(qrsrc, (i * NW * 64 + tid) * 16, row * RB, 0));
    lse = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lrsrc, lane * 4, row * 4, 0));
    if (++head == p.heads) head = 0, pos += KW_ROWS;
  };
  auto store = [&](int slot, int slot4) __attribute__((always_inline)) {
    // rows that give nothing: their queries may hold anything
    static_assert(KW_ROWS == 64, "a lane a row");
    const unsigned long long none = __ballot(lse == -INFINITY);
    if (none) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
        if (none >> ((i * NW * 64 + tid) / C::NCH) & 1) chunk[i] = i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) store_row_chunk<DT, D>(tile[slot], i * NW * 64 + tid, chunk[i]);
    if (tid < KW_ROWS) top[slot4][tid] = lse != -INFINITY ? lse * 1.4426950408889634f : INFINITY;
  };

  float sum[NB] = {};
  const int kswz = k_swz<DT_BF16, D>(i32);
  const int key0 = k0 + wave * KEYS;  // this wave's first key
  // a lane's operands of the first half of tile 0; the others lie at constant offsets
  const uint8_t* qlane[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) qlane[t] = tile[0] + i32 * B16::RB + (((2 * t + g) ^ kswz) << 4);
  auto operand = [&](int slot, int half, int t) __attribute__((always_inline)) {
    return *(const bf16x8*)(qlane[t] + (slot * KW_ROWS + half * HALF) * B16::RB);
  };
  auto row_top = [&](f32x4 (&e)[4], int slot4, int half) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 4; ++x) e[x] = *(const f32x4*)&top[slot4][half * HALF + 8 * x + 4 * g];
  };
  // scores of half a tile with this wave's keys
  auto scores = [&](f32x16 (&s)[NB], int slot, int half) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const bf16x8 a = operand(slot, half, t);
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, keys[kb].x[t], t == 0 ? f32x16{0.0f} : s[kb], 0, 0, 0);
    }
  };
  // the weights of s (half a tile, of which `left` rows are real, the first in
  // row r0 of its run) added up, without those of keys that a row does not see
  auto weigh_masked = [&](f32x16 (&s)[NB], int slot4, int half, int r0, int left) __attribute__((always_inline)) {
    f32x4 e[4];
    row_top(e, slot4, half);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int r = 8 * (j >> 2) + 4 * g + (j & 3);
      const int at = by_head ? r0 + r : (r0 + r) % p.Sq;
      const int last = r >= left ? -1 : p.causal ? shift + at : n - 1;
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][j], p.c1, -e[j >> 2][j & 3]));
        sum[kb] += key0 + 32 * kb + i32 <= last ? w : 0.0f;
      }
    }
  };
  // the weights of s, all of which count, and between them the scores of
  // another half in s_next: a step, held in this order by the fences, has the
  // two products of 16 channels and a share of the 32 weights
  auto weigh_whole = [&](f32x16 (&s)[NB], int slot4, int half, f32x16 (&s_next)[NB], int slot_next,
                         int half_next) __attribute__((always_inline)) {
    constexpr int SHARE = 16 * NB / NQ;
    f32x4 e[4];
    row_top(e, slot4, half);
    bf16x8 a[NQ];
    a[0] = operand(slot_next, half_next, 0);
    a[1] = operand(slot_next, half_next, 1);
    a[2] = operand(slot_next, half_next, 2);
    float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      if (t + 3 < NQ) a[t + 3] = operand(slot_next, half_next, t + 3);
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
        s_next[kb] =
            __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[t], keys[kb].x[t], t == 0 ? f32x16{0.0f} : s_next[kb], 0, 0, 0);
#pragma unroll
      for (int x = t * SHARE; x < (t + 1) * SHARE; ++x) {
        const int kb = x >> 4, j = x & 15;
        part[x & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][j], p.c1, -e[j >> 2][j & 3]));
        if (j == 15) {
          sum[kb] += (part[0] + part[1]) + (part[2] + part[3]);
          part[0] = part[1] = part[2] = part[3] = 0.0f;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  int run = 0, at = first * KW_ROWS;  // the tile of this turn: its run and first row there
  auto half_turn = [&](f32x16 (&s)[NB], int slot4, int half, f32x16 (&s_next)[NB], int slot_next,
                       int half_next) __attribute__((always_inline)) {
    const int r0 = at + half * HALF, left = p.hrows - r0;
    // whole: every row of the half sees all of this wave's keys; none: no row any
    const bool whole = left >= HALF && key0 + KEYS <= n && (!p.causal || (by_head && key0 + KEYS - 1 <= shift + r0));
    const bool none = left <= 0 || key0 >= n || (p.causal && by_head && key0 > shift + r0 + HALF - 1);
    if (whole) {
      weigh_whole(s, slot4, half, s_next, slot_next, half_next);
    } else {
      if (!none) weigh_masked(s, slot4, half, r0, left);
      scores(s_next, slot_next, half_next);
    }
  };

  f32x16 s0[NB], s1[NB];
  load();
  store(0, 0);
  load();
  // the keys are waited for here: first used in the loop, they would have every
  // turn of it wait for the tile that it has just asked for
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int t = 0; t < NQ; ++t) asm volatile("" : "+v"(keys[kb].x[t]));
  lds_barrier();
  scores(s0, 0, 0);
  // Turn i: tile i + 1 to LDS, i + 2 on its way, the weights of tile i.  (Past
  // the barrier everyone has read the second half of tile i, and tile i + 1 is
  // whole.  Its slot was last read before the barrier of turn i - 1; its
  // log-sums have four slots, since the last ones are read after it.)
  auto turn = [&](int i4) __attribute__((always_inline)) {  // i4 = i % 4: every LDS address is a constant
    store((i4 + 1) & 1, (i4 + 1) & 3);
    load();
    half_turn(s0, i4, 0, s1, i4 & 1, 1);
    lds_barrier();
    half_turn(s1, i4, 1, s0, (i4 + 1) & 1, 0);
    if (++run == p.heads) run = 0, at += KW_ROWS;
  };
#pragma unroll 1
  for (int i = 0;; i += 4) {
    if (i >= turns) break;
    turn(0);
    if (i + 1 >= turns) break;
    turn(1);
    if (i + 2 >= turns) break;
    turn(2);
    if (i + 3 >= turns) break;
    turn(3);
  }
#pragma unroll
  for (int kb = 0; kb < NB; ++kb) {
    float x, y;
    with_partner(sum[kb], x, y);
    const float got = x + y;
    const int key = key0 + 32 * kb + i32;
    if (g == 0 && key < n) {
      if (p.parts > 1) {
        p.part[((size_t)part * p.B * p.Hkv + bh) * (size_t)p.Sk + key] = got;
      } else {
        float* const to = p.acc + (size_t)bh * p.Sk_cap + key;
        *to = (p.decay == 0.0f ? 0.0f : p.decay * *to) + got;
      }
    }
  }
}

// Up to KW_FEW_ROWS query rows of a KV head: they stay in LDS, and each wave
// streams its own run of keys past them, straight from memory into operand
// registers, the next unit of 64 keys on its way while one is weighed.  No
// barrier after the rows are in.  (Products between the weights, as above, gained
// 6% with 256 rows and cost a decode step 10%.)
template <int DT, int D>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_key_weights_few(
    WeightsParams p) {
  using C = Cfg<DT, D>;
  using B16 = Cfg<DT_BF16, D>;  // rows in LDS
  constexpr int RB = C::RB, KEYS = KW_FEW_KEYS, NB = KEYS / 32, CH = C::NCH / 2, NQ = D / 16;
  __shared__ __attribute__((aligned(16))) uint8_t rows[KW_FEW_ROWS * B16::RB];
  __shared__ __attribute__((aligned(16))) float top[KW_FEW_ROWS];  // lse log2(e) of the row, +inf for none
  __shared__ __attribute__((aligned(16))) int dead[NW];  // whether a wave's rows hold one with lse = -inf
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the blocks are rotated from one (batch, KV head) to the next: with a number
  // of them that is a multiple of 8 an XCD would always have the same ones, and
  // those behind the end of short caches would leave it idle (B16 8K, ragged: 50
  // -> 43 us with blocks of 24 units)
  const int bh = blockIdx.x / p.blocks, block = (blockIdx.x - bh * p.blocks + bh) % p.blocks;
  const int b = bh / p.Hkv, h = bh - b * p.Hkv;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  if (block * NW * p.span * KEYS >= n) return;
  const int k0 = (block * NW + wave) * p.span * KEYS;  // this wave's keys
  const int nk = max(min(n - k0, p.span * KEYS), 0);
  const size_t at = (size_t)bh * (size_t)p.Sk_cap + (size_t)(nk ? k0 : 0);
  const __amdgpu_buffer_rsrc_t krsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.k + at * RB), (short)0, nk * RB, BUF_DWORD3);
  const __amdgpu_buffer_rsrc_t arsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.acc + at), (short)0, p.decay == 0.0f ? 0 : nk * 4, BUF_DWORD3);
  // keys beyond the run read as zero and touch no memory
  i32x4 k[NB][CH];
  float old[NB];
  auto load = [&](int u) __attribute__((always_inline)) {
    const int row = min(u * KEYS, nk);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
      for (int t = 0; t < CH; ++t)
        k[kb][t] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                 krsrc, (32 * kb + i32) * RB + 32 * t + 16 * g, row * RB, 0));
      old[kb] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(arsrc, (32 * kb + i32) * 4, row * 4, 0));
    }
  };
  load(0);
  // ---- the query rows into LDS, 32 at a time; rows beyond the last are zero and
  // weigh nothing
  const int nrows = p.G * p.Sq, ntiles = (nrows + HALF - 1) / HALF;
  const size_t row0 = ((size_t)b * p.Hq + (size_t)h * p.G) * (size_t)p.Sq;
  const __amdgpu_buffer_rsrc_t qrsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.q + row0 * RB), (short)0, nrows * RB, BUF_DWORD3);
  const __amdgpu_buffer_rsrc_t lrsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)(p.lse + row0), (short)0, nrows * 4, BUF_DWORD3);
  // (four chunks of a thread are asked for before the first is stored; a single
  // tile has one or two)
  constexpr int BATCH = 4;
  for (int c0 = tid; ntiles > 1 && c0 - tid < ntiles * HALF * C::NCH; c0 += BATCH * NW * 64) {
    i32x4 x[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      x[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(qrsrc, (c0 + i * NW * 64) * 16, 0, 0));
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (c0 + i * NW * 64 < ntiles * HALF * C::NCH) store_row_chunk<DT, D>(rows, c0 + i * NW * 64, x[i]);
  }
  for (int c = tid; ntiles == 1 && c < HALF * C::NCH; c += NW * 64) {
    const i32x4 x = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(qrsrc, c * 16, 0, 0));
    store_row_chunk<DT, D>(rows, c, x);
  }
  if (tid < ntiles * HALF) {
    const float e = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lrsrc, tid * 4, 0, 0));
    const bool none = e == -INFINITY;
    top[tid] = tid < nrows && !none ? e * 1.4426950408889634f : INFINITY;
    const bool some = __ballot(none) != 0;
    if (lane == 0) dead[wave] = some ? 1 : 0;
  } else if (lane == 0) {
    dead[wave] = 0;
  }
  __syncthreads();
  const i32x4 any = *(const i32x4*)dead;
  if (any[0] | any[1] | any[2] | any[3]) {
    // rows that give nothing: their queries may hold anything
    for (int c = tid; c < ntiles * HALF * B16::NCH; c += NW * 64)
      if (top[c / B16::NCH] == INFINITY) *(i32x4*)(rows + c * 16) = i32x4{0, 0, 0, 0};
    __syncthreads();
  }
  const int open = p.causal ? n - p.Sq + 1 : n;  // keys from here on are not seen by every row
  const int kswz = k_swz<DT_BF16, D>(i32);
  const uint8_t* qlane[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) qlane[t] = rows + i32 * B16::RB + (((2 * t + g) ^ kswz) << 4);
#pragma unroll 1
  for (int u = 0; u * KEYS < nk; ++u) {
    const int key0 = k0 + u * KEYS;
    RowOperand<DT, D> keys[NB];
    float was[NB], sum[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
      for (int t = 0; t < CH; ++t) keys[kb].set(t, k[kb][t]);
#pragma unroll
      for (int t = 0; t < NQ; ++t) asm volatile("" : "+v"(keys[kb].x[t]));
      was[kb] = old[kb];
      sum[kb] = 0.0f;
    }
    load(u + 1);
#pragma unroll 1
    for (int tile = 0; tile < ntiles; ++tile) {
      f32x16 s[NB];
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const bf16x8 a = *(const bf16x8*)(qlane[t] + tile * HALF * B16::RB);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, keys[kb].x[t], t == 0 ? f32x16{0.0f} : s[kb], 0, 0, 0);
      }
      f32x4 e[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) e[x] = *(const f32x4*)&top[tile * HALF + 8 * x + 4 * g];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          s[kb][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][j], p.c1, -e[j >> 2][j & 3]));
        if (p.causal && key0 + KEYS > open) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int r = tile * HALF + 8 * (j >> 2) + 4 * g + (j & 3);
            if (key0 + 32 * kb + i32 >= open + r % p.Sq) s[kb][j] = 0.0f;
          }
        }
        float a[4] = {s[kb][0], s[kb][1], s[kb][2], s[kb][3]};
#pragma unroll
        for (int j = 4; j < 16; ++j) a[j & 3] += s[kb][j];
        sum[kb] += (a[0] + a[1]) + (a[2] + a[3]);
      }
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
      float x, y;
      with_partner(sum[kb], x, y);
      if (g == 0 && key0 + 32 * kb + i32 < n)
        p.acc[at + u * KEYS + 32 * kb + i32] = (p.decay == 0.0f ? 0.0f : p.decay * was[kb]) + (x + y);
    }
  }
}

// acc of each key from the sums of the row parts, in their order
__global__ __launch_bounds__(256) void attn_key_weights_add(WeightsParams p) {
  const int per = (p.Sk + 255) / 256;
  const int bh = blockIdx.x / per, key = (blockIdx.x - bh * per) * 256 + threadIdx.x;
  const int b = bh / p.Hkv;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  if (key >= n) return;
  float* const to = p.acc + (size_t)bh * p.Sk_cap + key;
  float sum = 0.0f;
  for (int i = 0; i < p.parts; ++i) sum += p.part[((size_t)i * p.B * p.Hkv + bh) * (size_t)p.Sk + key];
  *to = (p.decay == 0.0f ? 0.0f : p.decay * *to) + sum;
}
}  // namespace

namespace h15 {

int launch_weights(const WeightsParams& p, int dtype, int d, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)(p.B * p.Hkv * p.parts * p.blocks)), block(NW * 64);
  const bool few = p.G * p.Sq <= KW_FEW_ROWS;
  auto launch = [&](auto dt, auto dd) {
    constexpr int DT = decltype(dt)::value, D = decltype(dd)::value;
    if (few) hipLaunchKernelGGL((attn_key_weights_few<DT, D>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((attn_key_weights_kernel<DT, D>), grid, block, 0, st, p);
  };
  using I = std::integral_constant<int, DT_BF16>;
  using F = std::integral_constant<int, DT_FP8>;
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (dtype == ATTN_BF16) {
    if (d == 128) launch(I{}, D128{});
    else launch(I{}, D64{});
  } else {
    if (d == 128) launch(F{}, D128{});
    else launch(F{}, D64{});
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.parts > 1) {
    hipLaunchKernelGGL(attn_key_weights_add, dim3((unsigned)(p.B * p.Hkv * ((p.Sk + 255) / 256))), dim3(256), 0, st, p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
