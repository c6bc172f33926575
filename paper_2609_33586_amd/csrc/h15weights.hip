// The attention weight that each cached key receives (attn_key_weights):
//   acc[b][hkv][j] = decay acc[b][hkv][j]
//                    + sum over the G query heads and their rows i that see j
//                      of exp(scale q_i . k_j - lse_i).
//
// S = Q K^T with the query rows as the matrix rows, so that a lane's 16 scores
// belong to one key and to 16 rows: their sum is 15 additions in the lane, and
// the two halves of a wave meet once at the end.
//
// One workgroup = 4 waves for 256 keys of one (batch, KV head), 64 keys a wave,
// which stay in registers, against a run of tiles of 32 query rows.  A tile
// (and each row's log-sum and last visible key) passes through LDS, where all
// four waves read it: two copies, the next tile being written while one is
// read, a third on its way in registers, one barrier a tile.  With few query
// rows the call reads K once and HBM bounds it; with many, a score costs an
// exponential, an fma and an addition on the VALU beside its share of the
// matrix core's work.
//
// FP8 operands are widened to BF16 (exact) on their way to LDS and registers:
// the FP8 products sum less exactly than the FP32 sums promised.
//
// Long runs of query rows are cut into parts, which write their sums to a
// workspace; a second launch adds them up in their order, so results do not
// depend on timing.
#include "cache_params.h"
#include "unit_device.h"

namespace {

constexpr int NW = 4;

template <int DT, int D>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_key_weights_kernel(
    WeightsParams p) {
  using C = Cfg<DT, D>;
  using B16 = Cfg<DT_BF16, D>;  // rows in LDS
  constexpr int RB = C::RB, NB = 2, NQ = D / 16;
  constexpr int STEPS = (KW_ROWS * C::NCH + NW * 64 - 1) / (NW * 64);  // 16-byte chunks a thread copies
  __shared__ __attribute__((aligned(16))) uint8_t tile[2][KW_ROWS * B16::RB];
  __shared__ __attribute__((aligned(16))) float top[2][KW_ROWS];  // lse log2(e) of the row, +inf for none
  __shared__ __attribute__((aligned(16))) int last[2][KW_ROWS];   // its last visible key
  const int tid = threadIdx.x, lane = tid & 63, i32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // key blocks outermost: with a causal mask the first ones see the most rows,
  // and the longest workgroups start first
  int u = blockIdx.x;
  const int bh = u % (p.B * p.Hkv);
  u /= p.B * p.Hkv;
  const int part = u % p.parts, block = u / p.parts;
  const int b = bh / p.Hkv, h = bh - b * p.Hkv;
  const int n = p.lens ? min(max(p.lens[b], 0), p.Sk) : p.Sk;
  const int k0 = block * KW_KEYS;
  if (k0 >= n) return;
  const int shift = p.causal ? n - p.Sq : n;  // position i sees the keys up to shift + i

  // ---- tiles of this workgroup: of each run of rows those from the first row
  // that sees key k0 (runs of one head: in a packed run positions repeat)
  const bool by_head = p.hrows == p.Sq;
  const int first = p.causal && by_head && k0 > shift ? (k0 - shift) / KW_ROWS : 0;
  const int end = (p.hrows + KW_ROWS - 1) / KW_ROWS, per = max(end - first, 0);
  const int total = p.heads * per;
  const int u0 = (int)((long long)total * part / p.parts), u1 = (int)((long long)total * (part + 1) / p.parts);

  // ---- keys: lane holds key 32 kb + i32
  const __amdgpu_buffer_rsrc_t krsrc = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(p.k + ((size_t)bh * (size_t)p.Sk_cap + (size_t)k0) * RB), (short)0, min(n - k0, KW_KEYS) * RB, BUF_DWORD3);
  RowOperand<DT, D> keys[NB];
#pragma unroll
  for (int kb = 0; kb < NB; ++kb)
#pragma unroll
    for (int t = 0; t < keys[kb].CHUNKS; ++t)
      keys[kb].set(t, __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                    krsrc, (wave * 64 + 32 * kb + i32) * RB + 32 * t + 16 * g, 0, 0)));

  // ---- query rows of this (batch, KV head): heads * hrows consecutive ones
  const size_t row0 = ((size_t)b * p.Hq + (size_t)h * p.G) * (size_t)p.Sq;
  const uint8_t* const qrows = p.q + row0 * RB;
  const float* const lrows = p.lse + row0;
  // Tile in flight: chunk `step * 256 + tid` of its rows, and the row's log-sum
  // (threads 0..31).  Rows beyond the run are zero and see no key.
  struct Tile {
    int row, pos, left;  // first row, its position (runs of one head), rows from there to the run's end
  };
  i32x4 chunk[STEPS];
  float lse = 0.0f;
  int head = per ? u0 / per : 0, it = per ? u0 - head * per + first : 0;  // the next tile to load
  auto load = [&](Tile& t) __attribute__((always_inline)) {
    t.pos = it * KW_ROWS;
    t.row = head * p.hrows + t.pos;
    t.left = p.hrows - t.pos;
    const int bytes = min(t.left, KW_ROWS) * RB;
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc((void*)(qrows + (size_t)t.row * RB), (short)0, bytes, BUF_DWORD3);
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      chunk[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (i * NW * 64 + tid) * 16, 0, 0));
    if (tid < KW_ROWS && tid < t.left) lse = lrows[t.row + tid];
    if (++it == end) it = first, ++head;
  };
  auto store = [&](const Tile& t, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int ch = i * NW * 64 + tid, r = ch / C::NCH, c = ch % C::NCH;
      if (STEPS * NW * 64 > KW_ROWS * C::NCH && r >= KW_ROWS) break;
      uint8_t* const row = tile[slot] + r * B16::RB;
      const int swz = k_swz<DT_BF16, D>(r);
      if constexpr (DT == DT_BF16) {
        *(i32x4*)(row + ((c ^ swz) << 4)) = chunk[i];
      } else {
        // operand order of RowOperand: chunk 2 t + g holds the operands 2 t and
        // 2 t + 1 of half g, which lie at 2 (2 t) + g and 2 (2 t + 1) + g
        const int t2 = c >> 1, g2 = c & 1;
        *(bf16x8*)(row + (((4 * t2 + g2) ^ swz) << 4)) = widen(chunk[i][0], chunk[i][1]);
        *(bf16x8*)(row + (((4 * t2 + 2 + g2) ^ swz) << 4)) = widen(chunk[i][2], chunk[i][3]);
      }
    }
    if (tid < KW_ROWS) {
      const bool real = tid < t.left;
      top[slot][tid] = real && lse != -INFINITY ? lse * 1.4426950408889634f : INFINITY;
      last[slot][tid] = !real ? -1 : !p.causal ? n - 1 : shift + (by_head ? t.pos + tid : (t.row + tid) % p.Sq);
    }
  };
  float sum[NB] = {0.0f, 0.0f};
  const int kswz = k_swz<DT_BF16, D>(i32);
  const int key0 = k0 + wave * 64;  // this wave's first key
  Tile now = {}, next = {};
  if (u0 < u1) {
    load(now);
    store(now, 0);
    if (u0 + 1 < u1) load(next);
  }
  __syncthreads();
#pragma unroll 1
  for (int x = u0; x < u1; ++x) {
    const int slot = (x - u0) & 1;
    // whole: every row of the tile sees all of this wave's keys; none: no row any
    const bool whole = now.left >= KW_ROWS && key0 + 64 <= n && (!p.causal || (by_head && key0 + 63 <= shift + now.pos));
    const bool none = key0 >= n || (p.causal && by_head && key0 > shift + now.pos + KW_ROWS - 1);
    if (!none) {
      const uint8_t* const q = tile[slot] + i32 * B16::RB;
      f32x16 s[NB];
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const bf16x8 a = *(const bf16x8*)(q + (((2 * t + g) ^ kswz) << 4));
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, keys[kb].x[t], t == 0 ? f32x16{0.0f} : s[kb], 0, 0, 0);
      }
      f32x4 e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = *(const f32x4*)&top[slot][8 * i + 4 * g];
#pragma unroll
      for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          s[kb][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][j], p.c1, -e[j >> 2][j & 3]));
        if (!whole) {
          const int key = key0 + 32 * kb + i32;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (key > last[slot][8 * (j >> 2) + 4 * g + (j & 3)]) s[kb][j] = 0.0f;
        }
        float a[4] = {s[kb][0], s[kb][1], s[kb][2], s[kb][3]};
#pragma unroll
        for (int j = 4; j < 16; ++j) a[j & 3] += s[kb][j];
        sum[kb] += (a[0] + a[1]) + (a[2] + a[3]);
      }
    }
    if (x + 1 < u1) {
      now = next;
      store(now, slot ^ 1);
      if (x + 2 < u1) load(next);
    }
    __syncthreads();
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
  if (dtype == ATTN_BF16) {
    if (d == 128) hipLaunchKernelGGL((attn_key_weights_kernel<DT_BF16, 128>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((attn_key_weights_kernel<DT_BF16, 64>), grid, block, 0, st, p);
  } else {
    if (d == 128) hipLaunchKernelGGL((attn_key_weights_kernel<DT_FP8, 128>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((attn_key_weights_kernel<DT_FP8, 64>), grid, block, 0, st, p);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.parts > 1) {
    hipLaunchKernelGGL(attn_key_weights_add, dim3((unsigned)(p.B * p.Hkv * ((p.Sk + 255) / 256))), dim3(256), 0, st, p);
    e = hipGetLastError();
  }
  return e == hipSuccess ? 0 : 1;
}

}  // namespace h15
