// Norms of queries and keys for each head with their position rotation
// (attn_rope), and the gradient of both (attn_rope_bwd).
//
// A row has d / 16 lanes of 16 channels each, two chunks of 16 bytes, chosen so
// that a lane has both channels of each of its 8 pairs: chunks l and l + rot / 16
// of the rotated channels for the half layout, l and l + d / 16 of all for the
// interleaved one (and of the channels that are not rotated, counted on their own).
// So a rotation takes no exchange between lanes, a norm's sum three (d = 128) or two,
// and each load of a wave covers whole runs of memory (2 x 4096 positions, interleaved: 35.6
// us, with neighbouring chunks 43.8).  A thread keeps its position and
// takes a run of heads one after the other: the sines and cosines of its 8 pairs are made
// once for all of them.
//
// Angles: turns = position * freq / 2 pi in FP64 (off by 2^-53 of it, 2^-23 of a
// turn at the farthest position), less the nearest whole number, and then the
// sine and cosine instructions, which take turns (off by at most 1.3e-7 over
// half a turn to either side).
//
// Everything between the operand and the one rounding of the output is FP32.
//
// What bounds it: HBM (2 x 4096 positions, 32 heads over 8, d = 128, norms: 201 MB in 37.4 us,
// 5.4 TB/s, where a large copy reaches 4.9 to 5.2; its gradient at 4 x 2048 positions: 285 MB in
// 63 us, 4 of them for the weights' sums), and the launch for a few positions (one of each of 64
// sequences 4.2 us).  Holding the gradient to 128 registers for a fourth wave on each
// SIMD costs more than the wave gives (64 us for 55 with inputs in cache).
#include "qkv_params.h"
#include "attn_device.h"

namespace {

// A thread's place: the channels of its two chunks, and its 8 pairs.
template <int D, bool INTER>
struct Place {
  static constexpr int LPR = D / 16;
  int c0, c1;
  bool r0, r1;  // the first four pairs are rotated, and the others
  int l;
  __device__ __forceinline__ Place(const RopeParams& p, bool turned) {
    const int rot = turned ? p.rot : 0;
    l = threadIdx.x % LPR;
    if constexpr (INTER) {
      c0 = 8 * l, c1 = D / 2 + 8 * l;
      r0 = c0 < rot, r1 = c1 < rot;
    } else {
      r0 = r1 = 16 * l < rot;
      c0 = r0 ? 8 * l : rot / 2 + 8 * l;
      c1 = r0 ? rot / 2 + 8 * l : D / 2 + 8 * l;
    }
  }
  // f(j, pair) for the rotated ones
  template <typename F>
  __device__ __forceinline__ void rotated_pairs(F f) const {
    if constexpr (INTER) {
      if (r0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f(j, 4 * l + j);
      }
      if (r1) {
#pragma unroll
        for (int j = 4; j < 8; ++j) f(j, D / 4 + 4 * l + j - 4);
      }
    } else if (r0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f(j, 8 * l + j);
    }
  }
};

// Cosines and sines of a thread's pairs, times the amplitude.
struct Turn {
  float c[8], s[8];
  template <typename P>
  __device__ __forceinline__ void set(const RopeParams& p, const P& at, int b, int s_at) {
    const double pos = !p.positions      ? (double)s_at
                       : p.each_position ? (double)p.positions[(size_t)b * p.S + s_at]
                                         : (double)p.positions[b] + (double)s_at;
    const double turns = pos * 0.15915494309189535;
    at.rotated_pairs([&](int j, int pair) __attribute__((always_inline)) {
      double t = turns * p.freqs[pair];
      t -= __builtin_rint(t);
      c[j] = p.amplitude * __builtin_amdgcn_cosf((float)t);
      s[j] = p.amplitude * __builtin_amdgcn_sinf((float)t);
    });
  }
};

// x turned by the angles (BACK: by their negatives).  A pair's channels among a thread's
// 16: neighbours if interleaved, else the same of both chunks.
template <bool INTER, bool BACK, typename P>
__device__ __forceinline__ void rotate(float (&x)[16], const Turn& t, const P& at) {
  at.rotated_pairs([&](int j, int) __attribute__((always_inline)) {
    const int a = INTER ? 2 * j : j, b = INTER ? 2 * j + 1 : 8 + j;
    const float xa = x[a], xb = x[b], s = BACK ? -t.s[j] : t.s[j];
    x[a] = __builtin_fmaf(xa, t.c[j], -(xb * s));
    x[b] = __builtin_fmaf(xb, t.c[j], xa * s);
  });
}

__device__ __forceinline__ void widen16(float (&x)[16], u32x4 a, u32x4 b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16);
    x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    x[8 + 2 * i] = __uint_as_float(b[i] << 16);
    x[8 + 2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
  }
}

// 16 bytes that are read once (a prompt of 201 MB in and out 43.3 us without the hint,
// 37.5 so, 39.9 with the outputs' stores hinted, too, which the attention reads next; its
// gradient 67.7 / 62)
__device__ __forceinline__ u32x4 stream_in(const uint16_t* p) { return __builtin_nontemporal_load((const u32x4*)p); }

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ u32x4 pack8(const float* x) {
  return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
}

// +-448 at most; NaN stays (the median of a NaN and two numbers is one of them)
__device__ __forceinline__ float held(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f); }
__device__ __forceinline__ u32x2 pack8_fp8(const float* x, float inv) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(held(x[4 * i] * inv), held(x[4 * i + 1] * inv), 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(held(x[4 * i + 2] * inv), held(x[4 * i + 3] * inv), w, true);
  }
  return r;
}

// Sum over a row's lanes, 8 or 4 neighbours, on the VALU: lanes i ^ 1, i ^ 2, and
// the other four of eight.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xF, 0xF, true));
}
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  if constexpr (D == 128) x += dpp<0x141>(x);
  return x;
}

// mean x^2 + eps
template <int D>
__device__ __forceinline__ float mean_square(const float (&x)[16], float eps) {
  float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i & 3] = __builtin_fmaf(x[i], x[i], a[i & 3]);
  return __builtin_fmaf(row_sum<D>((a[0] + a[1]) + (a[2] + a[3])), 1.0f / D, eps);
}

// f and `down` with f * down = 1 / sqrt(mean x^2 + eps) and x times `down`, so that x f is
// the normalised row.  `down` is 1, and 2^-70 for a row whose mean (or eps) leaves FP32: the
// squares of BF16's largest values add up to less than 2^124 then, and what other channels
// lose below FP32 is less than BF16's least step, before the weight.  (All lanes of a row see
// the same mean.)
template <int D>
__device__ __forceinline__ float inverse_rms(float (&x)[16], float eps, float& down) {
  float mean = mean_square<D>(x, eps);
  down = 1.0f;
  if (mean == INFINITY) {
    down = 0x1p-70f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= down;
    mean = mean_square<D>(x, eps * 0x1p-140f);
    // (an infinity is among them: a root of 0 would make zeros of the others)
    if (mean == INFINITY) mean = __builtin_nanf("");
  }
  return __builtin_amdgcn_rsqf(mean);
}

// A thread's 16 weights.
__device__ __forceinline__ void load_weights(float (&w)[16], const void* from, bool bf16, int c0, int c1) {
  if (bf16) {
    const uint16_t* f = (const uint16_t*)from;
    widen16(w, *(const u32x4*)(f + c0), *(const u32x4*)(f + c1));
  } else {
    const float* f = (const float*)from;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = f[c0 + i], w[8 + i] = f[c1 + i];
  }
}

// Where a thread's two loads and stores of 16 bytes lie.
//   OWN    its own chunks;
//   MIXED  chunks l and l + d / 16 of its row, where a part of the head in halves would
//          leave each load of a wave runs of memory in both lines of a row of 128 channels
//          (2 x 4096 positions, 32 channels: 42.5 -> 37.5 us, their gradient 66 -> 56.5);
//   ROWS   a chunk of a row, and the same of the one 8 positions on, where a load of 64
//          channels' chunks would take half of each row's line (2 x 4096 positions: 24.8 ->
//          19.7 us, their gradient with norms 36.4 -> 31.6).
// In the last two a wave's threads exchange them in LDS, whose instructions a wave carries
// out in order.
enum { OWN = 0, MIXED = 1, ROWS = 2 };

template <int D, bool INTER, int KIND>
struct Memory {
  static constexpr int BYTES = KIND == OWN ? 16 : ROPE_THREADS * 32;
  int t0, t1, c0, c1;  // tokens (ROWS) and channels
  bool on;
  u32x4* slots;  // the wave's 128
  int f0, f1, k0, k1;
  __device__ __forceinline__ Memory(const Place<D, INTER>& at, bool mixed, uint8_t* lds)
      : t0(0), t1(0), c0(at.c0), c1(at.c1), on(KIND == ROWS || (KIND == MIXED && mixed)) {
    if constexpr (KIND != OWN) {
      const int lane = threadIdx.x & 63;
      slots = (u32x4*)lds + (threadIdx.x >> 6) * 128;
      const int row = lane / (D / 16) * (D / 8);
      k0 = row + at.c0 / 8, k1 = row + at.c1 / 8;
      if constexpr (KIND == ROWS) {
        f0 = lane, f1 = lane + 64;
        t0 = (threadIdx.x >> 6) * 16 + (lane >> 3), t1 = t0 + 8;
        c0 = c1 = 8 * (lane & 7);
      } else {
        f0 = row + at.l, f1 = f0 + D / 16;
        if (on) c0 = 8 * at.l, c1 = D / 2 + 8 * at.l;
      }
    }
  }
  __device__ __forceinline__ void pass(u32x4& a, u32x4& b, int from0, int from1, int to0, int to1) const {
    slots[from0] = a, slots[from1] = b;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    a = slots[to0], b = slots[to1];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
  // what was loaded, into the thread's own chunks; and back
  __device__ __forceinline__ void own(u32x4& a, u32x4& b) const {
    if constexpr (KIND != OWN)
      if (on) pass(a, b, f0, f1, k0, k1);
  }
  __device__ __forceinline__ void back(u32x4& a, u32x4& b) const {
    if constexpr (KIND != OWN)
      if (on) pass(a, b, k0, k1, f0, f1);
  }
};

// A thread's tokens of a tile: its own, and those of its loads and stores (beyond the
// last one: the last, and nothing is stored).
template <int D, int KIND>
struct Tokens {
  int own, m0, m1;
  bool live, w0, w1;
  template <typename M>
  __device__ __forceinline__ Tokens(const M& mem, int tile, int total) {
    const int first = tile * rope_tokens(D);
    own = first + threadIdx.x / (D / 16);
    live = own < total;
    own = min(own, total - 1);
    m0 = m1 = own;
    w0 = w1 = live;
    if constexpr (KIND == ROWS) {
      w0 = first + mem.t0 < total, w1 = first + mem.t1 < total;
      m0 = min(first + mem.t0, total - 1), m1 = min(first + mem.t1, total - 1);
    }
  }
};

// Offsets of a token's row of head h in [B][S][H][d] of the strides and in [B][H][S][d]
__device__ __forceinline__ int64_t strided(const RopeParams& p, int64_t sb, int64_t ss, int token) {
  const int b = token / p.S;
  return (int64_t)b * sb + (int64_t)(token - b * p.S) * ss;
}
__device__ __forceinline__ size_t plain(const RopeParams& p, int heads, int h, int D, int token) {
  const int b = token / p.S;
  return (((size_t)b * heads + h) * (size_t)p.S + (token - b * p.S)) * D;
}

// Tensor and first head of the run of heads `r`.
__device__ __forceinline__ int tensor_of(const RopeParams& p, int& r) {
  int i = 0;
  while (i < 2 && r >= p.t[i].runs) r -= p.t[i++].runs;
  return i;
}

template <int D, int DT, bool INTER, int KIND>
__global__ __launch_bounds__(ROPE_THREADS) void attn_rope_kernel(RopeParams p) {
  using Mem = Memory<D, INTER, KIND>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[Mem::BYTES];
  int r = blockIdx.y;
  const RopeTensor& t = p.t[tensor_of(p, r)];
  const Place<D, INTER> at(p, t.turned);
  const Mem mem(at, t.turned, lds);
  const Tokens<D, KIND> k(mem, blockIdx.x, p.B * p.S);
  if (KIND != ROWS && !k.live) return;  // (a row's lanes leave together)
  const int b = k.own / p.S, s = k.own - b * p.S, h0 = r * t.run, h1 = min(h0 + t.run, t.heads);
  const uint16_t* i0 = t.in + strided(p, t.sb, t.ss, k.m0) + (int64_t)h0 * t.sh + mem.c0;
  const uint16_t* i1 = i0 + (mem.c1 - mem.c0);
  if constexpr (KIND == ROWS) i1 = t.in + strided(p, t.sb, t.ss, k.m1) + (int64_t)h0 * t.sh + mem.c1;
  u32x4 a0 = stream_in(i0), a1 = stream_in(i1);
  Turn turn;
  turn.set(p, at, b, s);
  float w[16];
  if (t.weight) load_weights(w, t.weight, p.weight_bf16, at.c0, at.c1);
  size_t o = plain(p, t.heads, h0, D, k.own), o0 = o + mem.c0, o1 = o + mem.c1;
  if constexpr (KIND == ROWS) o0 = plain(p, t.heads, h0, D, k.m0) + mem.c0, o1 = plain(p, t.heads, h0, D, k.m1) + mem.c1;
  const size_t next = (size_t)p.S * D;
#pragma unroll 1
  for (int h = h0; h < h1; ++h, o += next, o0 += next, o1 += next) {
    float x[16];
    mem.own(a0, a1);
    widen16(x, a0, a1);
    if (h + 1 < h1) {
      i0 += t.sh;
      i1 += t.sh;
      a0 = stream_in(i0);
      a1 = stream_in(i1);
    }
    if (t.weight) {
      float down;
      const float f = inverse_rms<D>(x, p.eps, down);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * f * w[i];
    }
    rotate<INTER, false>(x, turn, at);
    if constexpr (DT == DT_BF16) {
      uint16_t* out = (uint16_t*)t.out;
      u32x4 y0 = pack8(x), y1 = pack8(x + 8);
      mem.back(y0, y1);
      if (KIND != ROWS || k.w0) *(u32x4*)(out + o0) = y0;
      if (KIND != ROWS || k.w1) *(u32x4*)(out + o1) = y1;
    } else if (KIND != ROWS || k.live) {
      uint8_t* out = (uint8_t*)t.out + o;
      *(u32x2*)(out + at.c0) = pack8_fp8(x, t.inv);
      *(u32x2*)(out + at.c1) = pack8_fp8(x + 8, t.inv);
    }
  }
}

// A workgroup takes every groups-th tile of positions for its run of heads; its
// part of a weight's gradient is one row of the workspace.
template <int D, bool INTER, int KIND>
__global__ __launch_bounds__(ROPE_THREADS) void attn_rope_bwd_kernel(RopeParams p) {
  using Mem = Memory<D, INTER, KIND>;
  constexpr int LPR = D / 16, TOKENS = rope_tokens(D);
  __shared__ float sums[TOKENS][D + 4];
  __shared__ __attribute__((aligned(16))) uint8_t lds[Mem::BYTES];
  int r = blockIdx.y;
  const RopeTensor& t = p.t[tensor_of(p, r)];
  const Place<D, INTER> at(p, t.turned);
  const Mem mem(at, t.turned && p.rot < D, lds);
  const int h0 = r * t.run, h1 = min(h0 + t.run, t.heads);
  float w[16], dw[16];
  if (t.weight) load_weights(w, t.weight, p.weight_bf16, at.c0, at.c1);
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i] = 0.0f;
#pragma unroll 1
  for (int tile = blockIdx.x; tile < p.tiles; tile += p.groups) {
    const Tokens<D, KIND> k(mem, tile, p.B * p.S);
    if (KIND != ROWS && !k.live) break;
    const int b = k.own / p.S, s = k.own - b * p.S;
    const int64_t far = mem.c1 - mem.c0;
    const uint16_t* g0 = (const uint16_t*)t.out + plain(p, t.heads, h0, D, k.m0) + mem.c0;
    const uint16_t* g1 = KIND == ROWS ? (const uint16_t*)t.out + plain(p, t.heads, h0, D, k.m1) + mem.c1 : g0 + far;
    const uint16_t* i0 = t.in + strided(p, t.sb, t.ss, k.m0) + (int64_t)h0 * t.sh + mem.c0;
    const uint16_t* i1 = KIND == ROWS ? t.in + strided(p, t.sb, t.ss, k.m1) + (int64_t)h0 * t.sh + mem.c1 : i0 + far;
    uint16_t* d0 = t.grad + strided(p, t.gb, t.gs, k.m0) + (int64_t)h0 * t.gh + mem.c0;
    uint16_t* d1 = KIND == ROWS ? t.grad + strided(p, t.gb, t.gs, k.m1) + (int64_t)h0 * t.gh + mem.c1 : d0 + far;
    u32x4 a0 = stream_in(g0), a1 = stream_in(g1), x0, x1;
    if (t.weight) x0 = stream_in(i0), x1 = stream_in(i1);
    Turn turn;
    turn.set(p, at, b, s);
#pragma unroll 1
    for (int h = h0; h < h1; ++h, d0 += t.gh, d1 += t.gh) {
      float e[16], u[16];
      mem.own(a0, a1);
      widen16(e, a0, a1);
      if (t.weight) {
        mem.own(x0, x1);
        widen16(u, x0, x1);
      }
      if (h + 1 < h1) {
        g0 += (size_t)p.S * D;
        g1 += (size_t)p.S * D;
        a0 = stream_in(g0);
        a1 = stream_in(g1);
        if (t.weight) {
          i0 += t.sh;
          i1 += t.sh;
          x0 = stream_in(i0);
          x1 = stream_in(i1);
        }
      }
      rotate<INTER, true>(e, turn, at);
      if (t.weight) {
        float down, m = 0.0f;
        const float f = inverse_rms<D>(u, p.eps, down);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          u[i] *= f;
          if (KIND != ROWS || k.live) dw[i] = __builtin_fmaf(e[i], u[i], dw[i]);
          e[i] *= w[i];
          m = __builtin_fmaf(e[i], u[i], m);
        }
        m = row_sum<D>(m) * (1.0f / D);
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = f * __builtin_fmaf(-m, u[i], e[i]);
        if (down != 1.0f) {
#pragma unroll
          for (int i = 0; i < 16; ++i) e[i] *= down;
        }
      }
      u32x4 y0 = pack8(e), y1 = pack8(e + 8);
      mem.back(y0, y1);
      if (KIND != ROWS || k.w0) *(u32x4*)d0 = y0;
      if (KIND != ROWS || k.w1) *(u32x4*)d1 = y1;
    }
  }
  if (!t.weight) return;
  float* const mine = sums[threadIdx.x / LPR];
#pragma unroll
  for (int i = 0; i < 8; ++i) mine[at.c0 + i] = dw[i], mine[at.c1 + i] = dw[8 + i];
  __syncthreads();
  if ((int)threadIdx.x < D) {
    float a = 0.0f;
#pragma unroll 8
    for (int i = 0; i < TOKENS; ++i) a += sums[i][threadIdx.x];
    p.part[((size_t)t.partials + (size_t)r * p.groups + blockIdx.x) * D + threadIdx.x] = a;
  }
}

// A weight's gradient from its workgroups' parts: 32 channels a workgroup, 128 parts
// at a time.
constexpr int SUM_THREADS = 1024;
template <int D>
__global__ __launch_bounds__(SUM_THREADS) void attn_rope_bwd_sum(RopeParams p) {
  constexpr int ROWS = SUM_THREADS / 8;
  __shared__ f32x4 sums[ROWS][8];
  const RopeTensor& t = p.t[blockIdx.y];
  if (!t.dweight) return;
  const int col = threadIdx.x & 7, row = threadIdx.x >> 3, n = t.runs * p.groups;
  const float* from = p.part + (size_t)t.partials * D + blockIdx.x * 32 + col * 4;
  f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = row; i < n; i += ROWS) {
    const f32x4 x = *(const f32x4*)(from + (size_t)i * D);
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] += x[e];
  }
  sums[row][col] = a;
  __syncthreads();
  // 128 -> 4 rows by a thread each, then one
  if (threadIdx.x < 128) {
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    float x = 0.0f;
#pragma unroll 8
    for (int i = 0; i < ROWS / 4; ++i) x += sums[q * (ROWS / 4) + i][c >> 2][c & 3];
    __syncthreads();
    ((float*)sums)[threadIdx.x] = x;
  } else {
    __syncthreads();
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const float* x = (const float*)sums + threadIdx.x;
    t.dweight[blockIdx.x * 32 + threadIdx.x] = (x[0] + x[32]) + (x[64] + x[96]);
  }
}

template <int D, int DT>
void launch_forward(const RopeParams& p, dim3 grid, hipStream_t st) {
  const dim3 block(ROPE_THREADS);
  constexpr int DIRECT = D == 64 ? ROWS : OWN, PART = D == 64 ? ROWS : MIXED;
  const bool part = p.rot > 0 && p.rot < D;
  // (the exchange's branches alone would cost a whole head in halves 2 us of 37)
  if (p.interleaved) hipLaunchKernelGGL((attn_rope_kernel<D, DT, true, DIRECT>), grid, block, 0, st, p);
  else if (part) hipLaunchKernelGGL((attn_rope_kernel<D, DT, false, PART>), grid, block, 0, st, p);
  else hipLaunchKernelGGL((attn_rope_kernel<D, DT, false, DIRECT>), grid, block, 0, st, p);
}

template <int D>
void launch_backward(const RopeParams& p, dim3 grid, hipStream_t st) {
  const dim3 block(ROPE_THREADS);
  if (p.interleaved) hipLaunchKernelGGL((attn_rope_bwd_kernel<D, true, D == 64 ? ROWS : OWN>), grid, block, 0, st, p);
  else hipLaunchKernelGGL((attn_rope_bwd_kernel<D, false, D == 64 ? ROWS : MIXED>), grid, block, 0, st, p);
  if (p.t[0].dweight || p.t[1].dweight)
    hipLaunchKernelGGL((attn_rope_bwd_sum<D>), dim3(D / 32, 2), dim3(SUM_THREADS), 0, st, p);
}
}  // namespace

namespace h15 {

int launch_rope(const RopeParams& p, int dtype, void* stream) {
  const dim3 grid((unsigned)p.tiles, (unsigned)(p.t[0].runs + p.t[1].runs + p.t[2].runs));
  hipStream_t st = (hipStream_t)stream;
  if (dtype == ATTN_BF16) p.d == 128 ? launch_forward<128, DT_BF16>(p, grid, st) : launch_forward<64, DT_BF16>(p, grid, st);
  else p.d == 128 ? launch_forward<128, DT_FP8>(p, grid, st) : launch_forward<64, DT_FP8>(p, grid, st);
  return hipGetLastError() == hipSuccess ? 0 : 1;
}

int launch_rope_bwd(const RopeParams& p, void* stream) {
  const dim3 grid((unsigned)p.groups, (unsigned)(p.t[0].runs + p.t[1].runs + p.t[2].runs));
  hipStream_t st = (hipStream_t)stream;
  p.d == 128 ? launch_backward<128>(p, grid, st) : launch_backward<64>(p, grid, st);
  return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace h15
