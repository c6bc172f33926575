// Host-side interface between the C entry points of h15qkv.h (qkv_api.cpp:
// argument checks, launch shapes, workspaces, plain C++) and their gfx950 kernels
// (h15rope.hip, h15append.hip, h15blocks.hip).  Nothing here depends on HIP, so
// the argument checks also build with a host compiler alone.
#ifndef H15ATTN_QKV_PARAMS_H
#define H15ATTN_QKV_PARAMS_H

#include <stddef.h>
#include <stdint.h>

#include "attn_params.h"

namespace h15 {

// Threads of a rope workgroup; d / 16 of them share a row.
constexpr int ROPE_THREADS = 256;
constexpr int rope_tokens(int d) { return ROPE_THREADS / (d / 16); }  // positions of a workgroup

// One of q, k, v (or its gradient) on its way.
struct RopeTensor {
  const uint16_t* in;  // [B][S][H][d] of the strides (backward: x, where there is a weight)
  void* out;           // [B][H][S][d] (backward: the incoming gradient)
  uint16_t* grad;      // backward: dx, [B][S][H][d] of the strides
  const void* weight;
  float* dweight;      // backward
  int64_t sb, ss, sh;  // strides of in
  int64_t gb, gs, gh;  // strides of grad
  float inv;           // 1 / descale
  int heads;           // 0: absent
  int runs;            // runs of `run` heads or fewer, each a workgroup's
  int run;             // heads that a thread takes one after the other
  int turned;          // rotated (q and k)
  int partials;        // first of its rows of partial sums in the workspace
};

struct RopeParams {
  RopeTensor t[3];
  const int32_t* positions;
  const double* freqs;
  float* part;  // backward: [groups][d] of the tensors with a weight
  int each_position, rot, interleaved, weight_bf16;
  float amplitude, eps;
  int B, S, d;
  int tiles;   // tiles of rope_tokens(d) positions
  int groups;  // workgroups of a run of heads: each takes every groups-th tile
};

// Writing new rows into a cache of 8-bit blocks.
struct AppendParams {
  const uint16_t* x[2];  // k, v
  uint8_t* cache[2];
  uint8_t* scales;
  const int32_t* lens;
  const int32_t* counts;
  int32_t* lens_out;
  int B, Hkv, n, cap, blocks;  // blocks: of a head's cache
  int reach;                   // blocks that n rows can lie in
};

// Query rows of a workgroup whose waves share each tile of keys.
constexpr int BLOCKS_ROWS = 4 * WROWS;
// Query rows of the wide form's, whose waves have two blocks of WROWS each.
constexpr int BLOCKS_WIDE = 16 * WROWS;

// Attention over a cache of 8-bit blocks.
struct BlocksParams {
  const uint8_t* q;
  const uint8_t* k;  // [B][Hkv][Sk_cap][d]
  const uint8_t* v;
  const uint8_t* scales;  // [B][Hkv][blocks][2]
  const int32_t* lens;
  uint16_t* o;
  float* lse;
  float* part_o;   // [rows][parts][d], unnormalised O of each part (several parts)
  float* part_ml;  // [rows][parts][2], (m, l) of each part (several parts)
  int B, Hq, Hkv, Sq, G, R;  // R = G Sq: query rows of a sequence and KV head
  int Sk, Sk_cap, causal;
  int blocks, shift;  // blocks of a head's cache, log2 of their keys
  int parts, split;   // parts and their keys
  int turn;           // log2 of 8 / gcd(8, parts)
  int rows;           // query rows of a workgroup: WROWS, BLOCKS_ROWS or BLOCKS_WIDE
  int row_blocks;     // of a sequence and KV head
  int longest;        // caches are taken in the order of their lengths (B <= 256)
  int stream;         // keys are read with a streaming hint (keys form)
  int groups;
  float c1, ck;
};

// Launchers, as those of attn_params.h.  The caller has checked every argument.
int launch_rope(const RopeParams& p, int dtype, void* stream);
int launch_rope_bwd(const RopeParams& p, void* stream);
int launch_append(const AppendParams& p, int d, int block, bool in_place, void* stream);
int launch_blocks(const BlocksParams& p, int d, int mode, void* stream);

}  // namespace h15

#endif  // H15ATTN_QKV_PARAMS_H
