// Host-side interface between the C entry points of h15cache.h (cache_api.cpp:
// argument checks, cuts, workspaces, plain C++) and their gfx950 kernels
// (h15prefix.hip, h15weights.hip, h15evict.hip).  Nothing here depends on HIP,
// so the argument checks also build with a host compiler alone.
#ifndef H15ATTN_CACHE_PARAMS_H
#define H15ATTN_CACHE_PARAMS_H

#include <stddef.h>
#include <stdint.h>

#include "attn_params.h"

namespace h15 {

// Query rows of a prefix workgroup whose waves share each tile of keys.
constexpr int PREFIX_ROWS = 4 * WROWS;

// Keys and query rows of a key-weights workgroup: four waves of 64 keys each,
// a tile of 64 query rows at a time.
constexpr int KW_KEYS = 4 * 64;
constexpr int KW_ROWS = 64;

// Up to this many query rows of a KV head stay in LDS (64 KB of it at d = 128,
// so that two workgroups share a compute unit), and each wave streams units of
// KW_FEW_KEYS keys past them.  Times of a call so / in the form of more rows (8 KV
// heads, BF16 d = 128): 2 caches of 16K keys, 4 rows 14 / 20 us, 64 16 / 22, 128 22 /
// 28, 256 rows as 4 heads of 64 positions 33 / 32, as 8 heads of 32 33 / 43, as one
// head 40 / 30; 16 caches of 8K, 4 rows 45 / 58, 128 61 / 85, 256 as 4 heads 93 / 97, as
// 16 heads 93 / 165, as one 109 / 96.  FP8 likewise.
constexpr int KW_FEW_ROWS = 256;
constexpr int KW_FEW_KEYS = 64;

// Decode over a shared prefix and each sequence's own cache.
struct PrefixParams {
  const uint8_t* q;
  const uint8_t* kp;  // [Hkv][P_cap][d]
  const uint8_t* vp;
  const uint8_t* k;  // [B][Hkv][Sk_cap][d]
  const uint8_t* v;
  const int32_t* lens;  // [B], or NULL: Sk keys each
  uint16_t* o;
  float* lse;
  float* part_o;   // [rows][parts][d], unnormalised O of each part (several parts)
  float* part_ml;  // [rows][parts][2], (m, l) of each part (several parts)
  int B, Hq, Hkv, Sq, G, R;  // R = G Sq: query rows of a sequence and KV head
  int P, P_cap, Sk, Sk_cap, causal;
  int p_parts, p_split;  // parts of the prefix (0: no prefix) and their keys
  int o_parts, o_split;  // parts of the own caches (0: none) and their keys
  int parts;             // p_parts + o_parts (chained: 1)
  int longest;           // own caches are taken in the order of their lengths (B <= 256)
  int chain;             // a workgroup of an own cache takes the prefix first (one part of each)
  int p_rows;            // query rows of a prefix workgroup: PREFIX_ROWS or WROWS
  int p_blocks, o_blocks;  // row blocks of a KV head's rows of all sequences, of one sequence
  int p_groups, o_groups;  // workgroups
  float c1, ck, vd;
};

// The attention weight that each cached key receives.
struct WeightsParams {
  const uint8_t* q;
  const uint8_t* k;
  const float* lse;
  const int32_t* lens;
  float* acc;
  float* part;  // [parts][B Hkv][Sk], several parts only
  int B, Hq, Hkv, Sq, G, Sk, Sk_cap, causal;
  int heads, hrows;  // runs of query rows that tiles stay within, and rows of each
  // row parts, their tiles of each run, blocks of KW_KEYS keys; with up to
  // KW_FEW_ROWS rows: 1, a wave's units of keys, blocks of 4 span units
  int parts, span, blocks;
  float c1, decay;
};

// A selection's parts have a multiple of EVICT_PART keys each, EVICT_PART_MOST of them
// at most; what its launches hand on about one.
constexpr int EVICT_PART = 4096;
constexpr int EVICT_PART_MOST = 15 * EVICT_PART;
constexpr int EVICT_PART_BYTES = 4 * (2 * 1024 + 512 + 4);

// The keys that stay in each cache.
struct EvictParams {
  const uint8_t* k;
  const uint8_t* v;
  const float* acc;
  const int32_t* lens;
  uint8_t* k_out;
  uint8_t* v_out;
  float* acc_out;
  int32_t* index;
  int32_t* lens_out;
  int B, Hkv, Sk, Sk_cap, keep, recent, out_cap, row_bytes;
  uint8_t* scratch;  // [B Hkv][parts] of EVICT_PART_BYTES (several parts only)
  int parts;         // of part_keys keys, a workgroup each
  int part_keys;
  int gather;        // the selecting workgroup copies the rows, too: no second launch
};

// Launchers, as those of attn_params.h.  The caller has checked every argument.
int launch_prefix(const PrefixParams& p, int dtype, int d, int mode, void* stream);
int launch_weights(const WeightsParams& p, int dtype, int d, void* stream);
int launch_evict(const EvictParams& p, void* stream);

}  // namespace h15

#endif  // H15ATTN_CACHE_PARAMS_H
