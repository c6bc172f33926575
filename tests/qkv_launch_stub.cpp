// Launchers for host-only builds of the entry points of h15qkv.h
// (tests/test_qkv_host.py): they launch nothing, count their calls, report a
// launch error, and keep the parameters of the last call.
#include <stdint.h>

#include "qkv_params.h"

static int g_launches = 0, g_in_place = 0;
static h15::RopeParams g_rope;
static h15::AppendParams g_append;
static h15::BlocksParams g_blocks;

namespace h15 {

int launch_rope(const RopeParams& p, int, void*) { return g_rope = p, ++g_launches, 1; }
int launch_rope_bwd(const RopeParams& p, void*) { return g_rope = p, ++g_launches, 1; }
int launch_append(const AppendParams& p, int, int, bool in_place, void*) {
  return g_append = p, g_in_place = in_place, ++g_launches, 1;
}
int launch_blocks(const BlocksParams& p, int, int, void*) { return g_blocks = p, ++g_launches, 1; }

}  // namespace h15

extern "C" {
int h15_stub_qkv_launches(void) { return g_launches; }
int h15_stub_rope(int what) {
  const int v[] = {g_rope.tiles, g_rope.t[0].run, g_rope.groups, g_rope.t[0].runs, g_rope.t[1].runs, g_rope.t[2].runs,
                   g_rope.t[0].partials, g_rope.t[1].partials, g_rope.weight_bf16, g_rope.t[1].run, g_rope.t[2].run};
  return v[what];
}
int h15_stub_append(int what) {
  const int v[] = {g_append.blocks, g_append.reach, g_in_place};
  return v[what];
}
int h15_stub_blocks(int what) {
  const int v[] = {g_blocks.parts, g_blocks.split, g_blocks.rows, g_blocks.row_blocks, g_blocks.groups,
                   g_blocks.causal, g_blocks.longest, g_blocks.blocks, g_blocks.shift, g_blocks.stream};
  return v[what];
}
}
