// Launchers for host-only builds of the entry points over shared and bounded
// caches (tests/test_cache_host.py): they launch nothing, count their calls,
// report a launch error, and keep the parameters of the last call.
#include <stdint.h>

#include "cache_params.h"

static int g_launches = 0;
static h15::PrefixParams g_prefix;
static h15::WeightsParams g_weights;
static h15::EvictParams g_evict;

namespace h15 {

int launch_prefix(const PrefixParams& p, int, int, int, void*) { return g_prefix = p, ++g_launches, 1; }
int launch_weights(const WeightsParams& p, int, int, void*) { return g_weights = p, ++g_launches, 1; }
int launch_evict(const EvictParams& p, void*) { return g_evict = p, ++g_launches, 1; }

}  // namespace h15

extern "C" {
int h15_stub_launches(void) { return g_launches; }
int h15_stub_prefix(int what) {
  const int v[] = {g_prefix.p_parts, g_prefix.o_parts, g_prefix.p_rows, g_prefix.p_groups, g_prefix.o_groups,
                   g_prefix.p_split, g_prefix.o_split, g_prefix.causal, g_prefix.chain, g_prefix.longest};
  return v[what];
}
int h15_stub_evict(int what) { return what == 0 ? g_evict.parts : g_evict.gather; }
int h15_stub_weights(int what) {
  const int v[] = {g_weights.heads, g_weights.hrows, g_weights.parts, g_weights.blocks, g_weights.causal};
  return v[what];
}
}
