// Attention of trees of drafted tokens over a paged cache: the kernel of attend.cuh with the nodes' bits for masks, in a
// translation unit of its own (either takes some ten seconds to compile).
#include "attend.cuh"

namespace misat {

int attend_tree_prepare(const misat_kv* kv) { return allow_pool<true>(kv); }

void launch_attend_tree(const misat_kv* kv, const runs::AttendArgs& a, const CUtensorMap& map_q, cudaStream_t st) {
  launch_pool<true>(kv, a, map_q, st);
}

}  // namespace misat
