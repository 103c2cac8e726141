// Device helpers of the tree kernels: who sees whom in a tree of drafted tokens, and where a cached token stands.
#ifndef RAZOR_TREE_CUH_
#define RAZOR_TREE_CUH_

#include <stdint.h>

#include "razor_spec.h"

namespace razor {

// The tree of one sequence in shared memory.  see[t]: bit n set when node n is node t or one of its ancestors; no bit
// at all for an absent node (a parent outside [-1, t), or an absent ancestor).
struct TreeMask {
  uint32_t see[kTreeMaxNodes][kTreeMaxNodes / 32];
  int32_t parent[kTreeMaxNodes];
  int32_t depth[kTreeMaxNodes];   // 0 for a node that follows the cached sequence directly
};

__device__ __forceinline__ void tree_mask_load(TreeMask& m, const int32_t* parent, int n_nodes, int tid, int n_threads) {
  for (int t = tid; t < n_nodes; t += n_threads) m.parent[t] = parent[t];
}
// A thread per node walks up to the root (a parent precedes its node, so the walk ends).  A barrier belongs between
// tree_mask_load and this, and one behind it.
__device__ __forceinline__ void tree_mask_walk(TreeMask& m, int n_nodes, int tid, int n_threads) {
  for (int t = tid; t < n_nodes; t += n_threads) {
    uint32_t w[kTreeMaxNodes / 32] = {};
    int n = t, depth = -1;
    while (n >= 0) {
#pragma unroll
      for (int k = 0; k < kTreeMaxNodes / 32; ++k) w[k] |= (n >> 5) == k ? 1u << (n & 31) : 0u;
      depth += 1;
      const int a = m.parent[n];
      if (a < -1 || a >= n) {   // absent
#pragma unroll
        for (int k = 0; k < kTreeMaxNodes / 32; ++k) w[k] = 0u;
        break;
      }
      n = a;
    }
#pragma unroll
    for (int k = 0; k < kTreeMaxNodes / 32; ++k) m.see[t][k] = w[k];
    m.depth[t] = depth;
  }
}
__device__ __forceinline__ bool tree_sees(const TreeMask& m, int t, int n) { return m.see[t][n >> 5] >> (n & 31) & 1u; }

// Position of the token in slot s of a head that has seen `total` tokens (Algorithm 1 keeps the sinks and a ring of the
// recent tokens).
__device__ __forceinline__ int slot_position(int s, int n_sink, const HeadState& st, int total) {
  if (st.window < 0 || st.n_drop == 0 || s < n_sink) return s;
  int j = s - n_sink - st.ring_head;
  if (j < 0) j += st.window;
  return total - st.window + j;
}

}  // namespace razor
#endif
