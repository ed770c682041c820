// sdv_tree.cuh - drafted trees: nodes in an order in which parents come before their children.
#pragma once

#include <cstdint>

#include "../../include/specdiff.h"

namespace sdv {

static_assert(SDV_MAX_TREE == 64, "a node's ancestors are the bits of a word, a warp holds two nodes a lane");

// A node's parent, or -1 for one without: a root, or (bad) one whose parent does not come before it.
__device__ __forceinline__ int parent_of(int p, int node, bool& bad) {
  if (p >= 0 && p < node) return p;
  bad |= p != -1;
  return -1;
}

// The ancestors of nodes lane and 32 + lane, themselves among them, by a warp: bit j for node j.  Each round joins a node's
// set with that of the node it has come to and doubles the way that it has come.
__device__ __forceinline__ void ancestors(int p0, int p1, int lane, uint64_t& a0, uint64_t& a1) {
  a0 = 1ull << lane;
  a1 = 1ull << (32 + lane);
#pragma unroll 1
  for (int round = 0; round < 6; ++round) {
    const auto at = [&](int p, uint64_t& set, int& next) {
      const uint64_t lo = __shfl_sync(0xffffffffu, a0, p & 31), hi = __shfl_sync(0xffffffffu, a1, p & 31);
      const int nlo = __shfl_sync(0xffffffffu, p0, p & 31), nhi = __shfl_sync(0xffffffffu, p1, p & 31);
      set = p < 0 ? 0ull : p < 32 ? lo : hi;
      next = p < 0 ? -1 : p < 32 ? nlo : nhi;
    };
    uint64_t s0, s1;
    int n0, n1;
    at(p0, s0, n0);
    at(p1, s1, n1);
    a0 |= s0;
    a1 |= s1;
    p0 = n0;
    p1 = n1;
  }
}

}  // namespace sdv
