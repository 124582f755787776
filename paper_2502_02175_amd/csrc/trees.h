// Ways through a tree of drafted tokens.
#pragma once
#include "common.h"

#ifdef __HIPCC__
// The nodes on the way from node `from` on, along the links (link_of(t), asked for with t from 0 to VLAC_TREE_MAX_NODES - 1; negative: the
// way ends there).  UP: links lead to nodes before their own, else behind.  A wave follows it: lane k has the bits of nodes 64 k .. 64 k + 63
// in `way`, and all have what it ends with.  Nodes go by 64 at a time, and their links are doubled, as are the sets of nodes that a
// link skips: a chain of 64 takes 6 rounds of three trips between lanes.  (A thread that walks through LDS, scalar reads of lanes one by
// one, this, us.  The choice of 32000 for a chain of 64: 21.5, 13.0, 11.6; the path accepted of 8 trees, 5 of 31 nodes: 2.6, 2.6, 2.8;
// 64 of 64: 5.4, 4.1, 2.9; 512 of 512: 28, 17.7, 7.9.)
template <bool UP, class F>
__device__ inline int follow(int from, F link_of, uint64_t& way) {
  const int lane = threadIdx.x & 63;
  way = 0;
  int x = from;
  while (x >= 0) {
    const int b = x & ~63, at = x & 63, to = link_of(b + lane);
    int link = to >= b && to < b + 64 ? to - b : -1;  // (inside the 64)
    uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);  // this node and those on its way to the link
    while (__builtin_amdgcn_readlane(link, at) >= 0) {
      const int other = link >= 0 ? link : lane;
      lo |= __shfl(lo, other);
      hi |= __shfl(hi, other);
      link = __shfl(link, other);
    }
    const uint64_t part = (uint64_t)__builtin_amdgcn_readlane(hi, at) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, at);
    if (lane == b >> 6) way = part;
    x = __builtin_amdgcn_readlane(to, UP ? __ffsll((unsigned long long)part) - 1 : 63 - __clzll((long long)part));
  }
  return x;
}
// ... and the bits of nodes 64 k .. 64 k + 63, in all lanes
__device__ inline uint64_t part_of(uint64_t way, int k) {
  return (uint64_t)__builtin_amdgcn_readlane((uint32_t)(way >> 32), k) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)way, k);
}
#endif
