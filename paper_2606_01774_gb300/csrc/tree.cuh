// A drafted tree's paths, by one warp.
#pragma once

#include <stdint.h>

namespace flare {

constexpr int kMaxNodes = 64;  // nodes of a tree, a bit each in a 64-bit set

__device__ __forceinline__ uint64_t shfl64(uint64_t x, int src) {
  const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)x, src);
  const uint32_t hi = __shfl_sync(0xffffffffu, (uint32_t)(x >> 32), src);
  return (uint64_t)hi << 32 | lo;
}

// Parents of nodes lane and lane + 32 (-1 past n); whether the row is a tree in
// topological order with node 0 its only root.  Called by a whole warp.
__device__ __forceinline__ bool warp_load_tree(const int32_t* __restrict__ parent, int n, int& p0,
                                               int& p1) {
  const int lane = threadIdx.x & 31;
  p0 = lane < n ? parent[lane] : -1;
  p1 = lane + 32 < n ? parent[lane + 32] : -1;
  bool ok = lane >= n || (lane == 0 ? p0 == -1 : (p0 >= 0 && p0 < lane));
  ok = ok && (lane + 32 >= n || (p1 >= 0 && p1 < lane + 32));
  return __all_sync(0xffffffffu, ok);
}

// A log-gate as it enters a path's sum.  From -104 down the gate is zero in fp32, and
// a larger sum would only lose the digits of the other gates: weights along a path
// are differences of two sums (-1e9 at a reset would leave none).  A NaN stays one.
__device__ __forceinline__ float tree_log_gate(float g) { return g < -104.f ? -104.f : g; }

// The paths of nodes lane and lane + 32 as bit sets (itself and its ancestors;
// empty past n), by pointer doubling: after k rounds a set holds the 2^k
// nearest members.  x0 and x1 become their sums over the paths.  The parents
// must have passed warp_load_tree.  NODES = 32: no node has an upper half.
template <int NODES>
__device__ __forceinline__ void warp_paths(int n, int p0, int p1, uint64_t& a0, uint64_t& a1,
                                           float& x0, float& x1) {
  const int lane = threadIdx.x & 31;
  a0 = lane < n ? 1ull << lane : 0ull;
  a1 = lane + 32 < n ? 1ull << (lane + 32) : 0ull;
#pragma unroll 1
  while (__any_sync(0xffffffffu, p0 >= 0 || p1 >= 0)) {
    const uint64_t l0 = shfl64(a0, p0 & 31), h0 = shfl64(a1, p0 & 31);
    const float xl0 = __shfl_sync(0xffffffffu, x0, p0 & 31);
    const float xh0 = __shfl_sync(0xffffffffu, x1, p0 & 31);
    const int ql0 = __shfl_sync(0xffffffffu, p0, p0 & 31);
    const int qh0 = __shfl_sync(0xffffffffu, p1, p0 & 31);
    if constexpr (NODES > 32) {
      const uint64_t l1 = shfl64(a0, p1 & 31), h1 = shfl64(a1, p1 & 31);
      const float xl1 = __shfl_sync(0xffffffffu, x0, p1 & 31);
      const float xh1 = __shfl_sync(0xffffffffu, x1, p1 & 31);
      const int ql1 = __shfl_sync(0xffffffffu, p0, p1 & 31);
      const int qh1 = __shfl_sync(0xffffffffu, p1, p1 & 31);
      if (p1 >= 0) {
        a1 |= p1 < 32 ? l1 : h1;
        x1 += p1 < 32 ? xl1 : xh1;
        p1 = p1 < 32 ? ql1 : qh1;
      }
    }
    if (p0 >= 0) {
      a0 |= p0 < 32 ? l0 : h0;
      x0 += p0 < 32 ? xl0 : xh0;
      p0 = p0 < 32 ? ql0 : qh0;
    }
  }
}

__device__ __forceinline__ void warp_paths(int n, int p0, int p1, uint64_t& a0, uint64_t& a1) {
  float x0 = 0.f, x1 = 0.f;
  warp_paths<kMaxNodes>(n, p0, p1, a0, a1, x0, x1);
}

}  // namespace flare
