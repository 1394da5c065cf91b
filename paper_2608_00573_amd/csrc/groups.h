// Rows sorted by group (expert): what every kernel over them derives from the groups'
// borders, which only the device knows.  Not part of the public ABI.
#pragma once

#include "gemm.h"

namespace trimmoe {

// offsets [E + 1] ascending (NULL: one group of all n rows).  Borders are held to
// [0, n] and each group to a non-empty range, so no border can lead out of the rows.
// Rows of no group lie before the first border (slot E + 1) and behind the last (slot
// E); `slots` counts them as groups where a kernel writes zeros there.
struct Groups {
  const int32_t* offsets;
  int E, n;
  __device__ __forceinline__ int2 rows(int e) const {  // first row, end
    if (!offsets) return e == 0 ? make_int2(0, n) : make_int2(n, n);
    const int last = min(max(offsets[E], 0), n);
    if (e == E) return make_int2(last, n);
    if (e == E + 1) return make_int2(0, min(min(max(offsets[0], 0), n), last));
    const int a = min(max(offsets[e], 0), n);
    return make_int2(a, max(a, min(max(offsets[e + 1], 0), n)));
  }
};
constexpr int kGroupSlots = TRIMMOE_MAX_EXPERTS + 2;

// The groups' row tiles: how many there are up to each group, in LDS
struct GroupTiles {
  int* first;  // [slots + 1]
  int slots;
  // by all threads of the block, which then may use it
  __device__ __forceinline__ void init(int* lds, const Groups& g, int n_slots, int tile) {
    first = lds;
    slots = n_slots;
    if (threadIdx.x < 64) {
      int sum = 0;
      for (int e0 = 0; e0 < n_slots; e0 += 64) {
        const int e = e0 + (int)threadIdx.x;
        int t = 0;
        if (e < n_slots) {
          const int2 r = g.rows(e);
          t = (r.y - r.x + tile - 1) / tile;
        }
        int s = t;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int up = __shfl_up(s, o);
          if ((int)threadIdx.x >= o) s += up;
        }
        if (e < n_slots) first[e] = sum + s - t;
        sum += __shfl(s, 63);
      }
      if (threadIdx.x == 0) first[n_slots] = sum;
    }
    __syncthreads();
  }
  __device__ __forceinline__ int total() const {
    return __builtin_amdgcn_readfirstlane(first[slots]);
  }
  // group of row tile t < total()
  __device__ __forceinline__ int group(int t) const {
    int lo = 0, hi = slots;  // first[lo] <= t < first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  }
};

// row tiles of n rows in E groups at most, with those of no group
inline long row_tiles_most(int n, int E, int tile) {
  const long more = (long)E + 2;
  return (n + tile - 1) / tile + (more < n ? more : n);
}

}  // namespace trimmoe
