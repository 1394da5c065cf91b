// Rows sorted by group (expert): what every kernel over them derives from the groups'
// borders, which only the device knows.  Not part of the public ABI.
#pragma once

#include "gemm.h"

namespace trimmoe {

// offsets [E + 1] ascending (NULL: one group of all n rows).  Borders are held to
// [0, n] and a group's end to its begin or more, so no border can lead out of the rows.
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

constexpr int kGroupChunks = (TRIMMOE_MAX_EXPERTS + 2 + 63) / 64;

// The groups' row tiles: lane l holds how many there are before groups l, 64 + l, ...
// (in registers: the large tiles leave no LDS)
struct GroupTiles {
  int first[kGroupChunks], n;
  __device__ __forceinline__ GroupTiles(const Groups& g, int slots, int tile) {
    const int lane = threadIdx.x & 63;
    n = 0;
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c) {
      first[c] = INT32_MAX;
      if (64 * c >= slots) continue;
      const int e = 64 * c + lane;
      int t = 0;
      if (e < slots) {
        const int2 r = g.rows(e);
        t = (r.y - r.x + tile - 1) / tile;
      }
      int s = t;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(s, o);
        if (lane >= o) s += up;
      }
      if (e < slots) first[c] = n + s - t;
      n += __builtin_amdgcn_readlane(s, 63);
    }
    // (borders that do not ascend could make more of them)
    n = min(n, g.n / tile + slots);
  }
  // group of row tile t < n, and the tile's number within it
  __device__ __forceinline__ int group(int t, int& within) const {
    int e = -1;
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c) e += (int)__popcll(__ballot(first[c] <= t));
    int f = 0;
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c)
      if (e >> 6 == c) f = __builtin_amdgcn_readlane(first[c], e & 63);
    within = t - f;
    return e;
  }
};

// The groups by their rows, most first (ties: the lower one): a launch whose tiles take
// their group's rows as K then ends on its shortest tiles
struct GroupOrder {
  int rank[kGroupChunks];
  __device__ __forceinline__ explicit GroupOrder(const Groups& g) {
    const int lane = threadIdx.x & 63;
    int rows[kGroupChunks];
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c) {
      rank[c] = INT32_MAX;
      if (64 * c >= g.E) continue;
      rows[c] = -1;
      if (64 * c + lane < g.E) {
        const int2 r = g.rows(64 * c + lane);
        rows[c] = r.y - r.x;
        rank[c] = 0;
      }
    }
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c)
      for (int l = 0; l < 64 && 64 * c + l < g.E; ++l) {
        const int other = __builtin_amdgcn_readlane(rows[c], l);
#pragma unroll
        for (int k = 0; k < kGroupChunks; ++k)
          if (64 * k < g.E && 64 * k + lane < g.E)
            rank[k] += other > rows[k] || (other == rows[k] && 64 * c + l < 64 * k + lane) ? 1 : 0;
      }
  }
  __device__ __forceinline__ int group(int r) const {
    int e = 0;
#pragma unroll
    for (int c = 0; c < kGroupChunks; ++c) {
      const unsigned long long m = __ballot(rank[c] == r);
      if (m) e = 64 * c + __ffsll(m) - 1;
    }
    return __builtin_amdgcn_readfirstlane(e);
  }
};

// Tiles of E groups, `per` each, dealt to a grid: every group's tiles are cut into one
// run per XCD (block b runs on XCD b % 8), the groups in order, the longer runs passed
// on from XCD to XCD.  Block i of an XCD takes every bx-th of its tiles from i on.
struct GroupWalk {
  int E, nx, bx, q, r;
  int rank, run, left;  // the next tile: its group's rank, the XCD's run there, its place in it
  __device__ __forceinline__ GroupWalk(int per, int E_) : E(E_), rank(0) {
    nx = min(8, (int)gridDim.x);
    run = blockIdx.x % nx;
    left = blockIdx.x / nx;
    bx = ((int)gridDim.x - run + nx - 1) / nx;
    // (the compiler divides in vector registers)
    run = __builtin_amdgcn_readfirstlane(run);
    left = __builtin_amdgcn_readfirstlane(left);
    bx = __builtin_amdgcn_readfirstlane(bx);
    q = __builtin_amdgcn_readfirstlane(per / nx);
    r = per - q * nx;
    settle();
  }
  __device__ __forceinline__ int length() const { return q + (run < r ? 1 : 0); }
  __device__ __forceinline__ void settle() {
    while (rank < E && left >= length()) {
      left -= length();
      run = run + 1 == nx ? 0 : run + 1;
      ++rank;
    }
  }
  __device__ __forceinline__ bool more() const { return rank < E; }
  __device__ __forceinline__ int tile() const { return run * q + min(run, r) + left; }  // of the group's
  __device__ __forceinline__ void next() {
    left += bx;
    settle();
  }
};

// row tiles of n rows in E groups at most, with those of no group
inline long row_tiles_most(int n, int E, int tile) {
  const long more = (long)E + 2;
  return (n + tile - 1) / tile + (more < n ? more : n);
}

}  // namespace trimmoe
