// Products of the training losses in fp32 matrix instructions: the tile (device
// code) and the launchers of products.hip.  Not part of the public ABI.
#pragma once

#include <algorithm>

#include "gemm.h"

namespace trimmoe {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ------------------------------------------------------------ fp32 products --
// C = A B^T in v_mfma_f32_32x32x2_f32 over operands of either order: K-contiguous
// ([rows][K]) or row-contiguous ([K][rows]), any leading dimension and
// alignment.  128 x 128 tiles of 4 wavefronts (64 x 64 each); 16-deep K slices
// go through registers into a k-major LDS image (two buffers, the next slice's
// loads in flight under the MFMAs), so a fragment read is 32 consecutive floats
// and the order of the operand in memory only changes how a slice is written.
namespace f32p {
constexpr int BM = 128, BN = 128, KS = 16, THREADS = 256;
constexpr int LS = 132;  // floats of an LDS row: four lanes of one row, 4 k apart, hit distinct banks
}  // namespace f32p

// operand: `rows` x K elements of type T.  KC: element (r, k) at r ld + k,
// else at k ld + r
template <typename T, bool KC>
struct Operand {
  const T* p;
  size_t ld;
  int rows, K;
  bool vec;  // groups of four elements are aligned
};

template <typename T>
struct alignas(4 * sizeof(T)) Vec4 {
  T e[4];
};

template <typename T, bool KC>
inline Operand<T, KC> operand(const void* p, size_t ld, int rows, int K) {
  const bool vec = ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0;
  return Operand<T, KC>{static_cast<const T*>(p), ld, rows, K, vec};
}

// this thread's eight elements of slice k0 of the tile's rows from r0
template <typename T, bool KC>
__device__ __forceinline__ void load_slice(const Operand<T, KC>& o, int r0, int k0, int k_end,
                                           float (&x)[2][4]) {
  using namespace f32p;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int r, k, lim;
    if constexpr (KC) {
      r = r0 + (threadIdx.x >> 2) + 64 * i;
      k = k0 + 4 * (threadIdx.x & 3);
      lim = r < o.rows ? k_end - k : 0;
    } else {
      k = k0 + (threadIdx.x >> 4);
      r = r0 + 4 * (threadIdx.x & 15) + 64 * i;
      lim = k < k_end ? o.rows - r : 0;
    }
    const T* p = o.p + (KC ? (size_t)r * o.ld + k : (size_t)k * o.ld + r);
    if (o.vec && lim >= 4) {
      const Vec4<T> v = *reinterpret_cast<const Vec4<T>*>(p);
#pragma unroll
      for (int u = 0; u < 4; ++u) x[i][u] = to_f32<T>(v.e[u]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) x[i][u] = u < lim ? to_f32<T>(p[u]) : 0.f;
    }
  }
}

template <bool KC>
__device__ __forceinline__ void store_slice(float* s, const float (&x)[2][4]) {
  using namespace f32p;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (KC) {
      const int r = (threadIdx.x >> 2) + 64 * i, k = 4 * (threadIdx.x & 3);
#pragma unroll
      for (int u = 0; u < 4; ++u) s[(k + u) * LS + r] = x[i][u];
    } else {
      const int k = threadIdx.x >> 4, r = 4 * (threadIdx.x & 15) + 64 * i;
      *reinterpret_cast<float4*>(s + k * LS + r) = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
    }
  }
}

using F32Acc = f32x16_t[2][2];

// acc = tile (rows r0 of A, rows n0 of B) over K [k0, k_end)
template <typename TA, bool AK, typename TB, bool BKC>
__device__ __forceinline__ void f32_tile(const Operand<TA, AK>& A, const Operand<TB, BKC>& B, int r0,
                                         int n0, int k0, int k_end, float* lds, F32Acc& acc) {
  using namespace f32p;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int ra = (wave >> 1) * 64 + (lane & 31), rb = (wave & 1) * 64 + (lane & 31), kk = lane >> 5;
  constexpr int BUF = 2 * KS * LS;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x16_t{};
  float xa[2][4], xb[2][4];
  load_slice(A, r0, k0, k_end, xa);
  load_slice(B, n0, k0, k_end, xb);
  store_slice<AK>(lds, xa);
  store_slice<BKC>(lds + KS * LS, xb);
  __syncthreads();
  int buf = 0;
  for (int k = k0; k < k_end; k += KS) {
    const bool more = k + KS < k_end;
    if (more) {
      load_slice(A, r0, k + KS, k_end, xa);
      load_slice(B, n0, k + KS, k_end, xb);
    }
    const float* sa = lds + buf * BUF;
    const float* sb = sa + KS * LS;
#pragma unroll
    for (int s = 0; s < KS; s += 2) {
      float fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = sa[(s + kk) * LS + ra + 32 * i];
        fb[i] = sb[(s + kk) * LS + rb + 32 * i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
    if (more) {
      store_slice<AK>(lds + (buf ^ 1) * BUF, xa);
      store_slice<BKC>(lds + (buf ^ 1) * BUF + KS * LS, xb);
    }
    __syncthreads();
    buf ^= 1;
  }
}

// tile row / column of accumulator element r of acc[i][j]
__device__ __forceinline__ int f32_row(int i, int r) {
  return ((int)threadIdx.x >> 7) * 64 + 32 * i + 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3);
}
__device__ __forceinline__ int f32_col(int j) {
  return ((threadIdx.x >> 6) & 1) * 64 + 32 * j + (threadIdx.x & 31);
}

// K splits of an m x n product over K on a 256-CU device: tiles for two blocks a
// CU, each at least 256 deep
inline int product_splits(int m, int n, int K) {
  const long tiles = (long)cdiv(m, f32p::BM) * cdiv(n, f32p::BN);
  int s = 1;
  while (s < 64 && tiles * s < 512 && K / (2 * s) >= 256) s *= 2;
  return s;
}

// out [A.rows, B.rows] = A B^T in `splits` runs of K: rounded to TO, or (TO =
// float) one slice of partials per run, added to what the slices hold (`add`)
template <typename TO, typename TA, bool AK, typename TB, bool BKC>
hipError_t launch_product(const Operand<TA, AK>& A, const Operand<TB, BKC>& B, int splits, bool add,
                          TO* out, hipStream_t st);

// out = sum of the S slices of n partials, rounded once
template <typename T>
hipError_t launch_sum_parts(const float* part, int S, size_t n, T* out, hipStream_t st);

}  // namespace trimmoe
