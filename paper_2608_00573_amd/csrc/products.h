// Products of the training losses in fp32 matrix instructions: the tile (device
// code) and the launchers of products.hip.  Not part of the public ABI.
#pragma once

#include <algorithm>
#include <type_traits>

#include "gemm.h"

namespace trimmoe {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ------------------------------------------------------------ fp32 products --
// C = A B^T in v_mfma_f32_16x16x4_f32 over operands of either order: K-contiguous
// ([rows][K]) or row-contiguous ([K][rows]), any leading dimension and
// alignment.  128 x 128 tiles of 4 wavefronts (64 x 64 each); 16-deep K slices
// go through registers into a k-major LDS image (two buffers, the next slice's
// loads in flight under the MFMAs), so a fragment read is 32 consecutive floats
// and the order of the operand in memory only changes how a slice is written.
namespace f32p {
constexpr int BM = 128, BN = 128, KS = 16, THREADS = 256;
// floats of an LDS row (one k); every fourth row starts 16 floats further on.  The
// 4 rows of 16 that a fragment reads hit distinct banks, and so do the four lanes
// that write one operand row's 16 k.
constexpr int LS = 176;
__device__ __forceinline__ constexpr int row(int k) { return k * LS + 16 * ((k >> 2) & 3); }
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

// This thread's part of an operand's slices: N groups of four elements, rows from
// r0.  Whole slices of aligned operands inside their bounds take one load a group;
// the others test every element (past the bounds: zeros).
template <int N, typename T, bool KC>
struct Fetch {
  const T* p[N];
  int lim[N];  // KC: > 0 for a valid row; else elements from r on that are valid
  int k;       // KC: first k of the thread's groups, else its row's k
  size_t step;
  bool whole;
  __device__ __forceinline__ Fetch(const Operand<T, KC>& o, int r0, int k0) {
    step = KC ? (size_t)f32p::KS : (size_t)f32p::KS * o.ld;
    whole = o.vec && r0 + 64 * N <= o.rows;
    k = k0 + (KC ? 4 * (threadIdx.x & 3) : threadIdx.x >> 4);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + 64 * i + (KC ? threadIdx.x >> 2 : 4 * (threadIdx.x & 15));
      lim[i] = o.rows - r;
      p[i] = o.p + (KC ? (size_t)min(r, o.rows - 1) * o.ld + k : (size_t)k * o.ld + r);
    }
    vec = o.vec;
  }
  bool vec;
  // the slice that begins at k0, and on to the next one
  __device__ __forceinline__ void next(int k0, int k_end, float (&x)[N][4]) {
    if (whole && k0 + f32p::KS <= k_end) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Vec4<T> v = *reinterpret_cast<const Vec4<T>*>(p[i]);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[i][u] = to_f32<T>(v.e[u]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = KC ? (lim[i] > 0 ? k_end - k : 0) : (k < k_end ? lim[i] : 0);
        if (vec && n >= 4) {
          const Vec4<T> v = *reinterpret_cast<const Vec4<T>*>(p[i]);
#pragma unroll
          for (int u = 0; u < 4; ++u) x[i][u] = to_f32<T>(v.e[u]);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) x[i][u] = u < n ? to_f32<T>(p[i][u]) : 0.f;
        }
      }
    }
    k += f32p::KS;
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] += step;
  }
};

template <bool KC, int N>
__device__ __forceinline__ void store_slice(float* s, const float (&x)[N][4]) {
  using namespace f32p;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (KC) {
      const int r = (threadIdx.x >> 2) + 64 * i, k = 4 * (threadIdx.x & 3);
#pragma unroll
      for (int u = 0; u < 4; ++u) s[row(k) + u * LS + r] = x[i][u];
    } else {
      const int k = threadIdx.x >> 4, r = 4 * (threadIdx.x & 15) + 64 * i;
      *reinterpret_cast<float4*>(s + row(k) + r) = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
    }
  }
}

constexpr int kTM = f32p::BM / 32, kTN = 4;  // accumulators of a wavefront: 16 x 16
using F32Acc = f32x4_t[kTM][kTN];

// acc = tile (rows r0 of A, rows n0 of B) over K [k0, k_end)
template <typename TA, bool AK, typename TB, bool BKC>
__device__ __forceinline__ void f32_tile(const Operand<TA, AK>& A, const Operand<TB, BKC>& B, int r0,
                                         int n0, int k0, int k_end, float* lds, F32Acc& acc) {
  using namespace f32p;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int ra = (wave >> 1) * 16 * kTM + (lane & 15), rb = (wave & 1) * 64 + (lane & 15), kk = lane >> 4;
  constexpr int BUF = 2 * KS * LS;
#pragma unroll
  for (int i = 0; i < kTM; ++i)
#pragma unroll
    for (int j = 0; j < kTN; ++j) acc[i][j] = f32x4_t{};
  // A slice's fragments are in registers when its MFMAs begin.  In the middle of
  // them: the barrier, after which the slice's own LDS buffer is free for the one
  // two slices on (whose loads were issued a slice ago), and the loads of the next;
  // in the second half the next slice's fragments are read, a few behind each row
  // of MFMAs, so that the matrix pipe is never left waiting for a phase to end.
  float xa[BM / 64][4], xb[BN / 64][4];
  Fetch<BM / 64, TA, AK> la(A, r0, k0);
  Fetch<BN / 64, TB, BKC> lb(B, n0, k0);
  const auto put = [&](int buf) {
    store_slice<AK>(lds + buf * BUF, xa);
    store_slice<BKC>(lds + buf * BUF + KS * LS, xb);
  };
  const auto fetch = [&](int k) {
    la.next(k, k_end, xa);
    lb.next(k, k_end, xb);
  };
  struct Frags {
    float a[KS / 4][kTM], b[KS / 4][kTN];
  };
  constexpr int NF = kTM + kTN;  // fragments of a k-step
  const auto read = [&](Frags& f, int buf, int n) {  // fragment n of the slice
    const int s = n / NF, i = n % NF;
    const float* p = lds + buf * BUF + row(4 * s) + kk * LS;
    if (i < kTM)
      f.a[s][i] = p[ra + 16 * i];
    else
      f.b[s][i - kTM] = p[KS * LS + rb + 16 * (i - kTM)];
  };
  fetch(k0);
  put(0);
  fetch(k0 + KS);  // (slices past the end are zeros)
  put(1);
  fetch(k0 + 2 * KS);
  __syncthreads();
  Frags f0, f1;
#pragma unroll
  for (int n = 0; n < KS / 4 * NF; ++n) read(f0, 0, n);
  // groups of 16 rows of this wavefront that hold a row: the last row tile's others
  // take no MFMAs
  const int groups = (A.rows - r0 - (wave >> 1) * 16 * kTM + 15) / 16;
  const auto slice = [&](auto whole, Frags& f, Frags& next, int k, int buf) {
    constexpr int ROWS = KS / 4 * kTM;  // rows of kTN MFMAs
#pragma unroll
    for (int g = 0; g < ROWS; ++g) {
      if (g == ROWS / 2) {
        lds_barrier();
        if (k + 2 * KS < k_end) {
          put(buf);
          fetch(k + 3 * KS);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (whole || g % kTM < groups)
#pragma unroll
        for (int j = 0; j < kTN; ++j)
          acc[g % kTM][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
              f.a[g / kTM][g % kTM], f.b[g / kTM][j], acc[g % kTM][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (g >= ROWS / 2) {
        constexpr int PER = KS / 4 * NF / (ROWS / 2);
#pragma unroll
        for (int n = 0; n < PER; ++n) read(next, buf ^ 1, (g - ROWS / 2) * PER + n);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto run = [&](auto whole) {
    for (int k = k0; k < k_end; k += 2 * KS) {
      slice(whole, f0, f1, k, 0);
      if (k + KS < k_end) slice(whole, f1, f0, k + KS, 1);
    }
  };
  if (groups >= kTM)
    run(std::true_type());
  else
    run(std::false_type());
  __syncthreads();
}

// tile row / column of accumulator element r of acc[i][j]
__device__ __forceinline__ int f32_row(int i, int r) {
  return ((int)threadIdx.x >> 7) * 16 * kTM + 16 * i + 4 * ((threadIdx.x & 63) >> 4) + r;
}
__device__ __forceinline__ int f32_col(int j) {
  return ((threadIdx.x >> 6) & 1) * 64 + 16 * j + (threadIdx.x & 15);
}

// K splits of an m x n product over K on a 256-CU device: the fewest slices on the
// busiest CU, a block's start and end counted as 16 of them, and a tenth more for a
// block that has no other one beside it
inline int product_splits(int m, int n, int K) {
  const long tiles = (long)cdiv(m, f32p::BM) * cdiv(n, f32p::BN);
  const int nk = cdiv(K, f32p::KS);
  int best = 1;
  long cost = 0;
  for (int s = 1; s <= 64 && (s == 1 || nk / s >= 16); ++s) {
    const long rounds = (tiles * s + 255) / 256;
    const long c = rounds * (cdiv(nk, s) + 16) * (rounds == 1 ? 11 : 10);
    if (s == 1 || c < cost) {
      best = s;
      cost = c;
    }
  }
  return best;
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
