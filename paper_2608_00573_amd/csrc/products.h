// Products of the training losses in fp32 matrix instructions: the tile (device
// code) and the launchers of products.hip.  Not part of the public ABI.
#pragma once

#include <type_traits>

#include "gemm.h"

namespace trimmoe {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ------------------------------------------------------------ fp32 products --
// C = A B^T in v_mfma_f32_16x16x4_f32 over operands of either order: K-contiguous
// ([rows][K]) or row-contiguous ([K][rows]), any leading dimension and
// alignment.  Blocks of 4 wavefronts, in tiles (A x B rows) of four kinds:
//   kSquare 128 x 128, kNarrow 64 x 256 (an A of no more than 64 rows): a wavefront
//     holds 64 x 64 of C.  16-deep K slices go through registers into a k-major LDS
//     image (two buffers, the next slices' loads in flight under the MFMAs), so a
//     fragment read is 32 consecutive floats and the order of the operand in memory
//     only changes how a slice is written.
//   kFew 128 x 64, kFewer 256 x 32 (few rows of B, a small batch of tokens), kSmall
//     128 x 32: the wavefronts lie along A and share none of it, so both operands go
//     straight to the registers (f32_stream): no LDS, no barrier, several slices in
//     flight.
namespace f32p {
constexpr int KS = 16, THREADS = 256;
// An LDS row (one k) of `rows` floats takes LS, and every fourth one starts 16 floats
// further on.  The 4 rows of 16 that a fragment reads hit distinct banks, and so do
// the four lanes that write one operand row's 16 k.
__host__ __device__ constexpr int ls(int rows) { return rows + 48; }
__device__ __forceinline__ constexpr int row(int k, int LS) { return k * LS + 16 * ((k >> 2) & 3); }

enum Kind { kNarrow, kSquare, kFew, kFewer, kSmall };
__host__ __device__ constexpr int tile_a(int kind) {
  return kind == kNarrow ? 64 : kind == kFewer ? 256 : 128;
}
__host__ __device__ constexpr int tile_b(int kind) {
  return kind == kNarrow ? 256 : kind == kSquare ? 128 : kind == kFew ? 64 : 32;
}
template <int KIND>
struct Tile {
  static constexpr bool STREAM = KIND >= kFew;
  static constexpr int A = tile_a(KIND), B = tile_b(KIND);  // rows
  static constexpr int WA = KIND == kNarrow ? 1 : KIND == kSquare ? 2 : 4;  // wavefronts
  static constexpr int WB = 4 / WA;
  static constexpr int NA = A / WA / 16, NB = B / WB / 16;  // a wavefront's 16-row groups
  static constexpr int BUF = KS * (ls(A) + ls(B)), FLOATS = STREAM ? A : 2 * BUF;
  static constexpr int OCC = STREAM ? 3 : 2;  // wavefronts a SIMD
};

inline long tiles(int kind, int a, int b) {
  return (long)cdiv(a, tile_a(kind)) * cdiv(b, tile_b(kind));
}

// the kind for a product of a x b rows
inline int shape_kind(int a, int b) {
  return a <= 64 ? kNarrow : b <= 32 ? kFewer : b <= 64 ? kFew : kSquare;
}
// ... that is not split along K: smaller tiles where they would leave half of the CUs
// without one (300 tokens, d 1316, vocabulary 530: 43 instead of 107 us)
inline int tile_kind(int a, int b) {
  const int k = shape_kind(a, b);
  if (k == kNarrow || tiles(k, a, b) > 128) return k;
  return k != kSquare || tiles(k, a, b) <= 64 ? kSmall : kFew;
}
// ... of launch_product: the streams take a K-contiguous B
inline int product_kind(bool b_k, int a, int b) {
  const int k = shape_kind(a, b);
  return k >= kFew && !b_k ? kSquare : k;
}

// f(integral constant of the kind)
template <typename F>
inline void with_kind(int kind, F f) {
  if (kind == kNarrow)
    f(std::integral_constant<int, kNarrow>());
  else if (kind == kSquare)
    f(std::integral_constant<int, kSquare>());
  else if (kind == kFew)
    f(std::integral_constant<int, kFew>());
  else if (kind == kSmall)
    f(std::integral_constant<int, kSmall>());
  else
    f(std::integral_constant<int, kFewer>());
}
}  // namespace f32p

// four floats at any address of a float
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// operand: `rows` x K floats.  KC: element (r, k) at r ld + k, else at k ld + r
template <bool KC>
struct Operand {
  const float* p;
  size_t ld;
  int rows, K;
};

// This thread's part of an operand's slices: N groups of four elements, rows from
// r0, in 16-byte loads.  Rows past the end hold anything: the last row's elements
// (KC), or a group moved back to end with the operand and turned when it is stored.
// Elements past the end of K are zeros.
template <int N, bool KC>
struct Fetch {
  const float* p[N];
  int sh[N];  // row-contiguous: rows the group was moved back by
  int k;      // KC: first k of the thread's groups, else its row's k
  int rows;
  bool turn, wide;
  size_t step;
  __device__ __forceinline__ Fetch(const Operand<KC>& o, int r0, int k0) {
    step = KC ? (size_t)f32p::KS : (size_t)f32p::KS * o.ld;
    rows = o.rows;
    turn = !KC && r0 + 64 * N > o.rows;
    wide = KC || o.rows >= 4;
    k = k0 + (KC ? 4 * (threadIdx.x & 3) : threadIdx.x >> 4);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + 64 * i + (KC ? threadIdx.x >> 2 : 4 * (threadIdx.x & 15));
      const int at = KC ? min(r, o.rows - 1) : min(r, max(o.rows - 4, 0));
      sh[i] = r - at;
      p[i] = o.p + (KC ? (size_t)at * o.ld + k : (size_t)k * o.ld + at);
    }
  }
  // the slice that begins at k0, and on to the next one
  __device__ __forceinline__ void next(int k0, int k_end, float (&x)[N][4]) {
    if (wide && k0 + f32p::KS <= k_end) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f32x4_any v = *reinterpret_cast<const f32x4_any*>(p[i]);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[i][u] = v[u];
      }
    } else {
      // elements of a group that may be read
      const int n = KC ? k_end - k : k < k_end ? (wide ? 4 : rows) : 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) x[i][u] = u < n ? p[i][u] : 0.f;
    }
    k += f32p::KS;
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] += step;
  }
  __device__ __forceinline__ void store(float* s, const float (&x)[N][4]) const {
    using namespace f32p;
    constexpr int LS = ls(64 * N);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (KC) {
        const int r = (threadIdx.x >> 2) + 64 * i, k = 4 * (threadIdx.x & 3);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[row(k, LS) + u * LS + r] = x[i][u];
      } else {
        const int k = threadIdx.x >> 4, r = 4 * (threadIdx.x & 15) + 64 * i;
        float4 v = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
        if (turn) {
          const int m = sh[i];
          v.x = m == 0 ? v.x : m == 1 ? v.y : m == 2 ? v.z : v.w;
          v.y = m == 0 ? v.y : m == 1 ? v.z : v.w;
          v.z = m == 0 ? v.z : v.w;
        }
        *reinterpret_cast<float4*>(s + row(k, LS) + r) = v;
      }
    }
  }
};

// A wavefront's part of a tile's product, 16 x 16 accumulators [A][B].  A tile cut
// short is shared out evenly: its 16-row groups of an operand go to the wavefronts in
// equal runs, and groups behind the last row take no MFMAs.
template <int KIND>
struct F32Tile {
  using T = f32p::Tile<KIND>;
  f32x4_t acc[T::NA][T::NB];
  int a, b;    // the wavefront's first rows of the operands
  int na, nb;  // its groups
  __device__ __forceinline__ F32Tile(int r0, int rows_a, int n0, int rows_b) {
    const int w = threadIdx.x >> 6, wave = T::STREAM ? __builtin_amdgcn_readfirstlane(w) : w;
    const int ga = (min(T::A, rows_a - r0) + 15) / 16, gb = (min(T::B, rows_b - n0) + 15) / 16;
    const int pa = (ga + T::WA - 1) / T::WA, pb = (gb + T::WB - 1) / T::WB;
    const int ia = wave % T::WA * pa, ib = wave / T::WA * pb;
    na = min(pa, ga - ia);
    nb = min(pb, gb - ib);
    a = r0 + 16 * ia;
    b = n0 + 16 * ib;
  }
  // row of A / of B of element r of acc[i][j] (i < na, j < nb)
  __device__ __forceinline__ int row_a(int i, int r) const {
    return a + 16 * i + 4 * ((threadIdx.x & 63) >> 4) + r;
  }
  __device__ __forceinline__ int row_b(int j) const { return b + 16 * j + (threadIdx.x & 15); }
};

// t.acc = tile (rows r0 of A, rows n0 of B) over K [k0, k_end)
template <int KIND, bool AK, bool BKC>
__device__ __forceinline__ void f32_tile(const Operand<AK>& A, const Operand<BKC>& B, int r0, int n0,
                                         int k0, int k_end, float* lds, F32Tile<KIND>& t) {
  using namespace f32p;
  using T = Tile<KIND>;
  constexpr int LA = ls(T::A), LB = ls(T::B);
  const int lane = threadIdx.x & 63, kk = lane >> 4;
  const int ra = t.a - r0 + (lane & 15), rb = t.b - n0 + (lane & 15);
  const int na = t.na, nb = t.nb;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) t.acc[i][j] = f32x4_t{};
  // A slice's fragments are in registers when its MFMAs begin.  In the middle of
  // them: the barrier, after which the slice's own LDS buffer is free for the one
  // two slices on (whose loads were issued two slices ago), and the loads of the one
  // two further on; in the second half the next slice's fragments are read, a few behind each row
  // of MFMAs, so that the matrix pipe is never left waiting for a phase to end.
  struct Regs {
    float a[T::A / 64][4], b[T::B / 64][4];
  };
  Fetch<T::A / 64, AK> la(A, r0, k0);
  Fetch<T::B / 64, BKC> lb(B, n0, k0);
  const auto put = [&](const Regs& x, int buf) {
    la.store(lds + buf * T::BUF, x.a);
    lb.store(lds + buf * T::BUF + KS * LA, x.b);
  };
  const auto fetch = [&](Regs& x, int k) {
    la.next(k, k_end, x.a);
    lb.next(k, k_end, x.b);
  };
  struct Frags {
    float a[KS / 4][4], b[KS / 4][4];
  };
  const auto read = [&](Frags& f, int buf, int n) {  // fragment n of the slice
    const int s = n / 8, i = n % 8;
    const float* p = lds + buf * T::BUF;
    if (i < 4)
      f.a[s][i] = p[row(4 * s, LA) + kk * LA + ra + 16 * i];
    else
      f.b[s][i - 4] = p[KS * LA + row(4 * s, LB) + kk * LB + rb + 16 * (i - 4)];
  };
  Regs x0, x1;
  fetch(x0, k0);
  fetch(x1, k0 + KS);  // (slices past the end are zeros)
  put(x0, 0);
  put(x1, 1);
  fetch(x0, k0 + 2 * KS);
  fetch(x1, k0 + 3 * KS);
  __syncthreads();
  Frags f0, f1;
#pragma unroll
  for (int n = 0; n < 2 * KS; ++n) read(f0, 0, n);
  const auto slice = [&](auto whole_a, auto whole_b, Frags& f, Frags& next, Regs& x, int k, int buf) {
#pragma unroll
    for (int g = 0; g < KS; ++g) {  // a row of MFMAs: k-step g / 4, group g % 4 of B
      if (g == KS / 2) {
        lds_barrier();
        if (k + 2 * KS < k_end) {
          put(x, buf);
          fetch(x, k + 4 * KS);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (whole_b || g % 4 < nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (whole_a || i < na)
            t.acc[i][g % 4] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.a[g / 4][i], f.b[g / 4][g % 4],
                                                                   t.acc[i][g % 4], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (g >= KS / 2) {
#pragma unroll
        for (int n = 0; n < 4; ++n) read(next, buf ^ 1, (g - KS / 2) * 4 + n);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto run = [&](auto whole_a, auto whole_b) {
    for (int k = k0; k < k_end; k += 2 * KS) {
      slice(whole_a, whole_b, f0, f1, x0, k, 0);
      if (k + KS < k_end) slice(whole_a, whole_b, f1, f0, x1, k + KS, 1);
    }
  };
  if (na >= 4 && nb >= 4)
    run(std::true_type(), std::true_type());
  else if (na >= 4)
    run(std::true_type(), std::false_type());
  else
    run(std::false_type(), std::false_type());
  __syncthreads();
}

// t.acc for few rows of B.  A lane's load is consecutive elements along the operand's
// contiguous axis, and the MFMAs take them in an order that suits it: any order of k
// will do if both operands share it, and lane (fr, q) gives MFMA u the k = 4 q + u of
// a slice.
//   * K-contiguous: element u of the 16 bytes of row 16 i + fr is MFMA u's;
//   * row-contiguous (A only): load u is k = 4 q + u, its element i row NA fr + i, so
//     element r of acc[i][j] is row NA (4 q + r) + i.  The last rows' loads are moved
//     back to end with A (A.rows >= NA).
// Wavefronts begin at different slices: rows that lie a power of two apart would
// otherwise be read from the same few memory channels at a time.  1.2 GB of w (rows of
// 8 KB) against 7 rows of h: 298 us (4.2 TB/s), 328 without that, 365 through LDS;
// against 20: 336 and 415 through LDS.
template <int NB, int DEPTH, int KIND, bool AK>
__device__ __forceinline__ void f32_stream_of(const Operand<AK>& A, const Operand<true>& B, int k0,
                                              int k_end, F32Tile<KIND>& t) {
  constexpr int KS = f32p::KS, NA = f32p::Tile<KIND>::NA;
  typedef float NaVec __attribute__((ext_vector_type(NA), aligned(4)));
  const int lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  const int a1 = min(t.a, A.rows - (AK ? 1 : NA));  // (a wavefront may lie behind A)
  const float* pa = A.p + (AK ? (size_t)a1 * A.ld + k0 : (size_t)k0 * A.ld + a1);
  const float* pb = B.p + (size_t)t.b * B.ld + k0;
  const size_t step = AK ? (size_t)KS : KS * A.ld;
  constexpr int LA = AK ? NA : 4;  // loads of a slice of A
  uint32_t oa[LA], ob[NB];
#pragma unroll
  for (int i = 0; i < LA; ++i)
    oa[i] = AK ? (uint32_t)(min(t.a + 16 * i + fr, A.rows - 1) - a1) * (uint32_t)A.ld + 4 * q
               : (uint32_t)(4 * q + i) * (uint32_t)A.ld + (min(t.a + NA * fr, A.rows - NA) - a1);
#pragma unroll
  for (int j = 0; j < NB; ++j)
    ob[j] = (uint32_t)(min(t.b + 16 * j + fr, B.rows - 1) - t.b) * (uint32_t)B.ld + 4 * q;
  struct Regs {
    float a[LA][AK ? 4 : NA], b[NB][4];
  };
  const int n = (k_end - k0) / KS, rest = k_end - k0 - n * KS;
  const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = n > 0 ? (int)((blockIdx.x * 4 + wave) * 7 % (unsigned)n) : 0;
  const auto load = [&](Regs& x, int s) {  // (past the last slice: it again, unused)
    s = min(s, n - 1) + first;
    s = s >= n ? s - n : s;
    const float *qa = pa + s * step, *qb = pb + s * KS;
#pragma unroll
    for (int i = 0; i < LA; ++i) {
      if constexpr (AK) {
        const f32x4_any v = *reinterpret_cast<const f32x4_any*>(qa + oa[i]);
#pragma unroll
        for (int u = 0; u < 4; ++u) x.a[i][u] = v[u];
      } else {
        const NaVec v = *reinterpret_cast<const NaVec*>(qa + oa[i]);
#pragma unroll
        for (int u = 0; u < NA; ++u) x.a[i][u] = v[u];
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const f32x4_any v = *reinterpret_cast<const f32x4_any*>(qb + ob[j]);
#pragma unroll
      for (int u = 0; u < 4; ++u) x.b[j][u] = v[u];
    }
  };
  const auto mma = [&](const Regs& x) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < NA; ++i)
          t.acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(AK ? x.a[i][u] : x.a[u][i], x.b[j][u],
                                                             t.acc[i][j], 0, 0, 0);
  };
  if (n > 0) {
    Regs x[DEPTH];
#pragma unroll
    for (int p = 0; p < DEPTH; ++p) load(x[p], p);
    int s = 0;
    for (; s + DEPTH <= n; s += DEPTH)
#pragma unroll
      for (int p = 0; p < DEPTH; ++p) {
        mma(x[p]);
        load(x[p], s + p + DEPTH);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
    for (int p = 0; p < DEPTH; ++p)
      if (s + p < n) mma(x[p]);
  }
  if (rest > 0) {  // (rest < 16: elements past the end are zeros)
    Regs x;
    const float *qa = pa + n * step, *qb = pb + n * KS;
#pragma unroll
    for (int i = 0; i < LA; ++i)
#pragma unroll
      for (int u = 0; u < (AK ? 4 : NA); ++u)
        x.a[i][u] = 4 * q + (AK ? u : i) < rest ? qa[oa[i] + u] : 0.f;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) x.b[j][u] = 4 * q + u < rest ? qb[ob[j] + u] : 0.f;
    mma(x);
  }
}
// (as many slices in flight as 168 registers hold)
template <int KIND, bool AK>
__device__ __forceinline__ void f32_stream(const Operand<AK>& A, const Operand<true>& B, int k0,
                                           int k_end, F32Tile<KIND>& t) {
  using T = f32p::Tile<KIND>;
#pragma unroll
  for (int i = 0; i < T::NA; ++i)
#pragma unroll
    for (int j = 0; j < T::NB; ++j) t.acc[i][j] = f32x4_t{};
  if constexpr (KIND == f32p::kFewer) {
    if (t.nb == 1)
      f32_stream_of<1, 4>(A, B, k0, k_end, t);
    else
      f32_stream_of<2, 4>(A, B, k0, k_end, t);
  } else if constexpr (KIND == f32p::kSmall) {
    f32_stream_of<2, 6>(A, B, k0, k_end, t);
  } else {
    if (t.nb == 3)
      f32_stream_of<3, 4>(A, B, k0, k_end, t);
    else
      f32_stream_of<4, 3>(A, B, k0, k_end, t);
  }
}

// the product of a tile in the way of its kind
template <int KIND, bool AK, bool BKC>
__device__ __forceinline__ void f32_product(const Operand<AK>& A, const Operand<BKC>& B, int r0,
                                            int n0, int k0, int k_end, float* lds,
                                            F32Tile<KIND>& t) {
  if constexpr (f32p::Tile<KIND>::STREAM)
    f32_stream(A, B, k0, k_end, t);
  else
    f32_tile<KIND>(A, B, r0, n0, k0, k_end, lds, t);
}

// K splits of an a x b product over K on a whole MI355X, 256 CUs (a plan for a workspace,
// not the current device's count): the fewest slices on the busiest CU, a block's start
// and end counted as 16 of them, a tenth more for a block that has no other one beside
// it, and the partials' sum as 4
inline int product_splits(int kind, int a, int b, int K) {
  const long tiles = f32p::tiles(kind, a, b);
  const int nk = cdiv(K, f32p::KS);
  int best = 1;
  long cost = 0;
  for (int s = 1; s <= 64 && (s == 1 || nk / s >= 6); ++s) {
    const long rounds = (tiles * s + 255) / 256;
    const long c = rounds * (cdiv(nk, s) + 16) * (rounds == 1 ? 11 : 10) + (s > 1 ? 40 : 0);
    if (s == 1 || c < cost) {
      best = s;
      cost = c;
    }
  }
  return best;
}

// out [B.rows, A.rows] = B A^T in `splits` runs of K, one slice of partials per run,
// added to what the slices hold (`add`)
template <bool BKC>
hipError_t launch_product(const Operand<false>& A, const Operand<BKC>& B, int splits, bool add,
                          float* out, hipStream_t st);

// out = sum of the S slices of n partials
hipError_t launch_sum_parts(const float* part, int S, size_t n, float* out, hipStream_t st);

}  // namespace trimmoe
