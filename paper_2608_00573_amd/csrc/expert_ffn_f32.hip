// The expert feed-forward block and its gradient in fp32 (formulas: expert_ffn.hip), on
// the fp32 tiles of products.h, operands of any leading dimension and alignment: 128 x 128
// through LDS, or 128 columns x 32 rows straight from memory where those are few.  Bound by
// the fp32 matrix rate, with few tiles by the chain of a tile's loads (777 rows over 4
// experts of 768 x 1000: da 38 us, 80 in 128 x 128 tiles; dx 52 and 163; the weights'
// gradients, 128 x 128 tiles of all experts in one launch, 55).  The 32-row tiles sum K in
// four chains, whose registers are free (one chain and four: forward of 1 row of 2048 x
// 5632 93 and 95 us, gradient of 9 rows of 3769 x 2870 156 and 146, forward of 3800 rows over
// 60 experts of 2048 x 1408 1284 and 1264): sums of random signs off by half as much,
// 5.5e-7 of their norm over K = 4096 (1.1e-6).
#include <math.h>

#include <algorithm>

#include "expert_ffn.h"
#include "products.h"

namespace trimmoe {

namespace {

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

constexpr int kChains = 4;

// the block's tile: a group's rows r0 .. (e >= E: rows of no group) times columns from m0
template <int KIND>
struct F32At {
  using T = f32p::Tile<KIND>;
  int e, r0, end, m0;
  // false: no such tile
  __device__ __forceinline__ bool init(const Groups& g, int slots, int M) {
    const GroupTiles t(g, slots, T::B);
    const int n_m = (M + T::A - 1) / T::A;
    const int mt = blockIdx.x / n_m;
    if (mt >= t.n) return false;
    m0 = (int)(blockIdx.x % n_m) * T::A;
    int within;
    e = t.group(mt, within);
    const int2 r = g.rows(e);
    r0 = uniform(r.x + within * T::B);
    end = uniform(r.y);
    return true;
  }
};

// A tile's sums, zero to begin with.  AK: whether A is K-contiguous; a stream of an A
// that is not mixes the rows of A of its groups (see f32_stream_of), in whole runs.
template <int KIND, bool AK>
struct F32Sums : F32Tile<KIND> {
  using T = f32p::Tile<KIND>;
  static constexpr bool MIXED = T::STREAM && !AK;
  __device__ __forceinline__ F32Sums(const F32At<KIND>& at, int M)
      : F32Tile<KIND>(at.m0, M, at.r0, at.end) {
    if (MIXED) this->a = at.m0 + 16 * T::NA * uniform(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
#pragma unroll
      for (int j = 0; j < T::NB; ++j) this->acc[i][j] = f32x4_t{};
  }
};

// f(row, column, how many, take) for each run of a lane's elements of a tile (rows, cols:
// the ends of both); take(sums, v) gives the run's values of a tile's sums
template <class S, typename F>
__device__ __forceinline__ void each(const S& t, int rows, int cols, F f) {
  using T = typename S::T;
#pragma unroll
  for (int j = 0; j < T::NB; ++j) {
    const int b = t.row_b(j);
    if (j >= t.nb || b >= rows) continue;
    if constexpr (S::MIXED) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // elements `at` .. at + NA - 1; those before c are another lane's
        const int c = t.a + T::NA * (4 * ((threadIdx.x & 63) >> 4) + r);
        if (c >= cols) continue;
        const int skip = c - min(c, cols - T::NA);
        f(b, c, T::NA - skip, [&](const S& s, float(&v)[4]) {
#pragma unroll
          for (int i = 0; i < T::NA; ++i)
#pragma unroll
            for (int k = 0; k <= i; ++k)
              if (k == i - skip) v[k] = s.acc[i][j][r];
        });
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::NA; ++i) {
        const int c = t.row_a(i, 0);
        if (i >= t.na || c >= cols) continue;
        f(b, c, min(4, cols - c), [&](const S& s, float(&v)[4]) {
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = s.acc[i][j][r];
        });
      }
    }
  }
}

__device__ __forceinline__ void put4(float* p, const float (&v)[4], int n) {
  if (n == 4) {
    *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 3; ++r)
      if (r < n) p[r] = v[r];
  }
}

struct F32Up {
  Groups groups;
  const float *w_up, *w_gate, *x;
  int d, F;
  float *a, *up, *gate;  // up, gate: NULL or [n, F]
};

template <int KIND, bool GATED>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_up_f32(F32Up a) {
  __shared__ __align__(16) float lds[f32p::Tile<KIND>::FLOATS];
  F32At<KIND> at;
  if (!at.init(a.groups, a.groups.E + 2, a.F)) return;
  F32Sums<KIND, true> u(at, a.F), g(at, a.F);
  if (at.e < a.groups.E) {
    const size_t w0 = (size_t)at.e * a.F * a.d;
    const Operand<true> x{a.x, (size_t)a.d, at.end, a.d};
    f32_product<KIND, kChains>(Operand<true>{a.w_up + w0, (size_t)a.d, a.F, a.d}, x, at.m0, at.r0, 0, a.d,
                               lds, u);
    if constexpr (GATED)
      f32_product<KIND, kChains>(Operand<true>{a.w_gate + w0, (size_t)a.d, a.F, a.d}, x, at.m0, at.r0, 0,
                                 a.d, lds, g);
  }
  each(u, at.end, a.F, [&](int row, int c, int n, auto take) {
    const size_t o = (size_t)row * a.F + c;
    float vu[4] = {}, vg[4] = {}, va[4];
    take(u, vu);
    if constexpr (GATED) take(g, vg);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (GATED) {
        va[r] = vg[r] / (1.f + expf(-vg[r])) * vu[r];
      } else {
        va[r] = vu[r] < 0.f ? 0.f : vu[r];  // (NaN stays)
      }
    }
    put4(a.a + o, va, n);
    if (a.up) put4(a.up + o, vu, n);
    if (GATED && a.gate) put4(a.gate + o, vg, n);
  });
}

// out [n, M]: y = a Wd^T (AK: Wd K-contiguous) or dx = du Wu + dg Wg.  Grid y: pieces of
// K (of both products in a row) into slices of their own, where tiles are few (forward of
// 1 row of 2048 x 5632, 16 tiles of y: 174 us, 89 with y in 16 pieces).
struct F32Rows {
  Groups groups;
  const float *w, *w2, *b, *b2;
  int M, K;
  float* out;  // [pieces][n, M]
};

// K of a piece
__host__ __device__ inline long piece_of(long K, int pieces) {
  return ((K + pieces - 1) / pieces + f32p::KS - 1) / f32p::KS * f32p::KS;
}

template <int KIND, bool AK, bool TWO>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_rows_f32(F32Rows a) {
  __shared__ __align__(16) float lds[f32p::Tile<KIND>::FLOATS];
  F32At<KIND> at;
  if (!at.init(a.groups, a.groups.E + 2, a.M)) return;
  F32Sums<KIND, AK> t(at, a.M), t2(at, a.M);
  if (at.e < a.groups.E) {
    const size_t w0 = (size_t)at.e * a.M * a.K, ld = AK ? a.K : a.M;
    const long all = (TWO ? 2l : 1l) * a.K, per = piece_of(all, gridDim.y);
    const long k0 = min(per * blockIdx.y, all), k1 = min(k0 + per, all);
    if (k0 < a.K)
      f32_product<KIND, kChains>(Operand<AK>{a.w + w0, ld, a.M, a.K},
                                 Operand<true>{a.b, (size_t)a.K, at.end, a.K}, at.m0, at.r0, (int)k0,
                                 (int)min(k1, (long)a.K), lds, t);
    if (TWO && k1 > a.K)
      f32_product<KIND, kChains>(Operand<AK>{a.w2 + w0, ld, a.M, a.K},
                                 Operand<true>{a.b2, (size_t)a.K, at.end, a.K}, at.m0, at.r0,
                                 (int)max(k0 - a.K, 0l), (int)(k1 - a.K), lds, t2);
  }
  each(t, at.end, a.M, [&](int row, int c, int n, auto take) {
    float v[4] = {}, v2[4] = {};
    take(t, v);
    if constexpr (TWO) take(t2, v2);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = TWO ? v[r] + v2[r] : v[r];
    put4(a.out + ((size_t)blockIdx.y * a.groups.n + row) * a.M + c, v, n);
  });
}

struct F32Dact {
  Groups groups;
  const float *w_down, *dy;
  int d, F;
  const void *up, *gate;
  const uint8_t *up_scale, *gate_scale;
  float *a, *du, *dg;
};

template <bool PACKED>
__device__ __forceinline__ float kept(const void* p, const uint8_t* scale, int blocks, int F, int row,
                                      int c) {
  const size_t o = (size_t)row * F + c;
  if constexpr (PACKED)
    return pack_value(static_cast<const int8_t*>(p)[o], scale[(size_t)row * blocks + c / kPackBlock]);
  else
    return static_cast<const float*>(p)[o];
}

template <int KIND, bool GATED, bool PACKED>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_dact_f32(F32Dact a) {
  __shared__ __align__(16) float lds[f32p::Tile<KIND>::FLOATS];
  F32At<KIND> at;
  if (!at.init(a.groups, a.groups.E, a.F)) return;
  F32Sums<KIND, false> t(at, a.F);
  f32_product<KIND, kChains>(Operand<false>{a.w_down + (size_t)at.e * a.d * a.F, (size_t)a.F, a.F, a.d},
                             Operand<true>{a.dy, (size_t)a.d, at.end, a.d}, at.m0, at.r0, 0, a.d, lds, t);
  const int blocks = (a.F + kPackBlock - 1) / kPackBlock;
  each(t, at.end, a.F, [&](int row, int c, int n, auto take) {
    float vd[4] = {}, va[4], vu[4], vg[4];
    take(t, vd);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int cr = min(c + min(r, n - 1), a.F - 1);
      const float da = vd[r], u = kept<PACKED>(a.up, a.up_scale, blocks, a.F, row, cr);
      if constexpr (GATED) {
        const float g = kept<PACKED>(a.gate, a.gate_scale, blocks, a.F, row, cr);
        const float s = 1.f / (1.f + expf(-g)), gs = g * s;
        va[r] = gs * u;
        vu[r] = da * gs;
        vg[r] = da * u * (s * (1.f + g * (1.f - s)));
      } else {
        va[r] = u < 0.f ? 0.f : u;
        vu[r] = u > 0.f ? da : 0.f;
      }
    }
    const size_t o = (size_t)row * a.F + c;
    put4(a.a + o, va, n);
    put4(a.du + o, vu, n);
    if constexpr (GATED) put4(a.dg + o, vg, n);
  });
}

struct F32Weights {
  Groups groups;
  int n_prod;
  const float *A[3], *B[3];
  int M[3], N[3];
  float* out[3];
};

// blockIdx.y: product, z: group; x: tile
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_weights_f32(F32Weights a) {
  using T = f32p::Tile<f32p::kSquare>;
  __shared__ __align__(16) float lds[T::FLOATS];
  const int p = blockIdx.y, e = blockIdx.z;
  const int M = p == 0 ? a.M[0] : p == 1 ? a.M[1] : a.M[2];
  const int N = p == 0 ? a.N[0] : p == 1 ? a.N[1] : a.N[2];
  const float* A = p == 0 ? a.A[0] : p == 1 ? a.A[1] : a.A[2];
  const float* B = p == 0 ? a.B[0] : p == 1 ? a.B[1] : a.B[2];
  float* out = (p == 0 ? a.out[0] : p == 1 ? a.out[1] : a.out[2]) + (size_t)e * M * N;
  const int n_m = (M + T::A - 1) / T::A;
  const int m0 = (int)(blockIdx.x % n_m) * T::A, n0 = (int)(blockIdx.x / n_m) * T::B;
  if (n0 >= N) return;
  const int2 r = a.groups.rows(e);
  const int r0 = uniform(r.x), k = uniform(r.y) - r0;
  F32Sums<f32p::kSquare, false> t({e, n0, N, m0}, M);
  if (k > 0)
    f32_tile<f32p::kSquare>(Operand<false>{A + (size_t)r0 * M, (size_t)M, M, k},
                            Operand<false>{B + (size_t)r0 * N, (size_t)N, N, k}, m0, n0, 0, k, lds, t);
  each(t, N, M, [&](int row, int c, int n, auto take) {
    float v[4] = {};
    take(t, v);
    put4(out + (size_t)row * M + c, v, n);
  });
}

template <int KIND>
dim3 tiles_of(const Groups& g, int M) {
  using T = f32p::Tile<KIND>;
  return dim3((unsigned)(row_tiles_most(g.n, g.E, T::B) * cdiv(M, T::A)));
}
// tiles of A x B of rows times M columns, about
long tiles_about(const Groups& g, int M, int A, int B) {
  return std::max(1l, ((long)g.n / B + std::min(g.E, g.n)) * cdiv(M, A));
}
bool small_tiles(const Groups& g, int M) {
  using T = f32p::Tile<f32p::kSquare>;
  return M >= 2 && (g.n <= 64l * g.E || tiles_about(g, M, T::A, T::B) < 256);
}
// f(integral constant of the tiles' kind) for rows times M columns: 128 x 128 tiles, or
// 128 columns x 32 rows straight from memory for few rows an expert and where the others
// leave CUs idle (a lane's loads of an operand along K take two columns at least).  56 rows
// over 8 experts of 4096 x 14336: 1672 us in 128 x 128 tiles, 1167 in these
template <typename F>
hipError_t with_tiles(const Groups& g, int M, F f) {
  if (small_tiles(g, M))
    f(std::integral_constant<int, f32p::kSmall>());
  else
    f(std::integral_constant<int, f32p::kSquare>());
  return hipGetLastError();
}
// pieces of K of small tiles: a block a CU, 256 of K each at least
int pieces_f32(const Groups& g, int M, long K) {
  using T = f32p::Tile<f32p::kSmall>;
  if (!small_tiles(g, M)) return 1;
  return (int)std::max(1l, std::min({256 / tiles_about(g, M, T::A, T::B), K / 256, 16l}));
}
// y or dx
template <bool AK, bool TWO>
hipError_t launch_rows_f32(F32Rows r, float* part, hipStream_t st) {
  const int pieces = pieces_f32(r.groups, r.M, (TWO ? 2l : 1l) * r.K);
  float* out = r.out;
  if (pieces > 1) r.out = part;
  hipError_t e = with_tiles(r.groups, r.M, [&](auto kind) {
    dim3 grid = tiles_of<kind>(r.groups, r.M);
    grid.y = pieces;
    hipLaunchKernelGGL((k_expert_rows_f32<kind, AK, TWO>), grid, dim3(f32p::THREADS), 0, st, r);
  });
  if (e == hipSuccess && pieces > 1)
    e = launch_sum_parts(part, pieces, (size_t)r.groups.n * r.M, out, st);
  return e;
}
const float* as_f32(const void* p) { return static_cast<const float*>(p); }

}  // namespace

size_t row_parts_f32(const Groups& g, int M, long K) {
  const int p = pieces_f32(g, M, K);
  return p > 1 ? ffn_align((size_t)p * g.n * M * 4) : 0;
}

hipError_t launch_expert_ffn_f32(const ExpertFfnArgs& a, hipStream_t st) {
  const int n = a.groups.n;
  const size_t act = ffn_array(n, a.F, 4);
  const bool packed = a.keep == TRIMMOE_KEEP_PACKED;
  F32Up u{a.groups, as_f32(a.w_up), as_f32(a.w_gate), as_f32(a.x), a.d, a.F,
          reinterpret_cast<float*>(a.ws), nullptr, nullptr};
  if (packed) {
    u.up = reinterpret_cast<float*>(a.ws + act);
    if (a.gated) u.gate = reinterpret_cast<float*>(a.ws + 2 * act);
  } else if (a.keep == TRIMMOE_KEEP_FULL) {
    u.up = static_cast<float*>(a.up);
    u.gate = static_cast<float*>(a.gate);
  }
  const dim3 block(f32p::THREADS);
  hipError_t e = with_tiles(a.groups, a.F, [&](auto kind) {
    const dim3 grid = tiles_of<kind>(a.groups, a.F);
    if (a.gated)
      hipLaunchKernelGGL((k_expert_up_f32<kind, true>), grid, block, 0, st, u);
    else
      hipLaunchKernelGGL((k_expert_up_f32<kind, false>), grid, block, 0, st, u);
  });
  if (e == hipSuccess && packed)
    e = launch_checkpoint_pack(false, n, a.F, u.up, static_cast<int8_t*>(a.up), a.up_scale, st);
  if (e == hipSuccess && packed && a.gated)
    e = launch_checkpoint_pack(false, n, a.F, u.gate, static_cast<int8_t*>(a.gate), a.gate_scale, st);
  if (e != hipSuccess) return e;
  const F32Rows r{a.groups, as_f32(a.w_down), nullptr, u.a, nullptr, a.d, a.F, static_cast<float*>(a.y)};
  return launch_rows_f32<true, false>(
      r, reinterpret_cast<float*>(a.ws + (packed ? (a.gated ? 3 : 2) : 1) * act), st);
}

hipError_t launch_expert_ffn_backward_f32(const ExpertFfnArgs& a, hipStream_t st) {
  const int n = a.groups.n;
  const size_t act = ffn_array(n, a.F, 4);
  const bool packed = a.keep == TRIMMOE_KEEP_PACKED;
  const dim3 block(f32p::THREADS);
  F32Dact t{a.groups, as_f32(a.w_down), as_f32(a.dy), a.d, a.F, a.up, a.gate, a.up_scale, a.gate_scale,
            reinterpret_cast<float*>(a.ws), reinterpret_cast<float*>(a.ws + act),
            a.gated ? reinterpret_cast<float*>(a.ws + 2 * act) : nullptr};
  const float* x = as_f32(a.x);
  hipError_t e;
  if (n > 0) {
    e = with_tiles(a.groups, a.F, [&](auto kind) {
      const dim3 grid = tiles_of<kind>(a.groups, a.F);
      if (a.gated && packed)
        hipLaunchKernelGGL((k_expert_dact_f32<kind, true, true>), grid, block, 0, st, t);
      else if (a.gated)
        hipLaunchKernelGGL((k_expert_dact_f32<kind, true, false>), grid, block, 0, st, t);
      else if (packed)
        hipLaunchKernelGGL((k_expert_dact_f32<kind, false, true>), grid, block, 0, st, t);
      else
        hipLaunchKernelGGL((k_expert_dact_f32<kind, false, false>), grid, block, 0, st, t);
    });
    if (e != hipSuccess) return e;
    if (a.x_scale && (a.dw_up || a.dw_gate)) {
      float* to = reinterpret_cast<float*>(a.ws + (a.gated ? 3 : 2) * act);
      e = launch_checkpoint_unpack(false, n, a.d, static_cast<const int8_t*>(a.x), a.x_scale, to, st);
      if (e != hipSuccess) return e;
      x = to;
    }
    if (a.dx) {
      const F32Rows r{a.groups, as_f32(a.w_up), as_f32(a.w_gate), t.du, t.dg, a.d, a.F,
                      static_cast<float*>(a.dx)};
      float* part = reinterpret_cast<float*>(a.ws + (a.gated ? 3 : 2) * act +
                                             (a.x_scale ? ffn_array(n, a.d, 4) : 0));
      e = a.gated ? launch_rows_f32<false, true>(r, part, st) : launch_rows_f32<false, false>(r, part, st);
      if (e != hipSuccess) return e;
    }
  }
  F32Weights w{};
  w.groups = a.groups;
  unsigned tiles = 0;
  const auto add = [&](const float* A, const float* B, int M, int N, void* out) {
    if (!out) return;
    const int p = w.n_prod++;
    w.A[p] = A;
    w.B[p] = B;
    w.M[p] = M;
    w.N[p] = N;
    w.out[p] = static_cast<float*>(out);
    tiles = std::max(tiles, (unsigned)cdiv(M, 128) * cdiv(N, 128));
  };
  add(t.a, t.dy, a.F, a.d, a.dw_down);
  add(x, t.du, a.d, a.F, a.dw_up);
  if (a.gated) add(x, t.dg, a.d, a.F, a.dw_gate);
  if (w.n_prod == 0) return hipSuccess;
  hipLaunchKernelGGL(k_expert_weights_f32, dim3(tiles, w.n_prod, a.groups.E), block, 0, st, w);
  return hipGetLastError();
}

}  // namespace trimmoe
