// The expert feed-forward block and its gradient in fp32 (formulas: expert_ffn.hip), on
// the fp32 tiles of products.h: 128 x 128 through LDS, operands of any leading dimension
// and alignment.  Bound by the fp32 matrix rate.
#include <math.h>

#include <algorithm>

#include "expert_ffn.h"
#include "products.h"

namespace trimmoe {

namespace {

using F32T = F32Tile<f32p::kSquare>;
using F32S = f32p::Tile<f32p::kSquare>;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// the block's tile: a group's rows r0 .. (e >= E: rows of no group) times columns from m0
struct F32At {
  int e, r0, end, m0;
  // false: no such tile
  __device__ __forceinline__ bool init(const Groups& g, int slots, int M) {
    const GroupTiles t(g, slots, F32S::B);
    const int n_m = (M + F32S::A - 1) / F32S::A;
    const int mt = blockIdx.x / n_m;
    if (mt >= t.n) return false;
    m0 = (int)(blockIdx.x % n_m) * F32S::A;
    int within;
    e = t.group(mt, within);
    const int2 r = g.rows(e);
    r0 = uniform(r.x + within * F32S::B);
    end = uniform(r.y);
    return true;
  }
};

// f(row, column, values, how many of the four) for what a lane holds of the tile
template <typename F>
__device__ __forceinline__ void each(const F32T& t, int rows, int cols, F f) {
#pragma unroll
  for (int j = 0; j < F32S::NB; ++j) {
    const int b = t.row_b(j);
    if (j >= t.nb || b >= rows) continue;
#pragma unroll
    for (int i = 0; i < F32S::NA; ++i) {
      const int c = t.row_a(i, 0);
      if (i >= t.na || c >= cols) continue;
      f(i, j, b, c, min(4, cols - c));
    }
  }
}

__device__ __forceinline__ void zero_tile(F32T& t) {
#pragma unroll
  for (int i = 0; i < F32S::NA; ++i)
#pragma unroll
    for (int j = 0; j < F32S::NB; ++j) t.acc[i][j] = f32x4_t{};
}

__device__ __forceinline__ void put4(float* p, const float (&v)[4], int n) {
  if (n == 4) {
    *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
  } else {
    for (int r = 0; r < n; ++r) p[r] = v[r];
  }
}

struct F32Up {
  Groups groups;
  const float *w_up, *w_gate, *x;
  int d, F;
  float *a, *up, *gate;  // up, gate: NULL or [n, F]
};

template <bool GATED>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_up_f32(F32Up a) {
  __shared__ __align__(16) float lds[F32S::FLOATS];
  F32At at;
  if (!at.init(a.groups, a.groups.E + 2, a.F)) return;
  F32T u(at.m0, a.F, at.r0, at.end), g(at.m0, a.F, at.r0, at.end);
  zero_tile(u);
  zero_tile(g);
  if (at.e < a.groups.E) {
    const size_t w0 = (size_t)at.e * a.F * a.d;
    const Operand<true> x{a.x, (size_t)a.d, at.end, a.d};
    f32_tile<f32p::kSquare>(Operand<true>{a.w_up + w0, (size_t)a.d, a.F, a.d}, x, at.m0, at.r0, 0, a.d,
                            lds, u);
    if constexpr (GATED)
      f32_tile<f32p::kSquare>(Operand<true>{a.w_gate + w0, (size_t)a.d, a.F, a.d}, x, at.m0, at.r0, 0,
                              a.d, lds, g);
  }
  each(u, at.end, a.F, [&](int i, int j, int row, int c, int n) {
    const size_t o = (size_t)row * a.F + c;
    float vu[4], vg[4], va[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      vu[r] = u.acc[i][j][r];
      if constexpr (GATED) {
        vg[r] = g.acc[i][j][r];
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

// out [n, M]: y = a Wd^T (AK: Wd K-contiguous) or dx = du Wu + dg Wg
struct F32Rows {
  Groups groups;
  const float *w, *w2, *b, *b2;
  int M, K;
  float* out;
};

template <bool AK, bool TWO>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_rows_f32(F32Rows a) {
  __shared__ __align__(16) float lds[F32S::FLOATS];
  F32At at;
  if (!at.init(a.groups, a.groups.E + 2, a.M)) return;
  F32T t(at.m0, a.M, at.r0, at.end), t2(at.m0, a.M, at.r0, at.end);
  zero_tile(t);
  zero_tile(t2);
  if (at.e < a.groups.E) {
    const size_t w0 = (size_t)at.e * a.M * a.K, ld = AK ? a.K : a.M;
    f32_tile<f32p::kSquare>(Operand<AK>{a.w + w0, ld, a.M, a.K},
                            Operand<true>{a.b, (size_t)a.K, at.end, a.K}, at.m0, at.r0, 0, a.K, lds, t);
    if constexpr (TWO)
      f32_tile<f32p::kSquare>(Operand<AK>{a.w2 + w0, ld, a.M, a.K},
                              Operand<true>{a.b2, (size_t)a.K, at.end, a.K}, at.m0, at.r0, 0, a.K, lds,
                              t2);
  }
  each(t, at.end, a.M, [&](int i, int j, int row, int c, int n) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = TWO ? t.acc[i][j][r] + t2.acc[i][j][r] : t.acc[i][j][r];
    put4(a.out + (size_t)row * a.M + c, v, n);
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

template <bool GATED, bool PACKED>
__global__ __launch_bounds__(f32p::THREADS, 2) void k_expert_dact_f32(F32Dact a) {
  __shared__ __align__(16) float lds[F32S::FLOATS];
  F32At at;
  if (!at.init(a.groups, a.groups.E, a.F)) return;
  F32T t(at.m0, a.F, at.r0, at.end);
  f32_tile<f32p::kSquare>(
      Operand<false>{a.w_down + (size_t)at.e * a.d * a.F, (size_t)a.F, a.F, a.d},
      Operand<true>{a.dy, (size_t)a.d, at.end, a.d}, at.m0, at.r0, 0, a.d, lds, t);
  const int blocks = (a.F + kPackBlock - 1) / kPackBlock;
  each(t, at.end, a.F, [&](int i, int j, int row, int c, int n) {
    float va[4], vu[4], vg[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int cr = min(c + r, a.F - 1);
      const float da = t.acc[i][j][r], u = kept<PACKED>(a.up, a.up_scale, blocks, a.F, row, cr);
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
  __shared__ __align__(16) float lds[F32S::FLOATS];
  const int p = blockIdx.y, e = blockIdx.z;
  const int M = p == 0 ? a.M[0] : p == 1 ? a.M[1] : a.M[2];
  const int N = p == 0 ? a.N[0] : p == 1 ? a.N[1] : a.N[2];
  const float* A = p == 0 ? a.A[0] : p == 1 ? a.A[1] : a.A[2];
  const float* B = p == 0 ? a.B[0] : p == 1 ? a.B[1] : a.B[2];
  float* out = (p == 0 ? a.out[0] : p == 1 ? a.out[1] : a.out[2]) + (size_t)e * M * N;
  const int n_m = (M + F32S::A - 1) / F32S::A;
  const int m0 = (int)(blockIdx.x % n_m) * F32S::A, n0 = (int)(blockIdx.x / n_m) * F32S::B;
  if (n0 >= N) return;
  const int2 r = a.groups.rows(e);
  const int r0 = uniform(r.x), k = uniform(r.y) - r0;
  F32T t(m0, M, n0, N);
  zero_tile(t);
  if (k > 0)
    f32_tile<f32p::kSquare>(Operand<false>{A + (size_t)r0 * M, (size_t)M, M, k},
                            Operand<false>{B + (size_t)r0 * N, (size_t)N, N, k}, m0, n0, 0, k, lds, t);
  each(t, N, M, [&](int i, int j, int row, int c, int n) {
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = t.acc[i][j][q];
    put4(out + (size_t)row * M + c, v, n);
  });
}

unsigned tiles_of(const Groups& g, int M) {
  return (unsigned)(row_tiles_most(g.n, g.E, F32S::B) * cdiv(M, F32S::A));
}
const float* as_f32(const void* p) { return static_cast<const float*>(p); }

}  // namespace

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
  const dim3 grid(tiles_of(a.groups, a.F)), block(f32p::THREADS);
  if (a.gated)
    hipLaunchKernelGGL(k_expert_up_f32<true>, grid, block, 0, st, u);
  else
    hipLaunchKernelGGL(k_expert_up_f32<false>, grid, block, 0, st, u);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && packed)
    e = launch_checkpoint_pack(false, n, a.F, u.up, static_cast<int8_t*>(a.up), a.up_scale, st);
  if (e == hipSuccess && packed && a.gated)
    e = launch_checkpoint_pack(false, n, a.F, u.gate, static_cast<int8_t*>(a.gate), a.gate_scale, st);
  if (e != hipSuccess) return e;
  const F32Rows r{a.groups, as_f32(a.w_down), nullptr, u.a, nullptr, a.d, a.F, static_cast<float*>(a.y)};
  hipLaunchKernelGGL((k_expert_rows_f32<true, false>), dim3(tiles_of(a.groups, a.d)), block, 0, st, r);
  return hipGetLastError();
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
    const dim3 grid(tiles_of(a.groups, a.F));
    if (a.gated && packed)
      hipLaunchKernelGGL((k_expert_dact_f32<true, true>), grid, block, 0, st, t);
    else if (a.gated)
      hipLaunchKernelGGL((k_expert_dact_f32<true, false>), grid, block, 0, st, t);
    else if (packed)
      hipLaunchKernelGGL((k_expert_dact_f32<false, true>), grid, block, 0, st, t);
    else
      hipLaunchKernelGGL((k_expert_dact_f32<false, false>), grid, block, 0, st, t);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.x_scale && (a.dw_up || a.dw_gate)) {
      float* to = reinterpret_cast<float*>(a.ws + (a.gated ? 3 : 2) * act);
      e = launch_checkpoint_unpack(false, n, a.d, static_cast<const int8_t*>(a.x), a.x_scale, to, st);
      if (e != hipSuccess) return e;
      x = to;
    }
    if (a.dx) {
      const F32Rows r{a.groups, as_f32(a.w_up), as_f32(a.w_gate), t.du, t.dg, a.d, a.F,
                      static_cast<float*>(a.dx)};
      const dim3 rows(tiles_of(a.groups, a.d));
      if (a.gated)
        hipLaunchKernelGGL((k_expert_rows_f32<false, true>), rows, block, 0, st, r);
      else
        hipLaunchKernelGGL((k_expert_rows_f32<false, false>), rows, block, 0, st, r);
      if ((e = hipGetLastError()) != hipSuccess) return e;
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
    tiles = std::max(tiles, (unsigned)cdiv(M, F32S::A) * cdiv(N, F32S::B));
  };
  add(t.a, t.dy, a.F, a.d, a.dw_down);
  add(x, t.du, a.d, a.F, a.dw_up);
  if (a.gated) add(x, t.dg, a.d, a.F, a.dw_gate);
  if (w.n_prod == 0) return hipSuccess;
  hipLaunchKernelGGL(k_expert_weights_f32, dim3(tiles, w.n_prod, a.groups.E), block, 0, st, w);
  return hipGetLastError();
}

}  // namespace trimmoe
