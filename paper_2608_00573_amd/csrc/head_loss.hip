// Cross entropy of a vocabulary head and its gradient, in pieces of the
// vocabulary: no [T, V] array of logits is ever whole.
//   z_tv = w_v . h_t + b_v,  lse_t = log sum_v exp z_tv,  loss_t = lse_t - z_{t, y_t}
//   D_tv = g_t (exp(z_tv - lse_t) - [v = y_t])
//   dh = D w,  dw = D^T h,  db_v = sum_t D_tv
// Rows whose target lies outside [0, V), and rows without a logit above -inf
// (lse_t = -inf), take no part: loss and D are zero.
//
// Forward: the product z is reduced in its epilogue to a (max z, sum exp(z -
// max z)) pair per (row, vocabulary tile); one wavefront a row joins the pairs
// and takes the target's logit from one more dot product.
// Backward, per piece of the vocabulary: z again with D as its epilogue, then
// the two products of D.  dh is summed over the pieces in fp32.
#include <math.h>

#include <algorithm>

#include "gemm.h"
#include "loss.h"
#include "products.h"

namespace trimmoe {

namespace {

// ------------------------------------------------------- forward, fp32 --
// A = w (vocabulary rows), B = h: a lane holds 32 vocabulary rows of a token
// column, so the pair of a column is a reduction over registers, one lane
// exchange and the two wavefronts of the column.  A NaN logit makes the sum NaN.
template <typename T>
__global__ __launch_bounds__(f32p::THREADS) void k_loss_f32(Operand<T, true> W, Operand<T, true> H,
                                                            const float* bias, int n_vt,
                                                            float2* part) {
  using namespace f32p;
  __shared__ __align__(16) float lds[4 * BK * LS];
  __shared__ float2 s_p[2][BN];
  const int vt = blockIdx.x, tt = blockIdx.y;
  const int v0 = vt * BM, t0 = tt * BN;
  F32Acc acc;
  f32_tile(W, H, v0, t0, 0, W.K, lds, acc);
  const float ninf = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float m = ninf;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int v = v0 + f32_row(i, r);
        float z = acc[i][j][r];
        if (bias) z += bias[min(v, W.rows - 1)];
        z = v < W.rows ? z : ninf;
        acc[i][j][r] = z;
        m = fmaxf(m, z);
      }
    m = fmaxf(m, __shfl_xor(m, 32));
    const float ms = m == ninf ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (in pairs: a chain would round each small term at the size of the largest)
      float e[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) e[r] = expf(acc[i][j][r] - ms);
#pragma unroll
      for (int n = 8; n > 0; n >>= 1)
#pragma unroll
        for (int r = 0; r < n; ++r) e[r] += e[r + n];
      sum += e[0];
    }
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 32) s_p[threadIdx.x >> 7][f32_col(j)] = make_float2(m, sum);
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c < BN && t0 + c < H.rows) {
    const float2 p0 = s_p[0][c], p1 = s_p[1][c];
    const float M = fmaxf(p0.x, p1.x), Ms = M == ninf ? 0.f : M;
    part[(size_t)(t0 + c) * n_vt + vt] =
        make_float2(M, p0.y * expf(p0.x - Ms) + p1.y * expf(p1.x - Ms));
  }
}

// One wavefront a row: joins the pairs and takes the target's logit from one
// more dot product (a gathered row of w; the pairs do not keep it).
template <typename T>
__global__ __launch_bounds__(256) void k_loss_join(const float2* part, int n_vt, int V, int d, int T_,
                                                   const T* w, const float* b, const T* h,
                                                   const int32_t* target, float* loss, float* lse) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= T_) return;
  const float ninf = -__builtin_inff();
  const float2* p = part + (size_t)t * n_vt;
  float m = ninf;
  for (int i = lane; i < n_vt; i += 64) m = fmaxf(m, p[i].x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float ms = m == ninf ? 0.f : m;
  float sum = 0.f;
  for (int i = lane; i < n_vt; i += 64) sum = fmaf(p[i].y, expf(p[i].x - ms), sum);
  const int y = target[t];
  const bool live = y >= 0 && y < V;
  float z = 0.f;
  if (live)
    for (int k = lane; k < d; k += 64)
      z = fmaf(to_f32<T>(h[(size_t)t * d + k]), to_f32<T>(w[(size_t)y * d + k]), z);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    sum += __shfl_xor(sum, o);
    z += __shfl_xor(z, o);
  }
  if (lane) return;
  const float L = m == ninf && sum == 0.f ? ninf : m + logf(sum);
  lse[t] = L;
  if (b && live) z += b[y];
  float x = L - z;
  x = x < 0.f ? 0.f : x;  // (rounding: a loss is not negative)
  loss[t] = live && L != ninf ? x : 0.f;
}

// ------------------------------------------------------ backward, fp32 --
// D of the tokens x a piece's columns (v0 ..), and per token tile the column
// sums of D (db); columns past the piece up to its leading dimension are zero
template <typename T>
__global__ __launch_bounds__(f32p::THREADS) void k_dz_f32(Operand<T, true> H, Operand<T, true> W,
                                                          const float* bias, const int32_t* target,
                                                          const float* lse, const float* dloss, int V,
                                                          int v0, float* D, size_t ldd,
                                                          float* db_part) {
  using namespace f32p;
  __shared__ __align__(16) float lds[4 * BK * LS];
  const int vt = blockIdx.x, tt = blockIdx.y;
  const int c0 = vt * BN, t0 = tt * BM;
  F32Acc acc;
  f32_tile(H, W, t0, c0, 0, H.K, lds, acc);
  float* s_sum = lds;  // [2][BN]; the tile ended on a barrier
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int c = c0 + f32_col(j);
    const float bj = bias && c < W.rows ? bias[c] : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int t = t0 + f32_row(i, r);
        float x = 0.f;
        if (t < H.rows) {
          const int y = target[t];
          const float L = lse[t];
          if (c < W.rows && y >= 0 && y < V && L != -__builtin_inff())
            x = dloss[t] * (expf(acc[i][j][r] + bj - L) - (v0 + c == y ? 1.f : 0.f));
          D[(size_t)t * ldd + c] = x;
        }
        sum += x;
      }
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 32) s_sum[(threadIdx.x >> 7) * BN + f32_col(j)] = sum;
  }
  __syncthreads();
  if (db_part && threadIdx.x < BN)
    db_part[(size_t)tt * ldd + c0 + threadIdx.x] = s_sum[threadIdx.x] + s_sum[BN + threadIdx.x];
}

// rows that take part, zeros for the others: an ignored row's h may hold
// anything, and 0 * NaN is NaN
template <typename T>
__global__ __launch_bounds__(256) void k_live_rows(const T* h, const int32_t* target,
                                                   const float* lse, int V, int d, T* out) {
  const size_t t = blockIdx.x;
  const int y = target[t];
  const bool live = y >= 0 && y < V && lse[t] != -__builtin_inff();
  for (int k = threadIdx.x; k < d; k += 256) out[t * d + k] = live ? h[t * d + k] : T(0);
}

__global__ __launch_bounds__(256) void k_db_sum(const float* part, int n_tt, size_t ld, int n,
                                                float* db) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n) return;
  float s = 0.f;
  for (int i = 0; i < n_tt; ++i) s += part[(size_t)i * ld + c];
  db[c] = s;
}

// ------------------------------------------------------------------ plan --
// bytes of D that a piece may take
constexpr size_t kPieceBytes = (size_t)256 << 20;
struct BackPlan {
  int Vc;          // columns of a piece (a multiple of the tile)
  int s_dh, s_dw;  // K splits of the two products
  bool direct_dh;  // one piece, one split: dh needs no partials
  size_t o_dh, o_dw, o_d, o_db, o_h, total;
};

BackPlan back_plan(int V, int d, int T) {
  BackPlan p;
  const size_t rows = T > 0 ? T : 1;
  const size_t fit = kPieceBytes / (4 * rows) / f32p::BN * f32p::BN;
  const int most = (int)std::min<size_t>(std::max<size_t>(fit, f32p::BN), (size_t)1 << 30);
  const int n_pieces = cdiv(V, most);
  p.Vc = cdiv(cdiv(V, n_pieces), f32p::BN) * f32p::BN;
  p.s_dh = product_splits(T, d, p.Vc);
  p.s_dw = product_splits(p.Vc, d, T);
  p.direct_dh = n_pieces == 1 && p.s_dh == 1;
  size_t o = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = o;
    o += align256(bytes);
    return at;
  };
  p.o_dh = take(p.direct_dh ? 0 : (size_t)p.s_dh * rows * d * 4);
  p.o_dw = take(p.s_dw == 1 ? 0 : (size_t)p.s_dw * p.Vc * d * 4);
  p.o_d = take(rows * p.Vc * 4);
  p.o_db = take((size_t)cdiv(rows, f32p::BM) * p.Vc * 4);
  p.o_h = take(rows * d * 4);
  p.total = o;
  return p;
}

template <typename T>
hipError_t loss_f32(const HeadLossArgs& a, hipStream_t st) {
  float2* part = reinterpret_cast<float2*>(a.ws);
  const int n_vt = cdiv(a.V, f32p::BM);
  hipLaunchKernelGGL(k_loss_f32<T>, dim3(n_vt, cdiv(a.T, f32p::BN)), dim3(f32p::THREADS), 0, st,
                     (operand<T, true>(a.w, a.d, a.V, a.d)), (operand<T, true>(a.h, a.d, a.T, a.d)),
                     a.b, n_vt, part);
  hipLaunchKernelGGL(k_loss_join<T>, dim3(cdiv(a.T, 4)), dim3(256), 0, st, part, n_vt, a.V, a.d, a.T,
                     static_cast<const T*>(a.w), a.b, static_cast<const T*>(a.h), a.target, a.loss,
                     a.lse);
  return hipGetLastError();
}

template <typename T>
hipError_t backward_f32(const HeadLossArgs& a, hipStream_t st) {
  using namespace f32p;
  const BackPlan p = back_plan(a.V, a.d, a.T);
  float* dh = reinterpret_cast<float*>(a.ws + p.o_dh);
  float* dw = reinterpret_cast<float*>(a.ws + p.o_dw);
  float* D = reinterpret_cast<float*>(a.ws + p.o_d);
  float* db = reinterpret_cast<float*>(a.ws + p.o_db);
  const int n_tt = cdiv(a.T, BM);
  const T* w = static_cast<const T*>(a.w);
  T* hl = reinterpret_cast<T*>(a.ws + p.o_h);
  if (a.dw && a.T > 0)
    hipLaunchKernelGGL(k_live_rows<T>, dim3(a.T), dim3(256), 0, st, static_cast<const T*>(a.h),
                       a.target, a.lse, a.V, a.d, hl);
  for (int v0 = 0; v0 < a.V; v0 += p.Vc) {
    const int nv = std::min(p.Vc, a.V - v0);
    const size_t ldd = (size_t)cdiv(nv, BN) * BN;
    const T* wp = w + (size_t)v0 * a.d;
    if (a.T > 0)
      hipLaunchKernelGGL(k_dz_f32<T>, dim3((unsigned)(ldd / BN), n_tt), dim3(THREADS), 0, st,
                       (operand<T, true>(a.h, a.d, a.T, a.d)), (operand<T, true>(wp, a.d, nv, a.d)),
                       a.b ? a.b + v0 : nullptr, a.target, a.lse, a.dloss, a.V, v0, D, ldd,
                       a.db ? db : nullptr);
    if (a.db)
      hipLaunchKernelGGL(k_db_sum, dim3(cdiv(nv, 256)), dim3(256), 0, st, db, n_tt, ldd, nv,
                         a.db + v0);
    if (a.dw) {
      const auto A = operand<float, false>(D, ldd, nv, a.T);
      const auto B = operand<T, false>(hl, a.d, a.d, a.T);
      T* out = static_cast<T*>(a.dw) + (size_t)v0 * a.d;
      hipError_t e = hipSuccess;
      if (p.s_dw == 1) {
        e = launch_product(A, B, 1, false, out, st);
      } else {
        e = launch_product(A, B, p.s_dw, false, dw, st);
        if (e == hipSuccess) e = launch_sum_parts(dw, p.s_dw, (size_t)nv * a.d, out, st);
      }
      if (e != hipSuccess) return e;
    }
    if (a.dh) {
      const auto A = operand<float, true>(D, ldd, a.T, nv);
      const auto B = operand<T, false>(wp, a.d, a.d, nv);
      const hipError_t e = p.direct_dh
                               ? launch_product(A, B, 1, false, static_cast<T*>(a.dh), st)
                               : launch_product(A, B, p.s_dh, v0 > 0, dh, st);
      if (e != hipSuccess) return e;
    }
  }
  if (a.dh && !p.direct_dh)
    return launch_sum_parts(dh, p.s_dh, (size_t)a.T * a.d, static_cast<T*>(a.dh), st);
  return hipGetLastError();
}

}  // namespace

size_t head_loss_ws(bool, int V, int, int T) {
  return align256((size_t)(T > 0 ? T : 1) * cdiv(V, f32p::BM) * sizeof(float2));
}
size_t head_loss_backward_ws(bool, int V, int d, int T) { return back_plan(V, d, T).total; }

hipError_t launch_head_loss(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? loss_f32<bf16_t>(a, st) : loss_f32<float>(a, st);
}

hipError_t launch_head_loss_backward(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? backward_f32<bf16_t>(a, st) : backward_f32<float>(a, st);
}

}  // namespace trimmoe
