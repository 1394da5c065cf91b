// Balance loss of a router, its per-expert counts and its gradients.
//   p_t = softmax(w h_t + b);  c_e = routed slots of expert e, S in all;
//   n = rows with a routed slot;  P_e = sum of p_te over those rows
//   L = E / (S n) sum_e c_e P_e         (1 where the load is even)
//   dz_te = g E / (S n) p_te (c_e - sum_j p_tj c_j), 0 in rows without a slot
//   dh = dz w,  dw = dz^T h,  db_e = sum_t dz_te        (counts held constant)
#include <math.h>

#include "loss.h"
#include "products.h"

namespace trimmoe {

namespace {

constexpr int EV = TRIMMOE_MAX_EXPERTS / 64;  // experts a lane holds
constexpr int kRowBlocks = 512;

int row_blocks(int T) { return std::min(kRowBlocks, cdiv(std::max(T, 1), 4)); }

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// whether row t has a routed slot
__device__ __forceinline__ bool row_live(const int16_t* target, int t, int k, int E) {
  bool live = false;
  for (int s = 0; s < k; ++s) {
    const int e = target[(size_t)t * k + s];
    live |= e >= 0 && e < E;
  }
  return live;
}

// softmax of the logits in `prob`, in place; one wavefront a row.  A block's
// sums of p over its rows with a slot, and its counts
__global__ __launch_bounds__(256) void k_balance_rows(float* prob, const float* b,
                                                      const int16_t* target, int T, int E, int k,
                                                      float* part_p, int32_t* part_c) {
  __shared__ float s_p[4][TRIMMOE_MAX_EXPERTS];
  __shared__ int32_t s_c[TRIMMOE_MAX_EXPERTS + 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int e = threadIdx.x; e <= E; e += 256) s_c[e] = 0;
  __syncthreads();
  float sum[EV] = {};
  for (int t = blockIdx.x * 4 + wave; t < T; t += 4 * gridDim.x) {
    float* p = prob + (size_t)t * E;
    float z[EV], m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      const int e = lane + 64 * i;
      z[i] = e < E ? p[e] + (b ? b[e] : 0.f) : -__builtin_inff();
      m = fmaxf(m, z[i]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    // (a row without a logit above -inf has p = 0; a NaN logit makes it NaN)
    const float ms = m == -__builtin_inff() ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      z[i] = lane + 64 * i < E ? expf(z[i] - ms) : 0.f;
      s += z[i];
    }
    s = wave_sum(s);
    s = s == 0.f ? 1.f : s;
    const bool live = row_live(target, t, k, E);
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      const int e = lane + 64 * i;
      if (e >= E) continue;
      const float x = z[i] / s;
      p[e] = x;
      if (live) sum[i] += x;
    }
    if (lane < k) {
      const int e = target[(size_t)t * k + lane];
      if (e >= 0 && e < E) atomicAdd(&s_c[e], 1);
    }
    if (lane == 0 && live) atomicAdd(&s_c[E], 1);
  }
#pragma unroll
  for (int i = 0; i < EV; ++i) s_p[wave][lane + 64 * i] = sum[i];
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 256) {
    part_c[(size_t)blockIdx.x * (E + 1) + e] = s_c[e];
    if (e < E)
      part_p[(size_t)blockIdx.x * E + e] = (s_p[0][e] + s_p[1][e]) + (s_p[2][e] + s_p[3][e]);
  }
}

// sums over the blocks, and the loss
__global__ __launch_bounds__(256) void k_balance_loss(const float* part_p, const int32_t* part_c,
                                                      int nb, int E, int32_t* counts, float* prob_sum,
                                                      float* loss) {
  __shared__ double s_l[256];
  __shared__ double s_n[256];
  double l = 0.0, slots = 0.0;
  int rows = 0;
  const int e = threadIdx.x;
  if (e < E) {
    double p = 0.0;
    int c = 0;
    for (int i = 0; i < nb; ++i) {
      p += part_p[(size_t)i * E + e];
      c += part_c[(size_t)i * (E + 1) + e];
    }
    counts[e] = c;
    prob_sum[e] = (float)p;
    l = p * c;
    slots = c;
  }
  if (e == 0) {
    for (int i = 0; i < nb; ++i) rows += part_c[(size_t)i * (E + 1) + E];
    counts[E] = rows;
  }
  s_l[e] = l;
  s_n[e] = slots;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (e < o) {
      s_l[e] += s_l[e + o];
      s_n[e] += s_n[e + o];
    }
    __syncthreads();
  }
  if (e == 0) *loss = rows > 0 ? (float)(E * s_l[0] / (s_n[0] * rows)) : 0.f;
}

// dz of every row, and a block's column sums (db)
__global__ __launch_bounds__(256) void k_balance_dz(const float* prob, const int16_t* target,
                                                    const int32_t* counts, const float* dloss, int T,
                                                    int E, int k, float* dz, float* part_db) {
  __shared__ float s_p[4][TRIMMOE_MAX_EXPERTS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // counts against their mean: sum_j p_tj = 1, so the mean drops out of
  // c_e - sum_j p_tj c_j and would only cost digits
  float c[EV], total = 0.f;
#pragma unroll
  for (int i = 0; i < EV; ++i) {
    const int e = lane + 64 * i;
    c[i] = e < E ? (float)counts[e] : 0.f;
    total += c[i];
  }
  total = wave_sum(total);
  const int n = counts[E];
  const float scale = n > 0 ? *dloss * (float)((double)E / ((double)total * n)) : 0.f;
  const float mean = total / E;
#pragma unroll
  for (int i = 0; i < EV; ++i) c[i] -= mean;
  float sum[EV] = {};
  for (int t = blockIdx.x * 4 + wave; t < T; t += 4 * gridDim.x) {
    const bool live = row_live(target, t, k, E);
    float p[EV], s = 0.f;
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      const int e = lane + 64 * i;
      p[i] = e < E ? prob[(size_t)t * E + e] : 0.f;
      s = fmaf(p[i], c[i], s);
    }
    s = wave_sum(s);
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      const int e = lane + 64 * i;
      if (e >= E) continue;
      const float x = live ? scale * p[i] * (c[i] - s) : 0.f;
      dz[(size_t)t * E + e] = x;
      sum[i] += x;
    }
  }
#pragma unroll
  for (int i = 0; i < EV; ++i) s_p[wave][lane + 64 * i] = sum[i];
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += 256)
    part_db[(size_t)blockIdx.x * E + e] = (s_p[0][e] + s_p[1][e]) + (s_p[2][e] + s_p[3][e]);
}

// rows with a slot, zeros for the others: an inactive row's h may hold
// anything, and 0 * NaN is NaN
template <typename T>
__global__ __launch_bounds__(256) void k_live_rows(const T* h, const int16_t* target, int E, int k,
                                                   int d, T* out) {
  const size_t t = blockIdx.x;
  const bool live = row_live(target, blockIdx.x, k, E);
  for (int i = threadIdx.x; i < d; i += 256) out[t * d + i] = live ? h[t * d + i] : T(0);
}

struct BackPlan {
  int s_dw;
  size_t o_dz, o_db, o_dw, o_h, total;
};

BackPlan back_plan(int E, int d, int T) {
  BackPlan p;
  const size_t rows = std::max(T, 1);
  p.s_dw = product_splits(E, d, T);
  p.o_dz = 0;
  p.o_db = align256(rows * E * 4);
  p.o_dw = p.o_db + align256((size_t)row_blocks(T) * E * 4);
  p.o_h = p.o_dw + (p.s_dw > 1 ? align256((size_t)p.s_dw * E * d * 4) : 0);
  p.total = p.o_h + align256(rows * d * 4);
  return p;
}

template <typename T>
hipError_t forward(const BalanceArgs& a, hipStream_t st) {
  const auto H = operand<T, true>(a.h, a.d, a.T, a.d);
  const auto W = operand<T, true>(a.w, a.d, a.E, a.d);
  if (a.T > 0) {
    const hipError_t e = launch_product(H, W, 1, false, a.prob, st);
    if (e != hipSuccess) return e;
  }
  const int nb = a.T > 0 ? row_blocks(a.T) : 0;
  float* part_p = reinterpret_cast<float*>(a.ws);
  int32_t* part_c =
      reinterpret_cast<int32_t*>(a.ws + align256((size_t)row_blocks(a.T) * a.E * 4));
  if (nb)
    hipLaunchKernelGGL(k_balance_rows, dim3(nb), dim3(256), 0, st, a.prob, a.b, a.target, a.T, a.E,
                       a.k, part_p, part_c);
  hipLaunchKernelGGL(k_balance_loss, dim3(1), dim3(256), 0, st, part_p, part_c, nb, a.E, a.counts,
                     a.prob_sum, a.loss);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const BalanceArgs& a, hipStream_t st) {
  const BackPlan p = back_plan(a.E, a.d, a.T);
  float* dz = reinterpret_cast<float*>(a.ws + p.o_dz);
  float* part_db = reinterpret_cast<float*>(a.ws + p.o_db);
  float* part_dw = reinterpret_cast<float*>(a.ws + p.o_dw);
  const int nb = row_blocks(a.T);
  hipLaunchKernelGGL(k_balance_dz, dim3(nb), dim3(256), 0, st, a.prob, a.target, a.counts, a.dloss,
                     a.T, a.E, a.k, dz, part_db);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.db) e = launch_sum_parts(part_db, nb, (size_t)a.E, a.db, st);
  if (e == hipSuccess && a.dh && a.T > 0)
    e = launch_product(operand<float, true>(dz, a.E, a.T, a.E),
                       operand<T, false>(a.w, a.d, a.d, a.E), 1, false, static_cast<T*>(a.dh), st);
  if (e == hipSuccess && a.dw) {
    const auto D = operand<float, false>(dz, a.E, a.E, a.T);
    T* hl = reinterpret_cast<T*>(a.ws + p.o_h);
    if (a.T > 0)
      hipLaunchKernelGGL(k_live_rows<T>, dim3(a.T), dim3(256), 0, st, static_cast<const T*>(a.h),
                         a.target, a.E, a.k, a.d, hl);
    const auto H = operand<T, false>(hl, a.d, a.d, a.T);
    T* dw = static_cast<T*>(a.dw);
    if (p.s_dw == 1) {
      e = launch_product(D, H, 1, false, dw, st);
    } else {
      e = launch_product(D, H, p.s_dw, false, part_dw, st);
      if (e == hipSuccess) e = launch_sum_parts(part_dw, p.s_dw, (size_t)a.E * a.d, dw, st);
    }
  }
  return e;
}

}  // namespace

size_t balance_ws(int E, int T) {
  const size_t nb = row_blocks(T);
  return align256(nb * E * 4) + align256(nb * (E + 1) * 4);
}
size_t balance_backward_ws(int E, int d, int T) { return back_plan(E, d, T).total; }

hipError_t launch_balance(const BalanceArgs& a, hipStream_t st) {
  return a.bf16 ? forward<bf16_t>(a, st) : forward<float>(a, st);
}
hipError_t launch_balance_backward(const BalanceArgs& a, hipStream_t st) {
  return a.bf16 ? backward<bf16_t>(a, st) : backward<float>(a, st);
}

}  // namespace trimmoe
