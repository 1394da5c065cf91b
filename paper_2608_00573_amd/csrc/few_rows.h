// What the kernels of the head loss's gradient share: row weights, and the
// arguments of the few-token path (head_loss.hip, skinny.hip).
#pragma once

#include <math.h>

#include "gemm.h"

namespace trimmoe {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// v plus the value of a lane of the same 16 (ROR: a DPP rotation)
template <int ROR>
__device__ __forceinline__ float row_add(float v) {
  const int i = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(i, ROR, 0xf, 0xf, false));
}
// the sum over the 16 lanes, in each of them
__device__ __forceinline__ float row16_sum(float v) {
  return row_add<0x121>(row_add<0x122>(row_add<0x124>(row_add<0x128>(v))));
}

// exp(z - lse) of a lane's logit.  The difference is taken first: it is small where the
// probability is not, and its rounding with it (z log2 e - lse log2 e would carry the
// rounding of lse log2 e, some 2^-20, into every term of a row).
__device__ __forceinline__ float softmax_of(float z, float lse) {
  return __builtin_amdgcn_exp2f((z - lse) * kLog2e);
}

// m, 2^-e and g / m of a weight g
__device__ __forceinline__ void row_weight(float g, float G, float& m, float& e, float& gm) {
  int x = 0;
  const float f = g == 0.f ? 0.5f : frexpf(g / G, &x);  // (NaN stays NaN)
  m = f == 0.f ? 1.f : 2.f * f;
  e = g == 0.f || f == 0.f ? 0.f : ldexpf(1.f, x - 1);
  gm = g / m;
}

// A row's part in the backward, by the lanes of a wavefront (t: the lane's row):
// its target, or -1 where it takes no part; lse; m, 2^-e and g / m of its
// weight, and the largest |g| of all rows
struct FewRow {
  int y;
  float lse, m, e, gm, G;
  __device__ __forceinline__ FewRow(const int32_t* target, const float* lses, const float* dloss,
                                    int V, int T, int t) {
    const bool in = t < T;
    const float L = in ? lses[t] : 0.f;
    y = in ? target[t] : -1;
    const bool live = y >= 0 && y < V && L != -__builtin_inff();
    if (!live) y = -1;
    lse = live ? L : 0.f;
    const float g = live ? dloss[t] : 0.f;
    G = fabsf(g);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) G = fmaxf(G, __shfl_xor(G, o));
    row_weight(g, G, m, e, gm);
  }
};

struct FewArgs {
  const bf16_t *w, *h;
  const float* b;
  const int32_t* target;
  const float *lse, *dloss;
  int V, d, T;
  bf16_t* D;
  float* db;
};

// D (z of rows_grad.h) in rows of 16 ET tokens in one stream of w (skinny.hip): ET 1 or,
// without db, 4
template <int ET>
hipError_t launch_dz_skinny(const FewArgs& a, int n_cu, hipStream_t st);

}  // namespace trimmoe
