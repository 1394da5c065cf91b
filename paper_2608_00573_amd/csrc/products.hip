// Products of the training losses in fp32 matrix instructions (any order,
// leading dimension and alignment of the operands; bf16 operands are widened).
#include "products.h"

namespace trimmoe {

// A B^T over split blockIdx.z of K: rounded to its output type, or into the
// split's slice of fp32 partials, added to what is there (`add`)
template <typename TO, typename TA, bool AK, typename TB, bool BKC>
__global__ __launch_bounds__(f32p::THREADS) void k_prod_f32(Operand<TA, AK> A, Operand<TB, BKC> B,
                                                            int k_per, TO* out, int add) {
  using namespace f32p;
  __shared__ __align__(16) float lds[4 * KS * LS];
  const int nt = blockIdx.y, mt = blockIdx.x;
  const int k0 = min((int)blockIdx.z * k_per, A.K), k1 = min(k0 + k_per, A.K);
  F32Acc acc;
  f32_tile(A, B, mt * BM, nt * BN, k0, k1, lds, acc);
  TO* o = out + (size_t)blockIdx.z * A.rows * B.rows;
#pragma unroll
  for (int j = 0; j < kTN; ++j) {
    const int c = nt * BN + f32_col(j);
    if (c >= B.rows) continue;
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = mt * BM + f32_row(i, r);
        if (m >= A.rows) continue;
        TO* q = o + (size_t)m * B.rows + c;
        *q = from_f32<TO>(add ? to_f32<TO>(*q) + acc[i][j][r] : acc[i][j][r]);
      }
  }
}

// out = sum of the S slices, rounded once
template <typename T>
__global__ __launch_bounds__(256) void k_sum_parts(const float* part, int S, size_t n, T* out) {
  const size_t step = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    float s = part[i];
    for (int k = 1; k < S; ++k) s += part[(size_t)k * n + i];
    out[i] = from_f32<T>(s);
  }
}

template <typename TO, typename TA, bool AK, typename TB, bool BKC>
hipError_t launch_product(const Operand<TA, AK>& A, const Operand<TB, BKC>& B, int splits, bool add,
                          TO* out, hipStream_t st) {
  using namespace f32p;
  const int k_per = cdiv(cdiv(A.K, splits), KS) * KS;
  const dim3 grid(cdiv(A.rows, BM), cdiv(B.rows, BN), splits);
  hipLaunchKernelGGL((k_prod_f32<TO, TA, AK, TB, BKC>), grid, dim3(THREADS), 0, st, A, B, k_per, out,
                     add ? 1 : 0);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_sum_parts(const float* part, int S, size_t n, T* out, hipStream_t st) {
  const dim3 grid((unsigned)std::min<size_t>((n + 255) / 256, 4096));
  hipLaunchKernelGGL(k_sum_parts<T>, grid, dim3(256), 0, st, part, S, n, out);
  return hipGetLastError();
}

#define PRODUCT(TO, TA, AK, TB, BKC)                                                             \
  template hipError_t launch_product<TO, TA, AK, TB, BKC>(const Operand<TA, AK>&,                \
                                                          const Operand<TB, BKC>&, int, bool, TO*, \
                                                          hipStream_t);
// logits; gradients of the rows (D w) and of the weights (D^T h), whole and in partials
PRODUCT(float, bf16_t, true, bf16_t, true)
PRODUCT(float, float, true, float, true)
PRODUCT(bf16_t, float, true, bf16_t, false)
PRODUCT(float, float, true, bf16_t, false)
PRODUCT(float, float, true, float, false)
PRODUCT(bf16_t, float, false, bf16_t, false)
PRODUCT(float, float, false, bf16_t, false)
PRODUCT(float, float, false, float, false)
#undef PRODUCT
template hipError_t launch_sum_parts<float>(const float*, int, size_t, float*, hipStream_t);
template hipError_t launch_sum_parts<bf16_t>(const float*, int, size_t, bf16_t*, hipStream_t);

}  // namespace trimmoe
