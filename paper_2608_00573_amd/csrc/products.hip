// Products of the training losses in fp32 matrix instructions (any order,
// leading dimension and alignment of the operands).
#include "products.h"

#include <algorithm>

namespace trimmoe {

// B A^T over split blockIdx.z of K into the split's slice of out, added to what is
// there (`add`): a lane holds 4 consecutive elements of a row
template <int KIND, bool BKC>
__global__ __launch_bounds__(f32p::THREADS, f32p::Tile<KIND>::OCC) void k_prod_f32(
    Operand<false> A, Operand<BKC> B, int k_per, float* out, int add) {
  using namespace f32p;
  using T = Tile<KIND>;
  __shared__ __align__(16) float lds[T::FLOATS];
  const int n_at = (A.rows + T::A - 1) / T::A;
  const int a0 = (int)(blockIdx.x % n_at) * T::A, b0 = (int)(blockIdx.x / n_at) * T::B;
  const int k0 = min((int)blockIdx.z * k_per, A.K), k1 = min(k0 + k_per, A.K);
  F32Tile<KIND> t(a0, A.rows, b0, B.rows);
  // (a stream's rows of all groups are mixed: whole runs of them)
  if (T::STREAM) t.a = a0 + 16 * T::NA * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32_product<KIND>(A, B, a0, b0, k0, k1, lds, t);
  float* o = out + (size_t)blockIdx.z * A.rows * B.rows;
#pragma unroll
  for (int j = 0; j < T::NB; ++j) {
    const int b = t.row_b(j);
    if (j >= t.nb || b >= B.rows) continue;
    if constexpr (T::STREAM) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // elements `at` .. at + NA - 1; those before `a` are another lane's
        const int a = t.a + T::NA * (4 * ((threadIdx.x & 63) >> 4) + r), at = min(a, A.rows - T::NA);
        float* q = o + (size_t)b * A.rows + at;
#pragma unroll
        for (int i = 0; i < T::NA; ++i)
          if (at + i >= a) q[i] = add ? q[i] + t.acc[i][j][r] : t.acc[i][j][r];
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < T::NA; ++i) {
      if (i >= t.na) continue;
      const int a = t.row_a(i, 0), n = A.rows - a;
      float* q = o + (size_t)b * A.rows + a;
      if (n >= 4) {
        f32x4_t x = t.acc[i][j];
        if (add) x += *reinterpret_cast<const f32x4_any*>(q);
        *reinterpret_cast<f32x4_any*>(q) = x;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r < n) q[r] = add ? q[r] + t.acc[i][j][r] : t.acc[i][j][r];
      }
    }
  }
}

__global__ __launch_bounds__(256) void k_sum_parts(const float* part, int S, size_t n, float* out) {
  const size_t step = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    float s = part[i];
    for (int k = 1; k < S; ++k) s += part[(size_t)k * n + i];
    out[i] = s;
  }
}

template <bool BKC>
hipError_t launch_product(const Operand<false>& A, const Operand<BKC>& B, int splits, bool add,
                          float* out, hipStream_t st) {
  using namespace f32p;
  const int k_per = cdiv(cdiv(A.K, splits), KS) * KS;
  with_kind(product_kind(BKC, A.rows, B.rows), [&](auto kind) {
    using T = Tile<kind>;
    if constexpr (kind != kSmall && (!T::STREAM || BKC)) {
      const dim3 grid((unsigned)cdiv(A.rows, T::A) * cdiv(B.rows, T::B), 1, splits);
      hipLaunchKernelGGL((k_prod_f32<kind, BKC>), grid, dim3(THREADS), 0, st, A, B, k_per, out,
                         add ? 1 : 0);
    }
  });
  return hipGetLastError();
}

hipError_t launch_sum_parts(const float* part, int S, size_t n, float* out, hipStream_t st) {
  const dim3 grid((unsigned)std::min<size_t>((n + 255) / 256, 4096));
  hipLaunchKernelGGL(k_sum_parts, grid, dim3(256), 0, st, part, S, n, out);
  return hipGetLastError();
}

// the gradients of the rows (D w) and of the weights (D^T h)
template hipError_t launch_product<true>(const Operand<false>&, const Operand<true>&, int, bool,
                                         float*, hipStream_t);
template hipError_t launch_product<false>(const Operand<false>&, const Operand<false>&, int, bool,
                                          float*, hipStream_t);

}  // namespace trimmoe
