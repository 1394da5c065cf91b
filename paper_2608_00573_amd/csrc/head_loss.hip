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
#include "mfma_core.h"
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
  __shared__ __align__(16) float lds[4 * KS * LS];
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

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// One wavefront a row: joins the pairs and takes the target's logit from one
// more dot product (a gathered row of w; the pairs do not keep it).
// BASE2: the pairs' maxima are in base 2 (z log2 e).
template <typename T, bool BASE2>
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
  for (int i = lane; i < n_vt; i += 64) {
    const float2 v = p[i];
    sum = fmaf(v.y, BASE2 ? exp2f(v.x - ms) : expf(v.x - ms), sum);
  }
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
  const float L = m == ninf && sum == 0.f ? ninf : (BASE2 ? m * kLn2 : m) + logf(sum);
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
  __shared__ __align__(16) float lds[4 * KS * LS];
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

// ------------------------------------------------------ backward, bf16 --
// Three products on the large-group core, whose operands are both K-contiguous,
// so whatever runs the other way is laid out once: h^T for dw (zeros in the rows
// that take no part, whose h may hold anything) and w^T of the piece for dh; D
// is written in both orders by its own epilogue.
//   * D enters the products in bf16.  Its order for dh holds softmax - onehot
//     without the row's weight g (applied to the fp32 sums), its order for dw
//     g / G times that, G the largest |g| (applied to the fp32 sums): weights
//     that are all alike are exact, and so is the -1 of an unlikely target,
//     which carries most of an untrained row's gradient.
//   * dh is summed in fp32 over pieces and K splits, then rounded once.

// row t's part in the backward: its target, or -1 where it takes no part; its
// weight and weight / G (0 there); lse log2 e.  One block.
__global__ __launch_bounds__(1024) void k_row_prep(const int32_t* target, const float* lse,
                                                   const float* dloss, int V, int T, int Tp,
                                                   int32_t* ys, float* gl, float* gs, float* l2,
                                                   float* G) {
  __shared__ float s_m[16];
  float m = 0.f;
  for (int t = threadIdx.x; t < Tp; t += 1024) {
    const int y = t < T ? target[t] : -1;
    const float L = t < T ? lse[t] : 0.f;
    const bool live = y >= 0 && y < V && L != -__builtin_inff();
    const float g = live ? dloss[t] : 0.f;
    ys[t] = live ? y : -1;
    gl[t] = g;
    l2[t] = live ? L * kLog2e : 0.f;
    m = fmaxf(m, fabsf(g));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) s_m[threadIdx.x >> 6] = m;
  __syncthreads();
  m = s_m[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, s_m[i]);
  if (threadIdx.x == 0) *G = m;
  // (each thread reads back its own rows)
  for (int t = threadIdx.x; t < Tp; t += 1024) {
    const float g = gl[t];
    gs[t] = g == 0.f ? 0.f : g / m;
  }
}

// out [C, Rp] = in [R, C] transposed, columns past R zero; rows with ys < 0 are
// zeros (ys may be NULL).  64 x 64 tiles: 128-byte runs on both sides.
__global__ __launch_bounds__(256) void k_transpose(const bf16_t* in, const int32_t* ys, int R, int C,
                                                   int Rp, bf16_t* out) {
  __shared__ __align__(16) bf16_t s[64][72];
  const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
  const int row = threadIdx.x >> 3, ch = 8 * (threadIdx.x & 7);
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int r = r0 + row + i;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < R && (!ys || ys[r] >= 0)) v = *reinterpret_cast<const uint4*>(in + (size_t)r * C + c0 + ch);
    *reinterpret_cast<uint4*>(&s[row + i][ch]) = v;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int c = row + i;
    uint32_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      w[u] = (uint32_t)s[ch + 2 * u][c] | (uint32_t)s[ch + 2 * u + 1][c] << 16;
    *reinterpret_cast<uint4*>(out + (size_t)(c0 + c) * Rp + r0 + ch) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace

__device__ __forceinline__ int cdiv_d(int a, int b) { return (a + b - 1) / b; }

// operand rows of a tile of the large-group core: A rows from m0 (m of them
// valid), B rows from n0, both K-contiguous with leading dimension ld, from
// column k0
__device__ __forceinline__ void big_rows(BigRows& q, const bf16_t* A, int m0, int m_valid,
                                         const bf16_t* B, int n0, int n_valid, int ld, int k0, int r0,
                                         int cc) {
  q.ra = buf_rsrc(A + (size_t)m0 * ld);
  q.rb0 = buf_rsrc(B + (size_t)n0 * ld);
  q.rb1 = q.rb0;
  q.none = buf_rsrc_empty(A);
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int r = r0 + big::RPP * u;
    q.off[u] = ((uint32_t)min(r, m_valid - 1) * ld + k0 + cc) * 2;
    q.off[8 + u] = ((uint32_t)min(r, n_valid - 1) * ld + k0 + cc) * 2;
  }
}

// the block's lane constants on that core
struct BigLane {
  int lane, wave, wm, wn, r0, cc;
  uint32_t a[2], b[2];
  __device__ __forceinline__ BigLane() {
    const int tid = threadIdx.x;
    lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    wm = wave >> 1;
    wn = wave & 1;
    r0 = tid >> 3;
    cc = 8 * ((tid & 7) ^ swz16(r0));
    const int fr = lane & 15, hk = lane >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const uint32_t ch = ((4 * ks + hk) ^ swz16(fr)) << 4;
      a[ks] = (wm * 128 + fr) * big::RB + ch;
      b[ks] = (wn * 128 + fr) * big::RB + ch;
    }
  }
};

__device__ __forceinline__ void big_zero(AccBig& acc) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{};
}

// LDS image of a 256 x 256 bf16 tile: rows padded by 16 bytes
constexpr int kImgRow = 2 * 256 + 16;
static_assert(256 * kImgRow <= big::LDS, "tile image fits the stages");

// the image's valid rows and columns (a multiple of 8) to out, rows ld apart
__device__ __forceinline__ void big_image_out(const char* lds, bf16_t* out, size_t ld, int rows,
                                              int cols) {
  lds_barrier();
#pragma unroll 4
  for (int idx = threadIdx.x; idx < 256 * 32; idx += big::THREADS) {
    const int r = idx >> 5, ch = idx & 31;
    if (r < rows && ch * 8 < cols)
      *reinterpret_cast<uint4*>(out + (size_t)r * ld + ch * 8) =
          *reinterpret_cast<const uint4*>(lds + r * kImgRow + ch * 16);
  }
  lds_barrier();
}

struct DzArgs {
  const bf16_t* w;    // the piece's first row
  const bf16_t* h;
  const float* bias;  // the piece's first row, or NULL
  const int32_t* ys;
  const float *gs, *l2;
  int nv, v0, d, T;
  int Vp, Tp;         // leading dimensions of D and D^T
  bf16_t *D, *DT;
  float* db_part;     // [token tiles][Vp] or NULL
};

// D of a piece: A = w (vocabulary rows), B = h, so that a lane holds 4
// consecutive vocabulary rows of one row t per accumulator
__global__ __launch_bounds__(big::THREADS) void k_dz_big(DzArgs a) {
  __shared__ __align__(16) char lds[big::LDS];
  const BigLane L;
  TileSched S;
  int ntiles;
  if (!S.init(a.Vp / big::BM, cdiv_d(a.T, big::BN), 1, ntiles)) return;
  const int nk = a.d / BK;
  AccBig acc;
  for (int jt = 0; jt < ntiles; ++jt) {
    int vt, tt, sp;
    S.decode(jt, vt, tt, sp);
    const int c0 = vt * big::BM, t0 = tt * big::BN;
    const int v_valid = min(big::BM, a.nv - c0), t_valid = min(big::BN, a.T - t0);
    {
      BigRows q;
      big_rows(q, a.w, c0, v_valid, a.h, t0, t_valid, a.d, 0, L.r0, L.cc);
      big_zero(acc);
      big_tile<false>(lds, q, nk, acc, L.a, L.b);
    }
    const int c = L.lane & 15, hq = L.lane >> 4;
    const int rl = L.wm * 128 + 4 * hq;  // the lane's first vocabulary row
    const float* bias = a.bias ? a.bias + c0 : nullptr;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tl = L.wn * 128 + 16 * j + c, t = min(t0 + tl, a.T - 1);
      const float l2 = a.l2[t];
      const int y = tl < t_valid ? a.ys[t] : -1;
      const int yr = y - a.v0 - c0 - rl;  // the target's row, relative to the lane's first
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f32x4_t x = acc[i][j];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float z = x[r];
          if (bias) z += bias[min(rl + 16 * i + r, v_valid - 1)];
          const float p = __builtin_amdgcn_exp2f(fmaf(z, kLog2e, -l2));
          const bool in = y >= 0 && rl + 16 * i + r < v_valid;
          x[r] = in ? p - (16 * i + r == yr ? 1.f : 0.f) : 0.f;
        }
        acc[i][j] = x;
        uint2 w;
        w.x = pack_bf16x2(x[0], x[1]);
        w.y = pack_bf16x2(x[2], x[3]);
        *reinterpret_cast<uint2*>(lds + tl * kImgRow + (rl + 16 * i) * 2) = w;
      }
    }
    big_image_out(lds, a.D + (size_t)t0 * a.Vp + c0, a.Vp, t_valid, 256);
    // the other order, weighted; column sums for db
    float sum[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[i][r] = 0.f;
    const bool odd = c & 1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tl = L.wn * 128 + 16 * j + c;
      const float g = a.gs[min(t0 + tl, a.T - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const float v0 = acc[i][j][r] * g, v1 = acc[i][j][r + 1] * g;
          sum[i][r] += v0;
          sum[i][r + 1] += v1;
          const float got = swap_pair(odd ? v0 : v1);
          const uint32_t w = odd ? pack_bf16x2(got, v1) : pack_bf16x2(v0, got);
          *reinterpret_cast<uint32_t*>(lds + (rl + 16 * i + r + (odd ? 1 : 0)) * kImgRow +
                                       (L.wn * 128 + 16 * j + (c & ~1)) * 2) = w;
        }
    }
    big_image_out(lds, a.DT + (size_t)c0 * a.Tp + t0, a.Tp, 256, min(big::BN, a.Tp - t0));
    if (a.db_part) {
      float* s_db = reinterpret_cast<float*>(lds);  // [2][256]
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = sum[i][r];
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o);
          if (c == 0) s_db[L.wn * 256 + rl + 16 * i + r] = v;
        }
      lds_barrier();
      a.db_part[(size_t)tt * a.Vp + c0 + threadIdx.x] = s_db[threadIdx.x] + s_db[256 + threadIdx.x];
      lds_barrier();
    }
  }
}

struct BigProdArgs {
  const bf16_t* A;  // [M, K]
  const bf16_t* B;  // [N, K]
  int M, N, K;
  const float* scale;  // PARTIAL: not read
  void* out;           // bf16 [M, N] times *scale, or fp32 slices [splits][M, N]
  int splits;
  int add;             // PARTIAL: added to what the slices hold
};

// A B^T on the large-group core
template <bool PARTIAL>
__global__ __launch_bounds__(big::THREADS) void k_prod_big(BigProdArgs a) {
  __shared__ __align__(16) char lds[big::LDS];
  const BigLane L;
  TileSched S;
  int ntiles;
  if (!S.init(cdiv_d(a.M, big::BM), cdiv_d(a.N, big::BN), a.splits, ntiles)) return;
  const int nk = a.K / BK;
  AccBig acc;
  for (int jt = 0; jt < ntiles; ++jt) {
    int mt, nt, sp;
    S.decode(jt, mt, nt, sp);
    const int m0 = mt * big::BM, n0 = nt * big::BN;
    const int m_valid = min(big::BM, a.M - m0), n_valid = min(big::BN, a.N - n0);
    const int ka = (int)((long)sp * nk / a.splits), kb = (int)((long)(sp + 1) * nk / a.splits);
    {
      BigRows q;
      big_rows(q, a.A, m0, m_valid, a.B, n0, n_valid, a.K, ka * BK, L.r0, L.cc);
      big_zero(acc);
      big_tile<false>(lds, q, kb - ka, acc, L.a, L.b);
    }
    const int c = L.lane & 15, hq = L.lane >> 4;
    const int rl = L.wm * 128 + 4 * hq;
    if constexpr (PARTIAL) {
      float* out = static_cast<float*>(a.out) + (size_t)sp * a.M * a.N + (size_t)m0 * a.N + n0;
      const int cl = L.wn * 128 + c;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (cl + 16 * j < n_valid)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (rl + 16 * i + r < m_valid) {
                float* o = out + (size_t)(rl + 16 * i + r) * a.N + cl + 16 * j;
                *o = a.add ? *o + acc[i][j][r] : acc[i][j][r];
              }
    } else {
      const float g = *a.scale;
      const bool odd = c & 1;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            const float v0 = acc[i][j][r] * g, v1 = acc[i][j][r + 1] * g;
            const float got = swap_pair(odd ? v0 : v1);
            const uint32_t w = odd ? pack_bf16x2(got, v1) : pack_bf16x2(v0, got);
            *reinterpret_cast<uint32_t*>(lds + (rl + 16 * i + r + (odd ? 1 : 0)) * kImgRow +
                                         (L.wn * 128 + 16 * j + (c & ~1)) * 2) = w;
          }
      big_image_out(lds, static_cast<bf16_t*>(a.out) + (size_t)m0 * a.N + n0, a.N, m_valid, n_valid);
    }
  }
}

namespace {

// dh = g_t times the sum of the S slices, rounded once; 4 elements a thread (d
// is a multiple of 64)
__global__ __launch_bounds__(256) void k_dh_finish(const float* part, int S, const float* gl, int T,
                                                   int d, bf16_t* dh) {
  const size_t n = (size_t)T * d, i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= n) return;
  float4 s = *reinterpret_cast<const float4*>(part + i);
  for (int k = 1; k < S; ++k) {
    const float4 x = *reinterpret_cast<const float4*>(part + (size_t)k * n + i);
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  const float g = gl[i / d];
  uint2 w;
  w.x = pack_bf16x2(s.x * g, s.y * g);
  w.y = pack_bf16x2(s.z * g, s.w * g);
  *reinterpret_cast<uint2*>(dh + i) = w;
}

// db of a piece from the token tiles' sums
__global__ __launch_bounds__(256) void k_db_finish(const float* part, int n_tt, int ld, int n,
                                                   const float* G, float* db) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n) return;
  float s = 0.f;
  for (int i = 0; i < n_tt; ++i) s += part[(size_t)i * ld + c];
  db[c] = s * *G;
}

// ------------------------------------------------------------------ plan --
// bytes of D that a piece may take
constexpr size_t kPieceBytes = (size_t)256 << 20;
constexpr int kCu = 256;
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
  hipLaunchKernelGGL((k_loss_join<T, false>), dim3(cdiv(a.T, 4)), dim3(256), 0, st, part, n_vt, a.V, a.d, a.T,
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

// bf16: a piece's D in both orders
struct BackPlanBf16 {
  int Vp, Tp, s_dh;  // columns of a piece, rows rounded up to a K slice, splits of dh
  size_t o_rows, o_ht, o_wt, o_d, o_dt, o_dh, o_db, total;
};

// K splits of an m x n product of nk slices on the large-group core: the fewest
// slices on the busiest CU, a doubling of the partials for no less than an eighth
int big_splits(int m, int n, int nk) {
  const long tiles = (long)cdiv(m, big::BM) * cdiv(n, big::BN);
  int best = 1;
  long cost = (tiles + kCu - 1) / kCu * nk;
  for (int s = 2; s <= 32 && nk / s >= 16; s *= 2) {
    const long c = (tiles * s + kCu - 1) / kCu * cdiv(nk, s);
    if (8 * c <= 7 * cost) {
      best = s;
      cost = c;
    }
  }
  return best;
}

BackPlanBf16 back_plan_bf16(int V, int d, int T) {
  BackPlanBf16 p;
  const size_t rows = T > 0 ? T : 1;
  p.Tp = (int)((rows + 63) / 64 * 64);
  const size_t fit = kPieceBytes / (4 * (size_t)p.Tp) / big::BM * big::BM;
  const int most = (int)std::min<size_t>(std::max<size_t>(fit, big::BM), (size_t)1 << 22);
  const int n_pieces = cdiv(V, most);
  p.Vp = cdiv(cdiv(V, n_pieces), big::BM) * big::BM;
  p.s_dh = big_splits((int)rows, d, p.Vp / BK);
  size_t o = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = o;
    o += align256(bytes);
    return at;
  };
  p.o_rows = take(4 * (size_t)p.Tp * 4 + 256);
  p.o_ht = take((size_t)d * p.Tp * 2);
  p.o_wt = take((size_t)d * p.Vp * 2);
  p.o_d = take(rows * p.Vp * 2);
  p.o_dt = take((size_t)p.Vp * p.Tp * 2);
  p.o_dh = take((size_t)p.s_dh * rows * d * 4);
  p.o_db = take((size_t)cdiv((int)rows, big::BN) * p.Vp * 4);
  p.total = o;
  return p;
}

hipError_t loss_bf16(const HeadLossArgs& a, hipStream_t st) {
  float2* part = reinterpret_cast<float2*>(a.ws);
  const int n_vt = exit_vtiles(true, false, exit_streams(true, true, a.T, a.V, a.d), a.T, a.V, a.n_cu);
  const hipError_t e =
      launch_head_loss_partials(a.w, a.b, a.h, a.T, a.V, a.d, n_vt, part, a.n_cu, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_loss_join<bf16_t, true>), dim3(cdiv(a.T, 4)), dim3(256), 0, st, part, n_vt,
                     a.V, a.d, a.T, static_cast<const bf16_t*>(a.w), a.b,
                     static_cast<const bf16_t*>(a.h), a.target, a.loss, a.lse);
  return hipGetLastError();
}

hipError_t backward_bf16(const HeadLossArgs& a, hipStream_t st) {
  const BackPlanBf16 p = back_plan_bf16(a.V, a.d, a.T);
  int32_t* ys = reinterpret_cast<int32_t*>(a.ws + p.o_rows);
  float* gl = reinterpret_cast<float*>(ys) + p.Tp;
  float *gs = gl + p.Tp, *l2 = gs + p.Tp, *G = l2 + p.Tp;
  bf16_t* ht = reinterpret_cast<bf16_t*>(a.ws + p.o_ht);
  bf16_t* wt = reinterpret_cast<bf16_t*>(a.ws + p.o_wt);
  bf16_t* D = reinterpret_cast<bf16_t*>(a.ws + p.o_d);
  bf16_t* DT = reinterpret_cast<bf16_t*>(a.ws + p.o_dt);
  float* dh = reinterpret_cast<float*>(a.ws + p.o_dh);
  float* db = reinterpret_cast<float*>(a.ws + p.o_db);
  const bf16_t* w = static_cast<const bf16_t*>(a.w);
  const bf16_t* h = static_cast<const bf16_t*>(a.h);
  const int n_tt = cdiv(a.T, big::BN);
  const auto grid = [&](long tiles) { return dim3((unsigned)std::min<long>(tiles, a.n_cu)); };
  hipLaunchKernelGGL(k_row_prep, dim3(1), dim3(1024), 0, st, a.target, a.lse, a.dloss, a.V, a.T, p.Tp,
                     ys, gl, gs, l2, G);
  if (a.dw)
    hipLaunchKernelGGL(k_transpose, dim3(p.Tp / 64, a.d / 64), dim3(256), 0, st, h, ys, a.T, a.d,
                       p.Tp, ht);
  for (int v0 = 0; v0 < a.V; v0 += p.Vp) {
    const int nv = std::min(p.Vp, a.V - v0), Vp = cdiv(nv, big::BM) * big::BM;
    const bf16_t* wp = w + (size_t)v0 * a.d;
    DzArgs z{wp, h, a.b ? a.b + v0 : nullptr, ys, gs, l2, nv, v0, a.d, a.T, Vp, p.Tp, D, DT,
             a.db ? db : nullptr};
    if (a.T > 0)
      hipLaunchKernelGGL(k_dz_big, grid((long)(Vp / big::BM) * n_tt), dim3(big::THREADS), 0, st, z);
    if (a.db)
      hipLaunchKernelGGL(k_db_finish, dim3(cdiv(nv, 256)), dim3(256), 0, st, db, n_tt, Vp, nv, G,
                         a.db + v0);
    if (a.dw) {
      BigProdArgs q{DT, ht, nv, a.d, a.T > 0 ? p.Tp : 0, G, static_cast<bf16_t*>(a.dw) + (size_t)v0 * a.d,
                    1, 0};
      hipLaunchKernelGGL(k_prod_big<false>, grid((long)cdiv(nv, big::BM) * cdiv(a.d, big::BN)),
                         dim3(big::THREADS), 0, st, q);
    }
    if (a.dh) {
      hipLaunchKernelGGL(k_transpose, dim3(Vp / 64, a.d / 64), dim3(256), 0, st, wp, nullptr, nv, a.d,
                         Vp, wt);
      BigProdArgs q{D, wt, a.T, a.d, Vp, nullptr, dh, p.s_dh, v0 > 0};
      hipLaunchKernelGGL(k_prod_big<true>, grid((long)n_tt * cdiv(a.d, big::BN) * p.s_dh),
                         dim3(big::THREADS), 0, st, q);
    }
  }
  if (a.dh) {
    const size_t n = (size_t)a.T * a.d / 4;
    hipLaunchKernelGGL(k_dh_finish, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, dh, p.s_dh,
                       gl, a.T, a.d, static_cast<bf16_t*>(a.dh));
  }
  return hipGetLastError();
}

}  // namespace

size_t head_loss_ws(bool bf16, int V, int, int T) {
  const int rows = T > 0 ? T : 1;
  return align256((size_t)rows * cdiv(V, bf16 ? exit_tile_rows(true, rows) : f32p::BM) *
                  sizeof(float2));
}
size_t head_loss_backward_ws(bool bf16, int V, int d, int T) {
  return bf16 ? back_plan_bf16(V, d, T).total : back_plan(V, d, T).total;
}

hipError_t launch_head_loss(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? loss_bf16(a, st) : loss_f32<float>(a, st);
}

hipError_t launch_head_loss_backward(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? backward_bf16(a, st) : backward_f32<float>(a, st);
}

}  // namespace trimmoe
