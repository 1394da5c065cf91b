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

#include "few_rows.h"
#include "gemm.h"
#include "loss.h"
#include "products.h"
#include "rows_grad.h"

namespace trimmoe {

namespace {

// ------------------------------------------------------- forward, fp32 --
// A = w (vocabulary rows), B = h: a lane holds 16 vocabulary rows of a token, so the
// pair of a token is a reduction over registers, two lane exchanges and the
// wavefronts along the vocabulary.  A NaN logit makes the sum NaN.  Bound by the fp32
// matrix rate or, for few tokens, by reading w: 3000 tokens, d 333, vocabulary 20001:
// 400 us (101 TFLOP/s); 7 tokens, d 2048, vocabulary 151936: 298 us (4.2 TB/s).
template <int KIND>
__global__ __launch_bounds__(f32p::THREADS, f32p::Tile<KIND>::OCC) void k_loss_f32(
    Operand<true> W, Operand<true> H, const float* bias, int n_vt, float2* part) {
  using T = f32p::Tile<KIND>;
  __shared__ __align__(16) float lds[T::FLOATS];
  __shared__ float2 s_p[T::WA][T::B];
  const int vt = blockIdx.x, tt = blockIdx.y;
  const int v0 = vt * T::A, t0 = tt * T::B;
  F32Tile<KIND> t(v0, W.rows, t0, H.rows);
  f32_product<KIND>(W, H, v0, t0, 0, W.K, lds, t);
  const float ninf = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < T::NB; ++j) {
    if (j >= t.nb) continue;
    float m = ninf;
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int v = t.row_a(i, r);
        float z = t.acc[i][j][r];
        if (bias) z += bias[min(v, W.rows - 1)];
        z = i < t.na && v < W.rows ? z : ninf;
        t.acc[i][j][r] = z;
        m = fmaxf(m, z);
      }
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float ms = m == ninf ? 0.f : m;
    // (in a tree: a chain would round each small term at the size of the largest)
    float e[4 * T::NA];
#pragma unroll
    for (int i = 0; i < T::NA; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) e[4 * i + r] = expf(t.acc[i][j][r] - ms);
#pragma unroll
    for (int n = 2 * T::NA; n > 0; n >>= 1)
#pragma unroll
      for (int r = 0; r < n; ++r) e[r] += e[r + n];
    float sum = e[0];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 16)
      s_p[(threadIdx.x >> 6) % T::WA][t.row_b(j) - t0] = make_float2(m, sum);
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c < T::B && t0 + c < H.rows) {
    float M = s_p[0][c].x;
#pragma unroll
    for (int i = 1; i < T::WA; ++i) M = fmaxf(M, s_p[i][c].x);
    const float Ms = M == ninf ? 0.f : M;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < T::WA; ++i) sum += s_p[i][c].y * expf(s_p[i][c].x - Ms);
    part[(size_t)(t0 + c) * n_vt + vt] = make_float2(M, sum);
  }
}

// One wavefront a row: joins the pairs and takes the target's logit from one
// more dot product (a gathered row of w; the pairs do not keep it).  Latency for few
// rows (5 us at 32 of 4096), the gathered rows for many (8192 of 4096: 23 us).
// BASE2: the pairs' maxima are in base 2 (z log2 e).
template <typename T, bool BASE2>
__global__ __launch_bounds__(256) void k_loss_join(const float2* part, int n_vt, int V, int d, int T_,
                                                   bool vec, const T* w, const float* b, const T* h,
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
  if (live) {
    const T *hr = h + (size_t)t * d, *wr = w + (size_t)y * d;
    constexpr int N = 16 / sizeof(T);  // elements of a 16-byte load
    struct alignas(16) Vec {
      T e[N];
    };
    if (vec) {
#pragma unroll 4
      for (int k = N * lane; k < d; k += 64 * N) {
        const Vec x = *reinterpret_cast<const Vec*>(hr + k), u = *reinterpret_cast<const Vec*>(wr + k);
#pragma unroll
        for (int i = 0; i < N; ++i) z = fmaf(to_f32<T>(x.e[i]), to_f32<T>(u.e[i]), z);
      }
    } else {
      for (int k = lane; k < d; k += 64) z = fmaf(to_f32<T>(hr[k]), to_f32<T>(wr[k]), z);
    }
  }
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
// D of the tokens x a piece's columns (v0 ..; a row's elements behind the piece hold
// anything), and per token tile the column sums of D (db).  A = w: a lane holds NA x 4
// consecutive columns of a token.  777 tokens, d 768, vocabulary 32128: 430 us (89
// TFLOP/s; the two products 385 and 360), bound by the fp32 matrix rate and the last
// round: 1757 tiles, two to a CU, are 3.4 rounds of 512.
template <int KIND>
__global__ __launch_bounds__(f32p::THREADS, f32p::Tile<KIND>::OCC) void k_dz_f32(
    Operand<true> W, Operand<true> H, const float* bias, const int32_t* target, const float* lse,
    const float* dloss, int V, int v0, float* D, size_t ldd, float* db_part) {
  using T = f32p::Tile<KIND>;
  __shared__ __align__(16) float lds[T::FLOATS];
  const int c0 = blockIdx.x * T::A, tt = blockIdx.y, t0 = tt * T::B;
  F32Tile<KIND> tile(c0, W.rows, t0, H.rows);
  f32_product<KIND>(W, H, c0, t0, 0, H.K, lds, tile);
  float* s_sum = lds;  // [T::WB][T::A]; the tile ended on a barrier
  // the lane's rows first: behind a store the compiler would wait for each
  int ty[T::NB];
  float tl[T::NB], tg[T::NB];
#pragma unroll
  for (int j = 0; j < T::NB; ++j) {
    const int t = min(tile.row_b(j), H.rows - 1), y = target[t];
    tl[j] = lse[t];
    const bool live = y >= 0 && y < V && tl[j] != -__builtin_inff();
    ty[j] = live && tile.row_b(j) < H.rows ? y - v0 : INT32_MIN;
    tg[j] = dloss[t];
  }
#pragma unroll
  for (int i = 0; i < T::NA; ++i) {
    if (i >= tile.na) continue;
    const int c = tile.row_a(i, 0);
    f32x4_t bi = {}, sum = {};
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (bias) bi[r] = bias[min(c + r, W.rows - 1)];
#pragma unroll
    for (int j = 0; j < T::NB; ++j) {
      if (j >= tile.nb) continue;
      const int t = tile.row_b(j);
      f32x4_t x;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[r] = ty[j] != INT32_MIN && c + r < W.rows
                   ? tg[j] * (expf(tile.acc[i][j][r] + bi[r] - tl[j]) - (c + r == ty[j] ? 1.f : 0.f))
                   : 0.f;
      if (t < H.rows) *reinterpret_cast<f32x4_t*>(D + (size_t)t * ldd + c) = x;
      sum += x;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float s = row16_sum(sum[r]);
      if ((threadIdx.x & 15) == 0) s_sum[(threadIdx.x >> 6) / T::WA * T::A + c + r - c0] = s;
    }
  }
  __syncthreads();
  if (db_part && threadIdx.x < T::A && c0 + (int)threadIdx.x < W.rows) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < T::WB; ++i) s += s_sum[i * T::A + threadIdx.x];
    db_part[(size_t)tt * ldd + c0 + threadIdx.x] = s;
  }
}

// rows that take part, zeros for the others: an ignored row's h may hold
// anything, and 0 * NaN is NaN
__global__ __launch_bounds__(256) void k_live_rows(const float* h, const int32_t* target,
                                                   const float* lse, int V, int d, float* out) {
  const size_t t = blockIdx.x;
  const int y = target[t];
  const bool live = y >= 0 && y < V && lse[t] != -__builtin_inff();
  for (int k = threadIdx.x; k < d; k += 256) out[t * d + k] = live ? h[t * d + k] : 0.f;
}

// Column c's sum over the n rows of a [n][ld] array (the tiles' parts of db), by the 8
// lanes of a column in a block of 32 of them: each takes every eighth row, in four sums
// (one chain over the 8192 tiles of 2^21 rows would lose 11 bits and wait for each
// load), then a tree.  The result is in the first 32 threads.
constexpr int kColBlock = 32;
__device__ __forceinline__ float col_sum(const float* part, int n, size_t ld, int c, bool in) {
  __shared__ float s_c[8][kColBlock];
  const int l = threadIdx.x & 31, r0 = threadIdx.x >> 5;
  float s[4] = {};
  if (in)
    for (int i = r0; i < n; i += 32)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + 8 * k < n) s[k] += part[(size_t)(i + 8 * k) * ld + c];
  s_c[r0][l] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = s_c[k][l];
  return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

__global__ __launch_bounds__(256) void k_db_sum(const float* part, int n_tt, size_t ld, int n,
                                                float* db) {
  const int c = blockIdx.x * kColBlock + (threadIdx.x & 31);
  const float s = col_sum(part, n_tt, ld, c, c < n);
  if (threadIdx.x < kColBlock && c < n) db[c] = s;
}

// ------------------------------------------------------ backward, bf16 --
// Three products on the large-group core.  D of a piece is written once and read
// in both orders: as it lies for dh, transposed out of LDS for dw (as are w for
// dh and h for dw: nothing is turned in memory).
//   * D and the scaled copy of h lie in panels of 256 columns, [panel][row][256]:
//     a 64-row slice of a tile is then one run of 32 KB.
//   * D enters the products in bf16, once rounded: dh and dw are some 2.0e-3 off
//     (relative to their norm), where two parts would leave the 1.7e-3 of the results'
//     own rounding for twice the MFMAs of both products.  A row's weight g is G m 2^-e
//     with G the largest |g| and |m| in [1, 2): D holds m (softmax - onehot), dh takes
//     g / m on its fp32 sums, dw G on its own and 2^-e on the rows of h, where it is
//     exact.  So weights that are all alike (m = 1) add no rounding to the -1 of an
//     unlikely target, which carries most of an untrained row's gradient.
//   * The scaled copy of h has zeros in the rows that take no part: their h may
//     hold anything, and 0 * NaN is NaN.
//   * dh is summed in fp32 over pieces and K splits, then rounded once.
// A tile's A rows are the columns of its result (4 consecutive ones a lane), so
// that results leave the registers in 16-byte pieces without a turn through LDS.
// Bound by MFMA issue at the clock that the power limit leaves: 8192 tokens, d 4096, a
// piece of 16128 columns: D 0.86 to 0.90 ms (1.26 to 1.21 PFLOP/s), dw 0.84 to 0.89, dh
// 0.80 to 0.84.  The kernels take every register and spill 12 to 38 (dh: 82) around the
// slice loop, none in it.  With short rows D's epilogue shows (256 exponentials a lane
// and 128 KB of stores a tile, which only the next tile's first loads overlap): 4096
// tokens, d 768, vocabulary 32128: D 0.28 to 0.30 ms (0.72 to 0.68 PFLOP/s), dw 0.21 to
// 0.22, dh 0.18.
// A piece's D is at most 256 MB, so that the products find part of it in the last-
// level cache; pieces are whole rounds of the grid where that fits (2047 tokens, d
// 2048, vocabulary 151936: 3.51 ms in equal pieces, 3.34 in whole rounds).

// a row's part in the backward
struct RowPart {
  int32_t* y;  // its target, or -1 where it takes no part
  float* lse;  // its lse
  float* m;    // m, 2^-e (0 for a weight of 0) and g / m (0 where it takes no part)
  float* e;
  float* gm;
  float* G;    // [1]
};

// The rows' parts, and hw = 2^-e h_t in panels, zeros in the rows that take no part (hw
// may be NULL).  A block takes a run of rows, and the largest weight of all rows by
// itself (a launch of one block for it cost 8 us at 4096 rows), its first loads of h in
// flight meanwhile.  Bound by memory: 8192 rows of 4096 34 us (4 TB/s), 4096 of 768 10.
constexpr int kPartBlocks = 1024, kPartRows = TRIMMOE_LOSS_MAX_ROWS / kPartBlocks;
__global__ __launch_bounds__(256) void k_row_parts(const int32_t* target, const float* lse,
                                                   const float* dloss, int V, int T, int d,
                                                   const bf16_t* h, RowPart p, bf16_t* hw) {
  __shared__ float s_m[4], s_e[kPartRows];  // s_e: -1 for a row that takes no part
  const int t0 = (int)((long)T * blockIdx.x / gridDim.x);
  const int n = (int)((long)T * (blockIdx.x + 1) / gridDim.x) - t0;
  // rows of d / 8 pieces of 16 bytes
  const int pieces = d / 8, all = hw ? n * pieces : 0;
  struct Pieces {
    union {
      uint4 v;
      bf16_t e[8];
      uint32_t w[4];
    } x[4];
  };
  const auto load = [&](Pieces& q, int i0) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + 256 * k < all)
        q.x[k].v = *reinterpret_cast<const uint4*>(h + (size_t)t0 * d + (size_t)8 * (i0 + 256 * k));
  };
  Pieces q;
  load(q, threadIdx.x);
  float G = 0.f;
  for (int t = threadIdx.x; t < T; t += 8 * 256) {
    // (eight rows' loads in flight; behind the last row: it again)
    int y[8];
    float L[8], g[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int tk = min(t + 256 * k, T - 1);
      y[k] = target[tk];
      L[k] = lse[tk];
      g[k] = dloss[tk];
    }
    sched_fence();
#pragma unroll
    for (int k = 0; k < 8; ++k)
      G = fmaxf(G, y[k] >= 0 && y[k] < V && L[k] != -__builtin_inff() ? fabsf(g[k]) : 0.f);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) G = fmaxf(G, __shfl_xor(G, o));
  if ((threadIdx.x & 63) == 0) s_m[threadIdx.x >> 6] = G;
  __syncthreads();
  G = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.G = G;
  for (int r = threadIdx.x; r < n; r += 256) {
    const int t = t0 + r;
    const int y = target[t];
    const float L = lse[t];
    const bool live = y >= 0 && y < V && L != -__builtin_inff();
    float m, e, gm;
    row_weight(live ? dloss[t] : 0.f, G, m, e, gm);
    p.y[t] = live ? y : -1;
    p.lse[t] = live ? L : 0.f;
    p.m[t] = m;
    p.e[t] = e;
    p.gm[t] = gm;
    s_e[r] = live ? e : -1.f;
  }
  __syncthreads();
  for (int i0 = threadIdx.x; i0 < all; i0 += 4 * 256) {
    Pieces next;
    load(next, i0 + 4 * 256);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + 256 * k;
      if (i >= all) break;
      const int r = i / pieces, c = 8 * (i - r * pieces);
      const float e = s_e[r];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        q.x[k].w[u] = e < 0.f ? 0u
                              : pack_bf16x2(bf2f(q.x[k].e[2 * u]) * e, bf2f(q.x[k].e[2 * u + 1]) * e);
      *reinterpret_cast<uint4*>(hw + ((size_t)(c >> 8) * T + t0 + r) * 256 + (c & 255)) = q.x[k].v;
    }
    q = next;
  }
}

}  // namespace

struct DzArgs {
  const bf16_t* w;    // the piece's first row
  const bf16_t* h;
  const float* bias;  // the piece's first row, or NULL
  RowPart rows;
  int nv, v0, d, T;
  int Vp;             // columns of D
  bf16_t* D;          // [Vp / 256][T][256]
  float* db_part;     // [token tiles][Vp] or NULL
};

// D of a piece: A = w (vocabulary rows), B = h.  BIAS: with a bias, db or both.
// A tile's epilogue runs while the next tile's first loads are in flight.
template <bool BIAS>
__global__ __launch_bounds__(big::THREADS) void k_dz_big(DzArgs a) {
  __shared__ __align__(16) char lds[big::LDS];
  const BigLane L;
  TileSched S;
  int ntiles;
  if (!S.init(a.Vp / big::BM, cdiv_d(a.T, big::BN), 1, ntiles)) return;
  uint32_t la[2], lb[2];
  L.rows(la, L.wm);
  L.rows(lb, L.wn);
  const int nk = a.d / BK;
  const auto start = [&](BigFeed<false, false>& q, int jt, int& vt, int& tt) {
    int sp;
    S.decode(jt, vt, tt, sp);
    const int c0 = vt * big::BM, t0 = tt * big::BN;
    q.a = L.across(a.w + (size_t)c0 * a.d, a.d, min(big::BM, a.nv - c0), 0, nk, 0);
    q.b = L.across(a.h + (size_t)t0 * a.d, a.d, min(big::BN, a.T - t0), 0, nk, 0);
    big_start(lds, q);
  };
  AccBig acc;
  BigFeed<false, false> q;
  int vt, tt;
  start(q, 0, vt, tt);
  for (int jt = 0; jt < ntiles; ++jt) {
    big_zero(acc);
    if (jt == 0)
      big_wait<0>();
    else
      big_wait<32>();  // (every wavefront issues the epilogue's 32 stores)
    big_run(lds, q, nk, acc, la, lb);
    const int c0 = vt * big::BM, t0 = tt * big::BN, tile = tt;
    const int v_valid = min(big::BM, a.nv - c0), t_valid = min(big::BN, a.T - t0);
    const int c = L.lane & 15, rl = L.wm * 128 + 4 * (L.lane >> 4);  // the lane's first row
    // rows of D past the last one lie behind the buffer's end and are dropped
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(
        a.D + ((size_t)vt * a.T + t0) * 256, (short)0, t_valid * 512, 0x00020000);
    // what the epilogue reads, before the next tile's loads (it would wait for
    // those too) and before its stores
    float b[BIAS ? 8 : 1][4], sum[BIAS ? 8 : 1][4];
    if constexpr (BIAS)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          b[i][r] = a.bias ? a.bias[c0 + min(rl + 16 * i + r, v_valid - 1)] : 0.f;
          sum[i][r] = 0.f;
        }
    int ty[8];
    float tL[8], tm[8], te[BIAS ? 8 : 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = min(t0 + L.wn * 128 + 16 * j + c, a.T - 1);
      ty[j] = a.rows.y[t];
      tL[j] = a.rows.lse[t];
      tm[j] = a.rows.m[t];
      if constexpr (BIAS) te[j] = a.rows.e[t];
    }
    sched_fence();
    if (jt + 1 < ntiles) start(q, jt + 1, vt, tt);
    const uint32_t col = (uint32_t)(L.wm * 128 + pack_col(L.lane));
    const int lim = v_valid - rl;  // the lane's row o (16 i + r) is valid for o < lim
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tl = L.wn * 128 + 16 * j + c, y = ty[j];
      const float lse = tL[j], m = tm[j], g = BIAS ? m * te[BIAS ? j : 0] : 0.f;
      const bool live = y >= 0 && tl < t_valid;
      const int yr = y - a.v0 - c0 - rl;  // the target's row, relative to the lane's first
      const uint32_t off = ((uint32_t)tl * 256 + col) * 2;
      // few tiles hold a target of these rows, one a piece is cut short
      const bool plain = v_valid == big::BM && __ballot((unsigned)yr < 128u) == 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float x[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float z = acc[i + k][j][r];
            x[k][r] = softmax_of(BIAS ? z + b[i + k][r] : z, lse);
          }
        if (!plain)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int o = 16 * (i + k) + r;
              x[k][r] = o == yr ? x[k][r] - 1.f : x[k][r];
              x[k][r] = o < lim ? x[k][r] : 0.f;
            }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = live ? x[k][r] : 0.f;
            x[k][r] = p * m;
            if constexpr (BIAS) sum[i + k][r] = fmaf(g, p, sum[i + k][r]);
          }
        // (no scalar offset: see mfma_core.h, pack_rows)
        __builtin_amdgcn_raw_buffer_store_b128(pack_rows(x[0], x[1]), ro, off + 32 * i, 0, 0);
      }
    }
    if constexpr (BIAS) {
      if (!a.db_part) continue;
      // [2][256], in the B stage that the next tile's loads do not reach before its
      // first barrier
      float* s_db = reinterpret_cast<float*>(lds + big::B0 + 2 * big::BB);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float v = row16_sum(sum[i][r]);
          if (c == 0) s_db[L.wn * 256 + rl + 16 * i + r] = v;
        }
      lds_barrier();
      a.db_part[(size_t)tile * a.Vp + c0 + threadIdx.x] = s_db[threadIdx.x] + s_db[256 + threadIdx.x];
    }
  }
}

// D where 256 x 256 tiles would leave half of the CUs without one: the first core's
// tiles of 128 x 128, the same outputs (db_part: a run of rows per column of
// wavefronts).  A lane holds runs of 4 columns of a token, and the two halves of a
// wavefront the neighbouring ones.
using MidTile = Tile<128, 128, 1, 4, 2>;
struct MidSrc {
  using T = MidTile;
  struct Desc {
    int mt, nt;
    static __device__ __forceinline__ Desc pick(bool c, const Desc& x, const Desc& y) {
      return Desc{c ? x.mt : y.mt, c ? x.nt : y.nt};
    }
  };
  const DzArgs& a;
  const TileSched& S;

  __device__ __forceinline__ Desc desc(int j) const {
    int mt, nt, sp;
    S.decode(j, mt, nt, sp);
    return Desc{mt, nt};
  }
  __device__ __forceinline__ void rows(const Desc& d, int (&src)[T::A_PT]) const {
    const int c0 = d.mt * T::BM, valid = min(T::BM, a.nv - c0);
#pragma unroll
    for (int i = 0; i < T::A_PT; ++i) src[i] = c0 + min(dma_row(i, T::ROWS_PER_PASS), valid - 1);
  }
  __device__ __forceinline__ void ptrs(DPtrs<T>& q, const Desc& d,
                                       const int (&src)[T::A_PT]) const {
    const int t0 = d.nt * T::BN;
    make_dptrs<T>(q, a.w, src, a.h, nullptr, t0, min(T::BN, a.T - t0), a.d, 0);
  }
  __device__ __forceinline__ void epilogue(const Desc& d, Acc<T>& acc) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / T::GN, wn = wave % T::GN;
    const int c0 = d.mt * T::BM, t0 = d.nt * T::BN;
    int ty[T::TN];
    float tL[T::TN], tm[T::TN], te[T::TN];
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
      const int t = min(t0 + acc_col<T>(wn, j, lane), a.T - 1);
      ty[j] = a.rows.y[t];
      tL[j] = a.rows.lse[t];
      tm[j] = a.rows.m[t];
      te[j] = a.rows.e[t];
    }
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      float b[16], sum[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        b[r] = a.bias ? a.bias[min(c0 + acc_row<T>(wm, i, r, lane), a.nv - 1)] : 0.f;
        sum[r] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < T::TN; ++j) {
        const int t = t0 + acc_col<T>(wn, j, lane), y = ty[j] - a.v0;
        const bool live = ty[j] >= 0 && t < a.T;
        const float m = tm[j], g = m * te[j];
#pragma unroll
        for (int r0 = 0; r0 < 16; r0 += 4) {
          const int c = c0 + acc_row<T>(wm, i, r0, lane);
          float x[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float p = softmax_of(acc[i][j][r0 + r] + b[r0 + r], tL[j]);
            p = c + r == y ? p - 1.f : p;
            p = live && c + r < a.nv ? p : 0.f;
            sum[r0 + r] = fmaf(g, p, sum[r0 + r]);
            x[r] = p * m;
          }
          uint2 v;
          v.x = pack_bf16x2(x[0], x[1]);
          v.y = pack_bf16x2(x[2], x[3]);
          if (t < a.T)
            *reinterpret_cast<uint2*>(a.D + ((size_t)(c >> 8) * a.T + t) * 256 + (c & 255)) = v;
        }
      }
      if (!a.db_part) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const LanePair p = lanes_xor16(row16_sum(sum[r]));
        if ((lane & 31) == 0)
          a.db_part[(size_t)(d.nt * T::GN + wn) * a.Vp + c0 + acc_row<T>(wm, i, r, lane)] = p.a + p.b;
      }
    }
  }
};
__global__ __launch_bounds__(MidTile::THREADS) void k_dz_mid(DzArgs a) {
  __shared__ __align__(16) char lds[DmaTile<MidTile>::LDS];
  TileSched S;
  int ntiles;
  if (!S.init(cdiv_d(a.nv, MidTile::BM), cdiv_d(a.T, MidTile::BN), 1, ntiles)) return;
  dma_gemm_stream<MidTile>(lds, ntiles, a.d / BK, MidSrc{a, S});
}

struct BigProdArgs {
  const bf16_t* A;  // [K, M], DW: in panels
  const bf16_t* B;  // D in panels: [K, N] (DW) or [N, K]
  int M, N, K;
  const float* scale;  // not PART
  void* out;           // PART: fp32 slices [splits][N, M]; else bf16 [N, M] times *scale
  int splits;
  int add;             // not DW: added to what the slices hold
};

// out = B' A with the sums over K: dw (DW: A = scaled h, B = D, both transposed)
// or dh (A = w transposed, B = D); PART: partials
template <bool DW, bool PART>
__global__ __launch_bounds__(big::THREADS) void k_prod_big(BigProdArgs a) {
  __shared__ __align__(16) char lds[big::LDS];
  const BigLane L;
  TileSched S;
  int ntiles;
  if (!S.init(cdiv_d(a.N, big::BN), cdiv_d(a.M, big::BM), a.splits, ntiles)) return;
  uint32_t la[2], lb[2];
  L.cols(la, L.wm);
  if constexpr (DW)
    L.cols(lb, L.wn);
  else
    L.rows(lb, L.wn);
  const int nk = cdiv_d(a.K, BK);
  struct At {
    int m0, n0, sp, nk;
  };
  const auto start = [&](BigFeed<true, DW>& q, int jt, At& t) {
    int nt, mt, sp;
    S.decode(jt, nt, mt, sp);
    const int m0 = mt * big::BM, n0 = nt * big::BN;
    const int ka = (int)((long)sp * nk / a.splits), kb = (int)((long)(sp + 1) * nk / a.splits);
    t = At{m0, n0, sp, kb - ka};
    if constexpr (DW) {
      q.a = L.along_panel(a.A, a.K, ka * BK, kb * BK, m0);
      q.b = L.along_panel(a.B, a.K, ka * BK, kb * BK, n0);
    } else {
      q.a = L.along(a.A, a.M, a.K, ka * BK, kb * BK, m0);
      q.b = L.across(a.B + (size_t)n0 * 256, 256, min(big::BN, a.N - n0), ka, kb - ka,
                     (uint32_t)a.N * 512);
    }
    big_start(lds, q);
  };
  static_assert(DW || PART, "dh is scaled by row");
  constexpr int ES = PART ? 4 : 2, STORES = PART ? 64 : 32;
  const float g = PART ? 0.f : *a.scale;
  const int c = L.lane & 15;
  AccBig acc;
  BigFeed<true, DW> q;
  At at;
  start(q, 0, at);
  for (int jt = 0; jt < ntiles; ++jt) {
    const int m0 = at.m0, n0 = at.n0, sp = at.sp;
    const int m_valid = min(big::BM, a.M - m0), n_valid = min(big::BN, a.N - n0);
    if (!DW && a.add) {
      // the sums so far in place of zeros
      const int m = L.wm * 128 + 4 * (L.lane >> 4);
      const float* was = static_cast<const float*>(a.out) + ((size_t)sp * a.N + n0) * a.M + m0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float* p = was + (size_t)min(L.wn * 128 + 16 * j + c, n_valid - 1) * a.M;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          acc[i][j] = *reinterpret_cast<const f32x4_t*>(p + (m + 16 * i < m_valid ? m + 16 * i : 0));
      }
    } else {
      big_zero(acc);
    }
    if (jt == 0)
      big_wait<0>();
    else
      big_wait<STORES>();  // (every wavefront issues all of the epilogue's stores)
    big_run(lds, q, at.nk, acc, la, lb);
    sched_fence();
    if (jt + 1 < ntiles) start(q, jt + 1, at);
    int M = a.M;
    asm volatile("" : "+s"(M));  // per-tile value: keeps the offsets below inside the tile loop
    const size_t o = ((size_t)(PART ? sp : 0) * a.N + n0) * M + m0;
    // rows past the last one lie behind the buffer's end; so do columns past it by
    // their offset (M is a multiple of 64: blocks of 32 are valid or not as a whole)
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(
        static_cast<char*>(a.out) + o * ES, (short)0, (int)((uint32_t)n_valid * M * ES), 0x00020000);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t row = (uint32_t)(L.wn * 128 + 16 * j + c) * M;
      const uint32_t off = (row + L.wm * 128 + (PART ? 4 * (L.lane >> 4) : pack_col(L.lane))) * ES;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint32_t at_i = L.wm * 128 + 16 * i < m_valid ? off : 0xffff0000u;
        if constexpr (!PART) {
          float x[2][4];
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[k][r] = acc[i + k][j][r] * g;
          __builtin_amdgcn_raw_buffer_store_b128(pack_rows(x[0], x[1]), ro, at_i + 32 * i, 0, 0);
        } else {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            f32x4_t x = acc[i + k][j];
            asm volatile("" : "+v"(x));  // through VGPRs (see big_store_partial_rows)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), ro,
                                                   at_i + 64 * (i + k), 0, 0);
          }
        }
      }
    }
  }
}

namespace {

// out [n / d, d] = scale times the sum of the S slices of n partials, rounded once; 4
// elements a thread (d is a multiple of 64).  scale: of a row, or one for all
struct SliceSum {
  const float* part;
  int S, d;
  size_t n;
  const float* scale;
  bool by_row;
  bf16_t* out;
  int blocks;
};
// the column sums of a piece from its token tiles', times *scale
struct ColSum {
  const float* part;
  int n_tt, ld, n;
  const float* scale;
  float* out;
};
// blocks: those of x, of y, then the columns'
__global__ __launch_bounds__(256) void k_finish(SliceSum x, SliceSum y, ColSum f) {
  const int b = blockIdx.x - x.blocks - y.blocks;
  if (b >= 0) {
    const int c = b * kColBlock + (threadIdx.x & 31);
    const float s = col_sum(f.part, f.n_tt, f.ld, c, c < f.n);
    if (threadIdx.x < kColBlock && c < f.n) f.out[c] = s * *f.scale;
    return;
  }
  const bool first = (int)blockIdx.x < x.blocks;
  const SliceSum& o = first ? x : y;
  const size_t step = (size_t)4 * 256 * o.blocks;
  for (size_t i = 4 * ((size_t)(blockIdx.x - (first ? 0 : x.blocks)) * 256 + threadIdx.x); i < o.n;
       i += step) {
    float4 s = *reinterpret_cast<const float4*>(o.part + i);
    for (int k = 1; k < o.S; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(o.part + (size_t)k * o.n + i);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
    const float g = o.scale[o.by_row ? i / o.d : 0];
    uint2 w;
    w.x = pack_bf16x2(s.x * g, s.y * g);
    w.y = pack_bf16x2(s.z * g, s.w * g);
    *reinterpret_cast<uint2*>(o.out + i) = w;
  }
}

// ------------------------------------ backward, bf16, a few tokens --
// Up to kSkinnyTokens rows every weight is used once per product, so w is read
// twice (for z and for dh; past the last-level cache both come from HBM) and dw
// written once, whatever the rows: three kernels, the second of them both
// products in one pass over w (rows_grad.h; its rows are the vocabulary's, its
// experts the tokens).  D lies [vocabulary row][part][token] in two bf16 parts: what
// counts here is w's way through memory, beside which the second part is small (one part:
// 17 to 32 tokens 1 to 6% faster, 33 to 64 5 to 10%, dh and dw 2.0e-3 off instead of the
// 1.7e-3 that their own rounding to bf16 leaves).
// us here and in the kernels of more tokens, d and vocabulary 4096 x 32000: 16 tokens
// 154 and 276; 2048 x 151936: 17 tokens 391 and 597, 64 478 and 617; 768 x 32128 with a
// bias: 48 and 77, 75 and 83; 128 x 1000 with a bias: 20 and 36, 26 and 38.
// D comes out of the weight-streaming kernel where the exit head's rule takes it (up
// to 16 rows with db, whose sum it then holds in one row of lanes), stream and tiles in
// us: 16 tokens of 4096 x 32000: 154 and 175 to 186, 2048 x 151936 342 and 384, 4096 x 4000
// 33 and 47; 64 tokens 197 and 206 to 211, 478 and 468.
// 16 tokens of 4096 x 32000: D 45 us (5.8 TB/s), the products 102 (5.1 TB/s).
// D: the first core's tiles of 128 vocabulary rows x 16 ET tokens (32 at least)
template <class T, int ET>
struct FewSrc {
  struct Desc {
    int mt;
    static __device__ __forceinline__ Desc pick(bool c, const Desc& x, const Desc& y) {
      return Desc{c ? x.mt : y.mt};
    }
  };
  const FewArgs& a;
  const TileSched& S;
  const int* s_y;
  const float *s_lse, *s_m, *s_e;
  float G;

  __device__ __forceinline__ Desc desc(int j) const {
    int mt, nt, sp;
    S.decode(j, mt, nt, sp);
    return Desc{mt};
  }
  __device__ __forceinline__ void rows(const Desc& d, int (&src)[T::A_PT]) const {
    const int v0 = d.mt * T::BM, valid = min(T::BM, a.V - v0);
#pragma unroll
    for (int i = 0; i < T::A_PT; ++i) src[i] = v0 + min(dma_row(i, T::ROWS_PER_PASS), valid - 1);
  }
  __device__ __forceinline__ void ptrs(DPtrs<T>& q, const Desc&, const int (&src)[T::A_PT]) const {
    make_dptrs<T>(q, a.w, src, a.h, nullptr, 0, min(T::BN, a.T), a.d, 0);
  }
  __device__ __forceinline__ void epilogue(const Desc& d, Acc<T>& acc) const {
    constexpr int W = 32 * ET;
    const int lane = threadIdx.x & 63, wm = threadIdx.x >> 6;
    const int v0 = d.mt * T::BM;
    float sum[T::TM][16];
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[i][r] = 0.f;
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
      const int t = acc_col<T>(0, j, lane);
      const int y = s_y[t];
      const float lse = s_lse[t], m = s_m[t], e = m * s_e[t];
#pragma unroll
      for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int v = v0 + acc_row<T>(wm, i, r, lane);
          float z = acc[i][j][r];
          if (a.b) z += a.b[min(v, a.V - 1)];
          float p = softmax_of(z, lse);
          p = v == y ? p - 1.f : p;
          p = y >= 0 && v < a.V ? p : 0.f;
          sum[i][r] = fmaf(e, p, sum[i][r]);
          const float x = p * m;
          bf16_t* o = a.D + (size_t)v * W + t;
          if (16 * ET >= T::BN || t < 16 * ET) {
            const bf16_t hi = f2bf(x);
            o[0] = hi;
            o[16 * ET] = f2bf(x - bf2f(hi));
          }
        }
    }
    if (!a.db) return;
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float s = row16_sum(sum[i][r]);
        const LanePair p = lanes_xor16(s);
        const int v = v0 + acc_row<T>(wm, i, r, lane);
        if ((lane & 31) == 0 && v < a.V) a.db[v] = (p.a + p.b) * G;
      }
  }
};

template <class T, int ET>
__global__ __launch_bounds__(T::THREADS) void k_dz_few(FewArgs a) {
  __shared__ __align__(16) char lds[DmaTile<T>::LDS];
  __shared__ int s_y[64];
  __shared__ float s_lse[64], s_m[64], s_e[64], s_G;
  TileSched S;
  int ntiles;
  if (!S.init((a.V + T::BM - 1) / T::BM, 1, 1, ntiles)) return;
  if (threadIdx.x < 64) {
    const int t = threadIdx.x;
    const FewRow r(a.target, a.lse, a.dloss, a.V, a.T, t);
    s_y[t] = r.y;
    s_lse[t] = r.lse;
    s_m[t] = r.m;
    s_e[t] = r.e;
    s_G = r.G;
  }
  __syncthreads();
  const FewSrc<T, ET> src{a, S, s_y, s_lse, s_m, s_e, s_G};
  dma_gemm_stream<T>(lds, ntiles, a.d / BK, src);
}

struct FewTokens {
  const bf16_t* h;
  const float* s_e;  // 2^-e of live rows, -1 of the others
  int T, d, V;
  float scale;
  __device__ __forceinline__ bf16_t w(int t, int c) const {
    const float e = s_e[t];
    return e >= 0.f ? f2bf(bf2f(h[(size_t)t * d + c]) * e) : bf16_t(0);
  }
  __device__ __forceinline__ unsigned long long mask(int tile) const {
    const int n = V - tile * kRowTile;
    return n >= 64 ? ~0ull : (1ull << n) - 1;
  }
};

template <int ET, int CW>
__global__ __launch_bounds__(256) void k_few_grad(FewArgs a, bf16_t* dw, float* part_dh) {
  __shared__ __align__(16) char lds[RowsGrad<ET, CW>::LDS];
  __shared__ float s_e[64], s_G;
  if (threadIdx.x < 64) {
    const FewRow r(a.target, a.lse, a.dloss, a.V, a.T, threadIdx.x);
    s_e[threadIdx.x] = r.y >= 0 ? r.e : -1.f;
    s_G = r.G;
  }
  __syncthreads();
  rows_grad<ET, CW>(lds, FewTokens{a.h, s_e, a.T, a.d, a.V, s_G}, a.w, a.D, a.V, a.T, a.d, dw,
                    part_dh, nullptr);
}

// dh_t = g / m times the sum of the S slices: 4 elements a thread, every eighth slice
// (a chain of 171 loads took 19 us at 40 tokens of 768)
__global__ __launch_bounds__(256) void k_few_finish(FewArgs a, const float* part, int S,
                                                    bf16_t* dh) {
  __shared__ float s_gm[64];
  __shared__ f32x4_t s_p[8][32];
  if (threadIdx.x < 64) {
    const FewRow r(a.target, a.lse, a.dloss, a.V, a.T, threadIdx.x);
    s_gm[threadIdx.x] = r.gm;
  }
  const int l = threadIdx.x & 31, n = a.T * a.d, i = 4 * (blockIdx.x * 32 + l);
  f32x4_t s = {};
  if (i < n)
#pragma unroll 4
    for (int k = threadIdx.x >> 5; k < S; k += 8)
      s += *reinterpret_cast<const f32x4_t*>(part + (size_t)k * n + i);
  s_p[threadIdx.x >> 5][l] = s;
  __syncthreads();
  if (threadIdx.x >= 32 || i >= n) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) s += s_p[k][l];
  const float g = s_gm[i / a.d];
  uint2 w;
  w.x = pack_bf16x2(s[0] * g, s[1] * g);
  w.y = pack_bf16x2(s[2] * g, s[3] * g);
  *reinterpret_cast<uint2*>(dh + i) = w;
}

// ------------------------------------------------------------------ plan --
// bytes of D that a piece may take
constexpr size_t kPieceBytes = (size_t)256 << 20;
// the plans (and with them the workspaces' sizes) are made for a whole MI355X, whatever
// device is current; the launches go by the device's own count
constexpr int kCu = 256;
struct BackPlan {
  int kind;        // of D's tiles (A = the vocabulary)
  int Vc;          // columns of a piece (a multiple of the tile)
  int s_dh, s_dw;  // K splits of the two products
  bool direct_dh;  // one piece, one split: dh needs no partials
  size_t o_dh, o_dw, o_d, o_db, o_h, total;
};

BackPlan back_plan(int V, int d, int T) {
  BackPlan p;
  const size_t rows = T > 0 ? T : 1;
  p.kind = f32p::tile_kind(V, T);
  const int BA = f32p::tile_a(p.kind), BB = f32p::tile_b(p.kind);
  const size_t fit = kPieceBytes / (4 * rows) / BA * BA;
  const int most = (int)std::min<size_t>(std::max<size_t>(fit, BA), (size_t)1 << 30);
  const int n_pieces = cdiv(V, most);
  p.Vc = cdiv(cdiv(V, n_pieces), BA) * BA;
  p.s_dh = product_splits(f32p::product_kind(true, d, T), d, T, p.Vc);
  p.s_dw = product_splits(f32p::product_kind(false, d, p.Vc), d, p.Vc, T);
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
  p.o_db = take((size_t)cdiv((int)rows, BB) * p.Vc * 4);
  p.o_h = take(rows * d * 4);
  p.total = o;
  return p;
}

hipError_t loss_f32(const HeadLossArgs& a, hipStream_t st) {
  float2* part = reinterpret_cast<float2*>(a.ws);
  const float *w = static_cast<const float*>(a.w), *h = static_cast<const float*>(a.h);
  const size_t d = a.d;
  const int kind = f32p::tile_kind(a.V, a.T), n_vt = cdiv(a.V, f32p::tile_a(kind));
  f32p::with_kind(kind, [&](auto c) {
    hipLaunchKernelGGL(k_loss_f32<c>, dim3(n_vt, cdiv(a.T, f32p::Tile<c>::B)), dim3(f32p::THREADS), 0,
                       st, (Operand<true>{w, d, a.V, a.d}), (Operand<true>{h, d, a.T, a.d}), a.b, n_vt,
                       part);
  });
  hipLaunchKernelGGL((k_loss_join<float, false>), dim3(cdiv(a.T, 4)), dim3(256), 0, st, part, n_vt,
                     a.V, a.d, a.T,
                     a.d % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.w) |
                                       reinterpret_cast<uintptr_t>(a.h)) & 15) == 0,
                     w, a.b, h, a.target, a.loss, a.lse);
  return hipGetLastError();
}

hipError_t backward_f32(const HeadLossArgs& a, hipStream_t st) {
  const BackPlan p = back_plan(a.V, a.d, a.T);
  float* part_dh = reinterpret_cast<float*>(a.ws + p.o_dh);
  float* part_dw = reinterpret_cast<float*>(a.ws + p.o_dw);
  float* D = reinterpret_cast<float*>(a.ws + p.o_d);
  float* db = reinterpret_cast<float*>(a.ws + p.o_db);
  float* hl = reinterpret_cast<float*>(a.ws + p.o_h);
  const float *w = static_cast<const float*>(a.w), *h = static_cast<const float*>(a.h);
  float *dh = static_cast<float*>(a.dh), *dw = static_cast<float*>(a.dw);
  const size_t d = a.d;
  const int BA = f32p::tile_a(p.kind), n_tt = cdiv(a.T, f32p::tile_b(p.kind));
  if (dw && a.T > 0)
    hipLaunchKernelGGL(k_live_rows, dim3(a.T), dim3(256), 0, st, h, a.target, a.lse, a.V, a.d, hl);
  for (int v0 = 0; v0 < a.V; v0 += p.Vc) {
    const int nv = std::min(p.Vc, a.V - v0);
    const size_t ldd = (size_t)cdiv(nv, BA) * BA;
    const float* wp = w + v0 * d;
    if (a.T > 0)
      f32p::with_kind(p.kind, [&](auto c) {
        hipLaunchKernelGGL(k_dz_f32<c>, dim3((unsigned)(ldd / BA), n_tt), dim3(f32p::THREADS), 0, st,
                           (Operand<true>{wp, d, nv, a.d}), (Operand<true>{h, d, a.T, a.d}),
                           a.b ? a.b + v0 : nullptr, a.target, a.lse, a.dloss, a.V, v0, D, ldd,
                           a.db ? db : nullptr);
      });
    if (a.db)
      hipLaunchKernelGGL(k_db_sum, dim3(cdiv(nv, kColBlock)), dim3(256), 0, st, db, n_tt, ldd, nv,
                         a.db + v0);
    if (dw) {
      const Operand<false> A{hl, d, a.d, a.T}, B{D, ldd, nv, a.T};
      float* out = dw + v0 * d;
      hipError_t e = launch_product(A, B, p.s_dw, false, p.s_dw == 1 ? out : part_dw, st);
      if (e == hipSuccess && p.s_dw > 1) e = launch_sum_parts(part_dw, p.s_dw, nv * d, out, st);
      if (e != hipSuccess) return e;
    }
    if (dh) {
      const Operand<false> A{wp, d, a.d, nv};
      const Operand<true> B{D, ldd, a.T, nv};
      const hipError_t e =
          launch_product(A, B, p.s_dh, !p.direct_dh && v0 > 0, p.direct_dh ? dh : part_dh, st);
      if (e != hipSuccess) return e;
    }
  }
  if (dh && !p.direct_dh) return launch_sum_parts(part_dh, p.s_dh, a.T * d, dh, st);
  return hipGetLastError();
}

// bf16, up to kSkinnyTokens rows
struct FewPlan {
  int et, R;  // token tiles of 16, slices of dh
  int cols;   // columns / 64 of a block of both products
  size_t o_dh, total;
};

FewPlan few_plan(int V, int d, int T) {
  FewPlan p;
  p.et = T <= 16 ? 1 : T <= 32 ? 2 : 4;
  const int n_t = cdiv(V, kRowTile);
  // Blocks of 256 columns where each has 12 tiles of rows and more to make up for its
  // start (us in 256 and 128 columns: 17 tokens of 2048 x 151936 391 and 418, of 4096 x
  // 32000 186 and 189, of 768 x 32128 50 and 45, of 128 x 100000 44 and 41); with 64 tokens
  // they take more than 256 registers (768 x 32128, one part of D: 96 and 65).
  p.cols = p.et < 4 && (long)n_t * cdiv(d, 256) >= 12 * 2 * kCu ? 4 : 2;
  const int n_c = cdiv(d, 64 * p.cols);
  p.R = std::max(1, std::min(n_t, cdiv(2 * kCu, n_c)));
  const size_t rows = cdiv(V, 128) * (size_t)128;
  p.o_dh = align256(rows * 64 * p.et);
  p.total = p.o_dh + align256((size_t)p.R * std::max(T, 1) * d * 4);
  return p;
}

struct BackPlanBf16 {
  int Vp;          // columns of a piece (a multiple of the tile)
  bool mid;        // D in tiles of 128 x 128
  int s_dh, s_dw;  // K splits of the two products
  size_t o_rows, o_hw, o_d, o_dh, o_dw, o_db, total;
};

// K splits of an m x n product of nk slices on the large-group core: the fewest slices
// on the busiest CU, a tile's start and end counted as 8 of them, plus the partials'
// way through memory at 5.5 TB/s (a slice takes about 1.5 us).  whole: one run
// needs no partials (dw); else (dh) it writes them as every other does.
int big_splits(int m, int n, int nk, bool whole) {
  const long tiles = (long)cdiv(m, big::BM) * cdiv(n, big::BN);
  const double part = (double)m * n * 4 / 8.25e6;
  int best = 1;
  double cost = 0;
  for (int s = 1; s <= 32 && (s == 1 || nk / s >= 4); ++s) {
    const double c = (double)((tiles * s + kCu - 1) / kCu) * (cdiv(nk, s) + 8) +
                     (whole ? (s > 1 ? 2 * s * part : 0) : s * part);
    if (s == 1 || c < cost) {
      best = s;
      cost = c;
    }
  }
  return best;
}

// vocabulary tiles of a piece, of `all` and at most `most`: as many pieces as
// `most` makes, rounded up (while that stays below it) to what fills whole rounds
// of the grid, with n_tt tiles each for D and n_dt for dw
int even_rounds(int all, int most, int n_tt, int n_dt) {
  int per = cdiv(all, cdiv(all, most));
  if (per == all) return per;
  for (int n : {n_dt, n_tt}) {
    int g = kCu;  // kCu / gcd(kCu, n)
    while (g > 1 && n % 2 == 0) {
      g /= 2;
      n /= 2;
    }
    const int up = cdiv(per, g) * g;
    if (up <= most) per = up;
  }
  return per;
}

// D of up to so many 256 x 256 tiles goes in tiles of 128 x 128.  us of the whole
// gradient, there and in the large tiles (tokens x vocabulary x d): 16 tiles, 300 x 2000
// x 768: 59 and 78; 58, 397 x 7286 x 2560: 111 and 148; 126, 228 x 32128 x 768: 109 and
// 118; 300 x 16000 (126): d 128 62 and 69, 768 80 and 90, 2048 132 and 148; 600 x 16000
// (189): d 128 74 and 78, 512 89 and 92, 768 98 and 100, 2048 183 and 177; 1000 x 16000
// (252): 83 and 83, 107 and 104, 121 and 115, 232 and 210; 2000 x 16000 (504): d 128 105 and
// 107, 768 188 and 176.  The length of the rows matters too (a tile's epilogue weighs more
// where they are short); the rule without it gives up no more than 5% (189 tiles).
constexpr int kMidTiles = 128;
BackPlanBf16 back_plan_bf16(int V, int d, int T) {
  BackPlanBf16 p;
  const size_t rows = T > 0 ? T : 1;
  const size_t fit = kPieceBytes / (2 * rows) / big::BM * big::BM;
  const int most = (int)std::min<size_t>(std::max<size_t>(fit, big::BM), (size_t)1 << 22);
  p.Vp = even_rounds(cdiv(V, big::BM), most / big::BM, cdiv((int)rows, big::BN), cdiv(d, big::BM)) *
         big::BM;
  p.mid = (long)(p.Vp / big::BM) * cdiv((int)rows, big::BN) <= kMidTiles;
  p.s_dh = big_splits((int)rows, d, p.Vp / BK, false);
  p.s_dw = big_splits(p.Vp, d, cdiv((int)rows, BK), true);
  size_t o = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = o;
    o += align256(bytes);
    return at;
  };
  p.o_rows = take(5 * rows * 4 + 4);
  p.o_hw = take(rows * cdiv(d, 256) * 512);
  p.o_d = take(rows * p.Vp * 2);
  p.o_dh = take((size_t)p.s_dh * rows * d * 4);
  p.o_dw = take(p.s_dw == 1 ? 0 : (size_t)p.s_dw * p.Vp * d * 4);
  p.o_db = take((size_t)(p.mid ? cdiv((int)rows, MidTile::BN) * MidTile::GN
                               : cdiv((int)rows, big::BN)) * p.Vp * 4);
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
                     a.V, a.d, a.T, true, static_cast<const bf16_t*>(a.w), a.b,
                     static_cast<const bf16_t*>(a.h), a.target, a.loss, a.lse);
  return hipGetLastError();
}

template <int ET>
hipError_t backward_few(const HeadLossArgs& a, const FewPlan& p, hipStream_t st) {
  using Tl = Tile<128, ET == 4 ? 64 : 32, 1, 4, 1>;
  const FewArgs f{static_cast<const bf16_t*>(a.w), static_cast<const bf16_t*>(a.h), a.b, a.target,
                  a.lse, a.dloss, a.V, a.d, a.T, reinterpret_cast<bf16_t*>(a.ws), a.db};
  float* part = a.dh ? reinterpret_cast<float*>(a.ws + p.o_dh) : nullptr;
  // (17 to 32 rows have no stream: the exit head's rule takes theirs for heads of up to 16
  // vocabulary rows only, a few units)
  bool stream = false;
  if constexpr (ET != 2) {
    stream = exit_streams(true, true, a.T, a.V, a.d) && (ET == 1 || !a.db);
    if (stream)
      if (const hipError_t e = launch_dz_skinny<ET>(f, a.n_cu, st); e != hipSuccess) return e;
  }
  if (!stream)
    hipLaunchKernelGGL((k_dz_few<Tl, ET>), dim3(std::min(cdiv(a.V, 128), a.n_cu)), dim3(Tl::THREADS),
                       0, st, f);
  if (a.dw || a.dh) {
    if (const dim3 g(cdiv(a.d, 64 * p.cols), p.R); p.cols == 2)
      hipLaunchKernelGGL((k_few_grad<ET, 2>), g, dim3(256), 0, st, f, static_cast<bf16_t*>(a.dw),
                         part);
    else if constexpr (ET < 4)
      hipLaunchKernelGGL((k_few_grad<ET, 4>), g, dim3(256), 0, st, f, static_cast<bf16_t*>(a.dw),
                         part);
  }
  if (a.dh)
    hipLaunchKernelGGL(k_few_finish, dim3(cdiv(a.T * a.d, 128)), dim3(256), 0, st, f, part, p.R,
                       static_cast<bf16_t*>(a.dh));
  return hipGetLastError();
}

hipError_t backward_bf16(const HeadLossArgs& a, hipStream_t st) {
  if (a.T > 0 && a.T <= kSkinnyTokens) {
    const FewPlan p = few_plan(a.V, a.d, a.T);
    return p.et == 1 ? backward_few<1>(a, p, st)
                     : p.et == 2 ? backward_few<2>(a, p, st) : backward_few<4>(a, p, st);
  }
  const BackPlanBf16 p = back_plan_bf16(a.V, a.d, a.T);
  const size_t rows = a.T > 0 ? a.T : 1;
  float* f = reinterpret_cast<float*>(a.ws + p.o_rows);
  const RowPart part{reinterpret_cast<int32_t*>(f), f + rows,     f + 2 * rows,
                     f + 3 * rows,                  f + 4 * rows, f + 5 * rows};
  bf16_t* hw = reinterpret_cast<bf16_t*>(a.ws + p.o_hw);
  bf16_t* D = reinterpret_cast<bf16_t*>(a.ws + p.o_d);
  float* dh = reinterpret_cast<float*>(a.ws + p.o_dh);
  float* dw = reinterpret_cast<float*>(a.ws + p.o_dw);
  float* db = reinterpret_cast<float*>(a.ws + p.o_db);
  const bf16_t* w = static_cast<const bf16_t*>(a.w);
  const bf16_t* h = static_cast<const bf16_t*>(a.h);
  const int n_tt = cdiv(a.T, big::BN), n_dt = cdiv(a.d, big::BM);
  const auto grid = [&](long tiles) { return dim3((unsigned)std::min<long>(tiles, a.n_cu)); };
  const dim3 block(256);
  static_assert(big::THREADS == 256, "one block shape");
  // (grids hold fewer than 2^32 threads: what runs over T d elements strides)
  const auto blocks = [](size_t n, size_t most) { return (unsigned)std::min((n + 255) / 256, most); };
  hipLaunchKernelGGL(k_row_parts, dim3((unsigned)std::min<size_t>(rows, kPartBlocks)), block, 0, st,
                     a.target, a.lse, a.dloss, a.V, a.T, a.d, h, part, a.dw ? hw : nullptr);
  SliceSum sum_dh{}, sum_dw{};
  for (int v0 = 0; v0 < a.V; v0 += p.Vp) {
    const int nv = std::min(p.Vp, a.V - v0), Vp = cdiv(nv, big::BM) * big::BM;
    const bf16_t* wp = w + (size_t)v0 * a.d;
    if (a.T > 0) {
      const DzArgs z{wp, h, a.b ? a.b + v0 : nullptr, part, nv, v0, a.d, a.T, Vp, D,
                     a.db ? db : nullptr};
      const dim3 g = grid((long)(Vp / big::BM) * n_tt);
      if (p.mid)
        hipLaunchKernelGGL(k_dz_mid,
                           grid((long)cdiv(nv, MidTile::BM) * cdiv(a.T, MidTile::BN)),
                           dim3(MidTile::THREADS), 0, st, z);
      else if (a.b || a.db)
        hipLaunchKernelGGL(k_dz_big<true>, g, block, 0, st, z);
      else
        hipLaunchKernelGGL(k_dz_big<false>, g, block, 0, st, z);
    }
    if (a.dw) {
      bf16_t* out = static_cast<bf16_t*>(a.dw) + (size_t)v0 * a.d;
      const dim3 g = grid((long)cdiv(nv, big::BN) * n_dt * p.s_dw);
      BigProdArgs q{hw, D, a.d, nv, a.T, part.G, out, 1, 0};
      if (p.s_dw == 1) {
        hipLaunchKernelGGL((k_prod_big<true, false>), g, block, 0, st, q);
      } else {
        q.out = dw;
        q.splits = p.s_dw;
        hipLaunchKernelGGL((k_prod_big<true, true>), g, block, 0, st, q);
        sum_dw = SliceSum{dw, p.s_dw, a.d, (size_t)nv * a.d, part.G, false, out, 0};
        sum_dw.blocks = (int)blocks(sum_dw.n / 4, (size_t)1 << 22);
      }
    }
    if (a.dh) {
      const BigProdArgs q{wp, D, a.d, a.T, nv, nullptr, dh, p.s_dh, v0 > 0};
      hipLaunchKernelGGL((k_prod_big<false, true>), grid((long)n_tt * n_dt * p.s_dh), block, 0, st,
                         q);
      if (v0 + p.Vp >= a.V) {
        sum_dh = SliceSum{dh, p.s_dh, a.d, (size_t)a.T * a.d, part.gm, true,
                          static_cast<bf16_t*>(a.dh), 0};
        sum_dh.blocks = (int)blocks(sum_dh.n / 4, (size_t)1 << 22);
      }
    }
    // one launch a piece for what is left of it
    const ColSum cols{db,     p.mid ? cdiv(a.T, MidTile::BN) * MidTile::GN : n_tt,
                      Vp,     a.db ? nv : 0,
                      part.G, a.db ? a.db + v0 : nullptr};
    const unsigned n = sum_dh.blocks + sum_dw.blocks + cdiv(cols.n, kColBlock);
    if (n > 0) hipLaunchKernelGGL(k_finish, dim3(n), block, 0, st, sum_dh, sum_dw, cols);
  }
  return hipGetLastError();
}

}  // namespace

size_t head_loss_ws(bool bf16, int V, int, int T) {
  const int rows = T > 0 ? T : 1;
  const int tile = bf16 ? exit_tile_rows(true, rows) : f32p::tile_a(f32p::tile_kind(V, T));
  return align256((size_t)rows * cdiv(V, tile) * sizeof(float2));
}
size_t head_loss_backward_ws(bool bf16, int V, int d, int T) {
  if (!bf16) return back_plan(V, d, T).total;
  return T > 0 && T <= kSkinnyTokens ? few_plan(V, d, T).total : back_plan_bf16(V, d, T).total;
}

hipError_t launch_head_loss(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? loss_bf16(a, st) : loss_f32(a, st);
}

hipError_t launch_head_loss_backward(const HeadLossArgs& a, hipStream_t st) {
  return a.bf16 ? backward_bf16(a, st) : backward_f32(a, st);
}

}  // namespace trimmoe
