// Balance loss of a router, its per-expert counts and its gradients.
//   p_t = softmax(w h_t + b);  c_e = routed slots of expert e, S in all;
//   n = rows with a routed slot;  P_e = sum of p_te over those rows
//   L = E / (S n) sum_e c_e P_e         (1 where the load is even)
//   dz_te = g E / (S n) p_te (c_e - sum_j p_tj c_j), 0 in rows without a slot
//   dh = dz w,  dw = dz^T h,  db_e = sum_t dz_te        (counts held constant)
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "loss.h"
#include "rows_grad.h"

namespace trimmoe {

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Rows are handled 16 lanes a row (experts l, l + 16, ...: ET of them a lane) and
// 64 a tile.
constexpr int kTile = kRowTile;
constexpr int kRowBlocks = 512;

template <typename T>
__device__ __forceinline__ T sum16(T x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float max16(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// the row's slot of this lane (-1: none), and whether the row has one
__device__ __forceinline__ int row_slot(const int16_t* target, size_t t, int k, int E, int l,
                                        bool& live) {
  int e = l < k ? target[t * k + l] : -1;
  e = e >= 0 && e < E ? e : -1;
  const unsigned long long m = __ballot(e >= 0);
  live = (m >> (threadIdx.x & 48) & 0xffff) != 0;
  return e;
}

// A row's logits z (in place: its probabilities), its slots counted and its
// probabilities to memory.  Returns whether it has a slot.
template <int ET>
__device__ __forceinline__ bool row_forward(float (&z)[ET], size_t t, const int16_t* target, int E,
                                            int k, float* prob, int32_t* s_c) {
  const int l = threadIdx.x & 15;
  float m = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    z[i] = l + 16 * i < E ? z[i] : -__builtin_inff();
    m = fmaxf(m, z[i]);
  }
  m = max16(m);
  // (a row without a logit above -inf has p = 0; a NaN logit makes it NaN)
  const float ms = m == -__builtin_inff() ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    z[i] = expf(z[i] - ms);
    s += z[i];
  }
  s = sum16(s);
  s = s == 0.f ? 1.f : s;
  bool live;
  const int e = row_slot(target, t, k, E, l, live);
  if (e >= 0) atomicAdd(&s_c[e], 1);
  if (l == 0 && live) atomicAdd(&s_c[E], 1);
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    z[i] /= s;
    if (l + 16 * i < E) prob[t * E + l + 16 * i] = z[i];
  }
  return live;
}

// Operand fragments straight from memory.  bf16: 8 of a row's elements a lane,
// one v_mfma_f32_16x16x32_bf16 a k-step of 32.  fp32: 4 a lane, four
// v_mfma_f32_16x16x4_f32 a k-step of 16 (the MFMA u takes element u of every
// lane, on both sides); rows of any length and alignment (vec: all of them start
// on 16 bytes).
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
  static constexpr int K = 32;
  typedef bf16x8_t V;
  static __device__ __forceinline__ V load(const bf16_t* row, int k, int q, int, bool) {
    return *reinterpret_cast<const V*>(row + k + 8 * q);
  }
  static __device__ __forceinline__ void mma(const V& a, const V& b, f32x4_t& c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Frag<float> {
  static constexpr int K = 16;
  typedef f32x4_t V;
  static __device__ __forceinline__ V load(const float* row, int k, int q, int d, bool vec) {
    const int at = k + 4 * q;
    if (vec && at + 4 <= d) return *reinterpret_cast<const V*>(row + at);
    V v;
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = at + u < d ? row[at + u] : 0.f;
    return v;
  }
  static __device__ __forceinline__ void mma(const V& a, const V& b, f32x4_t& c) {
#pragma unroll
    for (int u = 0; u < 4; ++u) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u], b[u], c, 0, 0, 0);
  }
};

struct LossOut {
  int32_t* counts;
  float* prob_sum;
  float* loss;
};

// sums over the nb blocks, and the loss: by one block of N threads.  Groups of EP
// threads (a power of two from E up) take every N / EP-th block's sums.  Latency of a
// few round trips and the tree: 5.6 us for 256 blocks.
template <int N>
__device__ void balance_loss(const float* part_p, const int32_t* part_c, int nb, int E, int EP,
                             const LossOut& o) {
  __shared__ double s_p[N];
  __shared__ int32_t s_c[N];
  __shared__ int32_t s_n;
  const int e = threadIdx.x & (EP - 1), g0 = threadIdx.x / EP, ng = N / EP;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  double p = 0.0;
  int c = 0, n = 0;
  if (e < E) {
#pragma unroll 8
    for (int i = g0; i < nb; i += ng) {
      p += part_p[(size_t)i * E + e];
      c += part_c[(size_t)i * (E + 1) + e];
    }
  }
  for (int i = threadIdx.x; i < nb; i += N) n += part_c[(size_t)i * (E + 1) + E];
  if (n) atomicAdd(&s_n, n);
  s_p[threadIdx.x] = p;
  s_c[threadIdx.x] = c;
  __syncthreads();
  for (int r = N / 2; r >= EP; r >>= 1) {
    if ((int)threadIdx.x < r) {
      s_p[threadIdx.x] += s_p[threadIdx.x + r];
      s_c[threadIdx.x] += s_c[threadIdx.x + r];
    }
    __syncthreads();
  }
  double l = 0.0;
  if ((int)threadIdx.x < E) {
    p = s_p[threadIdx.x];
    c = s_c[threadIdx.x];
    o.counts[threadIdx.x] = c;
    o.prob_sum[threadIdx.x] = (float)p;
    l = p * c;
  }
  __syncthreads();
  // the loss: sum of p c over the experts, and the slots
  if ((int)threadIdx.x < EP) s_p[threadIdx.x] = l;
  __syncthreads();
  for (int r = EP / 2; r > 0; r >>= 1) {
    if ((int)threadIdx.x < r) {
      s_p[threadIdx.x] += s_p[threadIdx.x + r];
      s_c[threadIdx.x] += s_c[threadIdx.x + r];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    o.counts[E] = s_n;
    *o.loss = s_n > 0 ? (float)(E * s_p[0] / ((double)s_c[0] * s_n)) : 0.f;
  }
}

__global__ __launch_bounds__(1024) void k_balance_loss(const float* part_p, const int32_t* part_c,
                                                       int nb, int E, int EP, LossOut o) {
  balance_loss<1024>(part_p, part_c, nb, E, EP, o);
}

// Logits of RT x 16 rows a block in MFMAs, K split over the NW wavefronts (h is
// read once; w comes from L2), then the rows' softmax and sums.  Bound by reading
// h: a block keeps its wavefronts' loads of several k-steps in flight.  A single
// block goes on to the loss itself.  8192 rows of 4096, 8 experts: 17 us (67 MB, in part
// from the last-level cache), of which some 4 are the first loads' and the last sums'
// latency; in fp32 38.  Routers of many experts are bound by w: every block reads it
// whole (1000 rows of 1000, 200 experts, fp32: 42 us).
template <typename TT, int ET, int RT, int NW>
__global__ __launch_bounds__(64 * NW) void k_balance_forward(
    const TT* w, const float* b, const TT* h, const int16_t* target, int T, int E, int EP2, int k,
    int d, bool vec, float* prob, float* part_p, int32_t* part_c, LossOut out) {
  using F = Frag<TT>;
  using V = typename F::V;
  constexpr int U = ET <= 2 ? 4 : ET <= 8 ? 2 : 1;  // k-steps in flight
  constexpr int EP = 16 * ET, ZS = EP + 4;  // floats of an LDS row
  // K parts, then probabilities
  __shared__ __align__(16) float s_z[NW * 16 * RT * ZS];
  __shared__ int32_t s_c[TRIMMOE_MAX_EXPERTS + 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  for (int e = threadIdx.x; e <= E; e += 64 * NW) s_c[e] = 0;
  const int steps = (d + F::K - 1) / F::K;
  const int ks0 = steps * wave / NW, ks1 = steps * (wave + 1) / NW;
  const TT* wp[ET];
#pragma unroll
  for (int i = 0; i < ET; ++i) wp[i] = w + (size_t)min(16 * i + fr, E - 1) * d;
  float sum = 0.f;  // of expert threadIdx.x
  for (int t0 = blockIdx.x * 16 * RT; t0 < T; t0 += 16 * RT * gridDim.x) {
    f32x4_t acc[RT][ET];
    const TT* hp[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      hp[r] = h + (size_t)min(t0 + 16 * r + fr, T - 1) * d;
#pragma unroll
      for (int i = 0; i < ET; ++i) acc[r][i] = f32x4_t{};
    }
    int s = ks0;
    for (; s + U <= ks1; s += U) {
      V fh[U][RT], fw[U][ET];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int r = 0; r < RT; ++r) fh[u][r] = F::load(hp[r], F::K * (s + u), q, d, vec);
#pragma unroll
        for (int i = 0; i < ET; ++i) fw[u][i] = F::load(wp[i], F::K * (s + u), q, d, vec);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int i = 0; i < ET; ++i) F::mma(fh[u][r], fw[u][i], acc[r][i]);
    }
    for (; s < ks1; ++s)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const V fh = F::load(hp[r], F::K * s, q, d, vec);
#pragma unroll
        for (int i = 0; i < ET; ++i)
          F::mma(fh, F::load(wp[i], F::K * s, q, d, vec), acc[r][i]);
      }
    __syncthreads();  // the last rows' probabilities are summed
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < ET; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s_z[(wave * 16 * RT + 16 * r + 4 * q + j) * ZS + 16 * i + fr] = acc[r][i][j];
    __syncthreads();
#pragma unroll
    for (int r0 = 0; r0 < 16 * RT; r0 += 4 * NW) {
      const int row = r0 + (threadIdx.x >> 4), t = t0 + row, l = threadIdx.x & 15;
      if (row >= 16 * RT) break;  // (whole wavefronts)
      float* zr = s_z + row * ZS + l;
      float z[ET];
#pragma unroll
      for (int i = 0; i < ET; ++i) {
        float x[NW];
#pragma unroll
        for (int n = 0; n < NW; ++n) x[n] = zr[16 * i + n * 16 * RT * ZS];
#pragma unroll
        for (int n = NW / 2; n > 0; n >>= 1)
#pragma unroll
          for (int m = 0; m < n; ++m) x[m] += x[m + n];
        z[i] = x[0];
        if (b) z[i] += b[min(l + 16 * i, E - 1)];
      }
      bool live = false;
      if (t < T) live = row_forward<ET>(z, t, target, E, k, prob, s_c);
#pragma unroll
      for (int i = 0; i < ET; ++i) zr[16 * i] = live ? z[i] : 0.f;
    }
    __syncthreads();
    if ((int)threadIdx.x < EP) {
      float p = 0.f;
#pragma unroll
      for (int r = 0; r < 16 * RT; ++r) p += s_z[r * ZS + threadIdx.x];
      sum += p;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 64 * NW) part_c[(size_t)blockIdx.x * (E + 1) + e] = s_c[e];
  if ((int)threadIdx.x < E) part_p[(size_t)blockIdx.x * E + threadIdx.x] = sum;
  if (gridDim.x == 1) {
    __syncthreads();
    balance_loss<64 * NW>(part_p, part_c, 1, E, EP2, out);
  }
}

// dz of 16 rows a block, with zeros past E and in rows past T, its column sums and
// its rows with a slot as a bit mask.  fp32: [row][16 ET].  bf16: [row][part][16 ET] in
// two parts, the value rounded to bf16 and what that leaves rounded again (together
// within 2^-16 of dz).  8191 rows, 60 experts: 5.5 us, launch and latency.
template <int ET, bool BF16>
__global__ __launch_bounds__(256) void k_balance_dz(const float* prob, const int16_t* target,
                                                    const int32_t* counts, const float* dloss, int T,
                                                    int E, int k, void* dz, uint16_t* mask,
                                                    float* part_db) {
  __shared__ float s_p[16][16 * ET + 1];
  __shared__ uint8_t s_live[16];
  const int row = threadIdx.x >> 4, l = threadIdx.x & 15;
  const size_t t = (size_t)blockIdx.x * 16 + row;
  bool live = false;
  if (t < (size_t)T) row_slot(target, t, k, E, l, live);
  int32_t n_e[ET];
  float c[ET], p[ET];
  double total = 0.0;
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    const bool in = l + 16 * i < E;
    n_e[i] = in ? counts[l + 16 * i] : 0;
    p[i] = in && t < (size_t)T ? prob[t * E + l + 16 * i] : 0.f;
    total += n_e[i];
  }
  // counts against their mean: sum_j p_tj = 1, so the mean drops out of
  // c_e - sum_j p_tj c_j and would only cost digits.  In 64 bits up to the difference,
  // which is rounded to fp32: counts of several ranks together pass 2^24
  total = sum16(total);
  const int n = counts[E];
  const float scale = n > 0 ? *dloss * (float)((double)E / (total * n)) : 0.f;
  const double mean = total / E;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    c[i] = (float)(n_e[i] - mean);
    s = fmaf(p[i], c[i], s);
  }
  s = sum16(s);
  if (l == 0) s_live[row] = live;
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    const int e = l + 16 * i;
    const float x = live && e < E ? scale * p[i] * (c[i] - s) : 0.f;
    if constexpr (BF16) {
      bf16_t* o = static_cast<bf16_t*>(dz) + t * (32 * ET) + e;
      const bf16_t hi = f2bf(x);
      o[0] = hi;
      o[16 * ET] = f2bf(x - bf2f(hi));
    } else {
      static_cast<float*>(dz)[t * (16 * ET) + e] = x;
    }
    s_p[row][e] = x;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const unsigned long long m = __ballot(threadIdx.x < 16 && s_live[threadIdx.x & 15]);
    if (threadIdx.x == 0) mask[blockIdx.x] = (uint16_t)m;
  }
  if ((int)threadIdx.x < E) {
    float x = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) x += s_p[r][threadIdx.x];
    part_db[(size_t)blockIdx.x * E + threadIdx.x] = x;
  }
}

// dh = dz w and dw = dz^T h (rows_grad.h): h read and dh written once.  8191 rows of
// 2048, 60 experts: 23 us for 67 MB: four tiles of rows a block, two barriers each, and
// 308 registers (4 expert tiles; 461 at 8): one wavefront a SIMD.
// A row without a slot is not read: its h may hold anything, and 0 * NaN is NaN.
struct RouterRows {
  const bf16_t* wp;
  const unsigned long long* m;
  int E, d;
  float scale;
  __device__ __forceinline__ bf16_t w(int e, int c) const {
    return e < E ? wp[(size_t)e * d + c] : bf16_t(0);
  }
  __device__ __forceinline__ unsigned long long mask(int tile) const { return m[tile]; }
};

template <int ET, int CW>
__global__ __launch_bounds__(256) void k_balance_grad(const bf16_t* w, const bf16_t* h,
                                                      const bf16_t* dz,
                                                      const unsigned long long* mask, int T, int E,
                                                      int d, bf16_t* dh, float* part_dw, bf16_t* dw,
                                                      const float* part_db, float* db) {
  __shared__ __align__(16) char lds[RowsGrad<ET, CW>::LDS];
  if (db && blockIdx.x == 0 && (int)threadIdx.x < E) {  // of a single tile
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) s += part_db[i * E + threadIdx.x];
    db[threadIdx.x] = s;
  }
  rows_grad<ET, CW>(lds, RouterRows{w, mask, E, d, 1.f}, h, dz, T, E, d, dh, part_dw, dw);
}

// The same in fp32, 16 x 16 x 4 MFMAs: a lane holds single elements, so both
// orders of an operand are plain LDS reads; d and the alignment of rows are any
// (vec: four columns at a time).
template <int ET, int CW>
struct GradF32 {
  static constexpr int BC = 64 * CW, EP = 16 * ET;
  static constexpr int HS = BC + 4, ZS = EP + 4;  // floats of an LDS row
  static constexpr int HL = kTile * BC / 4 / 256, ZL = kTile * EP / 4 / 256;  // loads a thread
};

template <int ET, int CW>
__global__ __launch_bounds__(256) void k_balance_grad_f32(const float* w, const float* h,
                                                          const float* dz,
                                                          const unsigned long long* mask, int T,
                                                          int E, int d, bool vec, float* dh,
                                                          float* part_dw, float* dw,
                                                          const float* part_db, float* db) {
  using G = GradF32<ET, CW>;
  __shared__ __align__(16) float s_h[kTile * G::HS];
  __shared__ __align__(16) float s_z[kTile * G::ZS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * G::BC, cw = 16 * CW * wave, c_valid = min(G::BC, d - c0);
  const int n_t = (T + kTile - 1) / kTile;
  // w: column cw + 16 j + fr, expert 4 s + q
  float fw[4 * ET][CW];
#pragma unroll
  for (int s = 0; s < 4 * ET; ++s)
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      const int c = cw + 16 * j + fr, e = 4 * s + q;
      fw[s][j] = e < E && c < c_valid ? w[(size_t)e * d + c0 + c] : 0.f;
    }
  f32x4_t acc[ET][CW];
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) acc[i][j] = f32x4_t{};
  f32x4_t xh[G::HL], xz[G::ZL];
  auto load = [&](int tile) {
    const unsigned long long live = mask[tile];
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / (G::BC / 4), c = 4 * (i % (G::BC / 4));
      const float* p = h + ((size_t)tile * kTile + r) * d + c0 + c;
      const int lim = live >> r & 1 ? c_valid - c : 0;  // (see k_balance_grad)
      xh[u] = f32x4_t{};
      if (vec && lim >= 4) {
        xh[u] = *reinterpret_cast<const f32x4_t*>(p);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < lim) xh[u][k] = p[k];
      }
    }
#pragma unroll
    for (int u = 0; u < G::ZL; ++u) {
      const int i = threadIdx.x + 256 * u;
      xz[u] = *reinterpret_cast<const f32x4_t*>(dz + (size_t)tile * kTile * G::EP + 4 * i);
    }
  };
  int tile = blockIdx.y;
  if (tile < n_t) load(tile);
  for (; tile < n_t; tile += gridDim.y) {
    __syncthreads();  // the last tile is read
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / (G::BC / 4), c = 4 * (i % (G::BC / 4));
      *reinterpret_cast<f32x4_t*>(s_h + r * G::HS + c) = xh[u];
    }
#pragma unroll
    for (int u = 0; u < G::ZL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / (G::EP / 4), c = 4 * (i % (G::EP / 4));
      *reinterpret_cast<f32x4_t*>(s_z + r * G::ZS + c) = xz[u];
    }
    __syncthreads();
    if (tile + (int)gridDim.y < n_t) load(tile + gridDim.y);
    // dw += dz^T h: 16 k-steps of 4 rows
#pragma unroll 4
    for (int s = 0; s < kTile / 4; ++s) {
      const int r = 4 * s + q;
      float fh[CW], fz[ET];
#pragma unroll
      for (int j = 0; j < CW; ++j) fh[j] = s_h[r * G::HS + cw + 16 * j + fr];
#pragma unroll
      for (int i = 0; i < ET; ++i) fz[i] = s_z[r * G::ZS + 16 * i + fr];
#pragma unroll
      for (int i = 0; i < ET; ++i)
#pragma unroll
        for (int j = 0; j < CW; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fh[j], fz[i], acc[i][j], 0, 0, 0);
    }
    // dh = dz w: 4 tiles of 16 rows
    if (dh) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4_t o[CW];
#pragma unroll
        for (int j = 0; j < CW; ++j) o[j] = f32x4_t{};
#pragma unroll
        for (int s = 0; s < 4 * ET; ++s) {
          const float fz = s_z[(16 * rt + fr) * G::ZS + 4 * s + q];
#pragma unroll
          for (int j = 0; j < CW; ++j)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[s][j], fz, o[j], 0, 0, 0);
        }
        const size_t t = (size_t)tile * kTile + 16 * rt + fr;
#pragma unroll
        for (int j = 0; j < CW; ++j) {
          const int c = cw + 16 * j + 4 * q;
          float* p = dh + t * d + c0 + c;
          if (t >= (size_t)T) continue;
          if (vec && c + 4 <= c_valid) {
            *reinterpret_cast<f32x4_t*>(p) = o[j];
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (c + k < c_valid) p[k] = o[j][k];
          }
        }
      }
    }
  }
  if (db && blockIdx.x == 0 && (int)threadIdx.x < E) {  // of a single tile
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kTile / 16; ++i) s += part_db[i * E + threadIdx.x];
    db[threadIdx.x] = s;
  }
  if (!part_dw && !dw) return;
  float* out = dw ? dw : part_dw + (size_t)blockIdx.y * E * d;
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = 16 * i + fr, c = cw + 16 * j + 4 * q + k;
        if (e < E && c < c_valid) out[(size_t)e * d + c0 + c] = acc[i][j][k];
      }
}

// dw from its R slices (4 elements a thread), then db from the blocks' sums (one
// wavefront an expert)
template <typename TT>
__global__ __launch_bounds__(256) void k_balance_finish(const float* part_dw, int R, size_t n,
                                                        int dw_blocks, TT* dw, const float* part_db,
                                                        int nb, int E, float* db) {
  if ((int)blockIdx.x < dw_blocks) {
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (n % 4 == 0) {
      if (i >= n) return;
      f32x4_t s = *reinterpret_cast<const f32x4_t*>(part_dw + i);
#pragma unroll 4
      for (int r = 1; r < R; ++r) s += *reinterpret_cast<const f32x4_t*>(part_dw + (size_t)r * n + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) dw[i + k] = from_f32<TT>(s[k]);
    } else {
      for (size_t k = i; k < min(i + 4, n); ++k) {
        float s = part_dw[k];
        for (int r = 1; r < R; ++r) s += part_dw[(size_t)r * n + k];
        dw[k] = from_f32<TT>(s);
      }
    }
    return;
  }
  const int e = ((int)blockIdx.x - dw_blocks) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (e >= E) return;
  float s = 0.f;
  for (int i = lane; i < nb; i += 64) s += part_db[(size_t)i * E + e];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) db[e] = s;
}

// ------------------------------------------------------------------ plan --
int expert_tiles(int E) {  // of 16, a power of two
  int et = 1;
  while (16 * et < E) et *= 2;
  return et;
}
// calls f(std::integral_constant<int, expert tiles>)
template <class F>
void with_tiles(int E, F f) {
  switch (expert_tiles(E)) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    default: f(std::integral_constant<int, 16>()); break;
  }
}
// wavefronts of a forward block: its K parts fit LDS
constexpr int wavefronts(int et) { return et == 16 ? 4 : 8; }
// columns / 64 of a gradient block: accumulators of dw and fragments of w in registers
template <typename TT>
constexpr int col_tiles(int et) {
  return sizeof(TT) == 2 ? (et == 16 ? 2 : 4) : (et >= 8 ? 1 : 2);
}

// fp32 rows that start on 16 bytes
bool rows_aligned(int d, const void* p, const void* q) {
  return d % 4 == 0 && ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) & 15) == 0;
}

struct Plan {
  int et, rt, nb;  // expert tiles, rows / 16 a forward block takes at once, its blocks
  size_t f_c, f_total;
  int n_t, R;  // tiles of 64 rows, slices of dw
  size_t b_mask, b_db, b_dw, b_total;
  Plan(bool bf16, int E, int d, int T) : et(expert_tiles(E)) {
    const int rows = std::max(T, 1);
    // Little work takes one block, whose passes cost less than the loss's own launch (30
    // rows, d 4096, 8 experts: 15 us, 18 in two blocks; 64 rows, d 1024, 200 experts: 48,
    // 28 in two).  Blocks of 16 rows while that gives no CU a second one (1000 rows, d
    // 1000, 200 experts, fp32: 52 us, 103 with 32 rows; 8191 rows, d 2048, 60 experts,
    // bf16: 30 and 22, as w is read by twice the blocks).
    const bool one = rows <= 64 && et * d * cdiv(rows, 32) <= 4096;
    rt = !one && cdiv(rows, 16) <= 256 ? 1 : 2;
    nb = one ? 1 : std::min(kRowBlocks, cdiv(rows, 16 * rt));
    f_c = align256((size_t)nb * E * 4);
    f_total = f_c + align256((size_t)nb * (E + 1) * 4);
    n_t = cdiv(rows, kTile);
    // blocks for every CU, and slices of dw no larger than 32 MB together
    const int n_c = cdiv(d, 64 * (bf16 ? col_tiles<bf16_t>(et) : col_tiles<float>(et)));
    const size_t most = ((size_t)32 << 20) / ((size_t)E * d * 4);
    R = std::max(1, std::min(std::min(n_t, cdiv(256, n_c)), (int)std::min<size_t>(most, 1 << 20)));
    b_mask = align256((size_t)n_t * kTile * 64 * et);  // (dz: 4 bytes, or two parts of 2)
    b_db = b_mask + align256((size_t)n_t * 8);
    b_dw = b_db + align256((size_t)n_t * (kTile / 16) * E * 4);
    b_total = b_dw + (R > 1 ? align256((size_t)R * E * d * 4) : 0);
  }
};

template <typename TT>
hipError_t forward(const BalanceArgs& a, hipStream_t st) {
  const Plan p(a.bf16, a.E, a.d, a.T);
  float* part_p = reinterpret_cast<float*>(a.ws);
  int32_t* part_c = reinterpret_cast<int32_t*>(a.ws + p.f_c);
  const LossOut out{a.counts, a.prob_sum, a.loss};
  int EP = 1;
  while (EP < a.E) EP *= 2;
  const int nb = a.T > 0 ? p.nb : 0;
  if (nb > 0)
    with_tiles(a.E, [&](auto c) {
      constexpr int ET = c;
      const auto run = [&](auto rt) {
        hipLaunchKernelGGL((k_balance_forward<TT, ET, rt, wavefronts(ET)>), dim3(nb),
                           dim3(64 * wavefronts(ET)), 0, st, static_cast<const TT*>(a.w), a.b,
                           static_cast<const TT*>(a.h), a.target, a.T, a.E, EP, a.k, a.d,
                           rows_aligned(a.d, a.w, a.h), a.prob, part_p, part_c, out);
      };
      if (p.rt == 1)
        run(std::integral_constant<int, 1>());
      else
        run(std::integral_constant<int, 2>());
    });
  if (nb != 1)
    hipLaunchKernelGGL(k_balance_loss, dim3(1), dim3(1024), 0, st, part_p, part_c, nb, a.E, EP, out);
  return hipGetLastError();
}

template <typename TT>
hipError_t backward(const BalanceArgs& a, hipStream_t st) {
  constexpr bool BF16 = sizeof(TT) == 2;
  const Plan p(a.bf16, a.E, a.d, a.T);
  unsigned long long* mask = reinterpret_cast<unsigned long long*>(a.ws + p.b_mask);
  float* part_db = reinterpret_cast<float*>(a.ws + p.b_db);
  float* part_dw = a.dw && p.R > 1 ? reinterpret_cast<float*>(a.ws + p.b_dw) : nullptr;
  TT *dh = static_cast<TT*>(a.dh), *dw = static_cast<TT*>(a.dw), *whole = p.R > 1 ? nullptr : dw;
  const TT *w = static_cast<const TT*>(a.w), *h = static_cast<const TT*>(a.h);
  const int nb = p.n_t * (kTile / 16);
  // a single tile's gradient kernel sums db as well
  float* one_db = p.n_t == 1 && (dh || dw) ? a.db : nullptr;
  with_tiles(a.E, [&](auto c) {
    constexpr int ET = c, CW = col_tiles<TT>(ET);
    hipLaunchKernelGGL((k_balance_dz<ET, BF16>), dim3(nb), dim3(256), 0, st, a.prob, a.target,
                       a.counts, a.dloss, a.T, a.E, a.k, a.ws, reinterpret_cast<uint16_t*>(mask),
                       part_db);
    if (!dh && !dw) return;
    const dim3 grid(cdiv(a.d, 64 * CW), p.R);
    if constexpr (BF16)
      hipLaunchKernelGGL((k_balance_grad<ET, CW>), grid, dim3(256), 0, st, w, h,
                         reinterpret_cast<const bf16_t*>(a.ws), mask, a.T, a.E, a.d, dh, part_dw,
                         whole, part_db, one_db);
    else
      hipLaunchKernelGGL((k_balance_grad_f32<ET, CW>), grid, dim3(256), 0, st, w, h,
                         reinterpret_cast<const float*>(a.ws), mask, a.T, a.E, a.d,
                         rows_aligned(a.d, a.h, a.dh), dh, part_dw, whole, part_db, one_db);
  });
  const size_t n = (size_t)a.E * a.d;
  const int dw_blocks = part_dw ? (int)((n + 1023) / 1024) : 0;
  const int db_blocks = a.db && !one_db ? cdiv(a.E, 4) : 0;
  if (dw_blocks + db_blocks > 0)
    hipLaunchKernelGGL(k_balance_finish<TT>, dim3(dw_blocks + db_blocks), dim3(256), 0, st, part_dw,
                       p.R, n, dw_blocks, dw, part_db, nb, a.E, a.db);
  return hipGetLastError();
}

}  // namespace

size_t balance_ws(bool bf16, int E, int d, int T) { return Plan(bf16, E, d, T).f_total; }
size_t balance_backward_ws(bool bf16, int E, int d, int T) { return Plan(bf16, E, d, T).b_total; }

hipError_t launch_balance(const BalanceArgs& a, hipStream_t st) {
  return a.bf16 ? forward<bf16_t>(a, st) : forward<float>(a, st);
}
hipError_t launch_balance_backward(const BalanceArgs& a, hipStream_t st) {
  return a.bf16 ? backward<bf16_t>(a, st) : backward<float>(a, st);
}

}  // namespace trimmoe
