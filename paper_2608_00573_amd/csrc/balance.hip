// Balance loss of a router, its per-expert counts and its gradients.
//   p_t = softmax(w h_t + b);  c_e = routed slots of expert e, S in all;
//   n = rows with a routed slot;  P_e = sum of p_te over those rows
//   L = E / (S n) sum_e c_e P_e         (1 where the load is even)
//   dz_te = g E / (S n) p_te (c_e - sum_j p_tj c_j), 0 in rows without a slot
//   dh = dz w,  dw = dz^T h,  db_e = sum_t dz_te        (counts held constant)
#include <math.h>

#include <type_traits>

#include "loss.h"
#include "mfma_core.h"
#include "products.h"

namespace trimmoe {

namespace {

// Rows are handled 16 lanes a row (experts l, l + 16, ...: ET of them a lane) and
// 64 a tile.
constexpr int kTile = 64;
constexpr int kRowBlocks = 512;

__device__ __forceinline__ float sum16(float x) {
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

// fp32: the rows' logits lie in S slices of partial sums
template <int ET>
__global__ __launch_bounds__(256) void k_balance_rows(const float* logits, int S, const float* b,
                                                      const int16_t* target, int T, int E, int k,
                                                      float* prob, float* part_p, int32_t* part_c) {
  __shared__ float s_p[16][16 * ET + 1];
  __shared__ int32_t s_c[TRIMMOE_MAX_EXPERTS + 1];
  const int row = threadIdx.x >> 4, l = threadIdx.x & 15;
  for (int e = threadIdx.x; e <= E; e += 256) s_c[e] = 0;
  __syncthreads();
  float sum[ET] = {};
  for (int t0 = blockIdx.x * 16; t0 < T; t0 += 16 * gridDim.x) {
    const int t = t0 + row;
    if (t >= T) break;  // (whole groups of 16 lanes)
    float z[ET];
#pragma unroll
    for (int i = 0; i < ET; ++i) {
      const int e = l + 16 * i;
      z[i] = 0.f;
      if (e < E) {
        for (int j = 0; j < S; ++j) z[i] += logits[((size_t)j * T + t) * E + e];
        if (b) z[i] += b[e];
      }
    }
    const bool live = row_forward<ET>(z, t, target, E, k, prob, s_c);
#pragma unroll
    for (int i = 0; i < ET; ++i)
      if (live) sum[i] += z[i];
  }
#pragma unroll
  for (int i = 0; i < ET; ++i) s_p[row][l + 16 * i] = sum[i];
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 256) {
    part_c[(size_t)blockIdx.x * (E + 1) + e] = s_c[e];
    float p = 0.f;
    if (e < E) {
#pragma unroll
      for (int r = 0; r < 16; ++r) p += s_p[r][e];
      part_p[(size_t)blockIdx.x * E + e] = p;
    }
  }
}

// bf16: logits of RT x 16 rows a block in 16 x 16 x 32 MFMAs, K split over the
// four wavefronts, operands straight from memory (h is read once; w, at most 2
// MB, comes from L2), then the rows' softmax and sums.  Bound by reading h:
// a block keeps 4 wavefronts' loads of several k-steps in flight.
template <int ET, int RT>
__global__ __launch_bounds__(256) void k_balance_forward(const bf16_t* w, const float* b,
                                                         const bf16_t* h, const int16_t* target,
                                                         int T, int E, int k, int d, float* prob,
                                                         float* part_p, int32_t* part_c) {
  constexpr int U = ET <= 2 ? 8 : ET == 4 ? 4 : ET == 8 ? 2 : 1;  // k-steps in flight
  constexpr int EP = 16 * ET, ZS = EP + 4;  // floats of an LDS row
  // K parts, then probabilities
  __shared__ __align__(16) float s_z[4 * 16 * RT * ZS];
  __shared__ int32_t s_c[TRIMMOE_MAX_EXPERTS + 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  for (int e = threadIdx.x; e <= E; e += 256) s_c[e] = 0;
  const int steps = d / 32, ks0 = steps * wave / 4, ks1 = steps * (wave + 1) / 4;
  const bf16_t* wp[ET];
#pragma unroll
  for (int i = 0; i < ET; ++i) wp[i] = w + (size_t)min(16 * i + fr, E - 1) * d + 8 * q;
  float sum = 0.f;  // of expert threadIdx.x
  for (int t0 = blockIdx.x * 16 * RT; t0 < T; t0 += 16 * RT * gridDim.x) {
    f32x4_t acc[RT][ET];
    const bf16_t* hp[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      hp[r] = h + (size_t)min(t0 + 16 * r + fr, T - 1) * d + 8 * q;
#pragma unroll
      for (int i = 0; i < ET; ++i) acc[r][i] = f32x4_t{};
    }
    int s = ks0;
    for (; s + U <= ks1; s += U) {
      bf16x8_t fh[U][RT], fw[U][ET];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
          fh[u][r] = *reinterpret_cast<const bf16x8_t*>(hp[r] + 32 * (s + u));
#pragma unroll
        for (int i = 0; i < ET; ++i)
          fw[u][i] = *reinterpret_cast<const bf16x8_t*>(wp[i] + 32 * (s + u));
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int i = 0; i < ET; ++i)
            acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh[u][r], fw[u][i], acc[r][i], 0, 0, 0);
    }
    for (; s < ks1; ++s)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const bf16x8_t fh = *reinterpret_cast<const bf16x8_t*>(hp[r] + 32 * s);
#pragma unroll
        for (int i = 0; i < ET; ++i)
          acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              fh, *reinterpret_cast<const bf16x8_t*>(wp[i] + 32 * s), acc[r][i], 0, 0, 0);
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
    for (int r = 0; r < RT; ++r) {
      const int row = 16 * r + (threadIdx.x >> 4), t = t0 + row, l = threadIdx.x & 15;
      float* zr = s_z + row * ZS + l;
      float z[ET];
#pragma unroll
      for (int i = 0; i < ET; ++i) {
        z[i] = (zr[16 * i] + zr[16 * i + 16 * RT * ZS]) +
               (zr[16 * i + 32 * RT * ZS] + zr[16 * i + 48 * RT * ZS]);
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
  for (int e = threadIdx.x; e <= E; e += 256) part_c[(size_t)blockIdx.x * (E + 1) + e] = s_c[e];
  if ((int)threadIdx.x < E) part_p[(size_t)blockIdx.x * E + threadIdx.x] = sum;
}

// sums over the blocks, and the loss.  One block: groups of threads of EP (a
// power of two from E up) experts take every 1024 / EP-th block's sums.
__global__ __launch_bounds__(1024) void k_balance_loss(const float* part_p, const int32_t* part_c,
                                                       int nb, int E, int EP, int32_t* counts,
                                                       float* prob_sum, float* loss) {
  __shared__ double s_p[1024];
  __shared__ int32_t s_c[1024];
  __shared__ int32_t s_n;
  const int e = threadIdx.x & (EP - 1), g0 = threadIdx.x / EP, ng = 1024 / EP;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  double p = 0.0;
  int c = 0, n = 0;
  if (e < E) {
#pragma unroll 4
    for (int i = g0; i < nb; i += ng) {
      p += part_p[(size_t)i * E + e];
      c += part_c[(size_t)i * (E + 1) + e];
    }
  }
  for (int i = threadIdx.x; i < nb; i += 1024) n += part_c[(size_t)i * (E + 1) + E];
  if (n) atomicAdd(&s_n, n);
  s_p[threadIdx.x] = p;
  s_c[threadIdx.x] = c;
  __syncthreads();
  for (int o = 512; o >= EP; o >>= 1) {
    if ((int)threadIdx.x < o) {
      s_p[threadIdx.x] += s_p[threadIdx.x + o];
      s_c[threadIdx.x] += s_c[threadIdx.x + o];
    }
    __syncthreads();
  }
  double l = 0.0;
  if ((int)threadIdx.x < E) {
    p = s_p[threadIdx.x];
    c = s_c[threadIdx.x];
    counts[threadIdx.x] = c;
    prob_sum[threadIdx.x] = (float)p;
    l = p * c;
  }
  __syncthreads();
  // the loss: sum of p c over the experts, and the slots
  if ((int)threadIdx.x < EP) s_p[threadIdx.x] = l;
  __syncthreads();
  for (int o = EP / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) {
      s_p[threadIdx.x] += s_p[threadIdx.x + o];
      s_c[threadIdx.x] += s_c[threadIdx.x + o];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    counts[E] = s_n;
    *loss = s_n > 0 ? (float)(E * s_p[0] / ((double)s_c[0] * s_n)) : 0.f;
  }
}

// dz of a tile of 64 rows a block and its column sums (db).  fp32: as it is.
// bf16: in two parts, the value rounded to bf16 and what that leaves rounded
// again (together within 2^-16 of dz), as [row][part][16 ET] with zeros past E
// and in rows past T; and the tile's rows with a slot as a bit mask.
template <int ET, bool BF16>
__global__ __launch_bounds__(256) void k_balance_dz(const float* prob, const int16_t* target,
                                                    const int32_t* counts, const float* dloss, int T,
                                                    int E, int k, void* dz, unsigned long long* mask,
                                                    float* part_db) {
  __shared__ float s_p[16][16 * ET + 1];
  __shared__ uint8_t s_live[kTile];
  const int row = threadIdx.x >> 4, l = threadIdx.x & 15;
  // counts against their mean: sum_j p_tj = 1, so the mean drops out of
  // c_e - sum_j p_tj c_j and would only cost digits
  float c[ET], total = 0.f;
#pragma unroll
  for (int i = 0; i < ET; ++i) {
    c[i] = l + 16 * i < E ? (float)counts[l + 16 * i] : 0.f;
    total += c[i];
  }
  total = sum16(total);
  const int n = counts[E];
  const float scale = n > 0 ? *dloss * (float)((double)E / ((double)total * n)) : 0.f;
  const float mean = total / E;
#pragma unroll
  for (int i = 0; i < ET; ++i) c[i] -= mean;
  float sum[ET] = {};
#pragma unroll
  for (int r = 0; r < kTile; r += 16) {
    const size_t t = (size_t)blockIdx.x * kTile + r + row;
    bool live = false;
    float p[ET], s = 0.f;
    if (t < (size_t)T) row_slot(target, t, k, E, l, live);
#pragma unroll
    for (int i = 0; i < ET; ++i) {
      p[i] = live && l + 16 * i < E ? prob[t * E + l + 16 * i] : 0.f;
      s = fmaf(p[i], c[i], s);
    }
    s = sum16(s);
    if (l == 0) s_live[r + row] = live;
#pragma unroll
    for (int i = 0; i < ET; ++i) {
      const int e = l + 16 * i;
      const float x = live && e < E ? scale * p[i] * (c[i] - s) : 0.f;
      sum[i] += x;
      if constexpr (BF16) {
        bf16_t* o = static_cast<bf16_t*>(dz) + t * (32 * ET) + e;
        const bf16_t hi = f2bf(x);
        o[0] = hi;
        o[16 * ET] = f2bf(x - bf2f(hi));
      } else if (t < (size_t)T && e < E) {
        static_cast<float*>(dz)[t * E + e] = x;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < ET; ++i) s_p[row][l + 16 * i] = sum[i];
  __syncthreads();
  if (BF16 && threadIdx.x < 64) {
    const unsigned long long m = __ballot(s_live[threadIdx.x]);
    if (threadIdx.x == 0) mask[blockIdx.x] = m;
  }
  if ((int)threadIdx.x < E) {
    float x = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) x += s_p[r][threadIdx.x];
    part_db[(size_t)blockIdx.x * E + threadIdx.x] = x;
  }
}

// dh = dz w and the block's part of dw = dz^T h, for 64 CW columns and every
// gridDim.y-th tile of 64 rows, in 16 x 16 x 32 MFMAs whose A rows are the
// columns.  h is read once and dh written once; w's fragments stay in
// registers (a lane's 8 experts of a column), those of h (8 rows of a column)
// come transposed out of LDS, as do dz's for dw.  The next tile's loads are in
// flight under a tile's products.
//   ET = 1: the two parts of dz are one k-step of 32 (16 experts each, w's
// fragment twice); else a k-step is 32 experts of a part.
template <int ET, int CW>
struct Grad {
  static constexpr int BC = 64 * CW;               // columns of a block
  static constexpr int HR = 2 * BC;                // LDS bytes of a row of h
  static constexpr int ZB = 64 * ET;               // bytes of a row of dz
  static constexpr int ZR = ZB + 32;               // ... in LDS: rows on distinct banks
  static constexpr int KS = ET == 1 ? 1 : ET / 2;  // fragments of w
  static constexpr int LDS = kTile * (HR + ZR);
  static constexpr int HL = kTile * HR / 16 / 256, ZL = kTile * ZB / 16 / 256;  // loads a thread
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

// fragment of an operand that lies row by row along K (see lds_read_tr): rows
// k .. k + 8 of this lane's column; a: LDS byte address of row k + i / 4, piece
// i % 4, of the 16 lanes' columns, and of the row 4 further on
__device__ __forceinline__ bf16x8_t read_tr(uint32_t a0, uint32_t a1) {
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a0);
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a1);
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int ET, int CW>
__global__ __launch_bounds__(256) void k_balance_grad(const bf16_t* w, const bf16_t* h,
                                                      const bf16_t* dz,
                                                      const unsigned long long* mask, int T, int E,
                                                      int d, bf16_t* dh, float* part_dw,
                                                      bf16_t* dw) {
  using G = Grad<ET, CW>;
  __shared__ __align__(16) char lds[G::LDS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * G::BC, cw = 16 * CW * wave;  // the block's and the wavefront's columns
  const int c_valid = min(G::BC, d - c0);
  const int n_t = (T + kTile - 1) / kTile;
  char* s_h = lds;
  char* s_z = lds + kTile * G::HR;
  const uint32_t ah = lds_addr(s_h), az = lds_addr(s_z);
  // fragments of w: column cw + 16 j + fr, experts 32 s + 8 q .. (ET = 1: 8 (q % 2) ..)
  bf16x8_t fw[G::KS][CW];
#pragma unroll
  for (int s = 0; s < G::KS; ++s)
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      union {
        bf16x8_t v;
        bf16_t e[8];
      } f;
      const int c = c0 + min(cw + 16 * j + fr, c_valid - 1);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int e = ET == 1 ? 8 * (q & 1) + u : 32 * s + 8 * q + u;
        f.e[u] = e < E ? w[(size_t)e * d + c] : bf16_t(0);
      }
      fw[s][j] = f.v;
    }
  f32x4_t acc[ET][CW];
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) acc[i][j] = f32x4_t{};

  constexpr int HC = G::HR / 16;  // 16-byte chunks of a row of h
  u32x4_t xh[G::HL], xz[G::ZL];
  auto load = [&](int tile) {
    const unsigned long long live = mask[tile];
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / HC, ch = i % HC;
      const size_t t = (size_t)tile * kTile + r;
      // a row without a slot may hold anything, and 0 * NaN is NaN (its bit is
      // off in rows past T too)
      xh[u] = u32x4_t{};
      if ((live >> r & 1) && 8 * ch < c_valid)
        xh[u] = *reinterpret_cast<const u32x4_t*>(h + t * d + c0 + 8 * ch);
    }
#pragma unroll
    for (int u = 0; u < G::ZL; ++u) {
      const int i = threadIdx.x + 256 * u;
      xz[u] = *reinterpret_cast<const u32x4_t*>(dz + (size_t)tile * kTile * (32 * ET) + 8 * i);
    }
  };
  int tile = blockIdx.y;
  if (tile < n_t) load(tile);
  for (; tile < n_t; tile += gridDim.y) {
    __syncthreads();  // the last tile is read
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / HC, ch = i % HC;
      const int at = r * G::HR + (((ch >> 1) ^ tr_swz(r)) << 5) + 16 * (ch & 1);
      *reinterpret_cast<u32x4_t*>(s_h + at) = xh[u];
    }
#pragma unroll
    for (int u = 0; u < G::ZL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / (4 * ET), ch = i % (4 * ET);
      *reinterpret_cast<u32x4_t*>(s_z + r * G::ZR + 16 * ch) = xz[u];
    }
    __syncthreads();
    if (tile + (int)gridDim.y < n_t) load(tile + gridDim.y);
    // dw += dz^T h: two k-steps of 32 rows
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int k = 32 * s + 8 * q + (fr >> 2);
      bf16x8_t fh[CW];
#pragma unroll
      for (int j = 0; j < CW; ++j) {
        const int piece = wave * CW + j;  // of 16 columns
        const uint32_t a = ah + k * G::HR + ((piece ^ tr_swz(k)) << 5) + 8 * (fr & 3);
        fh[j] = read_tr(a, a + 4 * G::HR);
      }
#pragma unroll
      for (int i = 0; i < ET; ++i)
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const uint32_t a = az + k * G::ZR + (part * ET + i) * 32 + 8 * (fr & 3);
          const bf16x8_t fz = read_tr(a, a + 4 * G::ZR);
#pragma unroll
          for (int j = 0; j < CW; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh[j], fz, acc[i][j], 0, 0, 0);
        }
    }
    // dh = dz w: 4 tiles of 16 rows
    if (dh) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4_t o[CW];
#pragma unroll
        for (int j = 0; j < CW; ++j) o[j] = f32x4_t{};
        const char* zr = s_z + (16 * rt + fr) * G::ZR + 16 * q;
#pragma unroll
        for (int s = 0; s < (ET == 1 ? 1 : ET); ++s) {
          const bf16x8_t fz = *reinterpret_cast<const bf16x8_t*>(zr + 64 * s);
#pragma unroll
          for (int j = 0; j < CW; ++j)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[s % G::KS][j], fz, o[j], 0, 0, 0);
        }
        const size_t t = (size_t)tile * kTile + 16 * rt + fr;
#pragma unroll
        for (int j = 0; j < CW; j += 2) {
          const float x[4] = {o[j][0], o[j][1], o[j][2], o[j][3]};
          const float y[4] = {o[j + 1][0], o[j + 1][1], o[j + 1][2], o[j + 1][3]};
          const u32x4_t v = pack_rows(x, y);
          const int c = cw + 16 * j + pack_col(lane);
          if (t < (size_t)T && c < c_valid) *reinterpret_cast<u32x4_t*>(dh + t * d + c0 + c) = v;
        }
      }
    }
  }
  if (!part_dw && !dw) return;
  // lane: columns 4 q .. + 4 of its 16, expert fr
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      const int e = 16 * i + fr, c = cw + 16 * j + 4 * q;
      if (e >= E || c >= c_valid) continue;
      if (dw) {
        uint2 v;
        v.x = pack_bf16x2(acc[i][j][0], acc[i][j][1]);
        v.y = pack_bf16x2(acc[i][j][2], acc[i][j][3]);
        *reinterpret_cast<uint2*>(dw + (size_t)e * d + c0 + c) = v;
      } else {
        *reinterpret_cast<f32x4_t*>(part_dw + ((size_t)blockIdx.y * E + e) * d + c0 + c) = acc[i][j];
      }
    }
}

// dw from its R slices (4 elements a thread), then db from the tiles' sums (one
// wavefront an expert)
__global__ __launch_bounds__(256) void k_balance_finish(const float* part_dw, int R, size_t n,
                                                        int dw_blocks, bf16_t* dw,
                                                        const float* part_db, int n_t, int E,
                                                        float* db) {
  if ((int)blockIdx.x < dw_blocks) {
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= n) return;
    f32x4_t s = *reinterpret_cast<const f32x4_t*>(part_dw + i);
#pragma unroll 4
    for (int r = 1; r < R; ++r) s += *reinterpret_cast<const f32x4_t*>(part_dw + (size_t)r * n + i);
    uint2 v;
    v.x = pack_bf16x2(s[0], s[1]);
    v.y = pack_bf16x2(s[2], s[3]);
    *reinterpret_cast<uint2*>(dw + i) = v;
    return;
  }
  const int e = ((int)blockIdx.x - dw_blocks) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (e >= E) return;
  float s = 0.f;
  for (int i = lane; i < n_t; i += 64) s += part_db[(size_t)i * E + e];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) db[e] = s;
}

// rows with a slot, zeros for the others: an inactive row's h may hold
// anything, and 0 * NaN is NaN
__global__ __launch_bounds__(256) void k_live_rows(const float* h, const int16_t* target, int E,
                                                   int k, int d, float* out) {
  const size_t t = blockIdx.x;
  bool live = false;
  for (int s = 0; s < k; ++s) {
    const int e = target[t * k + s];
    live |= e >= 0 && e < E;
  }
  for (int i = threadIdx.x; i < d; i += 256) out[t * d + i] = live ? h[t * d + i] : 0.f;
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
// rows / 16 a forward block takes at once: w passes the block once for them
constexpr int row_tiles(int et) { return et >= 8 ? 2 : 1; }
// columns / 64 of a gradient block: accumulators of dw and fragments of w in registers
constexpr int col_tiles(int et) { return et == 16 ? 2 : 4; }

struct Plan {
  bool bf16;
  int E, d, T, et;
  int nb;     // forward blocks
  int s_z;    // fp32: K splits of the logits
  size_t f_c, f_z, f_total;  // forward: counts, logits
  int n_t;    // tiles of 64 rows
  int R;      // bf16: slices of dw; fp32: K splits of dw
  size_t b_mask, b_db, b_dw, b_h, b_total;
  Plan(bool bf, int E_, int d_, int T_) : bf16(bf), E(E_), d(d_), T(T_), et(expert_tiles(E_)) {
    const int rows = std::max(T, 1), per = bf16 ? 16 * row_tiles(et) : 16;
    nb = std::min(kRowBlocks, cdiv(rows, per));
    s_z = bf16 ? 1 : product_splits(rows, E, d);
    f_c = align256((size_t)nb * E * 4);
    f_z = f_c + align256((size_t)nb * (E + 1) * 4);
    f_total = f_z + (bf16 ? 0 : align256((size_t)s_z * rows * E * 4));
    n_t = cdiv(rows, kTile);
    size_t dz;
    if (bf16) {
      // two blocks a CU, and slices of dw no larger than 32 MB together
      const int n_c = cdiv(d, 64 * col_tiles(et));
      const size_t most = ((size_t)32 << 20) / ((size_t)E * d * 4);
      R = std::max(1, std::min(std::min(n_t, cdiv(512, n_c)), (int)std::min<size_t>(most, 1 << 20)));
      dz = (size_t)n_t * kTile * 64 * et;
    } else {
      R = product_splits(E, d, rows);
      dz = (size_t)rows * E * 4;
    }
    b_mask = align256(dz);
    b_db = b_mask + align256((size_t)n_t * 8);
    b_dw = b_db + align256((size_t)n_t * E * 4);
    b_h = b_dw + (R > 1 ? align256((size_t)R * E * d * 4) : 0);
    b_total = b_h + (bf16 ? 0 : align256((size_t)rows * d * 4));
  }
};

hipError_t forward(const BalanceArgs& a, hipStream_t st) {
  const Plan p(a.bf16, a.E, a.d, a.T);
  float* part_p = reinterpret_cast<float*>(a.ws);
  int32_t* part_c = reinterpret_cast<int32_t*>(a.ws + p.f_c);
  float* z = reinterpret_cast<float*>(a.ws + p.f_z);
  if (a.T > 0 && !a.bf16) {
    const hipError_t e = launch_product(operand<float, true>(a.h, a.d, a.T, a.d),
                                        operand<float, true>(a.w, a.d, a.E, a.d), p.s_z, false, z, st);
    if (e != hipSuccess) return e;
  }
  if (a.T > 0)
    with_tiles(a.E, [&](auto c) {
      constexpr int ET = c;
      constexpr int RT = row_tiles(ET);
      if (a.bf16)
        hipLaunchKernelGGL((k_balance_forward<ET, RT>), dim3(p.nb), dim3(256), 0, st,
                           static_cast<const bf16_t*>(a.w), a.b,
                           static_cast<const bf16_t*>(a.h), a.target, a.T, a.E, a.k, a.d, a.prob,
                           part_p, part_c);
      else
        hipLaunchKernelGGL(k_balance_rows<ET>, dim3(p.nb), dim3(256), 0, st, z, p.s_z, a.b, a.target,
                           a.T, a.E, a.k, a.prob, part_p, part_c);
    });
  int EP = 1;
  while (EP < a.E) EP *= 2;
  hipLaunchKernelGGL(k_balance_loss, dim3(1), dim3(1024), 0, st, part_p, part_c, a.T > 0 ? p.nb : 0,
                     a.E, EP, a.counts, a.prob_sum, a.loss);
  return hipGetLastError();
}

hipError_t backward(const BalanceArgs& a, hipStream_t st) {
  const Plan p(a.bf16, a.E, a.d, a.T);
  unsigned long long* mask = reinterpret_cast<unsigned long long*>(a.ws + p.b_mask);
  float* part_db = reinterpret_cast<float*>(a.ws + p.b_db);
  float* part_dw = reinterpret_cast<float*>(a.ws + p.b_dw);
  with_tiles(a.E, [&](auto c) {
    constexpr int ET = c;
    if (a.bf16)
      hipLaunchKernelGGL((k_balance_dz<ET, true>), dim3(p.n_t), dim3(256), 0, st, a.prob, a.target,
                         a.counts, a.dloss, a.T, a.E, a.k, a.ws, mask, part_db);
    else
      hipLaunchKernelGGL((k_balance_dz<ET, false>), dim3(p.n_t), dim3(256), 0, st, a.prob, a.target,
                         a.counts, a.dloss, a.T, a.E, a.k, a.ws, nullptr, part_db);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.bf16) {
    bf16_t* dw = static_cast<bf16_t*>(a.dw);
    const bool whole = p.R == 1;
    if (a.dh || a.dw)
      with_tiles(a.E, [&](auto c) {
        constexpr int ET = c;
        using G = Grad<ET, col_tiles(ET)>;
        hipLaunchKernelGGL((k_balance_grad<ET, col_tiles(ET)>), dim3(cdiv(a.d, G::BC), p.R), dim3(256),
                           0, st, static_cast<const bf16_t*>(a.w),
                           static_cast<const bf16_t*>(a.h), reinterpret_cast<const bf16_t*>(a.ws),
                           mask, a.T, a.E, a.d, static_cast<bf16_t*>(a.dh),
                           a.dw && !whole ? part_dw : nullptr, whole ? dw : nullptr);
      });
    const size_t n = (size_t)a.E * a.d;
    const int dw_blocks = a.dw && !whole ? (int)((n / 4 + 255) / 256) : 0;
    const int db_blocks = a.db ? cdiv(a.E, 4) : 0;
    if (dw_blocks + db_blocks > 0)
      hipLaunchKernelGGL(k_balance_finish, dim3(dw_blocks + db_blocks), dim3(256), 0, st, part_dw, p.R,
                         n, dw_blocks, dw, part_db, p.n_t, a.E, a.db);
    return hipGetLastError();
  }
  const float* dz = reinterpret_cast<const float*>(a.ws);
  if (a.db)
    hipLaunchKernelGGL(k_balance_finish, dim3(cdiv(a.E, 4)), dim3(256), 0, st, nullptr, 0, (size_t)0, 0,
                       nullptr, part_db, p.n_t, a.E, a.db);
  e = hipGetLastError();
  if (e == hipSuccess && a.dh)
    e = launch_product(operand<float, true>(dz, a.E, a.T, a.E),
                       operand<float, false>(a.w, a.d, a.d, a.E), 1, false,
                       static_cast<float*>(a.dh), st);
  if (e == hipSuccess && a.dw) {
    float* hl = reinterpret_cast<float*>(a.ws + p.b_h);
    if (a.T > 0)
      hipLaunchKernelGGL(k_live_rows, dim3(a.T), dim3(256), 0, st, static_cast<const float*>(a.h),
                         a.target, a.E, a.k, a.d, hl);
    const auto D = operand<float, false>(dz, a.E, a.E, a.T);
    const auto H = operand<float, false>(hl, a.d, a.d, a.T);
    float* dw = static_cast<float*>(a.dw);
    if (p.R == 1) {
      e = launch_product(D, H, 1, false, dw, st);
    } else {
      e = launch_product(D, H, p.R, false, part_dw, st);
      if (e == hipSuccess) e = launch_sum_parts(part_dw, p.R, (size_t)a.E * a.d, dw, st);
    }
  }
  return e;
}

}  // namespace

size_t balance_ws(bool bf16, int E, int d, int T) { return Plan(bf16, E, d, T).f_total; }
size_t balance_backward_ws(bool bf16, int E, int d, int T) { return Plan(bf16, E, d, T).b_total; }

hipError_t launch_balance(const BalanceArgs& a, hipStream_t st) { return forward(a, st); }
hipError_t launch_balance_backward(const BalanceArgs& a, hipStream_t st) { return backward(a, st); }

}  // namespace trimmoe
