// Both products of a tall thin matrix z [rows, E] (E <= 256) in one pass over the
// rows x [rows, d] that belong to it: out = z w, [rows, d], and z^T x, [E, d].
// The gradients of a router (z = dz, x = h) and those of a vocabulary head for a
// few tokens (rows of the vocabulary, E the tokens) have this form.
//
// A block takes 64 CW columns and every gridDim.y-th tile of 64 rows, in 16 x 16 x
// 32 MFMAs whose A rows are the columns.  x is read once and out written once;
// w's fragments stay in registers (a lane's 8 experts of a column), those of x (8
// rows of a column) come transposed out of LDS, as do z's for z^T x.  The next
// tile's loads are in flight under a tile's products.
//   z in two parts of bf16 (what bf16 holds of it and of the rest: within 2^-16; added up
// in the products), [row][part][16 ET].  ET = 1: both are one k-step of 32 (16 experts
// each, w's fragment twice); else a k-step is 32 experts of a part.
#pragma once

#include "mfma_core.h"

namespace trimmoe {

constexpr int kRowTile = 64;
constexpr int kZParts = 2;

template <int ET, int CW>
struct RowsGrad {
  static constexpr int BC = 64 * CW;                // columns of a block
  static constexpr int HR = 2 * BC;                 // LDS bytes of a row of x
  static constexpr int ZB = 32 * kZParts * ET;      // bytes of a row of z
  static constexpr int ZR = ZB + 32;                // ... in LDS: rows on distinct banks
  static constexpr int KS = ET == 1 ? 1 : ET / 2;   // fragments of w
  static constexpr int ZS = ET * kZParts / 2;       // k-steps of out
  static constexpr int LDS = kRowTile * (HR + ZR);
  static constexpr int HL = kRowTile * HR / 16 / 256, ZL = kRowTile * ZB / 16;  // 16-byte loads
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

// fragment of an operand that lies row by row along K (see lds_read_tr): 8 rows
// of this lane's column; a0: LDS byte address of row i / 4, piece i % 4 (lane i of
// 16) of the first four, a1 of the next four
__device__ __forceinline__ bf16x8_t read_tr(uint32_t a0, uint32_t a1) {
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a0);
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a1);
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// P: w(e, c) element of w (0 past E and in rows that take no part), mask(tile) the
// tile's rows to read (the others are zeros), scale of out.  out [rows, d], part
// [gridDim.y][E, d] fp32, whole [E, d] bf16 (instead of part): each may be NULL.
template <int ET, int CW, class P>
__device__ __forceinline__ void rows_grad(char* lds, const P& p, const bf16_t* x, const bf16_t* z,
                                          int rows, int E, int d, bf16_t* out, float* part,
                                          bf16_t* whole) {
  using G = RowsGrad<ET, CW>;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, fr = lane & 15, q = lane >> 4;
  const int c0 = blockIdx.x * G::BC, cw = 16 * CW * wave;  // first columns: block, wavefront
  const int c_valid = min(G::BC, d - c0);
  const int n_t = (rows + kRowTile - 1) / kRowTile;
  char* s_x = lds;
  char* s_z = lds + kRowTile * G::HR;
  const uint32_t ax = lds_addr(s_x), az = lds_addr(s_z);
  // fragments of w: column cw + 16 j + fr, experts 32 s + 8 q .. (ET = 1: 8 (q % 2) ..)
  bf16x8_t fw[G::KS][CW];
  if (out) {
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
        for (int u = 0; u < 8; ++u)
          f.e[u] = p.w(ET == 1 ? 8 * (q & 1) + u : 32 * s + 8 * q + u, c);
        fw[s][j] = f.v;
      }
  }
  f32x4_t acc[ET][CW];
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) acc[i][j] = f32x4_t{};

  constexpr int XC = G::HR / 16;                    // 16-byte chunks of a row of x
  constexpr int ZN = (G::ZL + 255) / 256;           // loads of z a thread
  u32x4_t xh[G::HL], xz[ZN];
  auto load = [&](int tile) {
    const unsigned long long live = p.mask(tile);
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / XC, ch = i % XC;
      const size_t t = (size_t)tile * kRowTile + r;
      xh[u] = u32x4_t{};
      if ((live >> r & 1) && 8 * ch < c_valid)
        xh[u] = *reinterpret_cast<const u32x4_t*>(x + t * d + c0 + 8 * ch);
    }
#pragma unroll
    for (int u = 0; u < ZN; ++u) {
      const int i = threadIdx.x + 256 * u;
      if (G::ZL % 256 == 0 || i < G::ZL)
        xz[u] = *reinterpret_cast<const u32x4_t*>(z + (size_t)tile * kRowTile * (G::ZB / 2) + 8 * i);
    }
  };
  int tile = blockIdx.y;
  if (tile < n_t) load(tile);
  for (; tile < n_t; tile += gridDim.y) {
    __syncthreads();  // the last tile is read
#pragma unroll
    for (int u = 0; u < G::HL; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / XC, ch = i % XC;
      const int at = r * G::HR + (((ch >> 1) ^ tr_swz(r)) << 5) + 16 * (ch & 1);
      *reinterpret_cast<u32x4_t*>(s_x + at) = xh[u];
    }
#pragma unroll
    for (int u = 0; u < ZN; ++u) {
      const int i = threadIdx.x + 256 * u, r = i / (G::ZB / 16), ch = i % (G::ZB / 16);
      if (G::ZL % 256 == 0 || i < G::ZL)
        *reinterpret_cast<u32x4_t*>(s_z + r * G::ZR + 16 * ch) = xz[u];
    }
    __syncthreads();
    if (tile + (int)gridDim.y < n_t) load(tile + gridDim.y);
    // z^T x: two k-steps of 32 rows
    if (part || whole) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int k = 32 * s + 8 * q + (fr >> 2);
        bf16x8_t fx[CW];
#pragma unroll
        for (int j = 0; j < CW; ++j) {
          const int piece = wave * CW + j;  // of 16 columns
          const uint32_t a = ax + k * G::HR + ((piece ^ tr_swz(k)) << 5) + 8 * (fr & 3);
          fx[j] = read_tr(a, a + 4 * G::HR);
        }
#pragma unroll
        for (int i = 0; i < ET; ++i)
#pragma unroll
          for (int n = 0; n < kZParts; ++n) {
            const uint32_t a = az + k * G::ZR + (n * ET + i) * 32 + 8 * (fr & 3);
            const bf16x8_t fz = read_tr(a, a + 4 * G::ZR);
#pragma unroll
            for (int j = 0; j < CW; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[j], fz, acc[i][j], 0, 0, 0);
          }
      }
    }
    // z w: 4 tiles of 16 rows
    if (out) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4_t o[CW];
#pragma unroll
        for (int j = 0; j < CW; ++j) o[j] = f32x4_t{};
        const char* zr = s_z + (16 * rt + fr) * G::ZR + 16 * q;
#pragma unroll
        for (int s = 0; s < G::ZS; ++s) {
          const bf16x8_t fz = *reinterpret_cast<const bf16x8_t*>(zr + 64 * s);
#pragma unroll
          for (int j = 0; j < CW; ++j)
            o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[s % G::KS][j], fz, o[j], 0, 0, 0);
        }
        const size_t t = (size_t)tile * kRowTile + 16 * rt + fr;
#pragma unroll
        for (int j = 0; j < CW; j += 2) {
          float u[4], v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            u[k] = o[j][k] * p.scale;
            v[k] = o[j + 1][k] * p.scale;
          }
          const u32x4_t w = pack_rows(u, v);
          const int c = cw + 16 * j + pack_col(lane);
          if (t < (size_t)rows && c < c_valid) *reinterpret_cast<u32x4_t*>(out + t * d + c0 + c) = w;
        }
      }
    }
  }
  if (!part && !whole) return;
  // lane: columns 4 q .. + 4 of its 16, expert fr
#pragma unroll
  for (int i = 0; i < ET; ++i)
#pragma unroll
    for (int j = 0; j < CW; ++j) {
      const int e = 16 * i + fr, c = cw + 16 * j + 4 * q;
      if (e >= E || c >= c_valid) continue;
      if (whole) {
        uint2 v;
        v.x = pack_bf16x2(acc[i][j][0], acc[i][j][1]);
        v.y = pack_bf16x2(acc[i][j][2], acc[i][j][3]);
        *reinterpret_cast<uint2*>(whole + (size_t)e * d + c0 + c) = v;
      } else {
        *reinterpret_cast<f32x4_t*>(part + ((size_t)blockIdx.y * E + e) * d + c0 + c) = acc[i][j];
      }
    }
}

}  // namespace trimmoe
