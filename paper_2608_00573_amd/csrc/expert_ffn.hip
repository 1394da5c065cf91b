// The expert feed-forward block on rows sorted by expert, and its gradient.
//   u = x Wu^T, g = x Wg^T, a = silu(g) u (gated) or relu(u), y = a Wd^T
//   da = dy Wd;  s = sigmoid(g):  du = da g s,  dg = da u s (1 + g (1 - s));
//   relu: du = da [u > 0]
//   dx = du Wu + dg Wg,  dWu = du^T x,  dWg = dg^T x,  dWd = dy^T a
// Forward: one kernel makes both projections and the activation (and keeps u and g, in
// bf16 or in 8 bits), one the product with Wd.  Backward: da with the activation's
// derivative in its epilogue (a, du, dg to the workspace, in bf16: they are operands of
// the products), then dx, then all weight gradients in one kernel.
// A tile's A side is the contiguous side of its result, so that a lane holds 4
// consecutive elements of a row and results leave the registers in 16-byte pieces.
//
// Rows are cut in tiles of 32, 128 or 256 by their number a group (rows_kind): the large-
// group core has the least LDS and L2 traffic an MFMA, but its tiles waste half a tile of
// rows a group and leave their registers with nothing else on the CU (da's epilogue reads
// and writes 5 values an element).  Traces of both sides: rows_kind.
#include "expert_ffn.h"

#include <algorithm>

#include "big_feed.h"

namespace trimmoe {

namespace {

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// a tile of rows times columns from c0 on; its group e (E and above: rows of no group,
// which have no product); which piece of its K
struct RowTile {
  int e, r0, valid, c0, piece;
  RowTile() = default;
  // tile L of the patch order
  __device__ __forceinline__ RowTile(const GroupTiles& t, const Groups& g, const TileSched& S, int L,
                                     int rows, int cols) {
    int mt, nt, within;
    S.decode_abs(L, mt, nt, piece);
    e = t.group(mt, within);
    const int2 r = g.rows(e);
    r0 = uniform(r.x + within * rows);
    valid = uniform(min(rows, r.y - r0));
    c0 = uniform(nt * cols);
    piece = uniform(piece);
  }
};
struct RowQueue {
  TileQueue<5> q;
  __device__ __forceinline__ int left() const { return q.n; }
  __device__ __forceinline__ void push(const RowTile& t) {
    q.push({{t.e, t.r0, t.valid, t.c0, t.piece}});
  }
  __device__ __forceinline__ RowTile pop() {
    const auto v = q.pop();
    RowTile t;
    t.e = v.v[0];
    t.r0 = v.v[1];
    t.valid = v.v[2];
    t.c0 = v.v[3];
    t.piece = v.v[4];
    return t;
  }
};

// sigmoid with the hardware exp2 and reciprocal (about 1 ulp each)
__device__ __forceinline__ float sigmoid_hw(float g) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-g * 1.4426950408889634f));
}

// 8 codes of a row, 8 bytes a lane, and the block's scale byte, from two accumulators'
// values (32 columns over 4 lanes)
__device__ __forceinline__ void store_codes(const float (&x)[2][4], bool in, int lane, int8_t* codes,
                                            uint8_t* scale) {
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = max(top, abs_bits(x[k][r]));
  LanePair p = lanes_xor16(__uint_as_float(top));
  top = max(__float_as_uint(p.a), __float_as_uint(p.b));
  p = lanes_xor32(__uint_as_float(top));
  top = max(__float_as_uint(p.a), __float_as_uint(p.b));
  const uint32_t s = pack_scale(top);
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t b[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) b[r] = pack_code_bits(x[k][r], s);
    // the lowest byte of each
    w[k] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
    w[k] = s == 255 ? 0u : w[k];
  }
  const auto q = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
  const uint32_t q0 = q[0], q1 = q[1];
  if (in) {
    *reinterpret_cast<uint2*>(codes + pack_col(lane)) = make_uint2(q0, q1);
    if (lane < 16) *scale = (uint8_t)s;
  }
}

// ---------------------------------------------------------------- forward --
struct UpArgs {
  Groups groups;
  const bf16_t *w_up, *w_gate, *x;
  int d, F;
  bf16_t* a;  // [n, F]
  void *up, *gate;
  uint8_t *up_scale, *gate_scale;
};

// A tile's first loads go out before the tile before it leaves its registers.  Bound by
// the MFMAs at the clock that the power limit leaves and, beside them, the activation and
// the codes of kept values (8192 rows, 4096 x 14336, kept in 8 bits: 1.89 ms, 1.02 PFLOP/s, a
// fifth of it the epilogue), with few rows by reading the weights (64 rows over 8 experts:
// 1.88 GB in 320 us, 5.9 TB/s).
template <class C, bool GATED, int KEEP>
__global__ __launch_bounds__(256, C::T::OCC) void k_expert_up(UpArgs a) {
  using T = typename C::T;
  __shared__ __align__(16) char lds[T::LDS];
  const GroupTiles tiles(a.groups, a.groups.E + 2, T::BN);
  TileSched S;
  int ntiles;
  if (!S.init(tiles.n, (a.F + T::ROWS_A - 1) / T::ROWS_A, 1, ntiles)) return;
  C core(lds);
  int jl = 0;
  RowQueue queue;
  auto load = [&] {
    if (jl == ntiles) return false;
    const RowTile at(tiles, a.groups, S, S.tb + S.i0 + jl++ * S.bx, T::BN, T::ROWS_A);
    queue.push(at);
    const int k = at.e < a.groups.E ? a.d : 0;
    const size_t w0 = ((size_t)(k ? at.e : 0) * a.F + at.c0) * a.d;
    tile_rows(core.a, a.w_up + w0, a.d, min(T::ROWS_A, a.F - at.c0), k, T::SPAN);
    if constexpr (GATED) core.a.p1 = reinterpret_cast<const char*>(a.w_gate + w0);
    tile_rows(core.b, a.x + (size_t)at.r0 * a.d, a.d, at.valid, k);
    core.left = max(k / T::KS, 1);
    return true;
  };
  constexpr int TMO = GATED ? T::TM / 2 : T::TM;  // 16-column groups of a wavefront
  core.first(load);
  while (queue.left()) {
    const RowTile was = queue.pop();
    typename C::Acc acc;
    core.run(was.e < a.groups.E ? a.d / T::KS : 1, acc, load);
    core.ahead(load);
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
      const int t = core.wn * T::WN + 16 * j + (core.lane & 15);
#pragma unroll
      for (int i = 0; i < TMO; i += 2) {
        const int c = was.c0 + core.wm * 16 * TMO + 16 * i;  // 32 columns, all of them or none in F
        const bool in = t < was.valid && c < a.F;
        const size_t o = (size_t)(was.r0 + t) * a.F + c;
        float u[2][4], g[2][4], v[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            u[k][r] = acc[i + k][j][r];
            if constexpr (GATED) {
              g[k][r] = acc[i + k + TMO][j][r];
              v[k][r] = g[k][r] * sigmoid_hw(g[k][r]) * u[k][r];
            } else {
              v[k][r] = u[k][r] < 0.f ? 0.f : u[k][r];  // (NaN stays)
            }
          }
        const int pc = pack_col(core.lane);
        const u32x4_t pv = pack_rows(v[0], v[1]);
        if (in) *reinterpret_cast<u32x4_t*>(a.a + o + pc) = pv;
        if constexpr (KEEP == TRIMMOE_KEEP_FULL) {
          const u32x4_t pu = pack_rows(u[0], u[1]);
          if (in) *reinterpret_cast<u32x4_t*>(static_cast<bf16_t*>(a.up) + o + pc) = pu;
          if constexpr (GATED) {
            const u32x4_t pg = pack_rows(g[0], g[1]);
            if (in) *reinterpret_cast<u32x4_t*>(static_cast<bf16_t*>(a.gate) + o + pc) = pg;
          }
        }
        if constexpr (KEEP == TRIMMOE_KEEP_PACKED) {
          store_codes(u, in, core.lane, static_cast<int8_t*>(a.up) + o, a.up_scale + o / kPackBlock);
          if constexpr (GATED)
            store_codes(g, in, core.lane, static_cast<int8_t*>(a.gate) + o,
                        a.gate_scale + o / kPackBlock);
        }
      }
    }
  }
  core.last();
}

// out [n, M] = rows times weights: y = a Wd^T (Wd K-contiguous) or, ATR, dx = du Wu (+
// dg Wg) (weights along K; the second product continues the first one's K).  Rows of no
// group get zeros.
// Few tiles leave CUs idle, so K is cut.  Small tiles: every tile in `splits` pieces
// whose sums k_join_slices adds.  The large-group core: the tiles of its last, partial
// round in as many pieces as its blocks make up (RowTail), which k_join_tail adds.
// 8192 rows over 8 experts (4096 x 14336), 2.25 rounds of 256 tiles: y 1043 to 860 us, dx
// 1977 to 1570; 2047 rows of 2048 x 5632, a quarter of a round: dx 230 to 118 us.  A slice
// of a 256 x 256 tile takes 1.5 to 1.6 us (1.34 PFLOP/s), what the power limit leaves.
struct RowsArgs {
  Groups groups;
  const bf16_t *w, *w2;  // expert 0; w2: NULL or the second product's
  const bf16_t *b, *b2;  // [n, K]
  int M, K;
  bf16_t* out;
  int splits;   // small tiles
  float* part;  // [splits][n, M], or of the tail [blocks][256][256]
};

// How the large-group core's blocks of an XCD share its tiles: `full` whole ones each,
// and the `tiles` of the last round in `pieces` each (1: whole).  A slice takes 1.5 us, the
// two launches that pieces need 10: short K is not cut (16384 rows over 60 experts, 22 and
// 44 slices: 157 and 280 us, 10 more with them).
constexpr int kTailSlices = 64;
struct RowTail {
  int full, tiles, pieces;
  __device__ __forceinline__ RowTail(int total, int slices, int grid, int x, int nx) {
    const int bx = (grid - x + nx - 1) / nx, n = total / nx + (x < total % nx ? 1 : 0);
    full = uniform(n / bx);
    tiles = uniform(n) - full * uniform(bx);
    pieces = tiles == 0 || slices < kTailSlices ? 1 : uniform(min(min(bx / max(tiles, 1), 8), slices / 8));
  }
  __device__ __forceinline__ bool cut() const { return pieces > 1; }
};

// A tile's results, bf16, 16 bytes a lane.  Rows past `valid` lie behind the buffer's
// end and are dropped, as are columns past M by their offset (M is a multiple of 64:
// blocks of 32 are valid or not as a whole), so that every wavefront issues STORES<C>
// stores.
template <class C>
constexpr int STORES = C::T::TM * C::T::TN / 2;
template <class C>
__device__ __forceinline__ void store_tile(const C& core, const typename C::Acc& acc, bf16_t* out, size_t row0,
                                           int valid, int m0, int M) {
  using T = typename C::T;
  m0 = uniform(m0);
  M = uniform(M);
  asm volatile("" : "+s"(M));  // per-tile value: keeps the offsets below inside the tile loop
  const __amdgpu_buffer_rsrc_t ro =
      uniform_rsrc(reinterpret_cast<const char*>(out + row0 * M + m0),
                   uniform((int)((uint32_t)min(valid, T::BN) * M * 2 - m0 * 2)));
  const uint32_t cw = core.wm * T::WM;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const uint32_t off =
        ((uint32_t)(core.wn * T::WN + 16 * j + (core.lane & 15)) * M + cw + pack_col(core.lane)) * 2;
#pragma unroll
    for (int i = 0; i < T::TM; i += 2) {
      float v[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[k][r] = acc[i + k][j][r];
      // (no scalar offset: see pack_rows)
      __builtin_amdgcn_raw_buffer_store_b128(
          pack_rows(v[0], v[1]), ro, ((int)(m0 + cw + 16 * i) < M ? off : 0xffff0000u) + 32 * i, 0, 0);
    }
  }
}

// the same as fp32 sums [.., ld]
template <class C>
__device__ __forceinline__ void store_part(const C& core, const typename C::Acc& acc, float* out, int valid,
                                           int cols, int ld) {
  using T = typename C::T;
  cols = uniform(cols);
  ld = uniform(ld);
  asm volatile("" : "+s"(ld));
  const __amdgpu_buffer_rsrc_t ro =
      uniform_rsrc(reinterpret_cast<const char*>(out),
                   uniform((int)(((uint32_t)(min(valid, T::BN) - 1) * ld + min(cols, T::BM)) * 4)));
  const uint32_t cw = core.wm * T::WM;
#pragma unroll
  for (int j = 0; j < T::TN; ++j) {
    const uint32_t off =
        ((uint32_t)(core.wn * T::WN + 16 * j + (core.lane & 15)) * ld + cw + 4 * (core.lane >> 4)) * 4;
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
      f32x4_t v = acc[i][j];
      asm volatile("" : "+v"(v));  // (through VGPRs: see gemm.hip, big_store_partial_rows)
      __builtin_amdgcn_raw_buffer_store_b128(
          __builtin_bit_cast(u32x4_t, v), ro,
          ((int)(cw + 16 * i) < cols ? off : 0xffff0000u) + 64 * i, 0, 0);
    }
  }
}

// PART: the pieces of cut tiles, else the whole tiles
template <class C, bool PART>
__global__ __launch_bounds__(256, C::T::OCC) void k_expert_rows(RowsArgs a) {
  using T = typename C::T;
  constexpr bool LARGE = T::OCC == 1;
  __shared__ __align__(16) char lds[T::LDS];
  const GroupTiles tiles(a.groups, a.groups.E + 2, T::BN);
  const int n_ct = (a.M + T::BM - 1) / T::BM, one = a.K / T::KS;
  const int slices = one * (T::ATR && a.w2 ? 2 : 1);
  TileSched S;
  int n = 0;  // the block's tiles, from index S.tb + S.i0 on
  if (!S.init(tiles.n, n_ct, !LARGE && PART ? a.splits : 1, n)) n = 0;
  int pieces = a.splits, piece = 0;
  if constexpr (LARGE) {
    const int nx = min(kXcd, (int)gridDim.x);
    const RowTail tail(tiles.n * n_ct, slices, gridDim.x, blockIdx.x % nx, nx);
    if (PART) {
      if (!tail.cut()) return;
      pieces = tail.pieces;
      piece = uniform(S.i0 / tail.tiles);
      n = piece < pieces ? 1 : 0;
      S.tb += tail.full * S.bx - piece * tail.tiles;
    } else if (tail.cut()) {
      n = tail.full;
    }
  }
  if (n == 0) return;
  C core(lds);
  const auto from = [&](int q) {  // first slice of a piece
    return PART ? uniform((int)((long)slices * q / pieces)) : q * slices;
  };
  int jl = 0;
  RowQueue queue;
  auto load = [&] {
    if (jl == n) return false;
    RowTile at(tiles, a.groups, S, S.tb + S.i0 + jl++ * S.bx, T::BN, T::BM);
    if (LARGE) at.piece = piece;
    queue.push(at);
    const int K = at.e < a.groups.E ? a.K : 0, s0 = PART && K ? from(at.piece) : 0;
    const bool second = PART && s0 >= one && s0 > 0;  // the piece begins in the second product
    const int k0 = (second ? s0 - one : s0) * T::KS, k = max(K - k0, 0);
    const size_t e0 = K ? (size_t)at.e * a.M * a.K : 0, b0 = (size_t)at.r0 * a.K;
    const bf16_t* w = second ? a.w2 : a.w;
    if constexpr (T::ATR)
      tile_along<T::BM, T::KS>(core.a, w + e0 + (size_t)k0 * a.M, a.M, at.c0, k);
    else
      tile_rows(core.a, w + e0 + (size_t)at.c0 * a.K + k0, a.K, min(T::BM, a.M - at.c0), k);
    tile_rows(core.b, (second ? a.b2 : a.b) + b0 + k0, a.K, at.valid, k);
    if (T::ATR && a.w2 && !second) {
      core.a.q = reinterpret_cast<const char*>(a.w2 + e0 + at.c0);
      core.b.q = reinterpret_cast<const char*>(a.b2 + b0);
      core.a.kq = core.b.kq = K;
    }
    core.left = K ? from(at.piece + 1) - s0 : 1;
    return true;
  };
  core.first(load);
  for (bool stored = false; queue.left(); stored = true) {
    const RowTile was = queue.pop();
    typename C::Acc acc;
    const int nk = was.e < a.groups.E ? from(was.piece + 1) - from(was.piece) : 1;
    if (stored && !PART)
      core.template run<STORES<C>>(nk, acc, load);
    else
      core.run(nk, acc, load);
    core.ahead(load);
    if constexpr (!PART)
      store_tile(core, acc, a.out, was.r0, was.valid, was.c0, a.M);
    else if constexpr (LARGE)
      store_part(core, acc, a.part + (size_t)blockIdx.x * T::BM * T::BN, was.valid, a.M - was.c0, T::BM);
    else
      store_part(core, acc, a.part + ((size_t)was.piece * a.groups.n + was.r0) * a.M + was.c0, was.valid,
                 a.M - was.c0, a.M);
  }
  core.last();
}

// 8 results, 16 bytes, from the sums of their pieces
__device__ __forceinline__ void join8(const float* p, size_t step, int pieces, bf16_t* out) {
  // (8 pieces at most, all loads in flight; one that is missing: the first again, unused)
  f32x4_t v[8], w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float* q = p + (i < pieces ? i : 0) * step;
    v[i] = *reinterpret_cast<const f32x4_t*>(q);
    w[i] = *reinterpret_cast<const f32x4_t*>(q + 4);
  }
  f32x4_t x = v[0], y = w[0];
#pragma unroll
  for (int i = 1; i < 8; ++i)
    if (i < pieces) {
      x += v[i];
      y += w[i];
    }
  *reinterpret_cast<u32x4_t*>(out) = u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                             pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

// The tail's tiles, 8 rows a block (32 of them: 29 us for 24 tiles in 8 pieces); grid.x as
// k_expert_rows had it
constexpr int kJoinRows = 8;
__global__ __launch_bounds__(256) void k_join_tail(RowsArgs a, int slices) {
  const GroupTiles tiles(a.groups, a.groups.E + 2, big::BN);
  const int n_ct = (a.M + big::BM - 1) / big::BM;
  const int nx = min(kXcd, (int)gridDim.x), x = blockIdx.x % nx;
  TileSched S;
  int ntiles;
  S.init(tiles.n, n_ct, 1, ntiles);
  const RowTail tail(tiles.n * n_ct, slices, gridDim.x, x, nx);
  if (!tail.cut() || S.i0 >= tail.tiles) return;
  const RowTile at(tiles, a.groups, S, S.tb + tail.full * S.bx + S.i0, big::BN, big::BM);
  constexpr size_t SLOT = (size_t)big::BM * big::BN;
  const int c = 8 * (threadIdx.x & 31), r = kJoinRows * blockIdx.y + (threadIdx.x >> 5);
  if (r < at.valid && at.c0 + c < a.M)
    join8(a.part + (size_t)blockIdx.x * SLOT + r * big::BM + c, (size_t)nx * tail.tiles * SLOT, tail.pieces,
          a.out + (size_t)(at.r0 + r) * a.M + at.c0 + c);
}

__global__ __launch_bounds__(256) void k_join_slices(const float* part, int splits, size_t n, bf16_t* out) {
  const size_t i = 8 * ((size_t)blockIdx.x * 256 + threadIdx.x);
  if (i < n) join8(part + i, n, splits, out + i);
}

// --------------------------------------------------------------- backward --
struct DactArgs {
  Groups groups;
  const bf16_t *w_down, *dy;
  int d, F;
  const void *up, *gate;
  const uint8_t *up_scale, *gate_scale;
  bf16_t *a, *du, *dg;  // [n, F]
};

// What was kept of one row of a tile: a lane's 4 consecutive columns of each 16.  All of a
// row's loads go out together, and the next row's before this one is used.
template <int TM, bool GATED, bool PACKED>
struct KeptRow {
  typedef std::conditional_t<PACKED, uint32_t, uint2> W;
  W u[TM], g[GATED ? TM : 1];
  uint8_t us[TM / 2], gs[TM / 2];
  // (columns past F: the row's first ones, unused)
  __device__ __forceinline__ void load(const DactArgs& a, size_t row, int c0, int lane) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int c = c0 + 16 * i < a.F ? c0 + 16 * i : 16 * (i & 1);
      const size_t o = row * a.F + c + 4 * (lane >> 4);
      constexpr int ES = PACKED ? 1 : 2;
      u[i] = *reinterpret_cast<const W*>(static_cast<const char*>(a.up) + o * ES);
      if constexpr (GATED) g[i] = *reinterpret_cast<const W*>(static_cast<const char*>(a.gate) + o * ES);
      if (PACKED && i % 2 == 0) {
        us[i / 2] = a.up_scale[o / kPackBlock];
        if constexpr (GATED) gs[i / 2] = a.gate_scale[o / kPackBlock];
      }
    }
  }
  static __device__ __forceinline__ void values(float (&v)[4], const W& w, uint32_t s) {
    if constexpr (PACKED) {
      // (exact at every scale: the whole number before the power of two.  An offset would
      // be scaled too, and 128 steps of the largest scale are past the range of fp32)
      const float step = pack_step(s);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = (float)(int8_t)(w >> (8 * r)) * step;
    } else {
      v[0] = __uint_as_float(w.x << 16);
      v[1] = __uint_as_float(w.x & 0xffff0000u);
      v[2] = __uint_as_float(w.y << 16);
      v[3] = __uint_as_float(w.y & 0xffff0000u);
    }
  }
};

// Bound by the MFMAs and by memory in turns (8192 rows, 4096 x 14336: 1.22 ms, of which 705
// MB written and 240 read take 0.2 to 0.4), with few rows by reading w_down (48 rows over
// 8 experts: 0.94 GB in 240 us, 3.9 TB/s: the columns of a tile are 256 bytes of each row).
template <class C, bool GATED, bool PACKED>
__global__ __launch_bounds__(256, C::T::OCC) void k_expert_dact(DactArgs a) {
  using T = typename C::T;
  __shared__ __align__(16) char lds[T::LDS];
  const GroupTiles tiles(a.groups, a.groups.E, T::BN);
  TileSched S;
  int ntiles;
  if (!S.init(tiles.n, (a.F + T::BM - 1) / T::BM, 1, ntiles)) return;
  C core(lds);
  int jl = 0;
  RowQueue queue;
  auto load = [&] {
    if (jl == ntiles) return false;
    const RowTile at(tiles, a.groups, S, S.tb + S.i0 + jl++ * S.bx, T::BN, T::ROWS_A);
    queue.push(at);
    tile_along<T::BM, T::KS>(core.a, a.w_down + (size_t)at.e * a.d * a.F, a.F, at.c0, a.d);
    tile_rows(core.b, a.dy + (size_t)at.r0 * a.d, a.d, at.valid, a.d);
    core.left = a.d / T::KS;
    return true;
  };
  core.first(load);
  while (queue.left()) {
    const RowTile was = queue.pop();
    typename C::Acc acc;
    core.run(a.d / T::KS, acc, load);
    const int c0 = was.c0 + core.wm * T::WM;
    const auto row_of = [&](int j) { return core.wn * T::WN + 16 * j + (core.lane & 15); };
    KeptRow<T::TM, GATED, PACKED> kept[2];
    const auto fetch = [&](int j) {
      kept[j & 1].load(a, (size_t)(was.r0 + min(row_of(j), was.valid - 1)), c0, core.lane);
    };
    // (the first before the next tile's loads, which it would wait for behind them)
    fetch(0);
    core.ahead(load);
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
      if (j + 1 < T::TN) fetch(j + 1);
      const int t = row_of(j);
      const auto& kj = kept[j & 1];
#pragma unroll
      for (int i = 0; i < T::TM; i += 2) {
        const int c = c0 + 16 * i;
        const bool in = t < was.valid && c < a.F;
        const size_t o = (size_t)(was.r0 + t) * a.F + c;
        float va[2][4], vu[2][4], vg[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float u[4], g[4];
          kj.values(u, kj.u[i + k], kj.us[i / 2]);
          if constexpr (GATED) kj.values(g, kj.g[i + k], kj.gs[i / 2]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float da = acc[i + k][j][r];
            if constexpr (GATED) {
              const float s = sigmoid_hw(g[r]), gs = g[r] * s;
              va[k][r] = gs * u[r];
              vu[k][r] = da * gs;
              vg[k][r] = da * u[r] * (s * (1.f + g[r] * (1.f - s)));
            } else {
              va[k][r] = u[r] < 0.f ? 0.f : u[r];
              vu[k][r] = u[r] > 0.f ? da : 0.f;
            }
          }
        }
        const int pc = pack_col(core.lane);
        const u32x4_t pa = pack_rows(va[0], va[1]), pu = pack_rows(vu[0], vu[1]);
        if (in) {
          *reinterpret_cast<u32x4_t*>(a.a + o + pc) = pa;
          *reinterpret_cast<u32x4_t*>(a.du + o + pc) = pu;
        }
        if constexpr (GATED) {
          const u32x4_t pg = pack_rows(vg[0], vg[1]);
          if (in) *reinterpret_cast<u32x4_t*>(a.dg + o + pc) = pg;
        }
      }
    }
  }
  core.last();
}

// Weight gradients: of group e and product p, out [N, M] = B^T A over the group's rows
// (dWd: A = a, B = dy; dWu, dWg: A = x, B = du, dg).  A group without rows gets zeros.
// K is a group's rows, few slices a tile, so what is between two tiles decides: the next
// tiles' loads are in flight throughout, two blocks a CU fill in for each other, and
// finding the next tile takes no division.  Tiles of 256 x 128 in 32-deep slices read the
// least LDS an MFMA that two blocks a CU leave room for.  16384 rows over 60 experts (2048
// x 1408): 510 to 580 us (128 x 128 tiles, 64-deep, a block a tile 984, blocks that stay 680, in
// 32-deep slices 690; the large-group core 665 to 740); 8192 rows over 8 experts (4096 x
// 14336): 2.87 ms (1.0 PFLOP/s; the large-group core 2.98); 48 rows: 600 us, 2.8 GB written
// at 4.7 TB/s (the 128 x 128 tiles 818 to 1025).
struct WeightArgs {
  Groups groups;
  int n_prod;
  const bf16_t *A[3], *B[3];
  int M[3], N[3];
  bf16_t* out[3];
};

template <class C>
__global__ __launch_bounds__(256, C::T::OCC) void k_expert_weights(WeightArgs a) {
  using T = typename C::T;
  __shared__ __align__(16) char lds[T::LDS];
  int first[4] = {0, 0, 0, 0};
#pragma unroll
  for (int p = 0; p < 3; ++p)
    first[p + 1] = first[p] + (p < a.n_prod ? ((a.M[p] + T::BM - 1) / T::BM) * ((a.N[p] + T::BN - 1) / T::BN)
                                            : 0);
  const GroupOrder order(a.groups);
  GroupWalk walk(first[3], a.groups.E);
  C core(lds);
  TileQueue<5> queue;  // group, product, first column and row of the result, K
  const auto of = [](const auto (&v)[3], int p) { return p == 0 ? v[0] : p == 1 ? v[1] : v[2]; };
  int rank = -1, e = 0, r0 = 0, k = 0;  // the group of the tile before
  auto load = [&] {
    if (!walk.more()) return false;
    if (walk.rank != rank) {
      rank = walk.rank;
      e = order.group(rank);
      const int2 r = a.groups.rows(e);
      r0 = uniform(r.x);
      k = uniform(r.y) - r0;
    }
    int L = uniform(walk.tile());
    walk.next();
    const int p = L >= first[2] ? 2 : L >= first[1] ? 1 : 0;
    const int M = of(a.M, p), N = of(a.N, p);
    L -= p == 0 ? 0 : p == 1 ? first[1] : first[2];
    // patches of 8 column tiles of the result
    const int n_mt = (N + T::BN - 1) / T::BN, n_nt = (M + T::BM - 1) / T::BM;
    const int g = uniform((int)((unsigned)L / (unsigned)(8 * n_nt))), w = L - g * 8 * n_nt;
    const int gm = min(8, n_mt - 8 * g);
    const int nt = gm == 8 ? w >> 3 : uniform((int)((unsigned)w / (unsigned)gm));
    const int mt = 8 * g + w - nt * gm;
    const int m0 = uniform(nt * T::BM), n0 = uniform(mt * T::BN);
    queue.push({{e, p, m0, n0, k}});
    tile_along<T::BM, T::KS>(core.a, of(a.A, p) + (size_t)r0 * M, M, m0, k);
    tile_along<T::BN, T::KS>(core.b, of(a.B, p) + (size_t)r0 * N, N, n0, k);
    core.left = max((k + T::KS - 1) / T::KS, 1);
    return true;
  };
  core.first(load);
  for (bool stored = false; queue.n; stored = true) {
    const auto at = queue.pop();
    const int(&was)[5] = at.v;
    const int p = was[1], M = of(a.M, p), N = of(a.N, p), nk = max((was[4] + T::KS - 1) / T::KS, 1);
    typename C::Acc acc;
    if (stored)
      core.template run<STORES<C>>(nk, acc, load);
    else
      core.run(nk, acc, load);
    core.ahead(load);
    store_tile(core, acc, of(a.out, p) + (size_t)was[0] * M * N, was[3], N - was[3], was[2], M);
  }
  core.last();
}

// --------------------------------------------------------------- launching --
// How the rows are cut: kFew 32-row tiles (groups of up to that many rows on average, or
// too few larger tiles), kMid 128-row tiles, kLarge the large-group core's 256 (groups of
// `large` rows on average, and tiles for most CUs; fewer where their K can be cut).  cols:
// columns of the tiles' A side.  us, by the rows alone and so (d 2048, F 5632, forward
// and gradient): 64 rows 43 and 28, 71 and 50; 110 rows 45 and 35, 78 and 59; 1736 rows over
// 4 experts of 640 x 192: 35 and 19, 57 and 41; 959 over 2 of 448 x 3264: 85 and 30.
// 128-row tiles and the large-group core (kernels' us with equal loads; in pieces of K
// with their sum):
//   rows an expert           up, gate       y             dx            da
//   60 x (2048 x 1408)  100  217   255      87   102      165   177     107   164
//                       150  283   263      121  107      216   180     161   170
//                       200  293   289      126  110      223   189     167   184
//                       273  363   392      177  171      318   311     219   265
//                       400  434   395      218  183      379   327     289   283
//                       500  447   424      233  189      406   339     312   298
//   8 x (4096 x 14336)  200  592   555      274  251      535   426     350   305
//                       400  1022  827      476  371      953   733     606   566
//                       1024 2057  1625     1041 709      2015  1371    1275  1066
//   1 x (2048 x 5632)   600  39    57       32   54       46    70      37    72
//                       1000 68    61       41   67       61    81      46    75
//                       2047 118   126      74   82       107   113     88    87
//                       4000 226   190      101  112      185   175     154   174
// The limits lie where up and gate change over, and da.  What they cost: y and dx of 150 to
// 255 rows an expert up to a quarter, y and dx of one expert of 1000 rows 26 and 20 us, da
// of 4000 rows of one expert 20.
enum Rows { kFew, kMid, kLarge };
constexpr long kLargeTiles = 160, kLargeCutTiles = 32, kMidTiles = 192;
Rows rows_kind(const Groups& g, long large, int cols, bool cut) {
  const auto tiles = [&](int rows, int width) {
    return ((long)g.n / rows + std::min(g.E, g.n)) * cdiv(cols, width);
  };
  if ((long)g.n <= 32l * g.E) return kFew;
  if ((long)g.n >= large * g.E && tiles(256, 256) >= (cut ? kLargeCutTiles : kLargeTiles)) return kLarge;
  return tiles(128, 128) >= (cut ? kMidTiles / 8 : kMidTiles) ? kMid : kFew;
}
constexpr long kLargeRows = 256, kLargeDactRows = 512;

template <int KIND, bool ATR, bool PAIR = false>
using CoreOf = std::conditional_t<
    KIND == kLarge, BigCore<BigTile<ATR, PAIR>>,
    std::conditional_t<KIND == kMid, MidCore<MidTile<128, 128, 2, ATR, false, PAIR>>,
                       MidCore<MidTile<128, 32, 3, ATR, false, PAIR>>>>;

// pieces of K of small tiles of the rows' products (M columns, `slices` of K): as many as
// two blocks a CU take at once, of 8 slices at least
int row_splits(const Groups& g, int M, int slices) {
  const Rows kind = rows_kind(g, kLargeRows, M, slices >= kTailSlices);
  if (kind == kLarge) return 1;
  const int tile = kind == kFew ? 32 : 128;
  const long tiles = std::max(1l, ((long)g.n / tile + std::min(g.E, g.n)) * cdiv(M, 128));
  return (int)std::max(1l, std::min({512 / tiles, (long)slices / 8, 8l}));
}
// bytes of the pieces' sums
constexpr int kTailBlocks = 256;
size_t row_parts(const Groups& g, int M, int slices) {
  if (rows_kind(g, kLargeRows, M, slices >= kTailSlices) == kLarge)
    return slices < kTailSlices ? 0 : (size_t)kTailBlocks * big::BM * big::BN * 4;
  const int s = row_splits(g, M, slices);
  return s > 1 ? ffn_align((size_t)s * g.n * M * 4) : 0;
}

// f(integral constant of the kind)
template <typename F>
hipError_t with_kind(Rows kind, F f) {
  if (kind == kFew)
    f(std::integral_constant<int, kFew>());
  else if (kind == kMid)
    f(std::integral_constant<int, kMid>());
  else
    f(std::integral_constant<int, kLarge>());
  return hipGetLastError();
}

// blocks of a launch over at most `tiles` tiles: as many as the CUs hold
template <class C>
dim3 grid_of(long tiles, int n_cu) {
  return dim3((unsigned)std::min(std::max(tiles, 1l), (long)n_cu * C::T::OCC));
}
// ... over row tiles, which take long enough that the hardware deals them out: a block
// each (but on the large-group core, whose blocks load their next tile early).  60 experts of
// 2048 x 1408, 100 rows each: up and gate 217 to 229 us, with blocks that stay 233, dx 164 to
// 174 and 174; 273 rows each: da 222 and 229
template <class C>
dim3 rows_grid(const Groups& g, int cols, int n_cu) {
  const long tiles = row_tiles_most(g.n, g.E, C::T::BN) * cdiv(cols, C::T::ROWS_A);
  return C::T::OCC == 1 ? grid_of<C>(tiles, n_cu) : dim3((unsigned)std::min(tiles, 1l << 20));
}

template <bool GATED, int KEEP>
hipError_t launch_up(const UpArgs& a, int n_cu, hipStream_t st) {
  return with_kind(rows_kind(a.groups, kLargeRows, GATED ? 2 * a.F : a.F, false), [&](auto kind) {
    using C = CoreOf<kind, false, GATED>;
    hipLaunchKernelGGL((k_expert_up<C, GATED, KEEP>), rows_grid<C>(a.groups, a.F, n_cu), dim3(256), 0, st, a);
  });
}

template <bool ATR>
hipError_t launch_rows(RowsArgs a, char* part, int n_cu, hipStream_t st) {
  const int slices = a.K / BK * (a.w2 ? 2 : 1);
  const Rows kind = rows_kind(a.groups, kLargeRows, a.M, slices >= kTailSlices);
  a.splits = row_splits(a.groups, a.M, slices);
  a.part = reinterpret_cast<float*>(part);
  unsigned blocks = 0;
  hipError_t e = with_kind(kind, [&](auto kind) {
    using C = CoreOf<kind, ATR>;
    dim3 grid = rows_grid<C>(a.groups, a.M, n_cu);
    if (kind == kLarge)
      grid.x = std::min(n_cu, kTailBlocks);
    else
      grid.x = std::min(grid.x * a.splits, 1u << 20);
    blocks = grid.x;
    if (kind == kLarge || a.splits == 1)
      hipLaunchKernelGGL((k_expert_rows<C, false>), grid, dim3(256), 0, st, a);
    if (kind == kLarge ? slices >= kTailSlices : a.splits > 1)
      hipLaunchKernelGGL((k_expert_rows<C, true>), grid, dim3(256), 0, st, a);
  });
  if (e != hipSuccess) return e;
  const size_t n = (size_t)a.groups.n * a.M;
  if (kind == kLarge && slices >= kTailSlices)
    hipLaunchKernelGGL(k_join_tail, dim3(blocks, big::BN / kJoinRows), dim3(256), 0, st, a, slices);
  else if (kind != kLarge && a.splits > 1)
    hipLaunchKernelGGL(k_join_slices, dim3((unsigned)((n / 8 + 255) / 256)), dim3(256), 0, st, a.part,
                       a.splits, n, a.out);
  return hipGetLastError();
}

template <bool GATED, bool PACKED>
hipError_t launch_dact(const DactArgs& a, int n_cu, hipStream_t st) {
  return with_kind(rows_kind(a.groups, kLargeDactRows, a.F, false), [&](auto kind) {
    using C = CoreOf<kind, true>;
    hipLaunchKernelGGL((k_expert_dact<C, GATED, PACKED>), rows_grid<C>(a.groups, a.F, n_cu), dim3(256), 0, st,
                       a);
  });
}

hipError_t launch_weights(const WeightArgs& a, int n_cu, hipStream_t st) {
  using C = MidCore<MidTile<256, 128, 3, true, true, false, 32>>;
  long tiles = 0;
  for (int p = 0; p < a.n_prod; ++p) tiles += (long)cdiv(a.M[p], C::T::BM) * cdiv(a.N[p], C::T::BN);
  hipLaunchKernelGGL((k_expert_weights<C>), grid_of<C>(tiles * a.groups.E, n_cu), dim3(256), 0, st, a);
  return hipGetLastError();
}

const bf16_t* as_bf16(const void* p) { return static_cast<const bf16_t*>(p); }

}  // namespace

size_t expert_ffn_ws(bool bf16, bool gated, int keep, int E, int d, int F, int n) {
  const size_t act = ffn_array(n, F, bf16 ? 2 : 4);
  if (bf16) return act + row_parts(Groups{nullptr, E, n}, d, F / BK);
  // (fp32 pre-activations are packed by a launch of their own)
  return act + (keep == TRIMMOE_KEEP_PACKED ? (gated ? 2 : 1) * act : 0) +
         row_parts_f32(Groups{nullptr, E, n}, d, F);
}

size_t expert_ffn_backward_ws(bool bf16, bool gated, bool x_packed, int E, int d, int F, int n) {
  const int elem = bf16 ? 2 : 4;
  return (gated ? 3 : 2) * ffn_array(n, F, elem) + (x_packed ? ffn_array(n, d, elem) : 0) +
         (bf16 ? row_parts(Groups{nullptr, E, n}, d, F / BK * (gated ? 2 : 1))
               : row_parts_f32(Groups{nullptr, E, n}, d, (gated ? 2l : 1l) * F));
}

hipError_t launch_expert_ffn(const ExpertFfnArgs& a, hipStream_t st) {
  if (a.groups.n == 0) return hipSuccess;
  if (!a.bf16) return launch_expert_ffn_f32(a, st);
  UpArgs u{};
  u.groups = a.groups;
  u.w_up = as_bf16(a.w_up);
  u.w_gate = as_bf16(a.w_gate);
  u.x = as_bf16(a.x);
  u.d = a.d;
  u.F = a.F;
  u.a = reinterpret_cast<bf16_t*>(a.ws);
  u.up = a.up;
  u.gate = a.gate;
  u.up_scale = a.up_scale;
  u.gate_scale = a.gate_scale;
  hipError_t e;
  if (a.gated)
    e = a.keep == TRIMMOE_KEEP_FULL     ? launch_up<true, TRIMMOE_KEEP_FULL>(u, a.n_cu, st)
        : a.keep == TRIMMOE_KEEP_PACKED ? launch_up<true, TRIMMOE_KEEP_PACKED>(u, a.n_cu, st)
                                        : launch_up<true, TRIMMOE_KEEP_NONE>(u, a.n_cu, st);
  else
    e = a.keep == TRIMMOE_KEEP_FULL     ? launch_up<false, TRIMMOE_KEEP_FULL>(u, a.n_cu, st)
        : a.keep == TRIMMOE_KEEP_PACKED ? launch_up<false, TRIMMOE_KEEP_PACKED>(u, a.n_cu, st)
                                        : launch_up<false, TRIMMOE_KEEP_NONE>(u, a.n_cu, st);
  if (e != hipSuccess) return e;
  RowsArgs r{};
  r.groups = a.groups;
  r.w = as_bf16(a.w_down);
  r.b = u.a;
  r.M = a.d;
  r.K = a.F;
  r.out = static_cast<bf16_t*>(a.y);
  return launch_rows<false>(r, a.ws + ffn_array(a.groups.n, a.F, 2), a.n_cu, st);
}

hipError_t launch_expert_ffn_backward(const ExpertFfnArgs& a, hipStream_t st) {
  if (!a.bf16) return launch_expert_ffn_backward_f32(a, st);
  const int n = a.groups.n;
  const size_t act = ffn_array(n, a.F, 2);
  DactArgs t{};
  t.groups = a.groups;
  t.w_down = as_bf16(a.w_down);
  t.dy = as_bf16(a.dy);
  t.d = a.d;
  t.F = a.F;
  t.up = a.up;
  t.gate = a.gate;
  t.up_scale = a.up_scale;
  t.gate_scale = a.gate_scale;
  t.a = reinterpret_cast<bf16_t*>(a.ws);
  t.du = reinterpret_cast<bf16_t*>(a.ws + act);
  t.dg = a.gated ? reinterpret_cast<bf16_t*>(a.ws + 2 * act) : nullptr;
  hipError_t e = hipSuccess;
  const bf16_t* x = as_bf16(a.x);
  if (n > 0) {
    if (a.gated)
      e = a.keep == TRIMMOE_KEEP_PACKED ? launch_dact<true, true>(t, a.n_cu, st)
                                        : launch_dact<true, false>(t, a.n_cu, st);
    else
      e = a.keep == TRIMMOE_KEEP_PACKED ? launch_dact<false, true>(t, a.n_cu, st)
                                        : launch_dact<false, false>(t, a.n_cu, st);
    if (e != hipSuccess) return e;
    if (a.x_scale && (a.dw_up || a.dw_gate)) {
      bf16_t* to = reinterpret_cast<bf16_t*>(a.ws + (a.gated ? 3 : 2) * act);
      e = launch_checkpoint_unpack(true, n, a.d, static_cast<const int8_t*>(a.x), a.x_scale, to, st);
      if (e != hipSuccess) return e;
      x = to;
    }
    if (a.dx) {
      RowsArgs r{};
      r.groups = a.groups;
      r.w = as_bf16(a.w_up);
      r.w2 = a.gated ? as_bf16(a.w_gate) : nullptr;
      r.b = t.du;
      r.b2 = t.dg;
      r.M = a.d;
      r.K = a.F;
      r.out = static_cast<bf16_t*>(a.dx);
      char* part = a.ws + (a.gated ? 3 : 2) * act + (a.x_scale ? ffn_array(n, a.d, 2) : 0);
      if ((e = launch_rows<true>(r, part, a.n_cu, st)) != hipSuccess) return e;
    }
  }
  WeightArgs w{};
  w.groups = a.groups;
  const auto add = [&](const bf16_t* A, const bf16_t* B, int M, int N, void* out) {
    if (!out) return;
    const int p = w.n_prod++;
    w.A[p] = A;
    w.B[p] = B;
    w.M[p] = M;
    w.N[p] = N;
    w.out[p] = static_cast<bf16_t*>(out);
  };
  add(t.a, t.dy, a.F, a.d, a.dw_down);
  add(x, t.du, a.d, a.F, a.dw_up);
  if (a.gated) add(x, t.dg, a.d, a.F, a.dw_gate);
  if (w.n_prod == 0) return hipSuccess;
  return launch_weights(w, a.n_cu, st);
}

}  // namespace trimmoe
