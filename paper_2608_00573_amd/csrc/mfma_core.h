// The two bf16 matrix cores: the direct-to-LDS pipeline with its tile scheduling
// (also in fp32) and the large-group core.  Kernels add their operand rows and
// epilogues (gemm.hip, head_loss.hip).
#pragma once

#include "gemm.h"

namespace trimmoe {

constexpr int BK = kGemmBK;  // 64 bf16 = one 128-byte row segment
constexpr int kPatch = 8;    // M-tiles per patch column in the tile order
constexpr int kXcd = 8;      // XCDs of an MI355X; blocks are dealt round-robin

static_assert(BK == 64, "the LDS layout assumes 128-byte row segments");

// ------------------------------------------------------------ tile shapes --
// BM x BN block tile, NB B operands sharing A, GM x GN wavefronts.  F32: the
// operands are fp32, seen as pairs of 2-byte words (K and strides count words).
template <int BM_, int BN_, int NB_, int GM_, int GN_, bool F32_ = false>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, NB = NB_, GM = GM_, GN = GN_;
  static constexpr bool F32 = F32_;
  static constexpr int THREADS = 64 * GM * GN;
  static constexpr int WM = BM / GM, WN = BN / GN;  // wavefront tile
  static constexpr int TM = WM / 32, TN = WN / 32;  // MFMA tiles per wavefront
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
  static constexpr int STAGE = A_BYTES + NB * B_BYTES;
  static constexpr int ROWS_PER_PASS = THREADS / 8;  // 8 threads per 128-byte row
  static constexpr int A_PT = BM / ROWS_PER_PASS, B_PT = BN / ROWS_PER_PASS;
  static_assert(WM % 32 == 0 && WN % 32 == 0, "wavefront tile");
  static_assert(BM % ROWS_PER_PASS == 0 && BN % ROWS_PER_PASS == 0, "load passes");
};

// accumulator element -> tile-local (row, col)
template <class T>
__device__ __forceinline__ int acc_row(int wm, int i, int r, int lane) {
  return wm * T::WM + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
}
template <class T>
__device__ __forceinline__ int acc_col(int wn, int j, int lane) {
  return wn * T::WN + j * 32 + (lane & 31);
}

// ------------------------------------------------ direct-to-LDS pipeline --
// gfx950's global_load_lds_dwordx4 moves a wavefront's 64 x 16 bytes from
// global memory straight into LDS at a wave-uniform base (lane l at base +
// 16 l): no staging VGPRs and no ds_write (the two things a register-staged
// operand path spends most of its non-MFMA issue time on).  Three LDS stages
// form a ring: slice g+2 is in flight while slice g is computed and slice
// g+1 has landed.  Lane l of the DMA that covers tile rows r..r+7 loads row
// r + l/8, chunk (l % 8) ^ swz16(row), so the LDS image is the same swizzled
// layout the fragment reads expect.
//
// Waits are explicit.  The compiler cannot tell that a DMA into one stage
// does not alias a read of another, and would wait for every outstanding DMA
// before each fragment read; the fragment reads are therefore inline-asm
// ds_read_b128, and
//   * lgkm_wait<N> (s_waitcnt lgkmcnt(N)) takes the fragments as in/out
//     operands, so the MFMAs that use them cannot be scheduled above it;
//   * slice_barrier<N> (s_waitcnt vmcnt(N) lgkmcnt(0); s_barrier) ends a
//     slice: this wave's DMAs older than the last N have landed and its
//     fragment reads are done, and after the barrier the same holds for all
//     waves, so the next stage may be read and the oldest one rewritten.
// Only LDS DMAs and rare stores are outstanding vector-memory operations in
// these loops; extra newer operations only make a vmcnt wait stricter.
__device__ __forceinline__ void dma16(const bf16_t* g, char* l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(g),
                                   (lds_byte*)(l), 16, 0, 0);
}

__device__ __forceinline__ bf16x8_t lds_read(uint32_t a) {
  bf16x8_t v;
  asm volatile("ds_read_b128 %0, %1" : "=v"(v) : "v"(a));
  return v;
}

// one k-step's fragments of a wavefront: TM A fragments (rows +32 i) and
// TN * NB B fragments (operand o, columns +32 j at index o * TN + j)
template <class T>
struct Frags {
  bf16x8_t a[T::TM];
  bf16x8_t b[T::TN * T::NB];
};

// ties every fragment register to the asm statement just before it (volatile
// asm keeps its order), so no MFMA reading one is scheduled above that wait
template <class T>
__device__ __forceinline__ void frags_after(Frags<T>& f) {
#pragma unroll
  for (int i = 0; i < T::TM; ++i) asm volatile("" : "+v"(f.a[i]));
#pragma unroll
  for (int j = 0; j < T::TN * T::NB; ++j) asm volatile("" : "+v"(f.b[j]));
}

template <int N, class T>
__device__ __forceinline__ void lgkm_wait(Frags<T>& f) {
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N));
  frags_after(f);
}

template <int N, class T>
__device__ __forceinline__ void slice_barrier(Frags<T>& f) {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
  frags_after(f);
}

// Ring depth: three stages (two slices in flight ahead of the one being
// computed) when they fit next to 8 KB of epilogue scratch, else two.
template <class T>
struct DmaTile {
  static constexpr int NF = T::TM + T::TN * T::NB;        // fragment reads per k-step
  static constexpr int NDMA = T::A_PT + T::B_PT * T::NB;  // DMAs per thread per slice
  static constexpr int STAGES = 3 * T::STAGE + 8 * 1024 <= 160 * 1024 ? 3 : 2;
  static constexpr int DEPTH = STAGES - 1;                // slices issued ahead
  static constexpr int LDS = STAGES * T::STAGE;
  static_assert(LDS + 8 * 1024 <= 160 * 1024, "stages plus epilogue scratch");
  static_assert(NF <= 15 && NDMA * (DEPTH - 1) <= 63, "waitcnt fields");
};

// per-lane global sources of one tile: A rows, then B0 rows (then B1 rows)
template <class T>
struct DPtrs {
  const bf16_t* a[T::A_PT];
  const bf16_t* b[T::B_PT * T::NB];
};

// tile row a thread's i-th A / B DMA covers, and the 16-byte chunk it loads
__device__ __forceinline__ int dma_row(int i, int rows_per_pass) {
  return ((int)threadIdx.x >> 3) + rows_per_pass * i;
}
__device__ __forceinline__ int dma_col(int row) { return 8 * (((int)threadIdx.x & 7) ^ swz16(row)); }

// A rows a_src[i] (matrix rows, already clamped) of A; B rows b_row0 + r,
// r clamped to b_valid - 1, of B0 (and B1); K columns from k_begin
template <class T>
__device__ __forceinline__ void make_dptrs(DPtrs<T>& q, const bf16_t* A, const int (&a_src)[T::A_PT],
                                           const bf16_t* B0, const bf16_t* B1, int b_row0,
                                           int b_valid, int K, int k_begin) {
#pragma unroll
  for (int i = 0; i < T::A_PT; ++i) {
    const int row = dma_row(i, T::ROWS_PER_PASS);
    q.a[i] = A + (size_t)a_src[i] * K + k_begin + dma_col(row);
  }
#pragma unroll
  for (int i = 0; i < T::B_PT; ++i) {
    const int row = dma_row(i, T::ROWS_PER_PASS);
    const size_t off = (size_t)(b_row0 + min(row, b_valid - 1)) * K + k_begin + dma_col(row);
    q.b[i] = B0 + off;
    if constexpr (T::NB == 2) q.b[T::B_PT + i] = B1 + off;
  }
}

// DMA slice kt of the tile into stage st
template <class T>
__device__ __forceinline__ void dma_slice(char* st, const DPtrs<T>& q, int kt) {
  const int w = threadIdx.x >> 6;
  const int o = kt * BK;
#pragma unroll
  for (int i = 0; i < T::A_PT; ++i) dma16(q.a[i] + o, st + (T::ROWS_PER_PASS * i + 8 * w) * 128);
#pragma unroll
  for (int i = 0; i < T::B_PT * T::NB; ++i)
    dma16(q.b[i] + o, st + T::A_BYTES + (i / T::B_PT) * T::B_BYTES +
                          (T::ROWS_PER_PASS * (i % T::B_PT) + 8 * w) * 128);
}

// per-lane LDS offsets of a wavefront's fragments within a stage
template <class T>
struct FragAddr {
  uint32_t a, b, ch[4];
  __device__ __forceinline__ FragAddr(int wm, int wn, int lane) {
    const int fr = lane & 31, hi = lane >> 5;
    a = (wm * T::WM + fr) * 128;
    b = T::A_BYTES + (wn * T::WN + fr) * 128;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) ch[ks] = ((2 * ks + hi) ^ swz16(fr)) << 4;
  }
  __device__ __forceinline__ void read(Frags<T>& f, uint32_t stage, int ks) const {
    const uint32_t pa = stage + a + ch[ks], pb = stage + b + ch[ks];
#pragma unroll
    for (int i = 0; i < T::TM; ++i) f.a[i] = lds_read(pa + i * 32 * 128);
#pragma unroll
    for (int o = 0; o < T::NB; ++o)
#pragma unroll
      for (int j = 0; j < T::TN; ++j) f.b[o * T::TN + j] = lds_read(pb + o * T::B_BYTES + j * 32 * 128);
  }
};

template <class T>
using Acc = f32x16_t[T::TM][T::TN * T::NB];

// acc[i][j] += A_i B_j^T for the k-step held in f.  fp32: the lane's 16 bytes
// are four consecutive K of its row; the two half-wavefronts hold neighbouring
// fours, so MFMA u multiplies K u and 4 + u of the k-step's eight
template <class T>
__device__ __forceinline__ void mma_step(const Frags<T>& f, Acc<T>& acc) {
  if constexpr (T::F32) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int j = 0; j < T::TN * T::NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(f32x4_t, f.a[i])[u],
                                                           __builtin_bit_cast(f32x4_t, f.b[j])[u],
                                                           acc[i][j], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int j = 0; j < T::TN * T::NB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  }
}

// One slice from stage cur (its k-step-0 fragments already in f0), with the
// next slice's k-step-0 fragments read from stage nxt under the last
// k-step's MFMAs.  `issue` starts the DMA of the slice DEPTH ahead; the
// barrier waits for the DMAs of the next slice only.
template <class T, class Issue>
__device__ __forceinline__ void dma_slice_mma(const FragAddr<T>& fa, uint32_t cur, uint32_t nxt,
                                              Frags<T>& f0, Frags<T>& f1, Acc<T>& acc,
                                              Issue issue) {
  using D = DmaTile<T>;
  issue();
  fa.read(f1, cur, 1);
  lgkm_wait<D::NF>(f0);
  mma_step<T>(f0, acc);
  fa.read(f0, cur, 2);
  lgkm_wait<D::NF>(f1);
  mma_step<T>(f1, acc);
  fa.read(f1, cur, 3);
  lgkm_wait<D::NF>(f0);
  mma_step<T>(f0, acc);
  slice_barrier<D::NDMA * (D::DEPTH - 1)>(f1);
  fa.read(f0, nxt, 0);
  mma_step<T>(f1, acc);
}

// ------------------------------------------------------- tile scheduling --
// Persistent grids: one block per CU (or fewer).  The live tiles (a count
// known only on the device) are split into contiguous ranges, one per XCD
// (hardware deals block b to XCD b % 8); block b walks tiles tb + i0,
// tb + i0 + bx, ... of its XCD's range (bx = blocks on that XCD), so the
// blocks of an XCD work on consecutive tiles and share its L2.  A tile index
// is read in patch order: kPatch M-tiles of one N-tile, then the next
// N-tile; the K split (if any) is the slowest index.
struct TileSched {
  int tb, i0, bx, n_mt, n_nt;
  // false when this block has no tile, else its tile count in ntiles
  __device__ __forceinline__ bool init(int n_mt_, int n_nt_, int n_split, int& ntiles) {
    return init_total(n_mt_ * n_nt_ * n_split, n_mt_, n_nt_, ntiles);
  }
  // the first `total` tile indices only
  __device__ __forceinline__ bool init_total(int total, int n_mt_, int n_nt_, int& ntiles) {
    n_mt = n_mt_;
    n_nt = n_nt_;
    const int nx = min(kXcd, (int)gridDim.x);  // fewer groups for a small grid
    const int x = blockIdx.x % nx;
    i0 = blockIdx.x / nx;
    bx = ((int)gridDim.x - x + nx - 1) / nx;
    const int q = total / nx, r = total % nx;
    tb = x * q + min(x, r);
    const int te = tb + q + (x < r ? 1 : 0);
    if (tb + i0 >= te) return false;
    ntiles = (te - (tb + i0) + bx - 1) / bx;
    return true;
  }
  __device__ __forceinline__ void decode(int j, int& mt, int& nt, int& sp) const {
    decode_abs(tb + i0 + j * bx, mt, nt, sp);
  }
  // tile index L of the whole patch order
  __device__ __forceinline__ void decode_abs(int L, int& mt, int& nt, int& sp) const {
    const int per = n_mt * n_nt;
    sp = L / per;
    L -= sp * per;
    const int span = kPatch * n_nt;
    const int g = L / span, w = L % span;
    const int gm = min(kPatch, n_mt - g * kPatch);
    nt = w / gm;
    mt = g * kPatch + w % gm;
  }
};

// The tiles from index `from` on as pieces of half their columns: piece q is
// half q % 2 of tile from + q / 2, and nt counts half-width column tiles
struct HalfSched {
  TileSched S;
  int from;
  __device__ __forceinline__ bool init(int from_, int n_mt, int n_nt, int& ntiles) {
    from = from_;
    return S.init_total(2 * (n_mt * n_nt - from), n_mt, n_nt, ntiles);
  }
  __device__ __forceinline__ void decode(int j, int& mt, int& nt, int& sp) const {
    const int q = S.tb + S.i0 + j * S.bx;
    S.decode_abs(from + (q >> 1), mt, nt, sp);
    nt = 2 * nt + (q & 1);
  }
};

// A persistent block's GEMM over its ntiles tiles of nk slices each: one
// continuous stream of K slices through the DMA ring, so the next tile's
// first slices are in flight while the current tile's epilogue runs.
// Src supplies, for tile j of the block:
//   Desc desc(int j)                      descriptor (may load from memory);
//                                         Desc::pick(c, x, y) = c ? x : y
//   void rows(const Desc&, int (&)[A_PT]) per-thread A source rows (may load)
//   void ptrs(DPtrs<T>&, const Desc&, const int (&)[A_PT])
//   void epilogue(const Desc&, Acc<T>&)
// Descriptors are loaded two tiles and rows one tile ahead of their use, so
// the compiler's load-count waits for them never drain the DMA ring.
template <class T, class Src>
__device__ __forceinline__ void dma_gemm_stream(char* lds, int ntiles, int nk, const Src& src) {
  using Desc = typename Src::Desc;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const FragAddr<T> fa(wave / T::GN, wave % T::GN, lane);
  const uint32_t st0 = lds_addr(lds);
  using D = DmaTile<T>;
  Acc<T> acc;
  const f32x16_t z = {};
  auto zero = [&] {
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int j = 0; j < T::TN * T::NB; ++j) acc[i][j] = z;
  };
  zero();

  // DMA side: slice dk of tile dj through pointers qp; n1 / n2 describe
  // tiles dj+1 / dj+2 and rn1 holds the A rows of dj+1
  // start-up: the three descriptor loads go out together, and the first
  // slice's DMA right after tile 0's rows, before tile 1's rows are needed
  const int last = ntiles - 1;
  DPtrs<T> qp;
  int rows[T::A_PT], rn1[T::A_PT];
  Desc c0 = src.desc(0);
  Desc n1 = src.desc(min(1, last));
  Desc n2 = src.desc(min(2, last));
  src.rows(c0, rows);
  src.ptrs(qp, c0, rows);
  int dj = 0, dk = 0;
  // compute side: c0 describes tile jc; c1 / c2 tiles jc+1 / jc+2 once the
  // DMA side has entered them (it runs at most DEPTH <= 2 slices ahead)
  Desc c1 = n1, c2 = n2;
  int jc = 0;
  // the DMA side enters a tile when it issues the tile's first slice, at
  // most DEPTH <= 2 slices ahead of the compute side, so dj - jc is 1 or 2
  auto issue = [&](int stage) {
    if (dk == nk) {
      if (dj == last) {  // past the end: the last slice again (in bounds, never read)
        dk = nk - 1;
      } else {
        ++dj;
        dk = 0;
        src.ptrs(qp, n1, rn1);
        const bool next = dj == jc + 1;  // field-wise selects: no indexed copy
        c1 = Desc::pick(next, n1, c1);
        c2 = Desc::pick(next, c2, n1);
        src.rows(n2, rn1);
        n1 = n2;
        n2 = src.desc(min(dj + 2, last));
      }
    }
    dma_slice<T>(lds + stage * T::STAGE, qp, dk);
    ++dk;
  };

  Frags<T> f0, f1;
  issue(0);
  src.rows(n1, rn1);  // first needed when the stream enters tile 1
#pragma unroll
  for (int s = 1; s < D::DEPTH; ++s) issue(s);
  slice_barrier<D::NDMA * (D::DEPTH - 1)>(f1);
  fa.read(f0, st0, 0);
  const int G = ntiles * nk;
  int sx = 0, kk = 0;  // stage of the slice being computed, its index in the tile
  for (int g = 0; g < G; ++g) {
    const int sn = sx + 1 == D::STAGES ? 0 : sx + 1;
    const int sp = (sx + D::DEPTH) % D::STAGES;  // stage of slice g + DEPTH
    dma_slice_mma<T>(fa, st0 + sx * T::STAGE, st0 + sn * T::STAGE, f0, f1, acc,
                     [&] { issue(sp); });
    if (++kk == nk) {
      src.epilogue(c0, acc);
      zero();
      c0 = c1;
      c1 = c2;
      ++jc;
      kk = 0;
    }
    sx = sn;
  }
}

// ------------------------------------------ large-group expert GEMMs --
// Expert groups of prefill batches (about a thousand rows or more per expert),
// the dense shared expert of large batches and the exit head of wide models
// (k_exit_big, below) use a second core with 256 x 256 block tiles and 4
// wavefronts, one per SIMD, each owning a 128 x 128 output patch: 8 x 8
// accumulators of 16 x 16 in AGPRs, multiplied in v_mfma_f32_16x16x32_bf16.
// A k-step of 32 reads 16 fragments for 64 MFMAs (half the LDS bytes per
// MFMA of the 64 x 64 patches) and a 64-wide K slice moves 64 KB for
// 256 x 256 outputs (2/3 of the bytes per MFMA of the 128 x 256 block).  The
// chip does not hold its peak clock under a dense MFMA load, and the
// 16 x 16 x 32 form keeps a higher one than 32 x 32 x 16 at nearly the same
// share of the cycles (a loop of MFMAs alone: about 2.1 GHz against 1.8),
// which is why this core uses it.  With one wavefront per SIMD no other
// wavefront fills the MFMA pipe while this one waits, so the instruction
// stream is laid out explicitly (sched_barrier keeps the compiler from
// regrouping it; the MFMAs are inline asm on AGPR operands, so the register
// allocator cannot move accumulators inside the loop):
//   * a k-step issues its 64 MFMAs row by row (tile (i, j) = (T / 8, T % 8)).
//     The next k-step's B fragments go to a second register set, read one
//     after each of the first 8 MFMAs; its a_i replaces this k-step's a_i
//     right after that fragment's last MFMA (8 i + 7), so A needs one set.
//     Each MFMA waits for its own fragments with a partial lgkmcnt;
//   * both operands go straight to LDS through buffer-to-LDS DMAs (a
//     wavefront's 64 x 16 bytes land at a wave-uniform base; 32-bit row
//     offsets, the K position in the scalar offset), so no VGPRs and no
//     ds_write are spent on them.  A (the gathered activations) has two
//     32 KB stages and B (the weights) a ring of three.  During slice g the
//     first k-step brings the second half of A of slice g + 1, the last
//     k-step (after the barrier, into the A stage slice g leaves) the first
//     half of A of slice g + 2, and both bring B of slice g + 2: 16 DMAs per
//     thread spread over the slice, since a DMA of a whole 64 KB slice at
//     once asks the texture path for about 128 B/clk per CU against the
//     ~50 B/clk it sustains, and its stalls land on the MFMA issue;
//   * one barrier per slice, before MFMA 32 of the last k-step: it waits for
//     this slice's reads and every DMA of slice g + 1, and the next slice's
//     first fragments are read after it, one after each following MFMA.
// Blocks are persistent and walk their XCD's contiguous tile range as the
// other core does; each tile runs its own prologue and epilogue.
namespace big {
constexpr int BM = 256, BN = 256, THREADS = 256;
constexpr int RB = 128;                  // bytes of a row segment (64 bf16)
constexpr int AB = BM * RB;              // A rows of a slice (32 KB)
constexpr int BB = BN * RB;              // B rows of a slice (32 KB)
constexpr int BS = 3;                    // B stages (DMA ring)
constexpr int B0 = 2 * AB;               // first B stage, after the two A stages
constexpr int LDS = 2 * AB + BS * BB;    // 160 KB
constexpr int RPP = THREADS / 8;         // rows per fetch pass (8 threads per 128-byte row)
}  // namespace big

// a wavefront's fragments of one 32-wide k-step: A rows +16 i, B columns +16 j
struct FragA {
  bf16x8_t a[8];
};
struct FragB {
  bf16x8_t b[8];
};
// its 128 x 128 patch: 8 x 8 accumulators of 16 x 16 (lane: column l % 16,
// rows 4 (l / 16) .. + 4)
using AccBig = f32x4_t[8][8];

__device__ __forceinline__ void sched_fence() { __builtin_amdgcn_sched_barrier(0); }

template <int N>
__device__ __forceinline__ void lgkm_le() {
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N));
}

// fragment read with a constant byte offset from a per-lane LDS address
template <int OFF>
__device__ __forceinline__ bf16x8_t lds_read_at(uint32_t a) {
  bf16x8_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(a), "n"(OFF));
  return v;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buf_rsrc(const void* p) {
  // raw buffer, no range limit: every offset is clamped to a valid row first
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)0xffffffff,
                                           0x00020000);
}

// a buffer of no records: every load from it returns zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buf_rsrc_empty(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, 0, 0x00020000);
}

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// A 32-wide k-step issues its 64 MFMAs row by row (tile (i, j) = (T / 8,
// T % 8)): a_i is last used by MFMA 8 i + 7, so the next k-step's a_i is read
// into the same registers right after it, while the b fragments alternate
// between two sets.  Per MFMA slot T: the fragment read after it (q = 2 n for
// a_n, 2 n + 1 for b_n; -1: none; the first k-step also reads the next a_0
// after MFMA 7), for the first k-step of a slice (0) and the last (1: its
// reads, of the next slice, follow the slice barrier before MFMA 32).
constexpr int kRead0[64] = {
     1,  3,  5,  7,  9, 11, 13, 15,  // MFMAs 0..7
    -1, -1, -1, -1, -1, -1, -1,  2,  // MFMAs 8..15
    -1, -1, -1, -1, -1, -1, -1,  4,  // MFMAs 16..23
    -1, -1, -1, -1, -1, -1, -1,  6,  // MFMAs 24..31
    -1, -1, -1, -1, -1, -1, -1,  8,  // MFMAs 32..39
    -1, -1, -1, -1, -1, -1, -1, 10,  // MFMAs 40..47
    -1, -1, -1, -1, -1, -1, -1, 12,  // MFMAs 48..55
    -1, -1, -1, -1, -1, -1, -1, 14   // MFMAs 56..63
};
constexpr int kRead1[64] = {
    -1, -1, -1, -1, -1, -1, -1, -1,  // MFMAs 0..7
    -1, -1, -1, -1, -1, -1, -1, -1,  // MFMAs 8..15
    -1, -1, -1, -1, -1, -1, -1, -1,  // MFMAs 16..23
    -1, -1, -1, -1, -1, -1, -1, -1,  // MFMAs 24..31
     0,  1,  2,  3,  4,  5,  6,  7,  // MFMAs 32..39
     8,  9, -1, 11, -1, 13, -1, 15,  // MFMAs 40..47
    10, -1, -1, -1, -1, -1, -1, -1,  // MFMAs 48..55
    12, -1, -1, -1, -1, -1, -1, 14   // MFMAs 56..63
};

// The lgkmcnt wait before each MFMA slot (-1: none): the LDS operations issued
// after the ones the slot needs, at most the counter's 15 (which only waits
// longer), where an earlier wait has not shown them landed.  The first k-step
// waits on the last k-step's read order and the last on the first's.  A
// fragment that is read transposed (BigRowsT) takes two operations.
struct BigWaits {
  int w[2][64];
};
constexpr BigWaits big_waits(bool atr, bool btr) {
  BigWaits out{};
  const int ops_a = atr ? 2 : 1, ops_b = btr ? 2 : 1;
  int end[2][16] = {};  // per k-step: operations issued up to the end of read q
  int issued = 0, landed = 0;
  for (int t = 0; t < 64; ++t)  // what is in flight when a slice begins
    if (kRead1[t] >= 0) {
      issued += kRead1[t] & 1 ? ops_b : ops_a;
      end[0][kRead1[t]] = issued;
    }
  for (int ks = 0; ks < 2; ++ks)
    for (int t = 0; t < 64; ++t) {
      if (ks == 1 && t == 32) landed = issued;  // the slice barrier
      const int ea = end[ks][2 * (t / 8)], eb = end[ks][2 * (t % 8) + 1];
      const int need = ea > eb ? ea : eb;
      out.w[ks][t] = -1;
      if (need > landed) {
        const int n = issued - need < 15 ? issued - need : 15;
        out.w[ks][t] = n;
        landed = issued - n;
      }
      const int q = ks ? kRead1[t] : kRead0[t];
      if (q >= 0) {
        issued += q & 1 ? ops_b : ops_a;
        end[1 - ks][q] = issued;
      }
      if (ks == 0 && t == 7) {
        issued += ops_a;
        end[1][0] = issued;
      }
    }
  return out;
}

// B fragment j of a wavefront: LDS row offset from its first B row.  DUAL:
// columns j = 0..3 of the up operand (rows 0..127 of the B stage), j = 4..7
// the same columns of the gate operand (rows 128..255).
template <bool DUAL>
constexpr int big_brow(int j) {
  return DUAL ? (j < 4 ? 16 * j : 128 + 16 * (j - 4)) : 16 * j;
}

// Transposed fragment read, of an operand that lies row by row along K: a slice
// is 64 rows (K) of 256 columns, 512 bytes each.  ds_read_b64_tr_b16 gives lane
// l of each 16 the 4 rows of column l out of what the 16 lanes address (lane i:
// 4 columns from 4 (i % 4) of row i / 4), so two of them, 4 rows apart, fill a
// fragment.  The 32-byte pieces of a row sit at piece n ^ (k % 4 + 4 (k / 8 % 2)):
// the rows that 32 lanes read together touch distinct banks, and fragment n's
// address is the lane's base ^ 32 n.
__device__ __forceinline__ bf16x8_t lds_read_tr(uint32_t a) {
  typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
  u32x2_t lo, hi;
  asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(lo) : "v"(a));
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:2048" : "=v"(hi) : "v"(a));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3));
}
// piece of a transposed operand's row k
__device__ __forceinline__ int tr_swz(int k) { return (k & 3) | ((k >> 3 & 1) << 2); }

// fragment read Q of a k-step: a_{Q/2} for even Q, b_{Q/2} for odd Q
template <bool DUAL, bool ATR, bool BTR, int Q>
__device__ __forceinline__ void big_read(FragA& fa, FragB& fb, uint32_t pa, uint32_t pb) {
  if constexpr (Q >= 0) {
    constexpr int n = Q >> 1;
    if constexpr (Q & 1) {
      if constexpr (BTR)
        fb.b[n] = lds_read_tr(pb ^ (n << 5));
      else
        fb.b[n] = lds_read_at<big_brow<DUAL>(n) * big::RB>(pb);
    } else {
      if constexpr (ATR)
        fa.a[n] = lds_read_tr(pa ^ (n << 5));
      else
        fa.a[n] = lds_read_at<n * 16 * big::RB>(pa);
    }
    sched_fence();
  }
}

// Per-thread operand rows of one tile: row u < 8 is A row r0 + 32 u (gathered,
// clamped), u >= 8 B row r0 + 32 (u - 8) (clamped to the valid columns); byte
// offsets of the thread's 16-byte chunk within their buffers at K = k0
struct BigRows {
  static constexpr bool ATR = false, BTR = false;
  __amdgpu_buffer_rsrc_t ra, rb0, rb1, none;
  uint32_t off[16];
};

// the buffers one slice is fetched from: a slice past the last one reads the
// empty buffer, so it lands as zeros and adds nothing
struct BigSrc {
  __amdgpu_buffer_rsrc_t ra, rb0, rb1;
  uint32_t ko;
  __device__ __forceinline__ BigSrc(const BigRows& q, int kt, int nk) {
    const bool live = kt < nk;
    ra = live ? q.ra : q.none;
    rb0 = live ? q.rb0 : q.none;
    rb1 = live ? q.rb1 : q.none;
    ko = live ? kt * big::RB : 0;
  }
};

// The operands of a tile as the head loss's products use the core: each
// K-contiguous, its K in one run or in panels of 256 (4 slices), or row by row
// along K (TR: fetched 64 rows a slice, read transposed; the buffer starts at the
// slice's first row, so its offsets stay within one slice, and ends with the
// operand, whose missing rows land as zeros).  The sources of the slice two ahead
// are made ready between the MFMAs of the slice before it, in a few scalar steps
// (a wavefront alone on its SIMD leaves the matrix pipe idle for every other
// instruction that it issues in a row).
template <bool TR>
struct BigOperand {
  const char* p;    // TR: the slice's first row; else the operand's first row at K = 0
  uint32_t off[8];  // of the thread's fetches
  int left;         // TR: rows from the slice on; else slices
  uint32_t row;     // TR: bytes of a row
  uint32_t cut;     // TR: bytes of a row before the tile's columns
  uint32_t ko;      // not TR: K offset of the slice
  uint32_t panel;   // not TR: bytes from the end of a panel's row to the next panel's
  uint32_t bytes;   // the buffer's
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc() const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, (int)bytes, 0x00020000);
  }
  __device__ __forceinline__ void limit() {
    if constexpr (TR) {
      const int n = min(left, 64);
      bytes = n > 0 ? (uint32_t)n * row - cut : 0;
    } else {
      // (the compiler selects all ones or zero in a vector register, which would turn
      // every fetch into a loop over lanes)
      bytes = __builtin_amdgcn_readfirstlane(left > 0 ? 0xffffffffu : 0);
    }
  }
  // to the next slice, in two steps
  __device__ __forceinline__ void step() {
    if constexpr (TR) {
      p += (size_t)row * 64;
      left -= 64;
    } else {
      left -= 1;
      ko += big::RB;
      ko += ko & 511 ? 0 : panel;
    }
  }
};
template <bool ATR_, bool BTR_>
struct BigFeed {
  static constexpr bool ATR = ATR_, BTR = BTR_;
  BigOperand<ATR> a;  // two slices ahead of the one computed; a1: one ahead
  BigOperand<BTR> b;
  __amdgpu_buffer_rsrc_t a1, a2, b2;
  uint32_t k1, k2, kb;
  __device__ __forceinline__ void take_a() {
    a2 = a.rsrc();
    k2 = ATR ? 0 : a.ko;
  }
  __device__ __forceinline__ void take_b() {
    b2 = b.rsrc();
    kb = BTR ? 0 : b.ko;
  }
  // what slot T of a slice's first k-step does for the next ones
  template <int T>
  __device__ __forceinline__ void slot() {
    if constexpr (T == 8) {
      a1 = a2;
      k1 = k2;
    } else if constexpr (T == 9) {
      a.step();
    } else if constexpr (T == 10) {
      a.limit();
    } else if constexpr (T == 11) {
      take_a();
    } else if constexpr (T == 12) {
      b.step();
    } else if constexpr (T == 13) {
      b.limit();
    } else if constexpr (T == 14) {
      take_b();
    }
    if constexpr (T >= 8 && T <= 14) sched_fence();
  }
};

// Row group u (0..7) of the wave straight into an LDS stage: lane l lands at
// stage + (8 w + 32 u) * 128 + 16 l, which is row 8 w + 32 u + l / 8, chunk slot
// l % 8 (the thread's fetch chunk is the swizzled one)
__device__ __forceinline__ void big_dma_group(uint32_t stage, int wave, __amdgpu_buffer_rsrc_t rs,
                                              uint32_t off, uint32_t ko, int u) {
  const uint32_t dst = stage + (uint32_t)((8 * wave + big::RPP * u) * big::RB);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_byte*)(uintptr_t)dst, 16, off, ko, 0, 0);
}
template <bool DUAL, class R, class Src>
__device__ __forceinline__ void big_dma(uint32_t bst, int wave, const R& q, const Src& b, int u) {
  if constexpr (DUAL)
    big_dma_group(bst, wave, u >= 4 ? b.rb1 : b.rb0, q.off[8 + u], b.ko, u);
  else
    big_dma_group(bst, wave, b.rb0, q.off[8 + u], b.ko, u);
}
template <class R, class Src>
__device__ __forceinline__ void big_dma_a(uint32_t ast, int wave, const R& q, const Src& b, int u) {
  big_dma_group(ast, wave, b.ra, q.off[u], b.ko, u);
}

struct BigNoFeed {
  template <int T>
  __device__ __forceinline__ void slot() {}
};

// MFMA slot T of a k-step (LAST: the second of the slice) from fragments fa,
// fb, with the next k-step's reads into fa (rotating) and fn: the wait, the
// MFMA, the reads; in the first k-step the A DMAs of the next slice (rows
// 4..7 of each thread) after MFMAs 16, 20, 24, 28; in the last the slice
// barrier before MFMA 32 and the A DMAs of the slice after next (rows 0..3,
// into the A stage this slice leaves) after MFMAs 32, 36, 40, 44; in both
// the B DMAs of the slice after next after MFMAs 18, 26, 50, 58 (rows 0..3
// in the first, 4..7 in the last).  The barrier waits for the next slice's
// A DMAs (the last issued at MFMA 28 of the first k-step, followed by 4 B
// DMAs) and its B DMAs (issued a slice earlier).
template <int T, bool LAST, bool DUAL, class R, class DmaA, class DmaB, class Feed>
__device__ __forceinline__ void big_slot(FragA& fa, FragB& fb, FragB& fn, AccBig& acc,
                                         uint32_t pa, uint32_t pb, DmaA& dma_a, DmaB& dma_b,
                                         Feed& feed) {
  constexpr int i = T / 8, j = T % 8;
  constexpr int w = big_waits(R::ATR, R::BTR).w[LAST ? 1 : 0][T];
  if constexpr (w >= 0) {
    lgkm_le<w>();
    asm volatile("" : "+v"(fa.a[i]), "+v"(fb.b[j]));
    sched_fence();
  }
  if constexpr (LAST && T == 32) {
    asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    asm volatile("" : "+v"(fa.a[i]), "+v"(fb.b[j]));
    sched_fence();
  }
  // the accumulators stay in AGPRs (with the builtin the allocator moved some
  // through VGPRs inside the loop)
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
               : "+a"(acc[i][j])
               : "v"(fa.a[i]), "v"(fb.b[j]));
  sched_fence();
  big_read<DUAL, R::ATR, R::BTR, LAST ? kRead1[T] : kRead0[T]>(fa, fn, pa, pb);
  // the first k-step's a_0 for the next k-step, after its last use
  if constexpr (!LAST && T == 7) big_read<DUAL, R::ATR, R::BTR, 0>(fa, fn, pa, pb);
  if constexpr (!LAST) feed.template slot<T>();
  if constexpr (!LAST && (T == 16 || T == 20 || T == 24 || T == 28)) {
    dma_a(4 + (T - 16) / 4);
    sched_fence();
  }
  if constexpr (LAST && (T == 32 || T == 36 || T == 40 || T == 44)) {
    dma_a((T - 32) / 4);
    sched_fence();
  }
  if constexpr (T == 18 || T == 26 || T == 50 || T == 58) {
    dma_b((LAST ? 4 : 0) + (T == 18 ? 0 : T == 26 ? 1 : T == 50 ? 2 : 3));
    sched_fence();
  }
  if constexpr (T < 63) big_slot<T + 1, LAST, DUAL, R>(fa, fb, fn, acc, pa, pb, dma_a, dma_b, feed);
}

// LDS of the large-group core: A stages at s0 and s0 + AB (slice parity), B
// stages at s0 + B0 + BB * (slice mod 3)
struct BigLds {
  uint32_t s0;
  __device__ __forceinline__ uint32_t a(int g) const { return s0 + (g & 1) * big::AB; }
  __device__ __forceinline__ uint32_t b(int g) const { return s0 + big::B0 + (g % 3) * big::BB; }
};

// One 64-wide slice g: two k-steps of 32 from A stage g & 1 and B stage
// g mod 3
template <bool DUAL, class R>
__device__ __forceinline__ void big_half(const BigLds& L, int g, int wave, const R& q,
                                         int nk, AccBig& acc, const uint32_t (&a_lane)[2],
                                         const uint32_t (&b_lane)[2], FragA& fa, FragB& fb0,
                                         FragB& fb1) {
  const uint32_t ca = L.a(g), cb = L.b(g), na = L.a(g + 1), nb = L.b(g + 1), db = L.b(g + 2);
  const BigSrc sa(q, g + 1, nk), sb(q, g + 2, nk);
  auto dma_a = [&](int u) { big_dma_a(na, wave, q, sa, u); };
  auto dma_a2 = [&](int u) { big_dma_a(ca, wave, q, sb, u); };
  auto dma_b = [&](int u) { big_dma<DUAL>(db, wave, q, sb, u); };
  BigNoFeed none;
  big_slot<0, false, DUAL, R>(fa, fb0, fb1, acc, ca + a_lane[1], cb + b_lane[1], dma_a, dma_b, none);
  big_slot<0, true, DUAL, R>(fa, fb1, fb0, acc, na + a_lane[0], nb + b_lane[0], dma_a2, dma_b, none);
}

// The same for a feed: stages of the slices (c: this one, n: the next, d: B of the
// one after) instead of their number
struct BigStages {
  uint32_t ca, na, cb, nb, db;
  __device__ __forceinline__ explicit BigStages(const BigLds& L)
      : ca(L.a(0)), na(L.a(1)), cb(L.b(0)), nb(L.b(1)), db(L.b(2)) {}
  __device__ __forceinline__ void next() {
    uint32_t t = ca;
    ca = na;
    na = t;
    t = cb;
    cb = nb;
    nb = db;
    db = t;
  }
};
template <class F>
__device__ __forceinline__ void big_slice(const BigStages& L, int wave, F& q, AccBig& acc,
                                          const uint32_t (&a_lane)[2], const uint32_t (&b_lane)[2],
                                          FragA& fa, FragB& fb0, FragB& fb1) {
  auto dma_a = [&](int u) { big_dma_group(L.na, wave, q.a1, q.a.off[u], q.k1, u); };
  auto dma_a2 = [&](int u) { big_dma_group(L.ca, wave, q.a2, q.a.off[u], q.k2, u); };
  auto dma_b = [&](int u) { big_dma_group(L.db, wave, q.b2, q.b.off[u], q.kb, u); };
  big_slot<0, false, false, F>(fa, fb0, fb1, acc, L.ca + a_lane[1], L.cb + b_lane[1], dma_a, dma_b, q);
  big_slot<0, true, false, F>(fa, fb1, fb0, acc, L.na + a_lane[0], L.nb + b_lane[0], dma_a2, dma_b, q);
}

// A tile's first loads: slice 0, B of slice 1 and the first half of its A.  LDS is
// free from the end of a tile on (the epilogue may use the last B stage).
template <bool DUAL, class R>
__device__ __forceinline__ void big_start(char* lds, const R& q, int nk) {
  const BigLds L{lds_addr(lds)};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BigSrc s0(q, 0, nk), s1(q, 1, nk);
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma_a(L.a(0), wave, q, s0, u);
    sched_fence();
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma<DUAL>(L.b(0), wave, q, s0, u);
    sched_fence();
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma<DUAL>(L.b(1), wave, q, s1, u);
    sched_fence();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    big_dma_a(L.a(1), wave, q, s1, u);
    sched_fence();
  }
}

// the first k-step's fragments, in the order the last k-step of a slice
// reads them (the first k-step's waits count on it)
template <bool DUAL, class R>
__device__ __forceinline__ void big_first_reads(FragA& fa, FragB& fb0, uint32_t pa, uint32_t pb) {
  big_read<DUAL, R::ATR, R::BTR, 0>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 1>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 2>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 3>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 4>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 5>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 6>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 7>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 8>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 9>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 11>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 13>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 15>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 10>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 12>(fa, fb0, pa, pb);
  big_read<DUAL, R::ATR, R::BTR, 14>(fa, fb0, pa, pb);
}

// what follows the last slice
__device__ __forceinline__ void big_close(FragA& fa, FragB& fb0, AccBig& acc) {
  // The last k-step read the first fragments of the slice past the end
  // (never used).  Those reads land whenever the LDS returns them, which the
  // compiler cannot see: the wait for them takes their registers as inputs,
  // so no other value is put there before they have landed.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)"
               :
               : "v"(fa.a[0]), "v"(fa.a[1]), "v"(fa.a[2]), "v"(fa.a[3]), "v"(fa.a[4]),
                 "v"(fa.a[5]), "v"(fa.a[6]), "v"(fa.a[7])
               : "memory");
  asm volatile("" ::"v"(fb0.b[0]), "v"(fb0.b[1]), "v"(fb0.b[2]), "v"(fb0.b[3]), "v"(fb0.b[4]),
               "v"(fb0.b[5]), "v"(fb0.b[6]), "v"(fb0.b[7]));
  // the last MFMAs' results must be in their AGPRs before anything reads
  // them, and the compiler does not see the inline MFMAs' write latency: the
  // wait states follow in an asm statement that takes the last row of
  // accumulators (the other rows were written at least 8 MFMAs earlier).
  // The compiler may still place its own accumulator copies between the
  // loop and this statement, so the emitted code is checked for any access
  // to an MFMA's destination within 19 wait states of it.
  asm volatile("s_barrier\n\ts_nop 7\n\ts_nop 7"
               : "+a"(acc[7][0]), "+a"(acc[7][1]), "+a"(acc[7][2]), "+a"(acc[7][3]),
                 "+a"(acc[7][4]), "+a"(acc[7][5]), "+a"(acc[7][6]), "+a"(acc[7][7])
               :
               : "memory");
}

// C tile += A rows x B rows over nk slices from the rows' K origin, after
// big_start and its wait; returns with every load landed and every wave past its
// last LDS access
template <bool DUAL, class R>
__device__ __forceinline__ void big_run(char* lds, const R& q, int nk, AccBig& acc,
                                        const uint32_t (&a_lane)[2],
                                        const uint32_t (&b_lane)[2]) {
  const BigLds L{lds_addr(lds)};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  FragA fa;
  FragB fb0, fb1;
  big_first_reads<DUAL, R>(fa, fb0, L.a(0) + a_lane[0], L.b(0) + b_lane[0]);
  for (int g = 0; g < nk; ++g)
    big_half<DUAL, R>(L, g, wave, q, nk, acc, a_lane, b_lane, fa, fb0, fb1);
  big_close(fa, fb0, acc);
}

// the same on a feed, whose operands end after nk slices
template <bool ATR, bool BTR>
__device__ __forceinline__ void big_start(char* lds, BigFeed<ATR, BTR>& q) {
  const BigLds L{lds_addr(lds)};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const auto take = [&] {
    q.a.limit();
    q.b.limit();
    q.take_a();
    q.take_b();
  };
  take();
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma_group(L.a(0), wave, q.a2, q.a.off[u], q.k2, u);
    sched_fence();
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma_group(L.b(0), wave, q.b2, q.b.off[u], q.kb, u);
    sched_fence();
  }
  q.a.step();
  q.b.step();
  take();
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    big_dma_group(L.b(1), wave, q.b2, q.b.off[u], q.kb, u);
    sched_fence();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    big_dma_group(L.a(1), wave, q.a2, q.a.off[u], q.k2, u);
    sched_fence();
  }
}
// (the last row's wait states come inside the loop, after its last slice: the
// compiler copies accumulators on the way out of it)
template <bool ATR, bool BTR>
__device__ __forceinline__ void big_run(char* lds, BigFeed<ATR, BTR>& q, int nk, AccBig& acc,
                                        const uint32_t (&a_lane)[2],
                                        const uint32_t (&b_lane)[2]) {
  BigStages L{BigLds{lds_addr(lds)}};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  FragA fa;
  FragB fb0, fb1;
  big_first_reads<false, BigFeed<ATR, BTR>>(fa, fb0, L.ca + a_lane[0], L.cb + b_lane[0]);
  for (int g = 0; g < nk; ++g) {
    big_slice(L, wave, q, acc, a_lane, b_lane, fa, fb0, fb1);
    L.next();
    if (g + 1 == nk)
      asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3"
                   : "+a"(acc[7][0]), "+a"(acc[7][1]), "+a"(acc[7][2]), "+a"(acc[7][3]),
                     "+a"(acc[7][4]), "+a"(acc[7][5]), "+a"(acc[7][6]), "+a"(acc[7][7]));
  }
  big_close(fa, fb0, acc);
}

// The wait between big_start and big_run: A and B of slice 0 have landed (12 newer
// loads, B of slice 1 and the first half of its A, and NEWER vector-memory
// operations issued since)
template <int NEWER>
__device__ __forceinline__ void big_wait() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(NEWER + 12 < 63 ? NEWER + 12 : 63)
               : "memory");
}

template <bool DUAL, class R>
__device__ __forceinline__ void big_tile(char* lds, const R& q, int nk, AccBig& acc,
                                         const uint32_t (&a_lane)[2],
                                         const uint32_t (&b_lane)[2]) {
  big_start<DUAL>(lds, q, nk);
  big_wait<0>();
  big_run<DUAL>(lds, q, nk, acc, a_lane, b_lane);
}

// Two accumulators' values of one row (columns 16 i .. and 16 (i + 1) ..; a lane
// holds 4 consecutive ones) as bf16, 8 consecutive columns a lane: lanes of even
// groups of 16 get the first block's pieces, those of odd groups the second's
// (A 16-byte buffer store of them takes its offset in the vector register and the
// instruction: with a scalar offset register, a VALU write to the data registers right
// behind the store reached its data, 4 bytes of a quarter of the lanes now and then, and
// the compiler keeps the distance only for stores without one.)
__device__ __forceinline__ u32x4_t pack_rows(const float (&x)[4], const float (&y)[4]) {
  const unsigned x0 = pack_bf16x2(x[0], x[1]), x1 = pack_bf16x2(x[2], x[3]);
  const unsigned y0 = pack_bf16x2(y[0], y[1]), y1 = pack_bf16x2(y[2], y[3]);
  const auto p = __builtin_amdgcn_permlane16_swap(x0, y0, false, false);
  const auto q = __builtin_amdgcn_permlane16_swap(x1, y1, false, false);
  const unsigned p0 = p[0], p1 = p[1], q0 = q[0], q1 = q[1];
  return u32x4_t{p0, q0, p1, q1};
}
// ... and where they go: column of the lane's piece within the two blocks
__device__ __forceinline__ int pack_col(int lane) {
  return 16 * (lane >> 4 & 1) + 8 * (lane >> 5);
}

__device__ __forceinline__ int cdiv_d(int a, int b) { return (a + b - 1) / b; }

// the block's lane constants on the large-group core: LDS offsets of fragments
// of a K-contiguous (a, b) and of a transposed operand (at, bt), fetch rows
struct BigLane {
  int lane, wave, wm, wn, r0, cc;
  __device__ __forceinline__ BigLane() {
    const int tid = threadIdx.x;
    lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    wm = wave >> 1;
    wn = wave & 1;
    r0 = tid >> 3;
    cc = 8 * ((tid & 7) ^ swz16(r0));
  }
  // fragment offsets of the operand whose half `half` of the tile this wavefront reads
  __device__ __forceinline__ void rows(uint32_t (&o)[2], int half) const {
    const int fr = lane & 15, hk = lane >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      o[ks] = (half * 128 + fr) * big::RB + (((4 * ks + hk) ^ swz16(fr)) << 4);
  }
  __device__ __forceinline__ void cols(uint32_t (&o)[2], int half) const {
    const int i = lane & 15, hk = lane >> 4, k = 8 * hk + (i >> 2);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      o[ks] = (32 * ks + k) * 512 + half * 256 + (tr_swz(k) << 5) + 8 * (i & 3);
  }
  // A TR operand of `rows` rows of ld elements along K, from row k0 (k1: the end of
  // the tile's run) and column c0
  __device__ __forceinline__ BigOperand<true> along(const bf16_t* p, int ld, int rows, int k0, int k1,
                                                    int c0) const {
    BigOperand<true> o;
    o.p = reinterpret_cast<const char*>(p + ((size_t)k0 * ld + c0));
    o.left = min(rows, k1) - k0;
    o.row = (uint32_t)ld * 2;
    o.cut = (uint32_t)c0 * 2;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = 2 * wave + 8 * u + (lane >> 5), c = lane & 31;
      o.off[u] = (uint32_t)((k * ld + 16 * ((c >> 1) ^ tr_swz(k)) + 8 * (c & 1)) * 2);
    }
    return o;
  }
  // ... that lies in panels of 256 columns
  __device__ __forceinline__ BigOperand<true> along_panel(const bf16_t* p, int rows, int k0, int k1,
                                                          int c0) const {
    return along(p + (size_t)c0 * rows, 256, rows, k0, k1, 0);
  }
  // a K-contiguous operand of ld elements a row, `valid` rows from p on, nk slices
  // from slice k0 on; panel: bytes from one panel of 256 to the next, or 0
  __device__ __forceinline__ BigOperand<false> across(const bf16_t* p, int ld, int valid, int k0,
                                                      int nk, uint32_t panel) const {
    BigOperand<false> o;
    o.p = reinterpret_cast<const char*>(p);
    o.left = nk;
    o.panel = panel ? panel - 512 : 0;
    o.ko = panel ? (uint32_t)(k0 >> 2) * panel + (uint32_t)(k0 & 3) * big::RB
                 : (uint32_t)k0 * big::RB;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      o.off[u] = ((uint32_t)min(r0 + big::RPP * u, valid - 1) * ld + cc) * 2;
    return o;
  }
};

__device__ __forceinline__ void big_zero(AccBig& acc) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{};
}

}  // namespace trimmoe
