// A bf16 matrix core for products whose operands lie in either order: C = A B^T on BM x
// BN tiles by four wavefronts, two or more blocks a CU.  Not part of the public ABI.
//
// An operand is K-contiguous ([rows][K]: slices of 64 elements land as rows of 128 bytes)
// or runs along K (TR, [K][rows]: a slice is 64 or 32 rows of BM or BN columns), and is read
// out of LDS as it lies or transposed (ds_read_b64_tr_b16).  Slices go straight to LDS by
// DMA into a ring of ST stages, ST - 1 of them in flight; one barrier a slice.  The
// MFMAs are 16 x 16 x 32.  An operand may go on in a second array where the first one's
// K ends.  Fragment reads are inline asm with explicit waits, as in the other cores: the
// compiler would wait for every DMA before each of them.
//
// Its bound is LDS: a 128 x 128 tile moves 96 KB in and out (768 cycles) for a 64-deep
// slice of 512 cycles of MFMAs a SIMD, a 256 x 128 tile 72 KB (576 cycles) for a 32-deep
// one of 512.  64-byte rows of K-contiguous operands cost more than that saves (up and
// gate of 16384 rows over 60 experts: 350 us in 128 x 128 tiles, 378 in 256 x 128), so the
// larger tiles are for operands along K.
#pragma once

#include "mfma_core.h"

namespace trimmoe {

// a buffer at p, which is the same in every lane (the compiler does not always see it,
// and would turn every fetch into a loop over lanes)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const char* p, uint32_t bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>((uint64_t)hi << 32 | lo), (short)0,
                                           (int)bytes, 0x00020000);
}

// K slices of an operand as a tile takes them.  Everything but off is wave-uniform.
template <int NP>  // DMAs a thread and slice
struct TileOperand {
  const char* p;     // not TR: row 0 at the slice; TR: the slice's first row, column 0 of the tile
  const char* p1;    // the second operand of a pair (see MidTile::PAIR)
  const char* q;     // where the second array begins (kq of it), or anything (kq 0)
  uint32_t inc;      // bytes from slice to slice
  uint32_t row, cut; // TR: bytes of a row, and of a row before the tile's columns
  int k, kq;         // K left from the slice on, in this array and in the next
  uint32_t off[NP];
  template <bool TR, int KS = BK>
  __device__ __forceinline__ uint32_t bytes() const {
    return __builtin_amdgcn_readfirstlane(k <= 0 ? 0u : TR ? (uint32_t)min(k, KS) * row - cut
                                                             : 0xffffffffu);
  }
  // to the next slice: on, and over to the next array at the end
  template <int KS = BK>
  __device__ __forceinline__ void go() {
    p += inc;
    p1 += inc;
    k -= KS;
  }
  __device__ __forceinline__ void turn() {
    if (k <= 0) {
      p = q;
      k = kq;
      kq = 0;
    }
  }
  template <int KS = BK>
  __device__ __forceinline__ void step() {
    go<KS>();
    turn();
  }
};

// PAIR: A holds two K-contiguous operands in turns of SPAN rows, so that a wavefront's
// fragments 0 .. TM / 2 - 1 are rows of the first and the rest the same rows of the second.
// KS: elements of K a slice (32 where both operands are along K).  OCC: blocks a CU.
template <int BM_, int BN_, int ST_, bool ATR_, bool BTR_, bool PAIR_ = false, int KS_ = BK>
struct MidTile {
  static constexpr int KS = KS_, OCC = 2, SPAN = PAIR_ ? BM_ / 4 : 0;
  static constexpr int BM = BM_, BN = BN_, ST = ST_;
  static constexpr bool ATR = ATR_, BTR = BTR_, PAIR = PAIR_;
  static constexpr int THREADS = 256, GM = 2, GN = 2;
  static constexpr int WM = BM / GM, WN = BN / GN, TM = WM / 16, TN = WN / 16;
  static constexpr int PA = BM * KS / 2048, PB = BN * KS / 2048;  // DMAs a thread
  static constexpr int A_BYTES = BM * KS * 2, STAGE = (BM + BN) * KS * 2, LDS = ST * STAGE;
  static constexpr int ROWS_A = PAIR ? BM / 2 : BM;  // rows of C's A side
  static_assert(KS == BK || (KS == 32 && ATR && BTR), "slices");
  static_assert(!PAIR || (!ATR && SPAN == 2048 / KS), "a pair's turns are one DMA each");
  static_assert(ST >= 2 && (PA + PB) * (ST - 2) < 64, "waits");
};

// 32-byte piece of a transposed operand's row k where its piece 0 sits (exclusive or):
// the eight rows that 32 lanes read together then touch distinct banks
template <int COLS>
__device__ __forceinline__ int mid_swz(int k) {
  static_assert(COLS >= 128, "a row of fewer pieces needs another order");
  return (k & 3) | ((k >> 3 & 1) << 2);
}

// this thread's DMA offsets: of a K-contiguous operand's rows (ld elements each, rows
// past `valid` repeat the last one; span: rows of a pair's turns, or 0) ...
template <int NP>
__device__ __forceinline__ void tile_rows(TileOperand<NP>& o, const bf16_t* p, int ld, int valid, int k,
                                         int span = 0) {
  constexpr int CH = BK / 8, RP = 256 / CH;  // 16-byte chunks of a row, rows of a DMA
  const int r0 = threadIdx.x / CH, c = (threadIdx.x % CH) ^ swz16(r0);
  o.p = reinterpret_cast<const char*>(p);
  o.inc = 2 * BK;
  o.row = o.cut = 0;
  o.k = k;
  o.kq = 0;
  o.q = o.p1 = o.p;
#pragma unroll
  for (int u = 0; u < NP; ++u) {
    // (the large core's pairs turn every two DMAs)
    const int r = span == RP       ? r0 + RP * (u >> 1)
                  : span == 2 * RP ? r0 + RP * (u & 1) + span * (u >> 2)
                                   : r0 + RP * u;
    o.off[u] = ((uint32_t)min(r, valid - 1) * (uint32_t)ld + 8 * c) * 2;
  }
}
// ... and of one along K, k rows of it from row 0 at p, from column c0 on
template <int COLS, int KS = BK, int NP>
__device__ __forceinline__ void tile_along(TileOperand<NP>& o, const bf16_t* p, int ld, int c0, int k) {
  o.p = reinterpret_cast<const char*>(p + c0);
  o.row = 2 * (uint32_t)ld;
  o.cut = 2 * (uint32_t)c0;
  o.inc = o.row * KS;
  o.k = k;
  o.kq = 0;
  o.q = o.p1 = o.p;
#pragma unroll
  for (int u = 0; u < NP; ++u) {
    const int i = u * 256 + (int)threadIdx.x, kr = i / (COLS / 8), c = i % (COLS / 8);
    o.off[u] = ((uint32_t)kr * (uint32_t)ld + 16 * ((c >> 1) ^ mid_swz<COLS>(kr)) + 8 * (c & 1)) * 2;
  }
}

// Up to three tiles (N numbers each) whose loads have begun, first in first out, in
// registers: selected number by number, for an indexed copy would lie in memory
template <int N>
struct TileQueue {
  struct At {
    int v[N];
  };
  int q0[N], q1[N], q2[N], n = 0;
  __device__ __forceinline__ void push(const At& at) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      q0[i] = n == 0 ? at.v[i] : q0[i];
      q1[i] = n == 1 ? at.v[i] : q1[i];
      q2[i] = n == 2 ? at.v[i] : q2[i];
    }
    ++n;
  }
  __device__ __forceinline__ At pop() {
    At at;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      at.v[i] = q0[i];
      q0[i] = q1[i];
      q1[i] = q2[i];
    }
    --n;
    return at;
  }
};

template <class T_>
struct MidCore {
  using T = T_;
  using Acc = f32x4_t[T::TM][T::TN];
  struct Frags {
    bf16x8_t a[T::TM], b[T::TN];
  };
  static constexpr int NDMA = T::PA + T::PB;
  static constexpr int OPS = T::TM * (T::ATR ? 2 : 1) + T::TN * (T::BTR ? 2 : 1);  // LDS reads a k-step
  int lane, wave, wm, wn;
  uint32_t s0, la[2], lb[2];
  TileOperand<T::PA> a;
  TileOperand<T::PB> b;

  __device__ __forceinline__ explicit MidCore(char* lds) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave >> 1;
    wn = wave & 1;
    s0 = lds_addr(lds);
    place<T::ATR, T::BM>(la, wm * T::WM);
    place<T::BTR, T::BN>(lb, wn * T::WN);
#pragma unroll
    for (int ks = 0; ks < T::KS / 32; ++ks) lb[ks] += T::A_BYTES;
  }
  // LDS offsets of the lane's part of fragment 0
  template <bool TR, int COLS>
  __device__ __forceinline__ void place(uint32_t (&o)[2], int first) const {
    const int fr = lane & 15, hk = lane >> 4;
#pragma unroll
    for (int ks = 0; ks < T::KS / 32; ++ks) {
      if constexpr (TR) {
        const int k = 32 * ks + 8 * hk + (fr >> 2);
        o[ks] = k * COLS * 2 + (((first >> 4) ^ mid_swz<COLS>(k)) << 5) + 8 * (fr & 3);
      } else {
        o[ks] = (first + fr) * BK * 2 + (((4 * ks + hk) ^ swz16(fr)) << 4);
      }
    }
  }
  template <bool TR, int COLS>
  static __device__ __forceinline__ bf16x8_t read1(uint32_t at, int n) {
    if constexpr (TR) {
      typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
      u32x2_t lo, hi;
      const uint32_t a = at ^ (uint32_t)(n << 5);
      asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(lo) : "v"(a));
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(hi) : "v"(a), "n"(4 * COLS * 2));
      return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3));
    } else {
      return lds_read(at + n * 16 * BK * 2);
    }
  }
  __device__ __forceinline__ void read(Frags& f, uint32_t stage, int ks) const {
#pragma unroll
    for (int i = 0; i < T::TM; ++i) f.a[i] = read1<T::ATR, T::BM>(stage + la[ks], i);
#pragma unroll
    for (int j = 0; j < T::TN; ++j) f.b[j] = read1<T::BTR, T::BN>(stage + lb[ks], j);
  }
  template <int N>
  static __device__ __forceinline__ void wait(Frags& f) {
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N < 15 ? N : 15));
#pragma unroll
    for (int i = 0; i < T::TM; ++i) asm volatile("" : "+v"(f.a[i]));
#pragma unroll
    for (int j = 0; j < T::TN; ++j) asm volatile("" : "+v"(f.b[j]));
  }
  static __device__ __forceinline__ void mma(const Frags& f, Acc& acc) {
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int j = 0; j < T::TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
  }
  template <bool TR, bool PAIR, int NP>
  __device__ __forceinline__ void issue1(uint32_t dst, const TileOperand<NP>& o) const {
    const uint32_t n = o.template bytes<TR, T::KS>();
    const auto rs = uniform_rsrc(o.p, n), r1 = uniform_rsrc(PAIR ? o.p1 : o.p, n);
#pragma unroll
    for (int u = 0; u < NP; ++u)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          PAIR && (u & 1) ? r1 : rs, (lds_byte*)(uintptr_t)(dst + (uint32_t)(u * 4096 + wave * 1024)), 16,
          o.off[u], 0, 0, 0);
  }
  __device__ __forceinline__ void issue(int stage) {
    const uint32_t s = s0 + stage * T::STAGE;
    issue1<T::ATR, T::PAIR>(s, a);
    issue1<T::BTR, false>(s + T::A_BYTES, b);
    a.template step<T::KS>();
    b.template step<T::KS>();
  }
  // The operands' slices of all of a block's tiles are one stream through the ring: the
  // next tiles' loads are in flight while a tile leaves its registers.  load() makes a,
  // b and left (at least 1) those of the next tile of the block (false: there is none;
  // the slices that follow are zeros).  Up to ST tiles have been loaded and not run.
  static_assert(T::ST <= 3, "TileQueue");
  int left, st, in;  // slices of the loading tile to come; stages of the next reads and loads
  template <class Load>
  __device__ __forceinline__ void next(Load& load) {
    if (left == 0 && !load()) left = INT32_MAX;
    issue(in);
    in = in + 1 == T::ST ? 0 : in + 1;
    --left;
  }
  template <class Load>
  __device__ __forceinline__ void first(Load& load) {
    left = st = in = 0;
    a.k = a.kq = b.k = b.kq = 0;
#pragma unroll
    for (int s = 0; s < T::ST - 1; ++s) next(load);
  }
  template <class Load>
  __device__ __forceinline__ void ahead(Load&) {}
  __device__ __forceinline__ void slice(Acc& acc) {
    const uint32_t s = s0 + st * T::STAGE;
    st = st + 1 == T::ST ? 0 : st + 1;
    Frags f0, f1;
    read(f0, s, 0);
    if constexpr (T::KS == BK) {
      read(f1, s, 1);
      wait<OPS>(f0);
      mma(f0, acc);
      wait<0>(f1);
      mma(f1, acc);
    } else {
      wait<0>(f0);
      mma(f0, acc);
    }
  }
  // acc = the tile's product over its nk slices.  NEWER: vector-memory operations that
  // every wavefront has issued since the last run, at least.
  template <int NEWER = 0, class Load>
  __device__ __forceinline__ void run(int nk, Acc& acc, Load& load) {
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
      for (int j = 0; j < T::TN; ++j) acc[i][j] = f32x4_t{};
    constexpr int W = NDMA * (T::ST - 2);
    int g = 0;
    // (the first ST - 1 slices were loaded before those operations)
    for (; g < min(nk, T::ST - 1); ++g) {
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(W + NEWER < 63 ? W + NEWER : 63) : "memory");
      next(load);
      slice(acc);
    }
    for (; g < nk; ++g) {
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(W) : "memory");
      next(load);
      slice(acc);
    }
  }
  // before the block ends: no load may land in LDS that is no longer its own
  __device__ __forceinline__ void last() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};

}  // namespace trimmoe
