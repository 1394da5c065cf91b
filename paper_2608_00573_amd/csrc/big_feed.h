// The large-group core (mfma_core.h) on the operands of mid_core.h: A in either order, B
// K-contiguous, a second array where the first one's K ends, and pairs of operands that
// share their rows.  Not part of the public ABI.
#pragma once

#include "mid_core.h"

namespace trimmoe {

template <bool ATR_, bool PAIR_ = false>
struct BigTile {
  static constexpr bool ATR = ATR_, BTR = false, PAIR = PAIR_;
  static constexpr int BM = big::BM, BN = big::BN, KS = BK, OCC = 1, SPAN = PAIR ? 64 : 0;
  static constexpr int THREADS = big::THREADS, WM = 128, WN = 128, TM = 8, TN = 8, PA = 8, PB = 8;
  static constexpr int LDS = big::LDS, ROWS_A = PAIR ? BM / 2 : BM;
};

// What the loop fetches from: A one slice ahead and both operands two ahead, made ready
// between the MFMAs of the slice before (see BigFeed).  PAIR: the operands of a take
// turns of 64 rows.
template <class T>
struct RunFeed {
  static constexpr bool ATR = T::ATR, BTR = T::BTR;
  TileOperand<8> a, b;
  __amdgpu_buffer_rsrc_t a1, a2, b2, g1, g2;
  uint32_t n;
  __device__ __forceinline__ void take_a() {
    a2 = uniform_rsrc(a.p, n);
    if constexpr (T::PAIR) g2 = uniform_rsrc(a.p1, n);
  }
  __device__ __forceinline__ void pass_a() {
    a1 = a2;
    if constexpr (T::PAIR) g1 = g2;
  }
  template <int S>
  __device__ __forceinline__ void slot() {
    if constexpr (S == 8) pass_a();
    if constexpr (S == 9) a.go();
    if constexpr (S == 10) a.turn();
    if constexpr (S == 11) n = a.template bytes<ATR>();
    if constexpr (S == 12) take_a();
    if constexpr (S == 13) b.go();
    if constexpr (S == 14) b.turn();
    if constexpr (S == 15) n = b.template bytes<BTR>();
    if constexpr (S == 16) b2 = uniform_rsrc(b.p, n);
    if constexpr (S >= 8 && S <= 16) sched_fence();
  }
  __device__ __forceinline__ void dma_a(uint32_t stage, int wave, bool next, int u) const {
    big_dma_group(stage, wave, T::PAIR && (u & 2) ? (next ? g1 : g2) : next ? a1 : a2, a.off[u], 0, u);
  }
  __device__ __forceinline__ void dma_b(uint32_t stage, int wave, int u) const {
    big_dma_group(stage, wave, b2, b.off[u], 0, u);
  }
};

template <class T_>
struct BigCore {
  using T = T_;
  using Acc = AccBig;
  char* lds;
  int lane, wave, wm, wn;
  uint32_t la[2], lb[2];
  RunFeed<T> f;
  TileOperand<8> a, b;  // of the tile that load() has made ready
  int left;
  __device__ __forceinline__ explicit BigCore(char* lds_) : lds(lds_) {
    const BigLane L;
    lane = L.lane;
    wave = L.wave;
    wm = L.wm;
    wn = L.wn;
    if constexpr (T::ATR)
      L.cols(la, wm);
    else
      L.rows(la, wm);
    L.rows(lb, wn);
  }
  // Every tile runs through its own slices; the next one's first loads (slice 0, B of
  // slice 1 and the first half of its A) go out before a tile leaves its registers.
  template <class Load>
  __device__ __forceinline__ void first(Load& load) {
    ahead(load);
  }
  template <class Load>
  __device__ __forceinline__ void ahead(Load& load) {
    if (!load()) return;
    f.a = a;
    f.b = b;
    const BigLds L{lds_addr(lds)};
    const auto take = [&] {
      f.n = f.a.template bytes<T::ATR>();
      f.take_a();
      f.n = f.b.template bytes<T::BTR>();
      f.b2 = uniform_rsrc(f.b.p, f.n);
    };
    take();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      f.dma_a(L.a(0), wave, false, u);
      sched_fence();
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      f.dma_b(L.b(0), wave, u);
      sched_fence();
    }
    f.a.step();
    f.b.step();
    take();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      f.dma_b(L.b(1), wave, u);
      sched_fence();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f.dma_a(L.a(1), wave, false, u);
      sched_fence();
    }
  }
  // acc = the tile's product over nk slices (see big_run).  NEWER: vector-memory
  // operations that every wavefront has issued since begin, at least
  template <int NEWER = 0, class Load>
  __device__ __forceinline__ void run(int nk, Acc& acc, Load&) {
    big_zero(acc);
    big_wait<NEWER>();
    BigStages L{BigLds{lds_addr(lds)}};
    FragA fa;
    FragB fb0, fb1;
    big_first_reads<false, RunFeed<T>>(fa, fb0, L.ca + la[0], L.cb + lb[0]);
    for (int g = 0; g < nk; ++g) {
      auto dma_a = [&](int u) { f.dma_a(L.na, wave, true, u); };
      auto dma_a2 = [&](int u) { f.dma_a(L.ca, wave, false, u); };
      auto dma_b = [&](int u) { f.dma_b(L.db, wave, u); };
      big_slot<0, false, false, RunFeed<T>>(fa, fb0, fb1, acc, L.ca + la[1], L.cb + lb[1], dma_a, dma_b,
                                            f);
      big_slot<0, true, false, RunFeed<T>>(fa, fb1, fb0, acc, L.na + la[0], L.nb + lb[0], dma_a2, dma_b,
                                           f);
      L.next();
      if (g + 1 == nk)
        asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3"
                     : "+a"(acc[7][0]), "+a"(acc[7][1]), "+a"(acc[7][2]), "+a"(acc[7][3]),
                       "+a"(acc[7][4]), "+a"(acc[7][5]), "+a"(acc[7][6]), "+a"(acc[7][7]));
    }
    big_close(fa, fb0, acc);
    sched_fence();
  }
  __device__ __forceinline__ void last() {}
};

}  // namespace trimmoe
