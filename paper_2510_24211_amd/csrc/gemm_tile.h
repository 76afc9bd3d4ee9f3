// A workgroup's tile of a matrix product whose operands both have k along their rows:
//   acc[a, b] = sum_k A[a, k] * B[b, k]        bf16 x bf16 or fp16 x fp16 -> fp32 (MFMA)
// HR rows of A x BN rows of B by eight wavefronts, k in tiles of 64, staged in LDS by loads that name no register.
#pragma once
#include "tile_loads.h"

namespace scd {
namespace {

template <int HR_, int BN_>
struct GemmTile {
  static constexpr int HR = HR_, BN = BN_;
  static constexpr int NW = 8, THREADS = NW * 64;
  static constexpr int CW = HR * BN <= 128 * 128 ? 32 : BN == 192 ? 96 : 64;   // rows of B per wavefront
  static constexpr int NC = CW / 32;
  static constexpr int WCOL = BN / CW, WROW = NW / WCOL;
  static constexpr int RW = HR / WROW;                        // rows of A per wavefront
  static constexpr int NB = RW / 32;
  static constexpr int AL = HR / 8 / NW, BL = BN / 8 / NW;    // loads per wavefront and k-tile
  static constexpr int AB = HR * 128, BB = BN * 128;          // bytes per stage
  static constexpr int SB = 3, SA = HR == 256 && BN > 128 ? 2 : 3;
  static constexpr int STAGES = SB * BB + SA * AB;
  static constexpr int kChain = 8;                            // k-tiles that a running sum holds where sums are folded
  static_assert(WCOL * WROW == NW && WROW * RW == HR && WCOL * CW == BN && AL * NW * 8 == HR && BL * NW * 8 == BN && STAGES <= 160 * 1024, "tile shape");
};

// One operand as a workgroup reads it: its first row, `rows` of them exist (past them the last one is read, and what
// comes of it is not to be stored), `bytes` from row to row.
struct TileOperand {
  uint64_t base;
  int rows;
  uint32_t bytes;
};

// acc += the k-tiles kt0 .. kt0 + KT - 1, walked cyclically from the `rot`-th of them, and `tail` (< 64, a multiple of 8)
// elements of the one behind.
//   * Tiles of 128 bytes per row go straight into LDS; lane l of a load writes slot l % 8 of row l / 8 and reads
//     chunk (l % 8) ^ ((row >> 1) & 7): operand reads are then free of bank conflicts without padding.
//   * One barrier per k-tile, in the middle of its last k-step: when it is passed the next tile is in LDS, its first
//     operands are read under the last MFMAs of this one, and the stage just read is free.
//   * Loads are issued one by one between MFMAs: eight wavefronts issuing all of theirs after the barrier would queue at
//     the one address unit with their MFMAs behind them.
// FOLDS: running sums go into whole ones every kChain k-tiles and start again, since one chain of 32-bit additions over k
// errs with its length; in the registers that small tiles have left.
// Ends with loads, MFMAs' operands and stages all settled for this wavefront; a barrier has to follow before LDS is reused.
template <class K, bool F16, bool FOLDS>
__device__ __forceinline__ void multiply_tile(unsigned char* const lds, const TileOperand& A, const TileOperand& B, const int kt0,
                                              const int KT, const int tail, const int rot, f32x16 (&acc)[K::NC][K::NB]) {
  constexpr int NC = K::NC, NB = K::NB, AL = K::AL, BL = K::BL, SA = K::SA, SB = K::SB;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wave % K::WCOL, wr = wave / K::WCOL;
  const int ln = lane & 31, lg = lane >> 5;

  auto piece_row = [&](int per_wave, int i) { return (wave * per_wave + i) * 8 + (lane >> 3); };
  auto piece_chunk = [&](int r) { return (lane & 7) ^ ((r >> 1) & 7); };
  uint32_t ao[AL], bo[BL];
#pragma unroll
  for (int i = 0; i < AL; ++i) {
    const int r = piece_row(AL, i);
    ao[i] = static_cast<uint32_t>(min(r, A.rows - 1)) * A.bytes + piece_chunk(r) * 16;
  }
#pragma unroll
  for (int i = 0; i < BL; ++i) {
    const int r = piece_row(BL, i);
    bo[i] = static_cast<uint32_t>(min(r, B.rows - 1)) * B.bytes + piece_chunk(r) * 16;
  }
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds));
  const uint32_t ldsB = lds0 + wave * BL * 1024, ldsA = lds0 + SB * K::BB + wave * AL * 1024;

  struct Walk {
    uint64_t at;          // the k-tile's column of the operand
    uint32_t lds;         // the stage it goes to
    int k, n;             // its index; tiles issued before it
  };
  auto column = [](const TileOperand& o, int k) { return o.base + static_cast<uint64_t>(static_cast<uint32_t>(k)) * 128u; };
  Walk aw{column(A, kt0 + rot), ldsA, kt0 + rot, 0}, bw{column(B, kt0 + rot), ldsB, kt0 + rot, 0};
  auto advance = [&](Walk& w, const TileOperand& o, uint32_t first, uint32_t bytes, int stages) {
    w.k = w.k + 1 == kt0 + KT ? kt0 : w.k + 1;
    w.at = column(o, w.k);
    w.lds = w.lds + bytes == first + bytes * stages ? first : w.lds + bytes;
    ++w.n;
  };
  auto piece = [&](auto qq, auto cond) {
    constexpr int q = decltype(qq)::value;
    constexpr bool COND = decltype(cond)::value;
    if constexpr (q < AL) {
      if (!COND || aw.n < KT) load_lds16<false, q * 1024>(aw.at, ao[q], aw.lds);
      if constexpr (q == AL - 1) advance(aw, A, ldsA, K::AB, SA);
    } else {
      if (!COND || bw.n < KT) load_lds16<false, (q - AL) * 1024>(bw.at, bo[q - AL], bw.lds);
      if constexpr (q == AL + BL - 1) advance(bw, B, ldsB, K::BB, SB);
    }
  };
  auto load_a = [&]() { static_for<AL>([&](auto i) { piece(i, TrueT{}); }); };
  auto load_b = [&]() { static_for<BL>([&](auto i) { piece(IntT<AL + decltype(i)::value>{}, TrueT{}); }); };

  u32x4 bq[2][NC], aq[2][NB];
  auto fetch = [&](int q, uint32_t sb, uint32_t sa, int kk) {
    const uint32_t slot = ((kk * 2 + lg) ^ ((ln >> 1) & 7)) * 16;
    const unsigned char* const Bt = lds + sb + (wc * K::CW + ln) * 128 + slot;
    const unsigned char* const At = lds + SB * K::BB + sa + (wr * K::RW + ln) * 128 + slot;
#pragma unroll
    for (int c = 0; c < NC; ++c) bq[q][c] = *reinterpret_cast<const u32x4*>(Bt + c * 4096);
#pragma unroll
    for (int i = 0; i < NB; ++i) aq[q][i] = *reinterpret_cast<const u32x4*>(At + i * 4096);
  };
  // the MFMAs of one k-step on operand set q, with quarter Q of a k-tile's loads between them (Q = 4: none)
  constexpr int NM = NC * NB, NP = AL + BL;
  auto mma = [&](int q, auto quarter, auto cond) {
    constexpr int Q = decltype(quarter)::value;
    constexpr int P0 = Q < 4 ? NP * Q / 4 : 0, P1 = Q < 4 ? NP * (Q + 1) / 4 : 0;
    static_for<NM>([&](auto ii) {
      constexpr int I = decltype(ii)::value, c = I / NB, i = I % NB;
      if constexpr (F16)
        acc[c][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, aq[q][i]), __builtin_bit_cast(f16x8, bq[q][c]),
                                                           acc[c][i], 0, 0, 0);
      else
        acc[c][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, aq[q][i]), __builtin_bit_cast(bf16x8, bq[q][c]),
                                                            acc[c][i], 0, 0, 0);
      constexpr int F = P0 + (P1 - P0) * I / NM, E = P0 + (P1 - P0) * (I + 1) / NM;
      if constexpr (E > F) {
        __builtin_amdgcn_sched_barrier(0);
        static_for<E - F>([&](auto k) { piece(IntT<F + decltype(k)::value>{}, cond); });
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x16 whole[NC][NB];
  auto fold = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        whole[c][i] += acc[c][i];
        acc[c][i] = f32x16{};
      }
  };
  if constexpr (FOLDS) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < NB; ++i) whole[c][i] = f32x16{};
  }
  if (KT > 0) {
    // Window t of the loads ends at the barrier of tile t; it brings B of tile t + 2 and A of tile t + SA - 1, A first (a
    // stage is free once the barrier of the tile that it held is passed).  At the barrier of tile t both parts of tile
    // t + 1 have to be in LDS; what was issued after them may be in flight.
    constexpr int AHEAD = BL + (SA == 3 ? AL : 0);
    uint32_t sb = 0, sa = 0;                           // stages of the tile whose operands are read next
    load_a();
    load_b();
    if constexpr (SA == 3) load_a();
    load_b();
    if (KT > 1) wait_loads<AHEAD>();
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    hard_fence();
    static_for<NP / 4>([&](auto i) { piece(i, TrueT{}); });
    fetch(0, 0, 0, 0);
    hard_fence();
    auto tile = [&](auto cond, bool more, bool next) {   // loads go on past this tile's barrier; a tile follows
      fetch(1, sb, sa, 1);
      __builtin_amdgcn_sched_barrier(0);
      mma(0, IntT<1>{}, cond);
      fetch(0, sb, sa, 2);
      __builtin_amdgcn_sched_barrier(0);
      mma(1, IntT<2>{}, cond);
      fetch(1, sb, sa, 3);
      __builtin_amdgcn_sched_barrier(0);
      mma(0, IntT<3>{}, cond);
      hard_fence();
      if (more) wait_loads<AHEAD>();
      else wait_loads<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this tile's operands are in registers
      __builtin_amdgcn_s_barrier();
      hard_fence();
      sb = sb + K::BB == SB * K::BB ? 0 : sb + K::BB;
      sa = sa + K::AB == SA * K::AB ? 0 : sa + K::AB;
      if (next) fetch(0, sb, sa, 0);
      hard_fence();
      mma(1, IntT<0>{}, cond);
      hard_fence();
    };
    int t = 0;
    if constexpr (FOLDS) {
#pragma unroll 1
      for (; t + K::kChain <= KT - 3; fold())
#pragma unroll 1
        for (const int end = t + K::kChain; t < end; ++t) tile(FalseT{}, true, true);
    }
#pragma unroll 1
    for (; t < KT - 3; ++t) tile(FalseT{}, true, true);
#pragma unroll 1
    for (; t < KT; ++t) tile(TrueT{}, t + 2 < KT, t + 1 < KT);
  }
  if (tail != 0) {
    // the ragged k-tile on its own: chunks past the end read the last one of the row and are zeroed in A (B is finite)
    // by the wavefront that loaded them
    const int nch = tail / 8;
    const uint64_t acol = column(A, kt0 + KT), bcol = column(B, kt0 + KT);
    __syncthreads();                                 // every wavefront has its operands: the stages are free
    static_for<AL>([&](auto ii) {
      constexpr int i = decltype(ii)::value;
      const int ch = piece_chunk(piece_row(AL, i));
      load_lds16<false, i * 1024>(acol, ao[i] - max(ch - (nch - 1), 0) * 16, ldsA);
    });
    static_for<BL>([&](auto ii) {
      constexpr int i = decltype(ii)::value;
      const int ch = piece_chunk(piece_row(BL, i));
      load_lds16<false, i * 1024>(bcol, bo[i] - max(ch - (nch - 1), 0) * 16, ldsB);
    });
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < AL; ++i)
      if (piece_chunk(piece_row(AL, i)) >= nch)
        *reinterpret_cast<u32x4*>(lds + SB * K::BB + (wave * AL + i) * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
    for (int kk = 0; kk * 2 < nch; ++kk) {
      fetch(0, 0, 0, kk);
      mma(0, IntT<4>{}, FalseT{});
    }
  }
  if constexpr (FOLDS) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[c][i] += whole[c][i];
  }
}

// Which tile a workgroup works on.  Workgroup ids go round robin over the 8 XCDs; an XCD takes a stretch of the tiles,
// four tiles of A's rows side by side, so that what its workgroups read together is shared in its L2.
struct TilePlace {
  int a, b, part;        // tile of A's rows, of B's rows, part of k; a < 0: none
};
__device__ __forceinline__ TilePlace tile_place(int MT, int NT, int KS) {
  const int tiles = MT * NT, all = tiles * KS, per = (all + 7) / 8;
  const int j = blockIdx.x / 8, idx = (blockIdx.x % 8) * per + j;
  if (j >= per || idx >= all) return {-1, 0, 0};
  const int part = idx / tiles, at = idx - part * tiles;
  const int group = at / (4 * NT), rest = at - group * 4 * NT, high = min(4, MT - group * 4);
  return {group * 4 + rest % high, rest / high, part};
}

}  // namespace
}  // namespace scd
