// LM head over 8-bit rows and weights, e4m3 with a scale for each block of 128:
//   logit[m, v] = sum over the blocks b of k  sh[m, b] * sw[v / 128, b] * sum over k in b of h[m, k] * W[v, k]
// then guidance mix and temperature as in the bf16 LM head.  The products of a block go to the matrix units, the block's sums times its
// scale are added to the logits in fp32: one multiplication per row and block, one fused multiply-add per logit and block.
//
// The matrix units' own 8-bit products do not do: they add products up with some 13 bits below the largest one of a step, which leaves
// errors of 1.5e-5 of the logits (normal rows and weights, 2-norm; 6e-5 where sizes spread more).  In fp16, which holds every code
// exactly, products are exact and sums keep fp32's bits (1e-8 to 7e-8 there).  So codes stay 8 bits wide in memory and LDS and are
// converted, two by an instruction, on their way from LDS to the MFMAs.
//
// Rows of h are the MFMA's columns: a lane has one row, and one scale of it; its columns' scale is one number, or two where a group of the
// table ends among them.  h, W and the scales of h go from memory straight into LDS, 128 bytes of a row to a stage; slot l % 8 of row l / 8 of a
// load holds chunk (l % 8) ^ ((row >> 1) & 7): operand reads are then free of bank conflicts.  Scales of h come for four blocks at a time (a word
// per row and block would ask the L2 for as many lines as h and W together: 5 % of the time), W's by way of the scalar cache.
//
//   What bounds it (d = 4096, guidance).  Few rows: memory.  One row x 65536 ids takes 45 us (268 MB of W: 6.0 TB/s), 32 x 2 rows 51 to 56; the bf16 head
// takes 82 for either.  Many rows: instructions.  512 x 2 rows x 8192 ids, one round of tiles, take 61 to 68 us (the bf16 head 61 to 63); with every vector
// instruction and load taken out of the loop 52 to 54 remained, 48 of them products at 1.43 PFLOP/s, the rate of a large product of 16 bits, 4 to
// 6 launch, first loads and stores.  512 x 2 x 64000 takes 490 to 518 us (1.04 to 1.1 PFLOP/s; the bf16 head 446 to 454): by counters the matrix pipes are
// busy half of the time (42 % in 480 x 2 x 8191), 64 cycles of a SIMD pass for each MFMA of 32, and 7.4 other vector instructions of 4 stand beside it.
//   What was tried: loads and conversions ahead of the MFMAs instead of between them 541 us; the sums of a block carried over the loop's end as copies
// (64 moves, and spilled offsets whose reloads wait for all loads) 880; all workgroups from block 0 on 65 instead of 59 (32 x 2 rows);
// logits turned in LDS for stores of whole lines: nothing; stores past the caches: 560.
#include "eights.h"
#include "launch_events.h"
#include "lm_head_rows.h"

#include <stdio.h>

#include <algorithm>

namespace scd {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Eight codes (two words) as fp16 numbers, which hold every e4m3 number, NaN among them.
__device__ __forceinline__ f16x8 to_f16(uint32_t a, uint32_t b) {
  const f16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true)};
  return f16x8{v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
}

// RB blocks of 32 window rows (times C with guidance) x BN columns by WCOL x WROW wavefronts; S stages
// of each of WK parts of k, which have wavefronts and stages of their own; NT: W past the caches
template <int C_, int RB_, int BN_, int WCOL_, int WROW_, int S_, int WK_ = 1, bool NT_ = false>
struct Fp8Cfg {
  static constexpr int C = C_, RB = RB_, BN = BN_, WCOL = WCOL_, WROW = WROW_, S = S_, WK = WK_;
  static constexpr bool NT = NT_;
  static int name(char* buf, size_t cap, bool borders) {
    return snprintf(buf, cap, "lm_head_fp8_kernel<Fp8Cfg<%d, %d, %d, %d, %d, %d, %d, %s>, %s>", C, RB, BN, WCOL, WROW, S, WK, NT ? "true" : "false",
                    borders ? "true" : "false");
  }
  static constexpr int NW = WCOL * WROW, THREADS = NW * WK * 64;
  static constexpr int HR = RB * C * 32;                   // rows of h
  static constexpr int CW = BN / WCOL, NC = CW / 32;       // columns per wavefront
  static constexpr int RBW = RB / WROW, NB = RBW * C;      // blocks of rows per wavefront
  static constexpr int AL = HR / 8 / NW, BL = BN / 8 / NW; // loads per wavefront and block of k
  static constexpr int AB = HR * 128, BB = BN * 128;       // bytes of a stage: h, W
  static constexpr int ALL = AL + BL;
  // Scales of h come four blocks at a time, SL loads per wavefront, behind the stages.
  static constexpr int SL = HR / 16 / NW, GB = HR * 16, GROUPS = (S + 3) / 4 + 1;
  static constexpr int PART = S * (AB + BB) + GROUPS * GB, LDS = WK * PART;       // LDS of a part of k, of all
  static constexpr int ACC = NC * NB == 1 ? 2 : 1;         // sums side by side: one alone would have every MFMA wait for the last
  static_assert((CW == 32 || CW == 64) && RBW * WROW == RB && AL * NW * 8 == HR && BL * NW * 8 == BN && SL * NW * 16 == HR, "tile shape");
  static_assert(LDS <= 160 * 1024 && PART >= NW * NC * NB * 4096 && S >= 2 && (S - 1) * ALL <= 63, "LDS, loads in flight");
};

struct Fp8Args {
  LmHeadArgs lm;               // h [B, C, L, d] codes
  const float* h_scales;       // [B, C, L, G]
  const uint8_t* W;            // [V, d] codes
  const float* W_scales;       // [ceil(V / 128), G]
  int v_lo;
};

// 4 bytes per lane from base + off (per lane) to LDS byte address lds + ADD + 4 * lane
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int ADD>
__device__ __forceinline__ void load_lds4(uint64_t base, uint32_t off, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base), "n"(ADD) : "memory", "m0", "scc");
}
#pragma clang diagnostic pop

// BORDERS: groups of the table may end among a wavefront's columns
template <class K, bool BORDERS>
__global__ __launch_bounds__(K::THREADS) __attribute__((amdgpu_waves_per_eu(2))) void lm_head_fp8_kernel(const Fp8Args f, const int WT, const int MT) {
  constexpr int C = K::C, RB = K::RB, NB = K::NB, NC = K::NC, AL = K::AL, BL = K::BL, S = K::S;
  __shared__ __attribute__((aligned(1024))) unsigned char whole[K::LDS];    // for each part of k: W's stages, then h's, then the scales'
  const LmHeadArgs& a = f.lm;
  // workgroups that share columns get ids 8 apart: the same XCD, the same L2
  const int id = blockIdx.x, mt = (id / 8) % MT, wt = id / (8 * MT) * 8 + id % 8;
  if (wt >= WT) return;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const int part = K::WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6) / K::NW;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) - part * K::NW;
  const int wc = wave % K::WCOL, wr = wave / K::WCOL;
  unsigned char* const lds = whole + part * K::PART;
  const int rows = a.B * a.L, d = a.d, KT = (d + 127) / 128, G = KT;
  const int k0 = KT * part / K::WK, count = KT * (part + 1) / K::WK - k0;      // the part's blocks of k; KT >= WK
  const int nch = d % 128 / 16;                          // 16-byte chunks of a ragged last block, 0: there is none
  const int p_base = mt * RB * 32;
  // columns are counted from the first allowed id, or from the multiple of 4 before it: a group of the table does not end among the four
  // columns of a quarter of a lane's registers then
  const int skip = BORDERS ? f.v_lo % 4 : 0, col_base = wt * K::BN - skip;
  RowState mine[K::RBW];
#pragma unroll
  for (int i = 0; i < K::RBW; ++i) mine[i] = row_state(a, p_base + (wr * K::RBW + i) * 32 + ln);

  // ---- where this lane's loads come from ----------------------------------------------------------------
  auto piece_row = [&](int per_wave, int i) { return (wave * per_wave + i) * 8 + (lane >> 3); };
  // (the rows of an even and of an odd piece: two chunks for all of a wavefront's loads)
  auto piece_chunk = [&](int odd) { return (lane & 7) ^ ((odd * 4 + (lane >> 4)) & 7); };
  auto odd_piece = [&](int per_wave, int i) { return per_wave % 2 == 0 ? i & 1 : (wave * per_wave + i) & 1; };
  const int h0 = first_h_row(p_base, C, a.L);
  const uint64_t hbase = reinterpret_cast<uint64_t>(a.h) + static_cast<uint64_t>(h0) * d;
  const int w0 = f.v_lo + col_base, w_last = f.v_lo + a.n - 1;       // row of W of the first column, and the last row that may be read
  const uint64_t wbase = reinterpret_cast<uint64_t>(f.W) + static_cast<uint64_t>(w0) * d;
  auto row_of_h = [&](int r) {                           // of row r of the tile: [RB][C][32]
    const int blk = r / 32, rb = blk / C;
    return h_row(min(p_base + rb * 32, rows - 1), r % 32, blk % C, C, a.L, rows);
  };
  uint32_t ao[AL], bo[BL];
#pragma unroll
  for (int i = 0; i < AL; ++i) {
    const int r = piece_row(AL, i);
    ao[i] = static_cast<uint32_t>(row_of_h(r) - h0) * static_cast<uint32_t>(d) + piece_chunk(odd_piece(AL, i)) * 16;
  }
#pragma unroll
  for (int i = 0; i < BL; ++i) {
    const int r = piece_row(BL, i);
    // (differences: behind the last id of a table of 2^31 - 1 there is no number)
    bo[i] = static_cast<uint32_t>(min(max(r, f.v_lo - w0), w_last - w0)) * static_cast<uint32_t>(d) + piece_chunk(odd_piece(BL, i)) * 16;
  }
  // scales of 16 rows x 4 blocks of k to a load
  const uint64_t sbase = reinterpret_cast<uint64_t>(f.h_scales) + static_cast<uint64_t>(h0) * G * 4;
  uint32_t so[K::SL];
#pragma unroll
  for (int i = 0; i < K::SL; ++i)
    so[i] = static_cast<uint32_t>(row_of_h((wave * K::SL + i) * 16 + (lane >> 2)) - h0) * static_cast<uint32_t>(G) * 4u;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds));
  const uint32_t ldsB = lds0 + wave * BL * 1024, ldsA = lds0 + S * K::BB + wave * AL * 1024,
                 ldsS = lds0 + S * (K::BB + K::AB) + wave * K::SL * 256;

  // Blocks are walked cyclically, from one that depends on the workgroup: rows are d bytes apart, and workgroups that all begin at block 0
  // ask the same few channels of the L2 for theirs.
  const int rot = k0 + (MT > 1 ? id % 8 : wt) * 5 % count;
  auto after = [&](int k) { return k + 1 == k0 + count ? k0 : k + 1; };
  // Past a ragged end a row's last chunk is read: offsets of the loads of block KT - 1, made before them and taken back behind.
  auto ragged_end = [&](int t, bool back) __attribute__((always_inline)) {
    if (t != KT - 1 || nch == 0) return;
    auto past = [&](int odd) { return static_cast<uint32_t>(max(piece_chunk(odd) - (nch - 1), 0) * 16); };
#pragma unroll
    for (int i = 0; i < AL; ++i) ao[i] += back ? past(odd_piece(AL, i)) : 0u - past(odd_piece(AL, i));
#pragma unroll
    for (int i = 0; i < BL; ++i) bo[i] += back ? past(odd_piece(BL, i)) : 0u - past(odd_piece(BL, i));
  };
  // Load q of block t.
  auto load = [&](auto qq, int t, uint32_t stage) {
    constexpr int Q = decltype(qq)::value;
    constexpr bool H = Q < AL;
    constexpr int I = H ? Q : Q - AL;
    load_lds16<!H && K::NT, I * 1024>((H ? hbase : wbase) + static_cast<uint64_t>(t) * 128, H ? ao[H ? I : 0] : bo[H ? 0 : I],
                                      H ? ldsA + stage * K::AB : ldsB + stage * K::BB);
  };
  // With the u-th block of the walk, where u is a multiple of 4: the scales of four blocks from there on.
  auto load_scales = [&](int u) __attribute__((always_inline)) {
    if (u % 4 != 0) return;
    int k = rot + min(u + (lane & 3), count - 1);
    k = k >= k0 + count ? k - count : k;
    static_for<K::SL>([&](auto i) {
      load_lds4<decltype(i)::value * 256>(sbase, so[decltype(i)::value] + static_cast<uint32_t>(k) * 4u, ldsS + u / 4 % K::GROUPS * K::GB);
    });
  };
  // What a ragged last block lacks counts as 0: in h, by the wavefront that has loaded it.
  auto clear_end = [&](int t, uint32_t stage) {
    if (t != KT - 1 || nch == 0) return;
#pragma unroll
    for (int i = 0; i < AL; ++i)
      if (piece_chunk(odd_piece(AL, i)) >= nch)
        *reinterpret_cast<u32x4*>(lds + S * K::BB + stage * K::AB + (wave * AL + i) * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
  };

  const unsigned char* const Bt = lds + (wc * K::CW + ln) * 128;
  const unsigned char* const At = lds + S * K::BB + (wr * NB * 32 + ln) * 128;
  const float* const St = reinterpret_cast<const float*>(lds + S * (K::BB + K::AB)) + (wr * NB * 32 + ln) * 4;
  u32x4 raw[2][NB + NC];                                  // codes of two chunks: NB blocks of rows, then NC of columns
  f16x8 op[2][NB + NC];                                   // operands of two MFMA steps
  f32x16 total[NC][NB], acc[K::ACC][NC][NB];
  // The wavefront's columns lie in one group of 128 of the table, or in two: those from `border` on have the second scale.
  const int first = w0 + min(wc * K::CW, w_last - w0), border = 128 - first % 128;
  float scale[NB], scale2[NB], sw = 0.f, sw2 = 0.f;
  const uint64_t wscales = reinterpret_cast<uint64_t>(f.W_scales) + static_cast<uint64_t>(first / 128) * G * 4;
  const int64_t more = first / 128 < w_last / 128 ? G : 0;
  int block_k = rot;                                      // the block of the walk's t-th step
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < NB; ++i) total[c][i] = f32x16{};

  auto fetch = [&](auto qq, uint32_t stage) {             // chunks 2 q and 2 q + 1: 16 k for each half of the wavefront
    constexpr int Q = decltype(qq)::value;
    const int slot = ((Q * 2 + lg) ^ ((ln >> 1) & 7)) * 16;
#pragma unroll
    for (int i = 0; i < NB; ++i) raw[Q & 1][i] = *reinterpret_cast<const u32x4*>(At + stage * K::AB + i * 4096 + slot);
#pragma unroll
    for (int c = 0; c < NC; ++c) raw[Q & 1][NB + c] = *reinterpret_cast<const u32x4*>(Bt + stage * K::BB + c * 4096 + slot);
  };
  auto convert = [&](auto step, auto from, auto to) {     // operands [from, to) of a step (of 8 in a block)
    constexpr int Q = decltype(step)::value / 2, E = decltype(step)::value % 2;
#pragma unroll
    for (int f = decltype(from)::value; f < decltype(to)::value; ++f) op[E][f] = to_f16(raw[Q & 1][f][2 * E], raw[Q & 1][f][2 * E + 1]);
  };
  auto add_up = [&](int c, int i) __attribute__((always_inline)) {       // the last block's sums, under its scale
#pragma unroll
    for (int q = 0; q < 4; ++q) {                         // (four neighbouring columns each)
      const float s = !BORDERS || c * 32 + q * 8 + lg * 4 < border ? scale[i] : scale2[i];
#pragma unroll
      for (int e = q * 4; e < q * 4 + 4; ++e)
        total[c][i][e] = __fmaf_rn(K::ACC == 2 ? acc[0][c][i][e] + acc[K::ACC - 1][c][i][e] : acc[0][c][i][e], s, total[c][i][e]);
    }
  };

  // Eight steps of 16 k make a block.  Between a step's MFMAs the next step's operands are converted, in a block's first step the sums of
  // the block before are added up, and behind the barrier the loads of a later block are issued, one or two at a time.  Every other step begins
  // with the reads of the next two steps' codes, which are converted behind its last MFMAs.  The barrier stands before the last step: all
  // codes of this block are in registers then, the next block has to be in LDS, and this block's stage is free.
  // (steps 1 to 7 of block t and step 0 of the next one: what a loop carries along is the MFMAs' own then)
  auto step = [&](auto which, int t, int coming, int loaded, uint32_t stage, uint32_t next, auto begins, auto last) {
    constexpr bool FIRST = decltype(begins)::value, LAST = decltype(last)::value;
      constexpr int X = decltype(which)::value, Q = X / 2, E = X % 2;
      if constexpr (X == 6 && !LAST) {
        hard_fence();
        if (t + S - 1 < count) wait_loads<(S - 2) * K::ALL>();      // h and W of blocks t + 2 .. t + S - 1 may be on their way
        else wait_loads<0>();
        clear_end(coming, next);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        hard_fence();
      }
      if constexpr (E == 0 && !(LAST && Q == 3)) fetch(IntT<(Q + 1) % 4>{}, Q == 3 ? next : stage);
      if constexpr (X == 4) {
        const float* const at = St + t / 4 % K::GROUPS * (K::GB / 4) + t % 4;
#pragma unroll
        for (int i = 0; i < NB; ++i) scale[i] = at[i * 128];
        // W's, alike for the whole wavefront, by way of the scalar cache: there before the seventh step, which waits for all of these
        const auto* const column = reinterpret_cast<const __attribute__((address_space(4))) float*>(wscales);
        sw = column[block_k];
        if (BORDERS) sw2 = column[more + block_k];
      }
      __builtin_amdgcn_sched_barrier(0);
      constexpr int NM = NC * NB, NF = NB + NC;
      if constexpr (X == 6 && !LAST) ragged_end(loaded, false);
      static_for<NM>([&](auto mm) {
        constexpr int M = decltype(mm)::value, c = M / NB, i = M % NB;
        if constexpr (X == 0 && !FIRST) add_up(c, i);
        f32x16& sum = acc[K::ACC == 2 ? E : 0][c][i];
        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(op[E][NB + c], op[E][i], X < K::ACC ? f32x16{} : sum, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (X >= 6 && !LAST) {
          constexpr int SLOT = (X - 6) * NM + M, FROM = K::ALL * SLOT / (2 * NM), TO = K::ALL * (SLOT + 1) / (2 * NM);
          if (t + S < count) {
            if constexpr (SLOT == 0) load_scales(t + S);
            static_for<TO - FROM>([&](auto j) { load(IntT<FROM + decltype(j)::value>{}, loaded, stage); });
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        constexpr int FROM = NF * M / NM, TO = NF * (M + 1) / NM;
        if constexpr (TO > FROM && !(LAST && X == 7)) convert(IntT<(X + 1) % 8>{}, IntT<FROM>{}, IntT<TO>{});
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (X == 7) {
        if constexpr (!LAST) ragged_end(loaded, true);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if (BORDERS) scale2[i] = scale[i] * sw2;
          scale[i] *= sw;
        }
      }
  };
  auto block = [&](int t, int coming, int loaded, uint32_t stage, uint32_t next, auto last) {
    static_for<7>([&](auto x) { step(IntT<decltype(x)::value + 1>{}, t, coming, loaded, stage, next, FalseT{}, last); });
    if constexpr (!decltype(last)::value) step(IntT<0>{}, t + 1, coming, loaded, next, next, FalseT{}, FalseT{});
  };

  int loaded = rot, coming = after(rot);                  // blocks to be loaded next, and to be multiplied next but one
  static_for<S>([&](auto t) {
    constexpr int T = decltype(t)::value;
    if (T < count) {
      ragged_end(loaded, false);
      load_scales(T);
      static_for<K::ALL>([&](auto q) { load(q, loaded, T); });
      ragged_end(loaded, true);
      loaded = after(loaded);
    }
  });
  if (count >= S) wait_loads<(S - 1) * K::ALL>();
  else wait_loads<0>();
  clear_end(rot, 0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  hard_fence();
  fetch(IntT<0>{}, 0);
  convert(IntT<0>{}, IntT<0>{}, IntT<NB + NC>{});
  step(IntT<0>{}, 0, 0, 0, 0, 0, TrueT{}, FalseT{});
  uint32_t stage = 0;
#pragma unroll 1
  for (int t = 0; t < count - 1; ++t) {
    const uint32_t next = stage + 1 == S ? 0 : stage + 1;
    block(t, coming, loaded, stage, next, FalseT{});
    stage = next;
    block_k = coming;
    coming = after(coming);
    loaded = after(loaded);
  }
  block(count - 1, 0, 0, stage, stage, TrueT{});
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < NB; ++i) add_up(c, i);
  if constexpr (K::WK > 1) {
    // the parts of k are joined in the stages' place, in order
    if (count < (KT + K::WK - 1) / K::WK) __builtin_amdgcn_s_barrier();        // a block less: the others have one more of its barriers
    f32x4* const sums = reinterpret_cast<f32x4*>(whole) + (wave * NC * NB * 4) * 64 + lane;
    constexpr int STRIDE = K::NW * NC * NB * 4 * 64;
    __syncthreads();
    if (part > 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sums[(part - 1) * STRIDE + ((c * NB + i) * 4 + q) * 64] = f32x4{total[c][i][q * 4], total[c][i][q * 4 + 1], total[c][i][q * 4 + 2], total[c][i][q * 4 + 3]};
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 0; p < K::WK - 1; ++p)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 v = sums[p * STRIDE + ((c * NB + i) * 4 + q) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) total[c][i][q * 4 + e] += v[e];
          }
  }

  // ---- logits: a lane has a window row, a register a column --------------------------------------------------
#pragma unroll
  for (int i = 0; i < K::RBW; ++i) {
    const int dest = row_dest(a, mine[i]);
    if (dest < 0) continue;
    float* const row = a.z + static_cast<int64_t>(dest) * a.n;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = col_base + wc * K::CW + c * 32 + q * 8 + lg * 4;
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          z[e] = processed_logit<C>(a, total[c][i * C][q * 4 + e], total[c][i * C + C - 1][q * 4 + e]);
        if (col >= 0 && col + 3 < a.n) store4(row + col, z[0], z[1], z[2], z[3]);
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e >= 0 && col + e < a.n) row[col + e] = z[e];
        }
      }
  }
}

// ---- the shape of workgroups for a call -------------------------------------------------------------------------
template <class K, class F>
void with(F&& go) { go(K{}); }
template <class K>
int64_t tiles_of(const LmHeadArgs& a, int v_lo) {
  return ((v_lo % 4 + static_cast<int64_t>(a.n) + K::BN - 1) / K::BN) * ((static_cast<int64_t>(a.B) * a.L + K::RB * 32 - 1) / (K::RB * 32));
}

template <int C, class F>
void choose_of(const LmHeadArgs& a, int v_lo, F&& go) {
  // 256 and 128 rows of h: a wavefront has 64 x 64 logits, which keeps its conversions below what the MFMAs hide.  64 rows: a stream of W, three
  // stages in each of two workgroups on a compute unit; narrow tiles with k in four parts where the others leave compute units idle (a
  // wavefront's chain of MFMAs is what a call of few tiles waits for).
  using Large = Fp8Cfg<C, 8 / C, 128, 2, 4, 3>;            // one workgroup on a compute unit
  using Medium = Fp8Cfg<C, 4 / C, 128, 2, 2, 2>;           // two
  using Few = Fp8Cfg<C, 2 / C, 128, 4, 1, 3>;              // two
  using FewParts = Fp8Cfg<C, 2 / C, 64, 2, 1, 2, 4>;       // one
  const int64_t rows = static_cast<int64_t>(a.B) * a.L * C;
  // W is read once, and larger than what the last cache keeps from one call to the next: past the caches 32 x 2 rows x 65536 x 4096 take 56 us, 58
  // by way of them, one row 54 and 58 (before other changes)
  const bool past = static_cast<int64_t>(a.n) * a.d >= (1 << 28);
  if constexpr (C == 1) {
    if (rows <= 32) {
      // Four parts of k while every compute unit has a workgroup of them (d > 384: a block of k for each part), one part of twice as many beyond.
      // One row, tables from memory, four parts and one (us): d = 512: 16384 ids 6.8 and 7.1, 16449 10.1 and 7.9, 32768 11.5 and 9.1; d = 1280: 8192 ids 8.7
      // and 10.2, 16384 9.9 and 10.5, 16449 14.9 and 12.4, 32768 17.6 and 13.6, 65000 32 and 19; d = 4096: 8192 ids 13.8 and 22.5, 16384 18.0 and 23.2,
      // 16449 26.8 and 28.2, 24000 29.1 and 29.3, 32768 33.0 and 30.2, 65000 60 and 53.  32 rows are alike; the choice is within 6 % of
      // the better one everywhere.
      if (tiles_of<Fp8Cfg<1, 1, 64, 2, 1, 3, 4>>(a, v_lo) <= 256 && a.d > 384) with<Fp8Cfg<1, 1, 64, 2, 1, 3, 4>>(go);
      else past ? with<Fp8Cfg<1, 1, 64, 2, 1, 3, 1, true>>(go) : with<Fp8Cfg<1, 1, 64, 2, 1, 3>>(go);
      return;
    }
  }
  // What rounds of tiles over 256 compute units take, measured at d = 4096 (us, 64 to 512 rows with guidance x 500 to 8000 ids): a round of the larger
  // shape 50 to 65, of two smaller tiles per compute unit 67, of one 35 to 42, of two streams 43, of one 26 to 30, of parts 14 each behind the
  // first.  64 x 2 rows x 1000: 50, 35, 26, 14 us; 512 x 2 x 8000: 65, 67, 83, 111.  Other lengths stand to each other alike: at d = 1024 16, 12, 9, 7 and 21, 21,
  // 25, 49 us, at d = 128 (no parts) 5.5, 5.2, 4.2 and 9.2, 8.9, 10.7.  Over 32 to 512 rows with guidance x 1000 to 16000 ids x d = 128 to 4096 the shape
  // that is chosen is within 8 % of the best of the four.
  auto halves = [](int64_t tiles, double two, double one) {
    const int64_t rest = tiles % 512;
    return static_cast<double>(tiles / 512) * two + (rest == 0 ? 0.0 : rest <= 256 ? one : two);
  };
  const double large = 62.0 * static_cast<double>((tiles_of<Large>(a, v_lo) + 255) / 256), medium = halves(tiles_of<Medium>(a, v_lo), 67.0, 42.0),
               few = halves(tiles_of<Few>(a, v_lo), 43.0, 29.5),
               parts = a.d > 384 ? 2.5 + 14.2 * static_cast<double>((tiles_of<FewParts>(a, v_lo) + 255) / 256) : 1e300;
  const double least = std::min(std::min(large, medium), std::min(few, parts));
  if (least == large) with<Large>(go);
  else if (least == medium) past && rows <= 128 ? with<Fp8Cfg<C, 4 / C, 128, 2, 2, 2, 1, true>>(go) : with<Medium>(go);
  else if (least == few) past && rows <= 64 ? with<Fp8Cfg<C, 2 / C, 128, 4, 1, 3, 1, true>>(go) : with<Few>(go);
  else with<FewParts>(go);
}
template <class F>
void choose(const LmHeadArgs& a, int v_lo, F&& go) {
  a.C == 2 ? choose_of<2>(a, v_lo, go) : choose_of<1>(a, v_lo, go);
}

// ---- weights in 8 bits ---------------------------------------------------------------------------------------------
// A workgroup takes a block of 128 x 128 of the table: 16 lanes to a row, eight elements each, eight rows of a thread.  Bound by memory: 65536 x 4096 take
// 146 us (805 MB: 5.5 TB/s), 16384 x 1280 12.2.
__global__ __launch_bounds__(256) void quantize_fp8_kernel(const uint16_t* __restrict__ W, int V, int d, uint8_t* __restrict__ codes,
                                                           float* __restrict__ scales) {
  __shared__ uint32_t ex[4];
  const int p = blockIdx.x * 16 + threadIdx.x % 16, pieces = d / 8;
  for (int group = blockIdx.y; group < (V - 1) / 128 + 1; group += gridDim.y) {
    Eight<false> v[8];
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = static_cast<int64_t>(group) * 128 + i * 16 + threadIdx.x / 16;
      const bool there = row < V && p < pieces;
      v[i] = load_eight<false>(W, there ? row * pieces + p : 0);
      most = max(most, there ? largest_bits(v[i].wide()) : 0u);
    }
    most = wave_max_u32(most);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) ex[threadIdx.x >> 6] = most;
    __syncthreads();
    const E4M3Scale s = e4m3_scale(fold_max<4>(ex));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = static_cast<int64_t>(group) * 128 + i * 16 + threadIdx.x / 16;
      if (row < V && p < pieces) reinterpret_cast<uint2*>(codes)[row * pieces + p] = to_e4m3(v[i].wide(), s);
    }
    if (threadIdx.x == 0) scales[static_cast<int64_t>(group) * gridDim.x + blockIdx.x] = s.scale;
  }
}

}  // namespace

namespace {
struct Grid {
  int64_t WT, MT, groups;
};
template <class K>
Grid grid_of(const LmHeadArgs& a, int v_lo) {
  const int64_t WT = (v_lo % 4 + static_cast<int64_t>(a.n) + K::BN - 1) / K::BN, MT = (static_cast<int64_t>(a.B) * a.L + K::RB * 32 - 1) / (K::RB * 32);
  return {WT, MT, (WT + 7) / 8 * 8 * MT};
}
}  // namespace

bool lm_head_fp8_fits(const LmHeadArgs& a, int v_lo) {
  bool fits = false;
  choose(a, v_lo, [&](auto k) {
    using K = decltype(k);
    fits = grid_of<K>(a, v_lo).groups * K::THREADS < static_cast<int64_t>(1) << 32;      // a launch's threads
  });
  return fits;
}

hipError_t launch_lm_head_fp8(const LmHeadArgs& a, const float* h_scales, const uint8_t* W, const float* W_scales, int v_lo, hipStream_t s,
                              hipEvent_t ev_start, hipEvent_t ev_stop) {
  const LaunchEvents ev{ev_start, ev_stop};
  const Fp8Args f{a, h_scales, W, W_scales, v_lo};
  choose(a, v_lo, [&](auto k) {
    using K = decltype(k);
    const Grid g = grid_of<K>(a, v_lo);
    launch_kernel(v_lo % 64 != 0 ? lm_head_fp8_kernel<K, true> : lm_head_fp8_kernel<K, false>, dim3(static_cast<unsigned>(g.groups)),
                  dim3(K::THREADS), s, ev, f, static_cast<int>(g.WT), static_cast<int>(g.MT));
  });
  return hipGetLastError();
}

int lm_head_fp8_kernel_name(const LmHeadArgs& a, int v_lo, char* buf, size_t cap) {
  int len = 0;
  choose(a, v_lo, [&](auto k) { len = decltype(k)::name(buf, cap, v_lo % 64 != 0); });
  return len;
}

hipError_t launch_quantize_fp8(const uint16_t* W, int V, int d, uint8_t* codes, float* scales, hipStream_t s) {
  hipLaunchKernelGGL(quantize_fp8_kernel, dim3((d + 127) / 128, (V - 1) / 128 + 1 > 65535 ? 65535 : (V - 1) / 128 + 1), dim3(256), 0, s, W, V, d,
                     codes, scales);
  return hipGetLastError();
}

}  // namespace scd
