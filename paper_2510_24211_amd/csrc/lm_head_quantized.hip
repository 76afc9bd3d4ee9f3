// LM head over 4-bit weights:
//   W[v, k] = s[v, k / G] * (q[v, k] - o[v, k / G])        q in 0 .. 15, s bf16, o = 8 or a zero point of 0 .. 15
//   logit[m, v] = sum_k h[m, k] * W[v, k]                   then guidance mix and temperature as in the bf16 LM head
//
// A code becomes the bf16 number 16 + q by one shift and one bitwise operation for two of them (q is put behind the leading
// mantissa bit), so the products go to the matrix units exactly:
//   sum over a group of h * (q - o) = sum h * (16 + q) - (16 + o) * sum h.
// The second sum is taken once per workgroup, by whoever loaded the rows.  It goes to the matrix units too, split into three
// bf16 terms of 8 bits each that hold all 24, times -(16 + o), which bf16 holds: one more MFMA for each four (C operands of that
// value would cost four times the LDS reads).  After every block of 64 k, or half of one where groups end inside, the accumulators are scaled
// and added to the fp32 logits, whatever the group's length: no weight is ever rounded.
//
// Layout.  Columns in tiles of 32, k in blocks of 64: a block of a tile is 1 KB, 16 bytes for each lane of a wavefront, which
// are its operands of four 32x32x16 MFMAs (lane l: column l % 32; word j: k = 16 j + 8 (l / 32) + 0 .. 7, even k in
// the low half, odd k in the high half of the word).  The blocks of a tile follow each other; behind all of them, per tile
// and group, the 32 columns' scales (2 bytes each; with zero points 4, the second two holding 16 + o as bf16).
//
// A workgroup of NW wavefronts owns NC * NW / (WK * WR) neighbouring column tiles, NC per wavefront; WK wavefronts share tiles and
// rows and take 1/WK of k each (their sums are added up at the end in a fixed order), WR share tiles and take a part of the rows
// each.  Weights and h rows go from memory straight into LDS, S stages deep.  The scales of the workgroup's columns are fetched whole at
// the start.
//   Bound by instruction issue: 32 rows with guidance x 65536 ids over 4096, groups of 128, take 54 to 58 us, of which the loads alone would take
// 25 to 30 (142 MB); a wavefront issues about 220 vector instructions per step of two tiles (64 convert codes, 64 scale, 30 add rows up) beside 20 MFMAs, and the
// matrix pipes are busy a quarter of the time.  With the offsets taken off by a product with ones it took 75, as C operands from LDS 63.
// The bf16 head takes 82 there.  Shorter groups bring more scales, which shut out the faster shapes of workgroups: groups of 64 take 64 us, with zero points
// 75, of 32 83, with zero points 231.  Batches are slower than the bf16 head too (480 rows with guidance x 8191: 114 to 117 us against 60):
// codes are converted by each of the four wavefronts that share columns.
#include "launch_events.h"
#include "lm_head_rows.h"
#include "tile_loads.h"

#include <stdio.h>

namespace scd {
namespace {

constexpr int kTileCols = 32, kBlockK = 64, kBlockBytes = 1024, kTilesPad = 8;

// rows per block of 32 that are really loaded: HRB; blocks of rows (guidance included) per wavefront: NB; KB of LDS it may take: KB
template <int C_, int RB_, int HRB_, int NC_, int NW_, int WK_, int KB_, int WR_ = 1>
struct QuantCfg {
  static constexpr int C = C_, RB = RB_, HRB = HRB_, NC = NC_, NW = NW_, WK = WK_, WR = WR_, LDS = KB_ * 1024;
  static int name(char* buf, size_t cap, int step, bool zeros) {
    return snprintf(buf, cap, "lm_head_quantized_kernel<QuantCfg<%d, %d, %d, %d, %d, %d, %d, %d>, %d, %s>", C, RB, HRB, NC, NW, WK, KB_, WR, step,
                    zeros ? "true" : "false");
  }
  static constexpr int THREADS = NW * 64, WC = NW / WK / WR, COLTILES = WC * NC, NB = RB * C / WR;
  static constexpr int HROWS = RB * C * HRB;             // h rows per part of k
  static constexpr int HI = WK * HROWS / 8;              // load instructions for the h rows of a step, all parts
  static constexpr int HL = (HI + NW - 1) / NW;          // per wavefront
  static constexpr int WP = COLTILES * WK, WL = (WP + NW - 1) / NW;      // blocks of weights of a step, per wavefront to be loaded
  static constexpr int WB = WP * kBlockBytes, HB = WK * HROWS * 128, STAGE = WB + HB;
  static constexpr int FIT = (LDS - LDS / 6) / STAGE, S = FIT > 7 ? 7 : FIT;
  static constexpr int RED = WK > 1 ? NW * NC * NB * 16 * 64 * 4 : 0;      // sums of the parts of k, in the place of the stages
  static constexpr int BASE = S * STAGE > RED ? S * STAGE : RED;
  static constexpr int TABLE = RB * 32 * 4;
  static constexpr int SUMS = 2 * WK * 2 * HROWS * 8;    // rows' sums of two steps, of the halves of a block
  static constexpr int SCALES = LDS - TABLE - SUMS - BASE;          // room for the columns' scales
  static_assert(NW % 2 == 0 && S >= 3 && SCALES >= COLTILES * 1024 && RB % WR == 0 && (WK == 1 || WR == 1), "LDS");
};

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// the eight codes of a word as bf16 numbers 16 + q
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t w) {
  auto two = [](uint32_t x) -> uint32_t { return __builtin_amdgcn_bitop3_b32(x, 0x00780078u, 0x41804180u, 0xEA); };      // (x & mask) | sixteen
  return u32x4{two(w << 3), two(w >> 1), two(w >> 5), two(w >> 9)};
}

// STEP: MFMAs between two applications of a scale (2: groups that end inside a block of k, 4: they do not)
template <class K, int STEP, bool ZEROS>
__global__ __launch_bounds__(K::THREADS) void lm_head_quantized_kernel(const LmHeadArgs a, const QuantizedArgs q, const int WT, const int MT) {
  constexpr int C = K::C, RB = K::RB, NB = K::NB, NC = K::NC, WL = K::WL, WR = K::WR, WK = K::WK, WC = K::WC, NW = K::NW;
  constexpr int S = K::S, HL = K::HL, HRB = K::HRB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[K::LDS];
  int* const table = reinterpret_cast<int*>(lds + K::BASE);
  uint2* const hsum = reinterpret_cast<uint2*>(lds + K::BASE + K::TABLE);     // [2][WK][2][HROWS]
  unsigned char* const slab = lds + K::BASE + K::TABLE + K::SUMS;
  // workgroups that share columns get ids 8 apart: the same XCD, the same L2
  const int id = blockIdx.x, mt = (id / 8) % MT, wt = id / (8 * MT) * 8 + id % 8;
  if (wt >= WT) return;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wave % WC, wr = wave / WC % WR, part = wave / (WC * WR);
  const int rows = a.B * a.L, p_base = mt * RB * 32, d = a.d;
  const int tile = (wt * WC + wc) * NC;                  // first column tile (the layout is padded to whole workgroups)
  const int KB = (d + kBlockK - 1) / kBlockK;
  const int nch = d % kBlockK / 8;                       // 16-byte chunks of a ragged last block, 0: there is none
  auto first_block = [&](int p) { return KB * p / WK; };
  const int T = (KB + WK - 1) / WK;                      // steps
  const int kb0 = first_block(part), count = first_block(part + 1) - kb0;
  const RowState mine = row_state(a, p_base + min(tid, RB * 32 - 1));

  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds));
  // ---- scales of the workgroup's columns ---------------------------------------------------------------
  constexpr int esize = ZEROS ? 4 : 2;
  const int tile_scales = q.groups * kTileCols * esize;
  {
    const uint64_t from = reinterpret_cast<uint64_t>(q.scales) + static_cast<uint64_t>(wt) * K::COLTILES * tile_scales;
    const int pieces = (K::COLTILES * tile_scales + 1023) / 1024;
    for (int i = wave; i < pieces; i += NW)
      load_lds16<false, 0>(from + static_cast<uint64_t>(i) * 1024, lane * 16, lds0 + K::BASE + K::TABLE + K::SUMS + i * 1024);
  }
  // ---- loads of a step: this wavefront's block of weights, its share of the h rows ---------------------------
  const uint64_t wbase = reinterpret_cast<uint64_t>(q.codes) + static_cast<uint64_t>(wt) * K::COLTILES * KB * kBlockBytes;
  const int h0 = first_h_row(p_base, C, a.L);
  const uint64_t hbase = reinterpret_cast<uint64_t>(a.h) + static_cast<uint64_t>(h0) * d * 2;
  // the chunk that a lane loads into slot lane % 8 of its row; the rows of its pieces are 8 NW apart: one swizzle
  const int hchunk = (lane & 7) ^ ((((K::HROWS > 8 ? wave & 1 : 0) * 8 + (lane >> 3)) >> 1) & 7);
  // Fewer pieces of h rows than wavefronts: the others load weights alone.  (Two that loaded a piece alike would not do: the one might clear
  // the end of a ragged block and add its rows up while the other's load is still to land.)
  const bool loads_h = K::HI >= NW || wave < K::HI;
  static_assert(K::HI < NW || K::HI % NW == 0, "pieces per wavefront");
  int hpart[HL];
  uint32_t hoff[HL], hlds[HL];
#pragma unroll
  for (int i = 0; i < HL; ++i) {
    const int piece = (wave + i * NW) % K::HI;
    const int r = piece % (K::HROWS / 8) * 8 + (lane >> 3), blk = r / HRB;
    hpart[i] = piece / (K::HROWS / 8);
    hoff[i] = static_cast<uint32_t>(h_row(min(p_base + (blk / C) * 32, rows - 1), r % HRB, blk % C, C, a.L, rows) - h0) *
                  static_cast<uint32_t>(d) * 2u +
              hchunk * 16;
    hlds[i] = lds0 + K::WB + piece * 1024;
  }
  // Every part walks its blocks cyclically from a start of the workgroup's own: rows of h are d * 2 bytes apart, and from one
  // start all of the chip would ask for the same address bits at the same time.  `at`: the block's index in its part; a part may
  // have one block less than T, and loads some other in its place.
  const int rot = wt * 5 % T;
  auto next_of = [&](int at) { return at + 1 == T ? 0 : at + 1; };
  int hfirst[HL];
#pragma unroll
  for (int i = 0; i < HL; ++i) hfirst[i] = first_block(hpart[i]);
  auto load_h = [&](int at, int stage) __attribute__((always_inline)) {
    if (!loads_h) return;
    static_for<HL>([&](auto ii) {
      constexpr int i = decltype(ii)::value;
      const int kb = __builtin_amdgcn_readfirstlane(min(hfirst[i] + at, KB - 1));
      uint32_t off = hoff[i];
      if (nch && kb == KB - 1) off -= max(hchunk - (nch - 1), 0) * 16;
      load_lds16<false, 0>(hbase + static_cast<uint32_t>(kb) * 128u, off, __builtin_amdgcn_readfirstlane(hlds[i]) + stage * K::STAGE);
    });
  };
  auto load_w = [&](int at, int stage) __attribute__((always_inline)) {
    static_for<WL>([&](auto ii) {
      const int piece = (wave * WL + decltype(ii)::value) % K::WP;       // (more wavefronts than blocks: some are loaded twice, alike)
      const int kb = __builtin_amdgcn_readfirstlane(min(first_block(piece / K::COLTILES) + at, KB - 1));
      load_lds16<false, 0>(wbase + (static_cast<uint64_t>(piece % K::COLTILES) * KB + kb) * kBlockBytes, lane * 16,
                           lds0 + piece * kBlockBytes + stage * K::STAGE);
    });
  };
  // the ragged block: chunks past the end are zeroed by the wavefront that loaded something in their place
  auto clear_ragged = [&](int at, int stage) __attribute__((always_inline)) {
    if (!loads_h) return;
#pragma unroll
    for (int i = 0; i < HL; ++i)
      if (hfirst[i] + at >= KB - 1 && hchunk >= nch)
        *reinterpret_cast<u32x4*>(lds + (hlds[i] - lds0) + stage * K::STAGE + lane * 16) = u32x4{0u, 0u, 0u, 0u};
  };

  // Sums of the h rows that this wavefront loaded: 8 lanes hold a row's block of k, 4 a half.
  auto add_rows = [&](int parity, int stage) __attribute__((always_inline)) {
    if (!loads_h) return;
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
#pragma unroll
    for (int i = 0; i < HL; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(lds + (hlds[i] - lds0) + stage * K::STAGE + lane * 16);
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = v[e];           // (a bit cast of the element itself takes the vector's first)
        s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, s, false);
      }
      // chunk c of the row sits in slot c ^ swizzle: the lanes of a half are those whose slots differ in the low two bits
      s += dpp_f32<kDppXor1>(s);
      s += dpp_f32<kDppXor2>(s);
      if (STEP == 4) s += dpp_f32<kDppHalfMirror>(s);
      const uint32_t first = __float_as_uint(s) & 0xFFFF0000u;
      const float r1 = s - __uint_as_float(first);
      const uint32_t second = __float_as_uint(r1) & 0xFFFF0000u;
      const float r2 = r1 - __uint_as_float(second);
      const int r = (hlds[i] - lds0 - K::WB) / 128 % K::HROWS + (lane >> 3);
      uint2* const to = hsum + (parity * WK + hpart[i]) * 2 * K::HROWS + r;
      const uint2 terms = make_uint2(first >> 16 | second, __float_as_uint(r2) >> 16);
      if (STEP == 4) {
        if ((lane & 7) == 0) to[0] = terms;
      } else {
        if ((lane & 3) == 0) to[(hchunk >> 2) * K::HROWS] = terms;
      }
    }
  };

  // What a step starts with, in registers: the weights' codes, the h rows' operands of the first half and, per half block with
  // STEP = 2, the terms of this lane's rows' sums and the scales (and zero points).
  constexpr int PER = 4 / STEP;
  struct Operands {
    u32x4 w[NC], h[2][NB];
    uint2 rows[PER][NB];
    uint32_t scale[PER][NC];
  };
  const int per_group = q.group / 32;                    // half blocks of k
  int g = 0, left = 0;                                   // group of the next half block; of it, left
  auto group_at = [&](int kb) __attribute__((always_inline)) {
    g = kb * 2 / per_group;
    left = per_group - kb * 2 % per_group;
  };
  const unsigned char* const hrows = lds + K::WB + (part * K::HROWS + wr * NB * HRB + ln % HRB) * 128;
  const unsigned char* const scales = slab + wc * NC * q.groups * (kTileCols * esize) + ln * esize;
  uint32_t hslot[4];                                     // of the first block's rows; rows 8 apart differ in bit 2 of the swizzle
#pragma unroll
  for (int j = 0; j < 4; ++j) hslot[j] = ((2 * j + lg) ^ ((ln % HRB >> 1) & 7)) * 16;
  auto read_h = [&](int stage, int j, int i) __attribute__((always_inline)) {
    const uint32_t slot = HRB == 8 && (i & 1) ? hslot[j] ^ 64u : hslot[j];
    return *reinterpret_cast<const u32x4*>(hrows + stage * K::STAGE + i * HRB * 128 + slot);
  };
  auto fetch = [&](int parity, int stage, uint32_t keep, Operands& x) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NC; ++c) x.w[c] = *reinterpret_cast<const u32x4*>(lds + stage * K::STAGE + (part * K::COLTILES + wc * NC + c) * kBlockBytes + lane * 16);
#pragma unroll
    for (int half = 0; half < PER; ++half) {
      const uint2* const hs = hsum + ((parity * WK + part) * 2 + half) * K::HROWS + wr * NB * HRB + ln % HRB;
#pragma unroll
      for (int i = 0; i < NB; ++i) x.rows[half][i] = hs[i * HRB];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        // (a half past the end of k has no group: its sums are zeros)
        const unsigned char* const from = scales + (c * q.groups + min(g, q.groups - 1)) * (kTileCols * esize);
        x.scale[half][c] = (ZEROS ? *reinterpret_cast<const uint32_t*>(from) : *reinterpret_cast<const uint16_t*>(from)) & keep;
      }
      left -= STEP / 2;
      if (left == 0) {
        ++g;
        left = per_group;
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < NB; ++i) x.h[j][i] = read_h(stage, j, i);
  };
  f32x16 sum[NC][NB];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < NB; ++i) sum[c][i] = f32x16{};
  // Products of a group and column tile go to one set of accumulators while those of the one before are scaled and added up in
  // the other, between the MFMAs: the wavefronts run in step, so what one does not overlap by itself is hardly overlapped at all.
  constexpr int SETS = NC * PER > 1 ? 2 : 1;
  auto compute = [&](const Operands& x, const u32x4 (&later)[2][NB], auto&& midway) __attribute__((always_inline)) {
    f32x16 acc[SETS][NB];
    float scale = 0.f;
    static_for<NC * PER>([&](auto pp) __attribute__((always_inline)) {
      constexpr int P = decltype(pp)::value, c = P / PER, half = P % PER, SET = P % SETS, BEFORE = (P + NC * PER - 1) % (NC * PER) / PER;
      const uint32_t o = ZEROS ? (x.scale[half][c] >> 16 ^ 0x8000u) : 0xC1C0u;  // -(16 + o): -24 without zero points
      u32x4 b{lg == 0 ? o | o << 16 : 0u, lg == 0 ? o : 0u, 0u, 0u};
      if constexpr (P > 0 && P == NC * PER - 1) midway();
      constexpr int M = (STEP + 1) * NB;
      static_for<M>([&](auto mm) __attribute__((always_inline)) {
        constexpr int m = decltype(mm)::value, j = half * STEP + m / NB - 1, i = m % NB;
        if constexpr (m < NB) acc[SET][i] = mfma(u32x4{x.rows[half][i].x, x.rows[half][i].y, 0u, 0u}, b, f32x16{});
        else acc[SET][i] = mfma(j < 2 ? x.h[j & 1][i] : later[j & 1][i], b, acc[SET][i]);
        if constexpr (i == NB - 1 && m < M - 1) b = codes_to_bf16(x.w[c][j + 1]);
        if constexpr (P > 0) {
          constexpr int E0 = NB * 16 * m / M, E1 = NB * 16 * (m + 1) / M;
          static_for<E1 - E0>([&](auto ee) __attribute__((always_inline)) {
            constexpr int e = E0 + decltype(ee)::value;
            sum[BEFORE][e / 16][e % 16] = __builtin_fmaf(scale, acc[SETS - 1 - SET][e / 16][e % 16], sum[BEFORE][e / 16][e % 16]);
          });
          __builtin_amdgcn_sched_barrier(0);
        }
      });
      scale = __uint_as_float(x.scale[half][c] << 16);
    });
    if constexpr (NC * PER == 1) midway();
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[NC - 1][i][e] = __builtin_fmaf(scale, acc[SETS - 1][i][e], sum[NC - 1][i][e]);
  };

  // Step t.  Its barrier says that the wavefronts are done with step t - 1 and that step t + 1's rows and their sums are in LDS, whose
  // first operands are fetched under this step's MFMAs.  The rows of step t + S - 1 go to the stage of step t - 1, and the weights
  // of step t + S to stage t, whose weights are in registers: they come from further away.  Late in the step
  // the rows of step t + 2, loaded by then, are added up.
  // all loads issued by step t but those behind the rows and weights of step t + 2
  auto wait_early_loads = [&]() __attribute__((always_inline)) {
    if (loads_h) wait_loads<(S - 3) * HL + (S - 2) * WL>();
    else wait_loads<(S - 2) * WL>();
  };
  int h_ahead = rot, w_ahead = rot;                      // indices of the blocks to be loaded next
#pragma unroll
  for (int t = 0; t < S; ++t) {
    if (t < S - 1 && t < T) {
      load_h(h_ahead, t);
      h_ahead = next_of(h_ahead);
    }
    if (t < T) {
      load_w(w_ahead, t);
      w_ahead = next_of(w_ahead);
    }
  }
  // the rows and weights of steps 0 and 1
  if (S <= T) wait_early_loads();
  else wait_loads<0>();
  int now = rot, rows_at = rot;                          // indices of the blocks to be multiplied and to be added up next
#pragma unroll
  for (int t = 0; t < 2; ++t)
    if (t < T) {
      if (nch) clear_ragged(rows_at, t);
      add_rows(t, t);
      rows_at = next_of(rows_at);
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  hard_fence();
  // (what a part loads in the place of a block that it has not gets a scale of 0)
  auto keep = [&](int at) { return at < count ? 0xFFFFFFFFu : 0xFFFF0000u; };
  Operands x[2];
  group_at(kb0 + rot);
  fetch(0, 0, keep(now), x[0]);
  int stage = 0;
  auto step = [&](auto odd, int t) __attribute__((always_inline)) {
    constexpr int ODD = decltype(odd)::value;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    hard_fence();
    const int then = next_of(now), one = stage + 1 == S ? 0 : stage + 1, two = one + 1 == S ? 0 : one + 1, last = stage == 0 ? S - 1 : stage - 1;
    u32x4 later[2][NB];                                  // this step's rows of the second half, ahead of the next one's in LDS's queue
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < NB; ++i) later[j][i] = read_h(stage, j + 2, i);
    __builtin_amdgcn_sched_barrier(0);
    if (t + S - 1 < T) {
      load_h(h_ahead, last);
      h_ahead = next_of(h_ahead);
    }
    if (t + S < T) {
      load_w(w_ahead, stage);
      w_ahead = next_of(w_ahead);
    }
    if (then == 0) group_at(kb0);
    fetch(1 - ODD, one, keep(then), x[1 - ODD]);         // (behind the last step: something that nobody uses)
    compute(x[ODD], later, [&]() __attribute__((always_inline)) {
      if (t + 2 >= T) return;
      if (t + S < T) wait_early_loads();
      else wait_loads<0>();
      if (nch) clear_ragged(rows_at, two);
      add_rows(ODD, two);
      rows_at = next_of(rows_at);
    });
    now = then;
    stage = one;
  };
#pragma unroll 1
  for (int t = 0; t < T; t += 2) {
    step(IntT<0>{}, t);
    if (t + 1 < T) step(IntT<1>{}, t + 1);
  }
  // ---- the parts of k added up, guidance mix, temperature, z ----------------------------------------------------
  if (tid < RB * 32) table[tid] = row_dest(a, mine);
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);
  if constexpr (WK > 1) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) red[(((wave * NC + c) * NB + i) * 16 + e) * 64 + lane] = sum[c][i][e];
    __syncthreads();
  }
  static_assert(16 % WK == 0, "elements per part");
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int v = (tile + c) * kTileCols + ln;
    if (v >= a.n) continue;
#pragma unroll
    for (int r = 0; r < RB / WR; ++r)
#pragma unroll
      for (int ee = 0; ee < 16 / WK; ++ee) {
        // the wavefronts of a tile store a share of its elements each
        const int e = WK > 1 ? part + ee * WK : ee;
        float cond, uncond;
        if constexpr (WK > 1) {
          cond = uncond = 0.f;
#pragma unroll
          for (int p = 0; p < WK; ++p) {
            const float* const from = red + (((p * WC + wc) * NC + c) * NB + r * C) * 1024 + e * 64 + lane;      // (WR is 1)
            cond += from[0];
            uncond += from[(C - 1) * 1024];
          }
        } else {
          cond = sum[c][r * C][ee];
          uncond = sum[c][r * C + C - 1][ee];
        }
        const int row = table[(wr * (RB / WR) + r) * 32 + (e >> 2) * 8 + lg * 4 + (e & 3)];
        if (row >= 0) a.z[static_cast<int64_t>(row) * a.n + v] = processed_logit<C>(a, cond, uncond);
      }
  }
}

// ---- quantisation and layout ---------------------------------------------------------------------------
// A wavefront per row and group.  Without zero points s = max(largest / 7, -smallest / 8), with them s = (largest -
// smallest) / 15 over a range that holds 0; s is rounded to bf16 first, the codes are the nearest under the rounded one.  Once per table, and
// not tuned: 65536 x 4096 in groups of 128 580 to 630 us, of 64 1130, of 32 2000 (two passes over the group, 4 bytes per lane and load, a
// division per weight; 0.67 GB, 131 us at a copy's rate).
__global__ __launch_bounds__(256) void quantize_kernel(const uint16_t* __restrict__ W, int64_t items, int d, int group, int groups,
                                                       uint8_t* __restrict__ codes, uint16_t* __restrict__ scales, uint8_t* __restrict__ zeros) {
  const int lane = threadIdx.x & 63;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); item < items; item += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t v = item / groups;
    const int g = static_cast<int>(item - v * groups), k0 = g * group, k1 = min(k0 + group, d);
    const uint32_t* const row = reinterpret_cast<const uint32_t*>(W + v * d);       // two weights each
    float lo = 0.f, hi = 0.f;
    for (int k = k0 / 2 + lane; k < k1 / 2; k += 64) {
      const uint32_t two = row[k];
      const float x = __uint_as_float(two << 16), y = __uint_as_float(two & 0xFFFF0000u);
      lo = fminf(lo, fminf(x, y));
      hi = fmaxf(hi, fmaxf(x, y));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      lo = fminf(lo, __shfl_xor(lo, o, 64));
      hi = fmaxf(hi, __shfl_xor(hi, o, 64));
    }
    // (halves, exactly: the range of finite weights may not be finite)
    const __bf16 sb = static_cast<__bf16>(zeros ? __fdiv_rn(0.5f * hi - 0.5f * lo, 7.5f) : fmaxf(__fdiv_rn(hi, 7.f), __fdiv_rn(-lo, 8.f)));
    const float s = static_cast<float>(sb);
    const int zero = zeros && s > 0.f ? static_cast<int>(fminf(rintf(__fdiv_rn(-lo, s)), 15.f)) : 8;
    auto code = [&](float x) {
      return s > 0.f ? static_cast<uint32_t>(fminf(fmaxf(rintf(__fdiv_rn(x, s)) + static_cast<float>(zero), 0.f), 15.f))
                     : static_cast<uint32_t>(zero);
    };
    for (int k = k0 / 2 + lane; k < k1 / 2; k += 64) {
      const uint32_t two = row[k];
      codes[v * (d / 2) + k] = static_cast<uint8_t>(code(__uint_as_float(two << 16)) | code(__uint_as_float(two & 0xFFFF0000u)) << 4);
    }
    if (lane == 0) {
      scales[item] = __builtin_bit_cast(uint16_t, sb);
      if (zeros) zeros[item] = static_cast<uint8_t>(zero);
    }
  }
}

// A wavefront per column tile and block of k: 16 bytes per lane.  Once per table: 65536 x 4096 90 to 100 us (52 at a copy's rate; a lane gathers
// 4 bytes from each of four places of its row), the scales 8.  (Tables of 64 GiB have more of them than a launch has threads for.)
__global__ __launch_bounds__(256) void pack_codes_kernel(const uint8_t* __restrict__ codes, int n, int d, int KB, int64_t blocks,
                                                         u32x4* __restrict__ to) {
  const int lane = threadIdx.x & 63;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); item < blocks; item += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t v = item / KB * kTileCols + (lane & 31);
    const int k0 = static_cast<int>(item % KB) * kBlockK + (lane >> 5) * 8;
    u32x4 out{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + j * 16;
      if (v < n && k < d) {                       // d is a multiple of 8
        const uint32_t in = *reinterpret_cast<const uint32_t*>(codes + v * (d / 2) + k / 2);      // code t at bits 4 t
        uint32_t w = 0u;
#pragma unroll
        for (int t = 0; t < 8; ++t) w |= (in >> (4 * t) & 15u) << ((t & 1) * 16 + (t >> 1) * 4);
        out[j] = w;
      }
    }
    to[item * 64 + lane] = out;
  }
}
__global__ __launch_bounds__(256) void pack_scales_kernel(const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, int n, int groups,
                                                          int64_t count, void* __restrict__ to) {
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < count; at += static_cast<int64_t>(gridDim.x) * 256) {
    // at: (tile, group, column)
    const int64_t tile = at / (static_cast<int64_t>(groups) * kTileCols), v = tile * kTileCols + at % kTileCols;
    const int64_t from = v * groups + at / kTileCols % groups;
    const uint32_t s = v < n ? scales[from] : 0u;
    if (zeros) {
      const float o = 16.f + (v < n ? static_cast<float>(min(static_cast<int>(zeros[from]), 15)) : 0.f);
      static_cast<uint32_t*>(to)[at] = s | (__float_as_uint(o) & 0xFFFF0000u);        // exact: o has five bits
    } else {
      static_cast<uint16_t*>(to)[at] = static_cast<uint16_t>(s);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------
constexpr int64_t kMostBlocks = 1 << 20;      // of kernels that loop over what is left
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline int64_t padded_tiles(int n) { return up(up(n, kTileCols) / kTileCols, kTilesPad); }
inline int k_blocks(int d) { return (d + kBlockK - 1) / kBlockK; }

template <class K>
bool scales_fit(const QuantizedArgs& q) {
  return up(static_cast<int64_t>(K::COLTILES) * q.groups * kTileCols * (q.zeros ? 4 : 2), 1024) <= K::SCALES;
}
// Two column tiles per wavefront leave no registers for groups that end inside a block: those have one.
inline bool whole_blocks(const QuantizedArgs& q) { return q.group % kBlockK == 0; }
template <class K, int STEP>
hipError_t launch(const LmHeadArgs& a, const QuantizedArgs& q, hipStream_t s, const LaunchEvents& ev) {
  const int64_t tiles = up(a.n, kTileCols) / kTileCols;
  const int WT = static_cast<int>((tiles + K::COLTILES - 1) / K::COLTILES), MT = (a.B * a.L + K::RB * 32 - 1) / (K::RB * 32);
  const dim3 grid((WT + 7) / 8 * 8 * MT);
  if (q.zeros) launch_kernel(lm_head_quantized_kernel<K, STEP, true>, grid, dim3(K::THREADS), s, ev, a, q, WT, MT);
  else launch_kernel(lm_head_quantized_kernel<K, STEP, false>, grid, dim3(K::THREADS), s, ev, a, q, WT, MT);
  return hipGetLastError();
}
// The instances for groups of whole blocks and for others.
struct Kernel {
  hipError_t (*launch)(const LmHeadArgs&, const QuantizedArgs&, hipStream_t, const LaunchEvents&);
  int (*name)(char*, size_t, int, bool);
  int step;
};
template <class K>
Kernel kernel_of(const QuantizedArgs& q) {
  if constexpr (K::NC == 2) return {launch<K, 4>, K::name, 4};
  else return whole_blocks(q) ? Kernel{launch<K, 4>, K::name, 4} : Kernel{launch<K, 2>, K::name, 2};
}
static_assert(QuantCfg<2, 1, 32, 1, 4, 4, 160>::SCALES >= kMaxGroups * kTileCols * 4 && QuantCfg<1, 2, 32, 1, 4, 4, 160>::SCALES >= kMaxGroups * kTileCols * 4,
              "the scales of one column tile always fit");
// Which workgroups serve a call: those whose rounds (of as many as run at once) cost least, among those that the scales of
// their columns fit into.  A round's cost is the time of one on d = 4096, it hardly depends on how full the round is:
// 32 rows with guidance x 8192 ids take 29 us with four wavefronts sharing a tile (Four), 34 with two (Two), 48 with two tiles per
// wavefront and k in two parts (Wide); x 16384 55 : 35 : 48, x 32768 105 : 37 : 49, x 65536 209 : 69 : 52; without guidance over
// 1280 x 8192 9.2 : 11.7 : 15.5, x 65536 61 : 24 : 18; one row x 8192 12.4 : 22.6 : 30, x 65536 87 : 48 : 35.  Tiles of 256 rows (Tall) keep up with
// Wide nowhere (480 rows with guidance x 8192 115 : 98), but serve groups whose scales do not fit it (groups of 64 with zero
// points, there 114 : 137 of Two).  One serves long rows of groups that end inside blocks.
template <class K>
int64_t cost_of(const LmHeadArgs& a, const QuantizedArgs& q, int resident, int round) {
  if (!scales_fit<K>(q)) return INT64_MAX;
  const int64_t tiles = up(a.n, kTileCols) / kTileCols, groups = (tiles + K::COLTILES - 1) / K::COLTILES;
  const int64_t row_tiles = (static_cast<int64_t>(a.B) * a.L + K::RB * 32 - 1) / (K::RB * 32);
  return (groups * row_tiles + resident - 1) / resident * round;
}
template <int C, int RB, int HRB>
Kernel best_of(const LmHeadArgs& a, const QuantizedArgs& q) {
  using Four = QuantCfg<C, RB, HRB, 1, 4, 4, 160>;
  using Two = QuantCfg<C, RB, HRB, 1, 8, 2, 160>;
  using One = QuantCfg<C, RB, HRB, 1, 8, 1, 160>;
  using Wide = QuantCfg<C, RB, HRB, 2, 8, 2, 160>;
  using Tall = QuantCfg<C, 8 / C, 32, 2, 8, 1, 160, 4>;          // a quarter of 256 rows per wavefront
  const bool whole = whole_blocks(q);
  Kernel best = kernel_of<Four>(q);
  int64_t least = cost_of<Four>(a, q, 256, HRB == 8 ? 13 : 29);
  auto consider = [&](int64_t cost, Kernel k) {
    if (cost < least) {
      least = cost;
      best = k;
    }
  };
  consider(cost_of<Two>(a, q, 256, HRB == 8 ? 23 : 35), kernel_of<Two>(q));
  consider(cost_of<One>(a, q, 256, HRB == 8 ? 40 : 57), kernel_of<One>(q));
  if (whole) consider(cost_of<Wide>(a, q, 256, HRB == 8 ? 31 : 51), kernel_of<Wide>(q));
  if constexpr (HRB == 8) {
    using Small = QuantCfg<C, RB, HRB, 1, 4, 4, 80>;             // two of them per CU
    consider(cost_of<Small>(a, q, 512, 15), kernel_of<Small>(q));
  } else {
    if (whole) consider(cost_of<Tall>(a, q, 256, 115), kernel_of<Tall>(q));
  }
  return best;
}
Kernel kernel_for(const LmHeadArgs& a, const QuantizedArgs& q) {
  const int rows = a.B * a.L;
  if (a.C == 2) return rows <= 8 ? best_of<2, 1, 8>(a, q) : best_of<2, 1, 32>(a, q);
  if (rows <= 8) return best_of<1, 1, 8>(a, q);
  return rows <= 32 ? best_of<1, 1, 32>(a, q) : best_of<1, 2, 32>(a, q);
}
QuantizedArgs quantized_args(const LmHeadArgs& a, const void* packed, int group, bool zeros) {
  const char* const codes = static_cast<const char*>(packed);
  return {codes, codes ? codes + padded_tiles(a.n) * k_blocks(a.d) * kBlockBytes : nullptr, group, (a.d + group - 1) / group, zeros};
}

}  // namespace

size_t quantized_bytes(int n, int d, int group, bool zeros) {
  const size_t tiles = padded_tiles(n), groups = (d + group - 1) / group;
  return tiles * k_blocks(d) * kBlockBytes + up(tiles * groups * kTileCols * (zeros ? 4 : 2), 256) + 1024;
}

hipError_t launch_quantize(const uint16_t* W, int V, int d, int group, uint8_t* codes, uint16_t* scales, uint8_t* zeros, hipStream_t s) {
  const int groups = (d + group - 1) / group;
  const int64_t items = static_cast<int64_t>(V) * groups;
  hipLaunchKernelGGL(quantize_kernel, dim3(static_cast<uint32_t>((items + 3) / 4 < kMostBlocks ? (items + 3) / 4 : kMostBlocks)), dim3(256), 0, s, W, items, d, group, groups, codes, scales, zeros);
  return hipGetLastError();
}

hipError_t launch_pack_quantized(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, int d, int group, void* packed,
                                 hipStream_t s) {
  const int64_t tiles = padded_tiles(n), blocks = tiles * k_blocks(d);
  const int groups = (d + group - 1) / group;
  hipLaunchKernelGGL(pack_codes_kernel, dim3(static_cast<uint32_t>((blocks + 3) / 4 < kMostBlocks ? (blocks + 3) / 4 : kMostBlocks)), dim3(256), 0, s, codes, n, d,
                     k_blocks(d), blocks, static_cast<u32x4*>(packed));
  const int64_t count = tiles * groups * kTileCols;
  hipLaunchKernelGGL(pack_scales_kernel, dim3(static_cast<uint32_t>((count + 255) / 256 < kMostBlocks ? (count + 255) / 256 : kMostBlocks)), dim3(256), 0, s, scales, zeros, n, groups, count,
                     static_cast<char*>(packed) + blocks * kBlockBytes);
  return hipGetLastError();
}

hipError_t launch_lm_head_quantized(const LmHeadArgs& a, const void* packed, int group, bool zeros, hipStream_t s, hipEvent_t ev_start,
                                    hipEvent_t ev_stop) {
  const QuantizedArgs q = quantized_args(a, packed, group, zeros);
  return kernel_for(a, q).launch(a, q, s, LaunchEvents{ev_start, ev_stop});
}

int lm_head_quantized_kernel_name(const LmHeadArgs& a, int group, bool zeros, char* buf, size_t cap) {
  const Kernel k = kernel_for(a, quantized_args(a, nullptr, group, zeros));
  return k.name(buf, cap, k.step, zeros);
}

}  // namespace scd
