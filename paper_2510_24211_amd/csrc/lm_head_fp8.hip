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
// Rows of h are the MFMA's columns: a lane has one row, and one scale.  Tiles of columns begin at multiples of 128 of the table, whatever
// the first allowed id, so that a wavefront's columns share theirs.  h, W and the scales go from memory straight into LDS, 128 bytes of a
// row to a stage; slot l % 8 of row l / 8 of a load holds chunk (l % 8) ^ ((row >> 1) & 7): operand reads are then free of bank conflicts.
#include "eights.h"
#include "launch_events.h"
#include "lm_head_rows.h"

#include <stdio.h>

namespace scd {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Eight codes (two words) as fp16 numbers, which hold every e4m3 number, NaN among them.
__device__ __forceinline__ f16x8 to_f16(uint32_t a, uint32_t b) {
  const f16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true)};
  return f16x8{v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
}

// RB blocks of 32 window rows (times C with guidance) x BN columns by WCOL x WROW wavefronts; SA stages of h and the scales, SB of W
template <int C_, int RB_, int BN_, int WCOL_, int WROW_, int SA_, int SB_>
struct Fp8Cfg {
  static constexpr int C = C_, RB = RB_, BN = BN_, WCOL = WCOL_, WROW = WROW_, SA = SA_, SB = SB_;
  static int name(char* buf, size_t cap) {
    return snprintf(buf, cap, "lm_head_fp8_kernel<Fp8Cfg<%d, %d, %d, %d, %d, %d, %d>>", C, RB, BN, WCOL, WROW, SA, SB);
  }
  static constexpr int NW = WCOL * WROW, THREADS = NW * 64;
  static constexpr int HR = RB * C * 32;                   // rows of h
  static constexpr int CW = BN / WCOL, NC = CW / 32;       // columns per wavefront
  static constexpr int RBW = RB / WROW, NB = RBW * C;      // blocks of rows per wavefront
  static constexpr int AL = HR / 8 / NW, BL = BN / 8 / NW; // loads per wavefront and block of k
  static constexpr int AB = HR * 128, BB = BN * 128, SCB = NW * 256;     // bytes of a stage: h, W, scales
  static constexpr int LDS = SA * (AB + SCB) + SB * BB;
  static_assert(CW % 32 == 0 && CW <= 128 && 128 % CW == 0 && RBW * WROW == RB && AL * NW * 8 == HR && BL * NW * 8 == BN, "tile shape");
  static_assert(LDS <= 160 * 1024 && NW * 64 >= HR + (BN + 127) / 128 && SB >= SA && SA >= 2, "LDS");
  static_assert((SA - 2) * (AL + BL + 1) + BL <= 63, "loads in flight");
};

struct Fp8Args {
  LmHeadArgs lm;               // h [B, C, L, d] codes
  const float* h_scales;       // [B, C, L, G]
  const uint8_t* W;            // [V, d] codes
  const float* W_scales;       // [ceil(V / 128), G]
  int v_lo;
};

// 4 bytes per lane from a lane's own address to LDS byte address lds + 4 * lane
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds4(uint64_t from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

template <class K>
__global__ __launch_bounds__(K::THREADS) void lm_head_fp8_kernel(const Fp8Args f, const int WT, const int MT) {
  constexpr int C = K::C, RB = K::RB, NB = K::NB, NC = K::NC, AL = K::AL, BL = K::BL, SA = K::SA, SB = K::SB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[K::LDS];      // W's stages, then h's, then the scales'
  const LmHeadArgs& a = f.lm;
  // workgroups that share columns get ids 8 apart: the same XCD, the same L2
  const int id = blockIdx.x, mt = (id / 8) % MT, wt = id / (8 * MT) * 8 + id % 8;
  if (wt >= WT) return;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wave % K::WCOL, wr = wave / K::WCOL;
  const int rows = a.B * a.L, d = a.d, KT = (d + 127) / 128, G = KT;
  const int nch = d % 128 / 16;                          // 16-byte chunks of a ragged last block, 0: there is none
  const int p_base = mt * RB * 32;
  const int col_base = (f.v_lo / 128) * 128 - f.v_lo + wt * K::BN;       // columns are counted from the first allowed id
  RowState mine[K::RBW];
#pragma unroll
  for (int i = 0; i < K::RBW; ++i) mine[i] = row_state(a, p_base + (wr * K::RBW + i) * 32 + ln);

  // ---- where this lane's loads come from ----------------------------------------------------------------
  auto piece_row = [&](int per_wave, int i) { return (wave * per_wave + i) * 8 + (lane >> 3); };
  auto piece_chunk = [&](int r) { return (lane & 7) ^ ((r >> 1) & 7); };
  const int h0 = first_h_row(p_base, C, a.L);
  const uint64_t hbase = reinterpret_cast<uint64_t>(a.h) + static_cast<uint64_t>(h0) * d;
  const int w0 = max(f.v_lo + col_base, f.v_lo), w_last = f.v_lo + a.n - 1;       // first and last row of W that may be read
  const uint64_t wbase = reinterpret_cast<uint64_t>(f.W) + static_cast<uint64_t>(w0) * d;
  auto row_of_h = [&](int r) {                           // of row r of the tile: [RB][C][32]
    const int blk = r / 32, rb = blk / C;
    return h_row(min(p_base + rb * 32, rows - 1), r % 32, blk % C, C, a.L, rows);
  };
  uint32_t ao[AL], bo[BL];
#pragma unroll
  for (int i = 0; i < AL; ++i) {
    const int r = piece_row(AL, i);
    ao[i] = static_cast<uint32_t>(row_of_h(r) - h0) * static_cast<uint32_t>(d) + piece_chunk(r) * 16;
  }
#pragma unroll
  for (int i = 0; i < BL; ++i) {
    const int r = piece_row(BL, i);
    const int v = min(max(f.v_lo + col_base + r, w0), w_last);
    bo[i] = static_cast<uint32_t>(v - w0) * static_cast<uint32_t>(d) + piece_chunk(r) * 16;
  }
  // a word per thread: the scales of h's rows, then those of the columns' groups of 128
  uint64_t so;
  if (tid < K::HR) so = reinterpret_cast<uint64_t>(f.h_scales) + static_cast<uint64_t>(row_of_h(tid)) * G * 4;
  else {
    const int group = (f.v_lo + col_base) / 128 + min(tid - K::HR, (K::BN - 1) / 128);
    so = reinterpret_cast<uint64_t>(f.W_scales) + static_cast<uint64_t>(min(group, w_last / 128)) * G * 4;
  }
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds));
  const uint32_t ldsB = lds0 + wave * BL * 1024, ldsA = lds0 + SB * K::BB + wave * AL * 1024,
                 ldsS = lds0 + SB * K::BB + SA * K::AB + wave * 256;

  auto back = [&](int t, int r) { return t == KT - 1 && nch != 0 ? max(piece_chunk(r) - (nch - 1), 0) * 16 : 0; };   // past a ragged end: its last chunk
  auto load_a = [&](int t) {
    const uint64_t at = hbase + static_cast<uint64_t>(t) * 128;
    const uint32_t to = ldsA + t % SA * K::AB;
    static_for<AL>([&](auto i) { load_lds16<false, decltype(i)::value * 1024>(at, ao[decltype(i)::value] - back(t, piece_row(AL, decltype(i)::value)), to); });
    load_lds4(so + static_cast<uint64_t>(t) * 4, ldsS + t % SA * K::SCB);
  };
  auto load_b = [&](int t) {
    const uint64_t at = wbase + static_cast<uint64_t>(t) * 128;
    const uint32_t to = ldsB + t % SB * K::BB;
    static_for<BL>([&](auto i) { load_lds16<false, decltype(i)::value * 1024>(at, bo[decltype(i)::value] - back(t, piece_row(BL, decltype(i)::value)), to); });
  };

  f32x16 total[NC][NB];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < NB; ++i) total[c][i] = f32x16{};

  // Window t of the loads ends at the barrier of block t; it brings h of block t + SA - 1 and W of t + SB - 1 (a stage is free once the
  // barrier behind the block that it held is passed).
  static_for<SB - 1>([&](auto t) {
    constexpr int T = decltype(t)::value;
    if constexpr (T < SA - 1) {
      if (T < KT) load_a(T);
    }
    if (T < KT) load_b(T);
  });
  // At the barrier of block t its h and W have to be there; what was issued behind h of block t may be in flight.
  constexpr int ALL = AL + BL + 1, AHEAD = (SA - 2) * ALL + (SB > SA ? BL : 0);
  auto multiply = [&](int t, auto ragged) {
    constexpr bool RAGGED = decltype(ragged)::value;
    const unsigned char* const Bt = lds + t % SB * K::BB + (wc * K::CW + ln) * 128;
    const unsigned char* const At = lds + SB * K::BB + t % SA * K::AB + (wr * NB * 32 + ln) * 128;
    const float* const St = reinterpret_cast<const float*>(lds + SB * K::BB + SA * K::AB + t % SA * K::SCB);
    const float sw = St[K::HR + wc * K::CW / 128];
    f32x16 acc[NC][NB];
    static_for<4>([&](auto qq) {
      constexpr int Q = decltype(qq)::value;               // chunks 2 Q and 2 Q + 1 of the block: 16 k for each half of the wavefront
      const int chunk = Q * 2 + lg, slot = (chunk ^ ((ln >> 1) & 7)) * 16;
      u32x4 w[NC], h[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        h[i] = *reinterpret_cast<const u32x4*>(At + i * 4096 + slot);
        if (RAGGED && chunk >= nch) h[i] = u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) w[c] = *reinterpret_cast<const u32x4*>(Bt + c * 4096 + slot);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        f16x8 hf[NB], wf[NC];
#pragma unroll
        for (int i = 0; i < NB; ++i) hf[i] = to_f16(h[i][2 * e], h[i][2 * e + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c) wf[c] = to_f16(w[c][2 * e], w[c][2 * e + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < NB; ++i)
            acc[c][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(wf[c], hf[i], Q == 0 && e == 0 ? f32x16{} : acc[c][i], 0, 0, 0);
      }
    });
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const float s = St[(wr * NB + i) * 32 + ln] * sw;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) total[c][i][e] = __fmaf_rn(acc[c][i][e], s, total[c][i][e]);
    }
  };
  auto step = [&](int t, auto ragged) {
    if (t + SB - 2 < KT) wait_loads<AHEAD>();            // the windows before brought all that they can
    else wait_loads<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the last block's operands are in registers
    __builtin_amdgcn_s_barrier();
    hard_fence();
    if (t + SA - 1 < KT) load_a(t + SA - 1);
    if (t + SB - 1 < KT) load_b(t + SB - 1);
    hard_fence();
    multiply(t, ragged);
    hard_fence();
  };
  const int full = nch != 0 ? KT - 1 : KT;
#pragma unroll 1
  for (int t = 0; t < full; ++t) step(t, FalseT{});
  if (nch != 0) step(KT - 1, TrueT{});

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

template <class F>
void choose(const LmHeadArgs& a, F&& go) {
  const int64_t rows = static_cast<int64_t>(a.B) * a.L;
  if (a.C == 2) {
    if (rows > 64) with<Fp8Cfg<2, 4, 128, 2, 4, 3, 3>>(go);
    else if (rows > 32) with<Fp8Cfg<2, 2, 128, 4, 1, 3, 4>>(go);
    else with<Fp8Cfg<2, 1, 128, 4, 1, 3, 3>>(go);
  } else {
    if (rows > 128) with<Fp8Cfg<1, 8, 128, 2, 4, 3, 3>>(go);
    else if (rows > 64) with<Fp8Cfg<1, 4, 128, 4, 1, 3, 4>>(go);
    else if (rows > 32) with<Fp8Cfg<1, 2, 128, 4, 1, 3, 3>>(go);
    else with<Fp8Cfg<1, 1, 64, 2, 1, 4, 4>>(go);
  }
}

// ---- weights in 8 bits ---------------------------------------------------------------------------------------------
// A workgroup takes a block of 128 x 128 of the table: 16 lanes to a row, eight elements each, eight rows of a thread.
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
      if (row < V && p < pieces) reinterpret_cast<uint2*>(codes)[row * pieces + p] = to_e4m3(v[i].wide(), s.inverse);
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
  const int64_t WT = (v_lo % 128 + static_cast<int64_t>(a.n) + K::BN - 1) / K::BN, MT = (static_cast<int64_t>(a.B) * a.L + K::RB * 32 - 1) / (K::RB * 32);
  return {WT, MT, (WT + 7) / 8 * 8 * MT};
}
}  // namespace

bool lm_head_fp8_fits(const LmHeadArgs& a) {
  bool fits = false;
  choose(a, [&](auto k) {
    using K = decltype(k);
    fits = grid_of<K>(a, 127).groups * K::THREADS < static_cast<int64_t>(1) << 32;      // a launch's threads
  });
  return fits;
}

hipError_t launch_lm_head_fp8(const LmHeadArgs& a, const float* h_scales, const uint8_t* W, const float* W_scales, int v_lo, hipStream_t s,
                              hipEvent_t ev_start, hipEvent_t ev_stop) {
  const LaunchEvents ev{ev_start, ev_stop};
  const Fp8Args f{a, h_scales, W, W_scales, v_lo};
  choose(a, [&](auto k) {
    using K = decltype(k);
    const Grid g = grid_of<K>(a, v_lo);
    launch_kernel(lm_head_fp8_kernel<K>, dim3(static_cast<unsigned>(g.groups)), dim3(K::THREADS), s, ev, f, static_cast<int>(g.WT), static_cast<int>(g.MT));
  });
  return hipGetLastError();
}

int lm_head_fp8_kernel_name(const LmHeadArgs& a, char* buf, size_t cap) {
  int len = 0;
  choose(a, [&](auto k) { len = decltype(k)::name(buf, cap); });
  return len;
}

hipError_t launch_quantize_fp8(const uint16_t* W, int V, int d, uint8_t* codes, float* scales, hipStream_t s) {
  hipLaunchKernelGGL(quantize_fp8_kernel, dim3((d + 127) / 128, (V - 1) / 128 + 1 > 65535 ? 65535 : (V - 1) / 128 + 1), dim3(256), 0, s, W, V, d,
                     codes, scales);
  return hipGetLastError();
}

}  // namespace scd
