// LM head over 4-bit weights:
//   W[v, k] = s[v, k / G] * (q[v, k] - o[v, k / G])        q in 0 .. 15, s bf16, o = 8 or a zero point of 0 .. 15
//   logit[m, v] = sum_k h[m, k] * W[v, k]                   then guidance mix and temperature as in the bf16 LM head
//
// A code becomes the bf16 number 16 + q by one shift and one bitwise operation for two of them (q is put behind the leading
// mantissa bit), so the products go to the matrix units exactly:
//   sum over a group of h * (q - o) = sum h * (16 + q) - (16 + o) * sum h,
// the second sum by a product of the same rows with ones.  At a group's end both are scaled and added to the
// fp32 logits: no weight is ever rounded.
//
// Layout.  Columns in tiles of 32, k in blocks of 64: a block of a tile is 1 KB, 16 bytes for each lane of a wavefront, which
// are its operands of four 32x32x16 MFMAs (lane l: column l % 32; word j: k = 16 j + 8 (l / 32) + 0 .. 7, even k in
// the low half, odd k in the high half of the word).  The blocks of a tile follow each other; behind all of them, per tile
// and group, the 32 columns' scales (2 bytes each; with zero points 4, the second two holding 16 + o as bf16).
//
// A workgroup of NW wavefronts owns NW / WK neighbouring column tiles; WK wavefronts share a tile and take 1/WK of k each
// (their sums are added up at the end in a fixed order).  Weights and h rows go from memory straight into
// LDS, S stages deep; a wavefront reads its own weights back, the h rows are shared.  The scales of the workgroup's columns are
// fetched whole at the start.
#include "lm_head_rows.h"
#include "tile_loads.h"

namespace scd {
namespace {

constexpr int kTileCols = 32, kBlockK = 64, kBlockBytes = 1024, kTilesPad = 8;
constexpr int kLdsBytes = 160 * 1024;

// rows per block of 32 that are really loaded: HRB; blocks per workgroup (guidance included): NB
template <int C_, int RB_, int HRB_, int NW_, int WK_>
struct QuantCfg {
  static constexpr int C = C_, RB = RB_, HRB = HRB_, NW = NW_, WK = WK_;
  static constexpr int THREADS = NW * 64, WC = NW / WK, NB = RB * C;
  static constexpr int HROWS = NB * HRB;                 // h rows per part of k
  static constexpr int HI = WK * HROWS / 8;              // load instructions for the h rows of a step, all parts
  static constexpr int HL = (HI + NW - 1) / NW;          // per wavefront
  static constexpr int WB = NW * kBlockBytes, HB = WK * HROWS * 128, STAGE = WB + HB;
  static constexpr int S = 120 * 1024 / STAGE < 2 ? 2 : 120 * 1024 / STAGE > 6 ? 6 : 120 * 1024 / STAGE;
  static constexpr int RED = WK > 1 ? NW * NB * 16 * 64 * 4 : 0;      // sums of the parts of k, in the place of the stages
  static constexpr int BASE = S * STAGE > RED ? S * STAGE : RED;
  static constexpr int TABLE = RB * 32 * 4;
  static constexpr int SCALES = kLdsBytes - TABLE - BASE;      // room for the columns' scales
  static_assert(SCALES >= WC * 4 * 1024, "LDS");
};

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// the eight codes of a word as bf16 numbers 16 + q
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
  return u32x4{(w << 3 & kMask) | kSixteen, (w >> 1 & kMask) | kSixteen, (w >> 5 & kMask) | kSixteen, (w >> 9 & kMask) | kSixteen};
}

// STEP: MFMAs between two applications of a scale (2: groups that end inside a block of k, 4: they do not)
template <class K, int STEP>
__global__ __launch_bounds__(K::THREADS) void lm_head_quantized_kernel(const LmHeadArgs a, const QuantizedArgs q, const int WT, const int MT) {
  constexpr int C = K::C, RB = K::RB, NB = K::NB, WK = K::WK, WC = K::WC, NW = K::NW, S = K::S, HL = K::HL, HRB = K::HRB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kLdsBytes];
  int* const table = reinterpret_cast<int*>(lds + K::BASE);
  unsigned char* const slab = lds + K::BASE + K::TABLE;
  // workgroups that share columns get ids 8 apart: the same XCD, the same L2
  const int id = blockIdx.x, mt = (id / 8) % MT, wt = id / (8 * MT) * 8 + id % 8;
  if (wt >= WT) return;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wave % WC, part = wave / WC;
  const int rows = a.B * a.L, p_base = mt * RB * 32, d = a.d;
  const int tile = wt * WC + wc;                         // column tile (the layout is padded to whole workgroups)
  const int KB = (d + kBlockK - 1) / kBlockK;
  const int nch = d % kBlockK / 8;                       // 16-byte chunks of a ragged last block, 0: there is none
  auto first_block = [&](int p) { return KB * p / WK; };
  const int T = (KB + WK - 1) / WK;                      // steps
  const int kb0 = first_block(part), count = first_block(part + 1) - kb0;
  const RowState mine = row_state(a, p_base + min(tid, RB * 32 - 1));

  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)lds));
  // ---- scales of the workgroup's columns ---------------------------------------------------------------
  const int esize = q.zeros ? 4 : 2, tile_scales = q.groups * kTileCols * esize;
  {
    const uint64_t from = reinterpret_cast<uint64_t>(q.scales) + static_cast<uint64_t>(wt) * WC * tile_scales;
    const int pieces = (WC * tile_scales + 1023) / 1024;
    for (int i = wave; i < pieces; i += NW)
      load_lds16<false, 0>(from + static_cast<uint64_t>(i) * 1024, lane * 16, lds0 + K::BASE + K::TABLE + i * 1024);
  }
  // ---- loads of a step: this wavefront's block of weights, its share of the h rows ---------------------------
  const uint64_t wbase = reinterpret_cast<uint64_t>(q.codes) + static_cast<uint64_t>(tile) * KB * kBlockBytes;
  const int h0 = first_h_row(p_base, C, a.L);
  const uint64_t hbase = reinterpret_cast<uint64_t>(a.h) + static_cast<uint64_t>(h0) * d * 2;
  int hpart[HL], hchunk[HL];
  uint32_t hoff[HL], hlds[HL];
#pragma unroll
  for (int i = 0; i < HL; ++i) {
    const int piece = (wave + i * NW) % K::HI;           // (fewer pieces than wavefronts: some are loaded twice, alike)
    const int r = piece % (K::HROWS / 8) * 8 + (lane >> 3), blk = r / HRB;
    hpart[i] = piece / (K::HROWS / 8);
    hchunk[i] = (lane & 7) ^ ((r >> 1) & 7);
    hoff[i] = static_cast<uint32_t>(h_row(min(p_base + (blk / C) * 32, rows - 1), r % HRB, blk % C, C, a.L, rows) - h0) *
              static_cast<uint32_t>(d) * 2u;
    hlds[i] = lds0 + K::WB + piece * 1024;
  }
  auto block_of = [&](int p, int t) {                    // block of k that part p works on in step t
    const int b0 = first_block(p), n = first_block(p + 1) - b0;
    return min(b0 + min(t, max(n - 1, 0)), KB - 1);
  };
  auto load = [&](int t, int stage) {
    static_for<HL>([&](auto ii) {
      constexpr int i = decltype(ii)::value;
      const int kb = block_of(hpart[i], t);
      const int chunk = nch && kb == KB - 1 ? min(hchunk[i], nch - 1) : hchunk[i];
      load_lds16<false, 0>(hbase + static_cast<uint32_t>(kb) * 128u, hoff[i] + chunk * 16, hlds[i] + stage * K::STAGE);
    });
    load_lds16<false, 0>(wbase + static_cast<uint64_t>(block_of(part, t)) * kBlockBytes, lane * 16, lds0 + wave * 1024 + stage * K::STAGE);
  };
  // the ragged block: chunks past the end are zeroed by the wavefront that loaded something in their place
  auto clear_ragged = [&](int t, int stage) {
#pragma unroll
    for (int i = 0; i < HL; ++i)
      if (block_of(hpart[i], t) == KB - 1 && hchunk[i] >= nch)
        *reinterpret_cast<u32x4*>(lds + (hlds[i] - lds0) + stage * K::STAGE + lane * 16) = u32x4{0u, 0u, 0u, 0u};
  };

  f32x16 sum[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) sum[i] = f32x16{};
  const int per_group = q.group / 32;                    // half blocks of k
  auto compute = [&](int kb, int stage) {
    const unsigned char* const Ht = lds + stage * K::STAGE + K::WB + part * (K::HROWS * 128);
    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + stage * K::STAGE + wave * 1024 + lane * 16);
    const u32x4 ones{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    u32x4 h[4][NB];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int r = i * HRB + ln % HRB;
        h[j][i] = *reinterpret_cast<const u32x4*>(Ht + r * 128 + (((2 * j + lg) ^ ((r >> 1) & 7)) * 16));
      }
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += STEP) {
      const int g = static_cast<int>(static_cast<uint32_t>(kb * 2 + j0 / 2) / static_cast<uint32_t>(per_group));
      const unsigned char* const at = slab + (wc * q.groups + g) * (kTileCols * esize) + ln * esize;
      float s, o;
      if (q.zeros) {
        const uint32_t both = *reinterpret_cast<const uint32_t*>(at);
        s = __uint_as_float(both << 16);
        o = __uint_as_float(both & 0xFFFF0000u);
      } else {
        s = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(at)) << 16);
        o = 24.f;
      }
      f32x16 acc[NB], all[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = all[i] = f32x16{};
#pragma unroll
      for (int j = j0; j < j0 + STEP; ++j) {
        const u32x4 b = codes_to_bf16(w[j]);
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[i] = mfma(h[j][i], b, acc[i]);
#pragma unroll
        for (int i = 0; i < NB; ++i) all[i] = mfma(h[j][i], ones, all[i]);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[i][e] = __builtin_fmaf(s, __builtin_fmaf(-o, all[i][e], acc[i][e]), sum[i][e]);
    }
  };

  // Step t: its loads are there (S - 2 steps' are still on their way), the barrier publishes them and says that every
  // wavefront is done with the stage of step t - 1, which takes the loads of step t + S - 1.
  constexpr int LPT = HL + 1;
#pragma unroll
  for (int t = 0; t < S - 1; ++t)
    if (t < T) load(t, t);
  int stage = 0, next = S - 1;
#pragma unroll 1
  for (int t = 0; t < T; ++t) {
    if (t + S - 2 < T) wait_loads<(S - 2) * LPT>();
    else wait_loads<0>();
    if (nch) clear_ragged(t, stage);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    hard_fence();
    if (t + S - 1 < T) load(t + S - 1, next);
    if (t < count) compute(kb0 + t, stage);
    hard_fence();
    stage = stage + 1 == S ? 0 : stage + 1;
    next = next + 1 == S ? 0 : next + 1;
  }
  // ---- the parts of k added up, guidance mix, temperature, z ----------------------------------------------------
  if (tid < RB * 32) table[tid] = row_dest(a, mine);
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);
  const int v = tile * kTileCols + ln;
  if constexpr (WK > 1) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) red[((wave * NB + i) * 16 + e) * 64 + lane] = sum[i][e];
    __syncthreads();
  }
  if (v >= a.n) return;
  static_assert(16 % WK == 0, "elements per part");
#pragma unroll
  for (int r = 0; r < RB; ++r)
#pragma unroll
    for (int ee = 0; ee < 16 / WK; ++ee) {
      // the wavefronts of a tile store a share of its elements each
      const int e = WK > 1 ? part + ee * WK : ee;
      float c, u;
      if constexpr (WK > 1) {
        c = u = 0.f;
#pragma unroll
        for (int p = 0; p < WK; ++p) {
          c += red[(((p * WC + wc) * NB + r * C) * 16 + e) * 64 + lane];
          u += red[(((p * WC + wc) * NB + r * C + C - 1) * 16 + e) * 64 + lane];
        }
      } else {
        c = sum[r * C][ee];
        u = sum[r * C + C - 1][ee];
      }
      const int row = table[r * 32 + (e >> 2) * 8 + lg * 4 + (e & 3)];
      if (row >= 0) a.z[static_cast<int64_t>(row) * a.n + v] = processed_logit<C>(a, c, u);
    }
}

// ---- quantisation and layout ---------------------------------------------------------------------------
// A wavefront per row and group.  Without zero points s = max(largest / 7, -smallest / 8), with them s = (largest -
// smallest) / 15 over a range that holds 0; s is rounded to bf16 first, the codes are the nearest under the rounded one.
__global__ __launch_bounds__(256) void quantize_kernel(const uint16_t* __restrict__ W, int64_t items, int d, int group, int groups,
                                                       uint8_t* __restrict__ codes, uint16_t* __restrict__ scales, uint8_t* __restrict__ zeros) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= items) return;
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
  const __bf16 sb = static_cast<__bf16>(zeros ? __fdiv_rn(hi - lo, 15.f) : fmaxf(__fdiv_rn(hi, 7.f), __fdiv_rn(-lo, 8.f)));
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

// A wavefront per column tile and block of k: 16 bytes per lane.
__global__ __launch_bounds__(256) void pack_codes_kernel(const uint8_t* __restrict__ codes, int n, int d, int KB, int64_t blocks,
                                                         u32x4* __restrict__ to) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (item >= blocks) return;
  const int lane = threadIdx.x & 63;
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
__global__ __launch_bounds__(256) void pack_scales_kernel(const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, int n, int groups,
                                                          int64_t count, void* __restrict__ to) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;        // (tile, group, column)
  if (at >= count) return;
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

// ---- host ----------------------------------------------------------------------------------------------
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline int64_t padded_tiles(int n) { return up(up(n, kTileCols) / kTileCols, kTilesPad); }
inline int k_blocks(int d) { return (d + kBlockK - 1) / kBlockK; }

template <class K>
bool scales_fit(const QuantizedArgs& q) {
  return up(static_cast<int64_t>(K::WC) * q.groups * kTileCols * (q.zeros ? 4 : 2), 1024) <= K::SCALES;
}
template <class K>
hipError_t launch(const LmHeadArgs& a, const QuantizedArgs& q, hipStream_t s) {
  const int64_t tiles = up(a.n, kTileCols) / kTileCols;
  const int WT = static_cast<int>((tiles + K::WC - 1) / K::WC), MT = (a.B * a.L + K::RB * 32 - 1) / (K::RB * 32);
  const dim3 grid((WT + 7) / 8 * 8 * MT), block(K::THREADS);
  if (q.group % kBlockK == 0) hipLaunchKernelGGL((lm_head_quantized_kernel<K, 4>), grid, block, 0, s, a, q, WT, MT);
  else hipLaunchKernelGGL((lm_head_quantized_kernel<K, 2>), grid, block, 0, s, a, q, WT, MT);
  return hipGetLastError();
}
// In how many parts k is dealt over the wavefronts of a workgroup: as few as leave enough workgroups, and as let the scales
// of its columns fit.
static_assert(QuantCfg<2, 1, 32, 4, 4>::SCALES >= kMaxGroups * kTileCols * 4 && QuantCfg<1, 2, 32, 4, 4>::SCALES >= kMaxGroups * kTileCols * 4,
              "the scales of one column tile always fit");
template <int C, int RB, int HRB>
hipError_t launch_parts(const LmHeadArgs& a, const QuantizedArgs& q, hipStream_t s) {
  const int64_t tiles = up(a.n, kTileCols) / kTileCols, row_tiles = (a.B * a.L + RB * 32 - 1) / (RB * 32);
  const int64_t work = tiles * row_tiles;
  using One = QuantCfg<C, RB, HRB, 8, 1>;
  using Two = QuantCfg<C, RB, HRB, 8, 2>;
  using Four = QuantCfg<C, RB, HRB, 4, 4>;
  if (work >= 2048 && scales_fit<One>(q)) return launch<One>(a, q, s);
  if (work >= 1024 && scales_fit<Two>(q)) return launch<Two>(a, q, s);
  return launch<Four>(a, q, s);
}

}  // namespace

size_t quantized_bytes(int n, int d, int group, bool zeros) {
  const size_t tiles = padded_tiles(n), groups = (d + group - 1) / group;
  return tiles * k_blocks(d) * kBlockBytes + up(tiles * groups * kTileCols * (zeros ? 4 : 2), 256) + 1024;
}

hipError_t launch_quantize(const uint16_t* W, int V, int d, int group, uint8_t* codes, uint16_t* scales, uint8_t* zeros, hipStream_t s) {
  const int groups = (d + group - 1) / group;
  const int64_t items = static_cast<int64_t>(V) * groups;
  hipLaunchKernelGGL(quantize_kernel, dim3(static_cast<uint32_t>((items + 3) / 4)), dim3(256), 0, s, W, items, d, group, groups, codes, scales, zeros);
  return hipGetLastError();
}

hipError_t launch_pack_quantized(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, int d, int group, void* packed,
                                 hipStream_t s) {
  const int64_t tiles = padded_tiles(n), blocks = tiles * k_blocks(d);
  const int groups = (d + group - 1) / group;
  hipLaunchKernelGGL(pack_codes_kernel, dim3(static_cast<uint32_t>((blocks + 3) / 4)), dim3(256), 0, s, codes, n, d, k_blocks(d), blocks,
                     static_cast<u32x4*>(packed));
  const int64_t count = tiles * groups * kTileCols;
  hipLaunchKernelGGL(pack_scales_kernel, dim3(static_cast<uint32_t>((count + 255) / 256)), dim3(256), 0, s, scales, zeros, n, groups, count,
                     static_cast<char*>(packed) + blocks * kBlockBytes);
  return hipGetLastError();
}

hipError_t launch_lm_head_quantized(const LmHeadArgs& a, const void* packed, int group, bool zeros, hipStream_t s) {
  QuantizedArgs q{};
  q.codes = packed;
  q.scales = static_cast<const char*>(packed) + padded_tiles(a.n) * k_blocks(a.d) * kBlockBytes;
  q.group = group; q.groups = (a.d + group - 1) / group; q.zeros = zeros;
  const int rows = a.B * a.L;
  if (a.C == 2) {
    if (rows <= 8) return launch_parts<2, 1, 8>(a, q, s);
    return launch_parts<2, 1, 32>(a, q, s);
  }
  if (rows <= 8) return launch_parts<1, 1, 8>(a, q, s);
  if (rows <= 32) return launch_parts<1, 1, 32>(a, q, s);
  return launch_parts<1, 2, 32>(a, q, s);
}

}  // namespace scd
