// Softmax cross entropy of hidden rows over the allowed ids of a vocabulary table, without keeping the logits:
//   z = h W^T / tau;  lse = log sum_v exp(z_v);  loss = lse - z_t
//   dz = weight * (exp(z - lse) - [v = t]) / tau;  dh = dz W;  dW = dz^T h
// Four matrix products of 2 * rows * n * d operations each (the logits are made again for the gradient), all on one tile
// routine that wants k along both operands' rows.
//   Forward: a tile of logits leaves (maximum, sum of exponentials) per row and the target's logit; finish_kernel joins a
// row's tiles.  Backward, for a piece of the vocabulary at a time: dz of the piece goes to the workspace as rows and as
// columns (k lies along ids for dh, along rows for dW), the piece of W and the rows of h are turned once for the same reason.
//   The products of the gradient take fp16 operands: dz has to be rounded for the matrix units, and bf16 would leave each of its
// terms an error as large as that of the bf16 results (2^-9 of the term, at 515 rows x 16395 ids 0.0025 of dh in the mean
// against 64 bits, where the rounding of the result alone makes 0.0017); fp16 errs by an eighth of it.  Its range is
// short, so every operand is brought under 2^15 by a power of two: W and the rows of h by the exponent of their largest finite
// element (range_kernel reads them once), dz, which lies in [-1, 1] without the rows' weights, by 2^14, and with
// the weights for dW by the exponent of the largest.  The elements of W and h, of 8 bits, stay exact down to 2^-31 of the
// largest; dz has its 11 bits down to 2^-28 of the largest weight, and an absolute error of 2^-39 of it below.  Where dW is kept in 32 bits
// dz enters its product as two terms, at the price of a fifth product: what the first one leaves, times 2^11, has sums of its own, which
// are brought down again before the first terms' are added to them.  So dz errs by 2^-22 of itself or 2^-50 of the largest
// weight, whichever is more.  Statistics and sums are fp32.
//   Bound by the matrix pipes: 4096 rows x 65536 ids over 4096 take 7.6 to 7.9 ms, the four products at 1.1 to 1.25 PFLOP/s (6.2 ms at the 1.42
// of a large library product), turning W 212 us, its largest element 98, dh's sums over the pieces about 100; the forward pass of 2304 rows
// 1.05 to 1.1 ms (1.13 to 1.18 PFLOP/s).  Few rows are bound by W: 77 x 16384 over 1280 16.5 to 17.5 us, 42 MB.
#include "gemm_tile.h"
#include "scd_device.h"
#include "scd_kernels.h"

#include <stdio.h>

namespace scd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// sum / maximum over the 32 lanes of a half wavefront, in every lane
template <class F>
__device__ __forceinline__ float half_fold(float v, F&& f) {
  auto other = [&](auto ctrl) { return __uint_as_float(dpp_u32<decltype(ctrl)::value>(__float_as_uint(v))); };
  v = f(v, other(IntT<kDppXor1>{}));
  v = f(v, other(IntT<kDppXor2>{}));
  v = f(v, other(IntT<kDppHalfMirror>{}));
  v = f(v, other(IntT<kDppMirror>{}));
  return f(v, __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x401F)));     // lane ^ 16
}

enum GemmUse { kLoss, kGradient, kRows, kTable, kTableTwoTerms };

// floor(log2) of the largest finite element of the allowed rows of W, of the rows of h and of the weights that count
struct Exponents {
  int W, h, weight;
};
constexpr int kTop = 14;     // operands of the gradient's products lie below 2^(kTop + 1)
constexpr int kRest = 11;    // the second terms of dz are stored times 2^kRest: what rounding to 11 bits leaves stays below the same bound

struct GemmArgs {
  const uint16_t* A;
  const uint16_t* B;
  int64_t lda, ldb;          // elements from row to row
  int M, N;                  // rows of A, of B
  int KT, tail;              // whole k-tiles, elements of the ragged one
  int MT, NT, KS;            // tiles, parts of k
  // kLoss, kGradient
  const int32_t* targets;
  float scale2, inv_tau;     // log2(e) / tau, 1 / tau
  int col0;                  // column of the first row of B
  float2* part;              // [M][NT]: largest product, sum of the exponentials of the logits' distances to its logit
  float* zt;                 // [M], the target's product
  const float* lse;
  const float* weight;
  uint16_t* dz;              // fp16 [M][ldz], 2^14 times dz without the rows' weights
  uint16_t* dzT;             // fp16 [N][ldT], with them: first terms, then (two_terms) the second ones `lo` columns on
  int64_t ldz, ldT;
  int lo;
  bool two_terms;            // to be written (kGradient); kTableTwoTerms takes both, on the same columns of B
  // kRows: sums [KS][M][N] in fp32, over the pieces of the vocabulary so far; it and the tables: result [M][N]
  float* sums;
  bool first, last;
  void* out;                 // bf16, kTableTwoTerms: fp32
  bool accumulate;
  const Exponents* exps;
};

// what multiplies a row of dz W: 0 where the row is left out, whatever its weight
__device__ __forceinline__ float row_factor(const int32_t* targets, const float* weight, float inv_tau, int row) {
  return targets[row] < 0 ? 0.f : (weight ? weight[row] : 1.f) * inv_tau;
}

template <class K>
constexpr int epilogue_bytes() {
  return 16 * K::HR + (K::HR * (K::BN + 8) > K::BN * (K::HR + 8) ? K::HR * (K::BN + 8) : K::BN * (K::HR + 8)) * 2;
}
template <class K>
constexpr int lds_bytes() {
  return K::STAGES > epilogue_bytes<K>() ? K::STAGES : epilogue_bytes<K>();
}

// element j of accumulator block i: this row of the wavefront's
__device__ __forceinline__ int block_row(int i, int j, int lg) { return i * 32 + (j >> 2) * 8 + lg * 4 + (j & 3); }
__device__ __forceinline__ uint16_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }
__device__ __forceinline__ uint16_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }
__device__ __forceinline__ float f16_value(uint16_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }
__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }

// The tile in LDS, `rows` lines of `cols` bf16 values (pitch cols + 8), to memory: lines below `line_end`, whole
// 16-byte pieces below column `col_end`.
template <int LINES, int COLS, int THREADS>
__device__ __forceinline__ void store_lines(const uint16_t* tile, uint16_t* to, int64_t ld, int line_end, int col_end) {
  constexpr int PER = COLS / 8;
  for (int p = threadIdx.x; p < LINES * PER; p += THREADS) {
    const int line = p / PER, col = p % PER * 8;
    if (line < line_end && col < col_end)
      *reinterpret_cast<u32x4*>(to + line * ld + col) = *reinterpret_cast<const u32x4*>(tile + line * (COLS + 8) + col);
  }
}

template <int HR, int BN, GemmUse USE>
__global__ __launch_bounds__(512) void gemm_kernel(const GemmArgs a) {
  using K = GemmTile<HR, BN>;
  constexpr int NC = K::NC, NB = K::NB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[lds_bytes<K>()];
  const TilePlace at = tile_place(a.MT, a.NT, a.KS);
  if (at.a < 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wave % K::WCOL, wr = wave / K::WCOL;
  const int ln = lane & 31, lg = lane >> 5;
  const int row0 = at.a * HR, col0 = at.b * BN, rows = a.M - row0, cols = a.N - col0;
  int kt0 = 0, KT = a.KT;
  if (a.KS > 1) {
    kt0 = static_cast<int>(static_cast<int64_t>(a.KT) * at.part / a.KS);
    KT = static_cast<int>(static_cast<int64_t>(a.KT) * (at.part + 1) / a.KS) - kt0;
  }
  f32x16 acc[NC][NB];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[c][i] = f32x16{};
  TileOperand A{reinterpret_cast<uint64_t>(a.A + row0 * a.lda), rows, static_cast<uint32_t>(a.lda * 2)};
  const TileOperand B{reinterpret_cast<uint64_t>(a.B + col0 * a.ldb), cols, static_cast<uint32_t>(a.ldb * 2)};
  // the workgroups of an XCD meet in its L2, the XCDs start at different columns
  const int rot = KT > 0 ? static_cast<int>(static_cast<int64_t>(blockIdx.x % 8) * KT / 8) : 0;
  // 2 rows x 2680 ids over 1688: the loss errs by 1.6e-6 rms in one chain, by 5.6e-7 folded, with no more time
  constexpr bool FOLDS = (USE == kLoss || USE == kGradient) && HR * BN <= 128 * 128;
  constexpr bool F16 = USE != kLoss && USE != kGradient;
  if constexpr (USE == kTableTwoTerms) {
    const uint64_t first = A.base;
    A.base += static_cast<uint64_t>(a.lo) * 2u;
#pragma unroll 1
    for (int term = 1; term >= 0; --term) {
      multiply_tile<K, F16, FOLDS>(lds, A, B, kt0, KT, a.tail, rot, acc);
      __syncthreads();
      A.base = first;
      const float down = term == 1 ? 1.f / (1 << kRest) : 1.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[c][i] *= down;
    }
  } else {
    multiply_tile<K, F16, FOLDS>(lds, A, B, kt0, KT, a.tail, rot, acc);
    __syncthreads();
  }

  if constexpr (USE == kLoss || USE == kGradient) {
    int* const target = reinterpret_cast<int*>(lds);
    float* const lse2 = reinterpret_cast<float*>(lds) + HR;
    float* const coef = lse2 + HR;
    for (int r = tid; r < HR; r += K::THREADS) {
      const int t = r < rows ? a.targets[row0 + r] : -1;
      target[r] = t < 0 ? -1 : t - a.col0 - col0 < 0 || t - a.col0 - col0 >= BN ? BN : t - a.col0 - col0;   // column of the tile
      if constexpr (USE == kGradient) {
        lse2[r] = r < rows ? a.lse[row0 + r] * kLog2e : 0.f;
        coef[r] = __builtin_ldexpf(r < rows && a.weight ? a.weight[row0 + r] : 1.f, -a.exps->weight);
      }
    }
    __syncthreads();
    const int c0 = wc * K::CW + ln;
    if constexpr (USE == kLoss) {
      float2* const joint = reinterpret_cast<float2*>(lds + 4 * HR);       // [WCOL][HR]
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = wr * K::RW + block_row(i, j, lg), t = target[r];
          float z[NC], m = -INFINITY, s = 0.f;
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (t == c0 + c * 32) a.zt[row0 + r] = acc[c][i][j];
            z[c] = c0 + c * 32 < cols ? acc[c][i][j] : -INFINITY;
            m = fmaxf(m, z[c]);
          }
          m = half_fold(m, [](float x, float y) { return fmaxf(x, y); });
          const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int c = 0; c < NC; ++c) s += exp2_fast((z[c] - ref) * a.scale2);
          s = half_fold(s, [](float x, float y) { return x + y; });
          if (ln == 0) joint[wc * HR + r] = make_float2(m, s);
        }
      __syncthreads();
      for (int r = tid; r < HR; r += K::THREADS) {
        if (r >= rows) continue;
        float2 w[K::WCOL];
        float m = -INFINITY, s = 0.f;
#pragma unroll
        for (int k = 0; k < K::WCOL; ++k) {
          w[k] = joint[k * HR + r];
          m = fmaxf(m, w[k].x);
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < K::WCOL; ++k) s += w[k].y * exp2_fast((w[k].x - ref) * a.scale2);
        a.part[static_cast<int64_t>(row0 + r) * a.NT + at.b] = make_float2(m, s);
      }
    } else {
      uint16_t* const tile = reinterpret_cast<uint16_t*>(lds + 16 * HR);
      // 2^14 dz, without the row's weight, replaces the logits
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = wr * K::RW + block_row(i, j, lg), t = target[r];
          const float l = lse2[r];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const float p = exp2_fast(__builtin_fmaf(acc[c][i][j], a.scale2, -l));
            const float v = (p - (t == c0 + c * 32 ? 1.f : 0.f)) * (1 << kTop);
            acc[c][i][j] = t < 0 || c0 + c * 32 >= cols ? 0.f : v;
          }
        }
      if (a.dz) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j)
#pragma unroll
            for (int c = 0; c < NC; ++c)
              tile[(wr * K::RW + block_row(i, j, lg)) * (BN + 8) + c0 + c * 32] = f16_bits(acc[c][i][j]);
        __syncthreads();
        store_lines<HR, BN, K::THREADS>(tile, a.dz + row0 * a.ldz + col0, a.ldz, rows, static_cast<int>(a.ldz) - col0);
        __syncthreads();
      }
      if (a.dzT) {
        const int stretch = a.lo;                       // columns of one term
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int r = wr * K::RW + block_row(i, j, lg);
            const bool there = target[r] >= 0;          // (a row that is left out may have any weight)
            const float g = coef[r];
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[c][i][j] = there ? acc[c][i][j] * g : 0.f;
          }
        for (int term = 0; term < (a.two_terms ? 2 : 1); ++term) {
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
              for (int c = 0; c < NC; ++c) {
                uint16_t b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  b[e] = f16_bits(acc[c][i][4 * g + e]);
                  acc[c][i][4 * g + e] = (acc[c][i][4 * g + e] - f16_value(b[e])) * (1 << kRest);       // exact
                }
                *reinterpret_cast<uint2*>(tile + (c0 + c * 32) * (HR + 8) + wr * K::RW + i * 32 + g * 8 + lg * 4) =
                    make_uint2(b[0] | static_cast<uint32_t>(b[1]) << 16, b[2] | static_cast<uint32_t>(b[3]) << 16);
              }
          __syncthreads();
          store_lines<BN, HR, K::THREADS>(tile, a.dzT + static_cast<int64_t>(col0) * a.ldT + term * stretch + row0, a.ldT, cols, stretch - row0);
          __syncthreads();
        }
      }
    }
  } else {
    const int c0 = wc * K::CW + ln;
    if constexpr (USE == kRows) {
      float* const sums = a.sums ? a.sums + (static_cast<int64_t>(at.part) * a.M + row0) * a.N + col0 : nullptr;
      if (!a.first || !a.last) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int r = wr * K::RW + block_row(i, j, lg);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (r >= rows || c0 + c * 32 >= cols) continue;
              float* const to = sums + static_cast<int64_t>(r) * a.N + c0 + c * 32;
              if (!a.first) acc[c][i][j] += *to;
              if (!a.last) *to = acc[c][i][j];
            }
          }
        if (!a.last) return;
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = min(wr * K::RW + block_row(i, j, lg), rows - 1);
          const float f = row_factor(a.targets, a.weight, a.inv_tau, row0 + r);
#pragma unroll
          for (int c = 0; c < NC; ++c) acc[c][i][j] = __builtin_ldexpf(acc[c][i][j], a.exps->W - 2 * kTop) * f;
        }
    } else {
      const int e = a.exps->h + a.exps->weight - 2 * kTop;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
          for (int c = 0; c < NC; ++c) acc[c][i][j] = __builtin_ldexpf(acc[c][i][j] * a.inv_tau, e);
    }
    constexpr bool F32 = USE == kTableTwoTerms;
    if (F32 || a.accumulate) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = wr * K::RW + block_row(i, j, lg);
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (r >= rows || c0 + c * 32 >= cols) continue;
            const int64_t to = static_cast<int64_t>(row0 + r) * a.N + col0 + c0 + c * 32;
            float v = acc[c][i][j];
            if constexpr (F32) {
              float* const p = static_cast<float*>(a.out) + to;
              if (a.accumulate) v += *p;
              *p = v;
            } else {
              uint16_t* const p = static_cast<uint16_t*>(a.out) + to;
              *p = bf16_bits(v + bf16_value(*p));
            }
          }
        }
      return;
    }
    uint16_t* const tile = reinterpret_cast<uint16_t*>(lds);
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          tile[(wr * K::RW + block_row(i, j, lg)) * (BN + 8) + c0 + c * 32] = bf16_bits(acc[c][i][j]);
    __syncthreads();
    store_lines<HR, BN, K::THREADS>(tile, static_cast<uint16_t*>(a.out) + static_cast<int64_t>(row0) * a.N + col0, a.N, rows, cols);
  }
}

// ---- a row's tiles joined -------------------------------------------------------------------------
__global__ __launch_bounds__(256) void finish_kernel(const float2* __restrict__ part, const float* __restrict__ zt,
                                                     const int32_t* __restrict__ targets, int rows, int n, int NT,
                                                     float scale2, float inv_tau, float* __restrict__ loss, float* __restrict__ lse) {
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= rows) return;
  const float2* const mine = part + static_cast<int64_t>(r) * NT;
  float m = -INFINITY, s = 0.f;
  for (int t = lane; t < NT; t += 64) {
    const float2 p = mine[t];
    const float high = fmaxf(m, p.x), ref = high == -INFINITY ? 0.f : high;
    s = s * exp2_fast((m - ref) * scale2) + p.y * exp2_fast((p.x - ref) * scale2);
    m = high;
  }
  float high = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) high = fmaxf(high, __shfl_xor(high, o, 64));
  const float ref = high == -INFINITY ? 0.f : high;
  s *= exp2_fast((m - ref) * scale2);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) {
    // the loss from the difference of the products, which is exact where the target's is about the largest: not from lse, whose
    // rounding is that of the logits' size
    const float log_s = logf(s);
    const int t = targets[r];
    lse[r] = __builtin_fmaf(high, inv_tau, log_s);
    loss[r] = t < 0 ? 0.f : t >= n ? INFINITY : __builtin_fmaf(high - zt[r], inv_tau, log_s);      // (an id outside the allowed ones has no probability)
  }
}

// ---- the largest elements ----------------------------------------------------------------------------
// Per workgroup the largest magnitude (as an integer: the order is the same) among the finite elements of its share of W,
// of the rows of h and of their weights.  The workgroups that turn the rows of h take the largest of those, each for itself, and
// the first leaves the exponents for the kernels behind it; settle_kernel where no rows are turned.
constexpr int kRangeBlocks = 512;
__device__ __forceinline__ uint32_t finite_magnitude16(uint32_t two) {            // the larger of two bf16 values'
  const uint32_t a = two & 0x7FFFu, b = two >> 16 & 0x7FFFu;
  return max(a < 0x7F80u ? a : 0u, b < 0x7F80u ? b : 0u);
}
__device__ __forceinline__ uint32_t finite_magnitude16(u32x4 v) {
  return max(max(finite_magnitude16(v[0]), finite_magnitude16(v[1])), max(finite_magnitude16(v[2]), finite_magnitude16(v[3])));
}
template <int NW>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* words) {
  v = wave_max_u32(v);
  if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0u;
#pragma unroll
  for (int w = 0; w < NW; ++w) v = max(v, words[w]);
  __syncthreads();
  return v;
}
__global__ __launch_bounds__(256) void range_kernel(const u32x4* __restrict__ W, int64_t pieces_W, const u32x4* __restrict__ h, int rows, int d8,
                                                    const float* __restrict__ weight, const int32_t* __restrict__ targets,
                                                    uint3* __restrict__ out) {
  __shared__ uint32_t words[4];
  uint32_t w = 0u, x = 0u, g = 0u;
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256, first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  constexpr int AHEAD = 8;
  for (int64_t i = first; i < pieces_W; i += AHEAD * step) {
    u32x4 v[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) v[k] = W[min(i + k * step, pieces_W - 1)];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) w = max(w, finite_magnitude16(v[k]));
  }
  for (int r = blockIdx.x; r < rows; r += gridDim.x) {
    if (targets[r] < 0) continue;
    for (int i = threadIdx.x; i < d8; i += 256) x = max(x, finite_magnitude16(h[static_cast<int64_t>(r) * d8 + i]));
    const uint32_t m = weight ? __float_as_uint(weight[r]) & 0x7FFFFFFFu : 0x3F800000u;
    g = max(g, m < 0x7F800000u ? m : 0u);
  }
  w = block_max<4>(w, words);
  x = block_max<4>(x, words);
  g = block_max<4>(g, words);
  if (threadIdx.x == 0) out[blockIdx.x] = make_uint3(w, x, g);
}
// the largest of them all, by a workgroup of 256
__device__ __forceinline__ Exponents settle(const uint3* in, int blocks, uint32_t* words) {
  uint32_t w = 0u, x = 0u, g = 0u;
  for (int i = threadIdx.x; i < blocks; i += 256) {
    const uint3 v = in[i];
    w = max(w, v.x);
    x = max(x, v.y);
    g = max(g, v.z);
  }
  w = block_max<4>(w, words);
  x = block_max<4>(x, words);
  g = block_max<4>(g, words);
  return Exponents{static_cast<int>(w >> 7) - 127, static_cast<int>(x >> 7) - 127, static_cast<int>(g >> 23) - 127};
}
__global__ __launch_bounds__(256) void settle_kernel(const uint3* __restrict__ in, int blocks, Exponents* __restrict__ out) {
  __shared__ uint32_t words[4];
  const Exponents e = settle(in, blocks, words);
  if (threadIdx.x == 0) *out = e;
}

// ---- to[c][r] = from[r][c] * 2^(kTop - exponent) in fp16 for r < rows, 0 for r up to rows_pad and where marks[r] < 0 ------
// ROWS: the rows of h, the exponents from `ranges`; else W, the exponents from `exps`.
constexpr int kTurn = 64;
template <bool ROWS>
__global__ __launch_bounds__(256) void turn_kernel(const uint16_t* __restrict__ from, int64_t ld_from, int rows, int cols,
                                                   uint16_t* __restrict__ to, int64_t ld_to, int rows_pad,
                                                   const int32_t* __restrict__ marks, const uint3* __restrict__ ranges, int blocks,
                                                   Exponents* __restrict__ exps) {
  __shared__ uint16_t tile[kTurn][kTurn + 2];
  __shared__ uint32_t words[4];
  const int r0 = blockIdx.x * kTurn, c0 = blockIdx.y * kTurn;
  int up;
  if constexpr (ROWS) {
    const Exponents e = settle(ranges, blocks, words);
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) *exps = e;
    up = kTop - e.h;
  } else {
    up = kTop - exps->W;
  }
  for (int p = threadIdx.x; p < kTurn * kTurn / 8; p += 256) {
    const int r = p / (kTurn / 8), c = p % (kTurn / 8) * 8;
    u32x4 v{0u, 0u, 0u, 0u};
    if (r0 + r < rows && c0 + c < cols && !(ROWS && marks[r0 + r] < 0))
      v = *reinterpret_cast<const u32x4*>(from + static_cast<int64_t>(r0 + r) * ld_from + c0 + c);
    uint32_t* const at = reinterpret_cast<uint32_t*>(&tile[r][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      at[e] = f16_bits(__builtin_ldexpf(bf16_value(v[e] & 0xFFFFu), up)) |
              static_cast<uint32_t>(f16_bits(__builtin_ldexpf(bf16_value(v[e] >> 16), up))) << 16;
  }
  __syncthreads();
  for (int p = threadIdx.x; p < kTurn * kTurn / 8; p += 256) {
    const int c = p / (kTurn / 8), r = p % (kTurn / 8) * 8;
    if (c0 + c >= cols || r0 + r >= rows_pad) continue;
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = tile[r + 2 * e][c] | static_cast<uint32_t>(tile[r + 2 * e + 1][c]) << 16;
    *reinterpret_cast<u32x4*>(to + static_cast<int64_t>(c0 + c) * ld_to + r0 + r) = v;
  }
}

// ---- dh from the parts of k ------------------------------------------------------------------------
__global__ __launch_bounds__(256) void join_rows_kernel(const float* __restrict__ sums, int parts, int64_t count, int d,
                                                        const int32_t* __restrict__ targets, const float* __restrict__ weight, float inv_tau,
                                                        const Exponents* __restrict__ exps, uint16_t* __restrict__ out) {
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= count) return;                       // count and d are multiples of 8
  float v[4] = {};
  for (int p = 0; p < parts; ++p) {
    const float4 t = *reinterpret_cast<const float4*>(sums + p * count + at);
    v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
  }
  const float f = row_factor(targets, weight, inv_tau, static_cast<int>(at / d));
  const int e = exps->W - 2 * kTop;
  uint16_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = bf16_bits(__builtin_ldexpf(v[i], e) * f);
  *reinterpret_cast<uint2*>(out + at) = make_uint2(b[0] | static_cast<uint32_t>(b[1]) << 16, b[2] | static_cast<uint32_t>(b[3]) << 16);
}

// ---- host --------------------------------------------------------------------------------------------
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Shape {
  int hr, bn;
};
// Tiles by what one round of a workgroup per CU costs, relative to each other as the LM head's were measured.  2304 rows x 8192 ids over 4096
// (288 tiles of 256 x 256) take 194 us in 387 tiles of 256 x 192, 201 in 576 of 256 x 128; the 144 tiles of dh's product there 212
// us, 198 of 256 x 192 176; 77 rows x 16384 ids over 1280 18.7 us in 128 tiles of 128 x 128, 15.2 in 256 of 128 x 64.
// A launch holds fewer than 2^32 threads: 2^30 ids are too many tiles of 128 columns.  (What is too many of any fits no memory either.)
constexpr int64_t kMostTiles = (1 << 23) - 8;
Shape choose(int64_t M, int64_t N) {
  struct Option { int hr, bn, cost; };
  constexpr Option options[] = {{128, 64, 18}, {128, 128, 27}, {256, 128, 40}, {256, 192, 56}, {256, 256, 73}};
  Shape best{256, 256};
  int64_t least = -1;
  for (const Option& o : options) {
    const int64_t tiles = (M + o.hr - 1) / o.hr * ((N + o.bn - 1) / o.bn), cost = (tiles + 255) / 256 * o.cost;
    if (tiles <= kMostTiles && (least < 0 || cost < least)) {
      least = cost;
      best = {o.hr, o.bn};
    }
  }
  return best;
}

template <GemmUse USE>
hipError_t launch_gemm(GemmArgs a, hipStream_t s) {
  const Shape t = choose(a.M, a.N);
  a.MT = (a.M + t.hr - 1) / t.hr;
  a.NT = (a.N + t.bn - 1) / t.bn;
  const int64_t all = static_cast<int64_t>(a.MT) * a.NT * a.KS;
  if (all == 0) return hipSuccess;
  const dim3 grid(static_cast<uint32_t>((all + 7) / 8 * 8)), block(512);
  if (t.bn == 64) hipLaunchKernelGGL((gemm_kernel<128, 64, USE>), grid, block, 0, s, a);
  else if (t.hr == 128) hipLaunchKernelGGL((gemm_kernel<128, 128, USE>), grid, block, 0, s, a);
  else if (t.bn == 192) hipLaunchKernelGGL((gemm_kernel<256, 192, USE>), grid, block, 0, s, a);
  else if (t.bn == 128) hipLaunchKernelGGL((gemm_kernel<256, 128, USE>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((gemm_kernel<256, 256, USE>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <bool ROWS>
hipError_t launch_turn(const uint16_t* from, int64_t ld_from, int rows, int cols, uint16_t* to, int64_t ld_to, int rows_pad,
                       const int32_t* marks, const uint3* ranges, int blocks, Exponents* exps, hipStream_t s) {
  if (rows_pad == 0) return hipSuccess;
  hipLaunchKernelGGL(turn_kernel<ROWS>, dim3((rows_pad + kTurn - 1) / kTurn, (cols + kTurn - 1) / kTurn), dim3(256), 0, s, from, ld_from, rows,
                     cols, to, ld_to, rows_pad, marks, ranges, blocks, exps);
  return hipGetLastError();
}

// What the backward pass keeps in the workspace.
struct Plan {
  int piece;                 // columns of a piece
  int parts;                 // of k in dh's product
  int64_t mpad, vpad;
  size_t ht, wt, dz, dzt, sums, total;
};
constexpr int64_t kPieceBytes = 400 << 20;       // dz both ways and the turned W of a piece
Plan make_plan(int rows, int n, int d, bool f32) {
  Plan p{};
  p.mpad = up(rows, 64);
  const int64_t per_column = 2 * (rows + p.mpad * (f32 ? 2 : 1) + d);
  int64_t piece = kPieceBytes / per_column / 256 * 256;
  if (piece < 256) piece = 256;
  // pieces of one size
  const int64_t count = (n + piece - 1) / piece;
  piece = up((n + count - 1) / count, 256);
  p.piece = static_cast<int>(piece < n ? piece : n);
  p.vpad = up(p.piece, 64);
  const Shape t = choose(rows, d);
  const int64_t tiles = up(rows, t.hr) / t.hr * (up(d, t.bn) / t.bn);
  // few tiles: k (a piece's ids) dealt over workgroups, at least 512 each
  p.parts = 1;
  while (tiles * p.parts * 2 <= 256 && p.vpad / 64 / (p.parts * 2) >= 8) p.parts *= 2;
  p.ht = up256(2 * d * p.mpad);
  p.wt = up256(2 * d * p.vpad);
  p.dz = up256(2 * rows * p.vpad);
  p.dzt = up256(2 * p.piece * p.mpad * (f32 ? 2 : 1));
  p.sums = p.piece < n || p.parts > 1 ? up256(sizeof(float) * p.parts * static_cast<size_t>(rows) * d) : 0;
  p.total = p.ht + p.wt + p.dz + p.dzt + p.sums + up256(sizeof(uint3) * kRangeBlocks) + 256;
  return p;
}

}  // namespace

size_t cross_entropy_bytes(int rows, int n) {
  const size_t tiles = (static_cast<size_t>(n) + 63) / 64;           // the narrowest tile's
  return up256(sizeof(float2) * tiles * rows) + up256(sizeof(float) * rows) + 256;
}

hipError_t launch_cross_entropy(const CrossEntropyArgs& c, hipStream_t s) {
  if (c.rows == 0) return hipSuccess;
  GemmArgs a{};
  a.A = c.h; a.B = c.W; a.lda = a.ldb = c.d;
  a.M = c.rows; a.N = c.n; a.KT = c.d / 64; a.tail = c.d % 64; a.KS = 1;
  a.targets = c.targets;
  a.inv_tau = 1.f / c.tau; a.scale2 = kLog2e / c.tau;
  a.zt = static_cast<float*>(c.ws);
  a.part = reinterpret_cast<float2*>(static_cast<char*>(c.ws) + up256(sizeof(float) * c.rows));
  if (hipError_t e = launch_gemm<kLoss>(a, s); e != hipSuccess) return e;
  const int bn = choose(c.rows, c.n).bn;
  hipLaunchKernelGGL(finish_kernel, dim3((c.rows + 3) / 4), dim3(256), 0, s, a.part, a.zt, c.targets, c.rows, c.n, (c.n + bn - 1) / bn,
                     a.scale2, a.inv_tau, c.loss, c.lse);
  return hipGetLastError();
}

int cross_entropy_kernel_names(int rows, int n, int d, bool f32, char* buf, size_t cap) {
  const Plan p = make_plan(rows, n, d, f32);
  const Shape l = choose(rows, n), g = choose(rows, p.piece), r = choose(rows, d), t = choose(p.piece, d);
  return snprintf(buf, cap,
                  "gemm_kernel<%d, %d, kLoss>; pieces of %d: gemm_kernel<%d, %d, kGradient>, gemm_kernel<%d, %d, kRows> in %d parts, "
                  "gemm_kernel<%d, %d, %s>",
                  l.hr, l.bn, p.piece, g.hr, g.bn, r.hr, r.bn, p.parts, t.hr, t.bn, f32 ? "kTableTwoTerms" : "kTable");
}

size_t cross_entropy_backward_bytes(int rows, int n, int d, bool f32) { return make_plan(rows, n, d, f32).total; }

hipError_t launch_cross_entropy_backward(const CrossEntropyArgs& c, hipStream_t s) {
  if (c.rows == 0 && (!c.dW || c.accumulate)) return hipSuccess;
  const Plan p = make_plan(c.rows, c.n, c.d, c.f32);
  char* at = static_cast<char*>(c.ws);
  auto take = [&](size_t bytes) {
    char* const q = at;
    at += bytes;
    return q;
  };
  uint16_t* const hT = reinterpret_cast<uint16_t*>(take(p.ht));
  uint16_t* const WT = reinterpret_cast<uint16_t*>(take(p.wt));
  uint16_t* const dz = reinterpret_cast<uint16_t*>(take(p.dz));
  uint16_t* const dzT = reinterpret_cast<uint16_t*>(take(p.dzt));
  float* const sums = p.sums ? reinterpret_cast<float*>(take(p.sums)) : nullptr;
  uint3* const ranges = reinterpret_cast<uint3*>(take(up256(sizeof(uint3) * kRangeBlocks)));
  Exponents* const exps = reinterpret_cast<Exponents*>(take(256));
  const int64_t pieces = c.dh ? static_cast<int64_t>(c.n) * c.d / 8 : 0;
  const int64_t want = (pieces + 256 * 8 - 1) / (256 * 8) > c.rows ? (pieces + 256 * 8 - 1) / (256 * 8) : c.rows;
  const int blocks = static_cast<int>(want < 1 ? 1 : want < kRangeBlocks ? want : kRangeBlocks);
  hipLaunchKernelGGL(range_kernel, dim3(blocks), dim3(256), 0, s, reinterpret_cast<const u32x4*>(c.W), pieces,
                     reinterpret_cast<const u32x4*>(c.h), c.rows, c.d / 8, c.weight, c.targets, ranges);
  hipError_t e = hipSuccess;
  if (c.dW && c.rows > 0) {
    e = launch_turn<true>(c.h, c.d, c.rows, c.d, hT, p.mpad, static_cast<int>(p.mpad), c.targets, ranges, blocks, exps, s);
  } else {
    hipLaunchKernelGGL(settle_kernel, dim3(1), dim3(256), 0, s, ranges, blocks, exps);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  const int terms = c.f32 ? 2 : 1;
  for (int v0 = 0; v0 < c.n; v0 += p.piece) {
    const int v = c.n - v0 < p.piece ? c.n - v0 : p.piece;
    const int64_t vpad = up(v, 64);
    const uint16_t* const W = c.W + static_cast<int64_t>(v0) * c.d;
    if (c.rows > 0) {
      GemmArgs a{};
      a.A = c.h; a.B = W; a.lda = a.ldb = c.d;
      a.M = c.rows; a.N = v; a.KT = c.d / 64; a.tail = c.d % 64; a.KS = 1;
      a.targets = c.targets; a.col0 = v0;
      a.inv_tau = 1.f / c.tau; a.scale2 = kLog2e / c.tau;
      a.lse = c.lse; a.weight = c.weight; a.exps = exps;
      a.dz = c.dh ? dz : nullptr; a.ldz = vpad;
      a.dzT = c.dW ? dzT : nullptr; a.ldT = p.mpad * terms; a.lo = static_cast<int>(p.mpad); a.two_terms = c.f32;
      if ((e = launch_gemm<kGradient>(a, s)) != hipSuccess) return e;
    }
    if (c.dh && c.rows > 0) {
      if ((e = launch_turn<false>(W, c.d, v, c.d, WT, vpad, static_cast<int>(vpad), nullptr, nullptr, 0, exps, s)) != hipSuccess) return e;
      GemmArgs a{};
      a.A = dz; a.B = WT; a.lda = a.ldb = vpad;
      a.M = c.rows; a.N = c.d; a.KT = static_cast<int>(vpad / 64); a.KS = p.parts;
      a.sums = sums; a.first = v0 == 0; a.last = p.parts == 1 && v0 + v == c.n;
      a.out = c.dh;
      a.targets = c.targets; a.weight = c.weight; a.inv_tau = 1.f / c.tau; a.exps = exps;
      if ((e = launch_gemm<kRows>(a, s)) != hipSuccess) return e;
    }
    if (c.dW) {
      GemmArgs a{};
      a.A = dzT; a.B = hT; a.lda = p.mpad * terms; a.ldb = p.mpad;
      a.M = v; a.N = c.d; a.KT = static_cast<int>(p.mpad / 64); a.KS = 1;
      a.lo = static_cast<int>(p.mpad);
      a.out = c.f32 ? static_cast<void*>(static_cast<float*>(c.dW) + static_cast<int64_t>(v0) * c.d)
                    : static_cast<void*>(static_cast<uint16_t*>(c.dW) + static_cast<int64_t>(v0) * c.d);
      a.accumulate = c.accumulate;
      a.inv_tau = 1.f / c.tau; a.exps = exps;
      if ((e = c.f32 ? launch_gemm<kTableTwoTerms>(a, s) : launch_gemm<kTable>(a, s)) != hipSuccess) return e;
    }
  }
  if (c.dh && c.rows > 0 && p.parts > 1) {
    const int64_t count = static_cast<int64_t>(c.rows) * c.d;
    hipLaunchKernelGGL(join_rows_kernel, dim3(static_cast<uint32_t>((count / 4 + 255) / 256)), dim3(256), 0, s, sums, p.parts, count, c.d,
                       c.targets, c.weight, 1.f / c.tau, exps, c.dh);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace scd
