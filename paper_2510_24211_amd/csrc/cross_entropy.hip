// Softmax cross entropy of hidden rows over the allowed ids of a vocabulary table, without keeping the logits:
//   z = h W^T / tau;  lse = log sum_v exp(z_v);  loss = lse - z_t
//   dz = weight * (exp(z - lse) - [v = t]) / tau;  dh = dz W;  dW = dz^T h
// Four matrix products of 2 * rows * n * d operations each (the logits are made again for the gradient), all on one tile
// routine that wants k along both operands' rows.
//   Forward: a tile of logits leaves (maximum, sum of exponentials) per row and the target's logit; finish_kernel joins a
// row's tiles.  Backward, for a piece of the vocabulary at a time: dz of the piece goes to the workspace as rows and as
// columns (k lies along ids for dh, along rows for dW), the piece of W and the rows of h are turned once for the same reason.
//   dz is rounded to bf16 for the matrix units: its terms err by up to 2^-8 of themselves, independently, as the bf16
// results do.  Where dW is kept in 32 bits dz enters that product as two bf16 terms (16 bits of its mantissa), at the
// price of a fifth product.  Statistics and sums are fp32.
#include "gemm_tile.h"
#include "scd_device.h"
#include "scd_kernels.h"

namespace scd {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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

enum GemmUse { kLoss, kGradient, kRows, kTable };

struct GemmArgs {
  const uint16_t* A;
  const uint16_t* B;
  int64_t lda, ldb;          // elements from row to row
  int M, N;                  // rows of A, of B
  int KT, tail, wrapB;       // whole k-tiles, elements of the ragged one; k-tiles after which B's columns begin again
  int MT, NT, KS;            // tiles, parts of k
  // kLoss, kGradient
  const int32_t* targets;
  float scale2, inv_tau;     // log2(e) / tau, 1 / tau
  int col0;                  // column of the first row of B
  float2* part;              // [M][NT]
  float* zt;                 // [M]
  const float* lse;
  const float* weight;
  uint16_t* dz;              // [M][ldz]
  uint16_t* dzT;             // [N][ldT]: hi terms, then (two_terms) lo terms `lo` columns on
  int64_t ldz, ldT;
  int lo;
  bool two_terms;
  // kRows: sums [KS][M][N] in fp32, over the pieces of the vocabulary so far; kRows, kTable: result [M][N]
  float* sums;
  bool first, last;
  void* out;
  bool f32, accumulate;
};

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
  const TileOperand A{reinterpret_cast<uint64_t>(a.A + row0 * a.lda), rows, static_cast<uint32_t>(a.lda * 2), 0x7FFFFFFF};
  const TileOperand B{reinterpret_cast<uint64_t>(a.B + col0 * a.ldb), cols, static_cast<uint32_t>(a.ldb * 2), a.wrapB};
  // the workgroups of an XCD meet in its L2, the XCDs start at different columns
  const int rot = KT > 0 ? static_cast<int>(static_cast<int64_t>(blockIdx.x % 8) * KT / 8) : 0;
  multiply_tile<K>(lds, A, B, kt0, KT, a.tail, rot, acc);
  __syncthreads();

  if constexpr (USE == kLoss || USE == kGradient) {
    int* const target = reinterpret_cast<int*>(lds);
    float* const lse2 = reinterpret_cast<float*>(lds) + HR;
    float* const coef = lse2 + HR;
    for (int r = tid; r < HR; r += K::THREADS) {
      const int t = r < rows ? a.targets[row0 + r] : -1;
      target[r] = t < 0 ? -1 : t - a.col0 - col0 < 0 || t - a.col0 - col0 >= BN ? BN : t - a.col0 - col0;   // column of the tile
      if constexpr (USE == kGradient) {
        lse2[r] = r < rows ? a.lse[row0 + r] * kLog2e : 0.f;
        coef[r] = (r < rows && a.weight ? a.weight[row0 + r] : 1.f) * a.inv_tau;
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
            if (t == c0 + c * 32) a.zt[row0 + r] = acc[c][i][j] * a.inv_tau;
            z[c] = c0 + c * 32 < cols ? acc[c][i][j] * a.scale2 : -INFINITY;
            m = fmaxf(m, z[c]);
          }
          m = half_fold(m, [](float x, float y) { return fmaxf(x, y); });
          const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int c = 0; c < NC; ++c) s += exp2_fast(z[c] - ref);
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
        for (int k = 0; k < K::WCOL; ++k) s += w[k].y * exp2_fast(w[k].x - ref);
        a.part[static_cast<int64_t>(row0 + r) * a.NT + at.b] = make_float2(m, s);
      }
    } else {
      uint16_t* const tile = reinterpret_cast<uint16_t*>(lds + 16 * HR);
      // dz replaces the logits
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = wr * K::RW + block_row(i, j, lg), t = target[r];
          const float l = lse2[r], g = coef[r];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const float p = exp2_fast(__builtin_fmaf(acc[c][i][j], a.scale2, -l));
            const float v = g * (p - (t == c0 + c * 32 ? 1.f : 0.f));
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
              tile[(wr * K::RW + block_row(i, j, lg)) * (BN + 8) + c0 + c * 32] = bf16_bits(acc[c][i][j]);
        __syncthreads();
        store_lines<HR, BN, K::THREADS>(tile, a.dz + row0 * a.ldz + col0, a.ldz, rows, static_cast<int>(a.ldz) - col0);
        __syncthreads();
      }
      if (a.dzT) {
        const int stretch = a.lo;                       // columns of one term
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
                  b[e] = bf16_bits(acc[c][i][4 * g + e]);
                  acc[c][i][4 * g + e] -= bf16_value(b[e]);       // the rest, for the second term
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
    }
    if (a.f32 || a.accumulate) {
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
            if (a.f32) {
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
                                                     float* __restrict__ loss, float* __restrict__ lse) {
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= rows) return;
  const float2* const mine = part + static_cast<int64_t>(r) * NT;
  float m = -INFINITY, s = 0.f;
  for (int t = lane; t < NT; t += 64) {
    const float2 p = mine[t];
    const float high = fmaxf(m, p.x), ref = high == -INFINITY ? 0.f : high;
    s = s * exp2_fast(m - ref) + p.y * exp2_fast(p.x - ref);
    m = high;
  }
  float high = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) high = fmaxf(high, __shfl_xor(high, o, 64));
  const float ref = high == -INFINITY ? 0.f : high;
  s *= exp2_fast(m - ref);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) {
    const float l = (high + __log2f(s)) * kLn2;
    const int t = targets[r];
    lse[r] = l;
    loss[r] = t < 0 ? 0.f : t >= n ? INFINITY : l - zt[r];       // an id outside the allowed ones has no probability
  }
}

// ---- to[c][r] = from[r][c] for r < rows, 0 for r up to rows_pad and for rows with a negative mark --------
constexpr int kTurn = 64;
__global__ __launch_bounds__(256) void turn_kernel(const uint16_t* __restrict__ from, int64_t ld_from, int rows, int cols,
                                                   uint16_t* __restrict__ to, int64_t ld_to, int rows_pad,
                                                   const int32_t* __restrict__ marks) {
  __shared__ uint16_t tile[kTurn][kTurn + 2];
  const int r0 = blockIdx.x * kTurn, c0 = blockIdx.y * kTurn;
  for (int p = threadIdx.x; p < kTurn * kTurn / 8; p += 256) {
    const int r = p / (kTurn / 8), c = p % (kTurn / 8) * 8;
    u32x4 v{0u, 0u, 0u, 0u};
    if (r0 + r < rows && c0 + c < cols && !(marks && marks[r0 + r] < 0))
      v = *reinterpret_cast<const u32x4*>(from + static_cast<int64_t>(r0 + r) * ld_from + c0 + c);
    uint32_t* const at = reinterpret_cast<uint32_t*>(&tile[r][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e) at[e] = v[e];
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
__global__ __launch_bounds__(256) void join_rows_kernel(const float* __restrict__ sums, int parts, int64_t count, uint16_t* __restrict__ out) {
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= count) return;                       // count is a multiple of 8
  float v[4] = {};
  for (int p = 0; p < parts; ++p) {
    const float4 t = *reinterpret_cast<const float4*>(sums + p * count + at);
    v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
  }
  *reinterpret_cast<uint2*>(out + at) = make_uint2(bf16_bits(v[0]) | static_cast<uint32_t>(bf16_bits(v[1])) << 16,
                                                   bf16_bits(v[2]) | static_cast<uint32_t>(bf16_bits(v[3])) << 16);
}

// ---- host --------------------------------------------------------------------------------------------
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Shape {
  int hr, bn;
};
// Tiles of which one round of a workgroup per CU costs `cost`: as in the LM head's choice.
Shape choose(int64_t M, int64_t N) {
  struct Option { int hr, bn, cost; };
  constexpr Option options[] = {{128, 128, 27}, {256, 128, 40}, {256, 256, 73}};
  Shape best{128, 128};
  int64_t least = -1;
  for (const Option& o : options) {
    const int64_t cost = ((M + o.hr - 1) / o.hr * ((N + o.bn - 1) / o.bn) + 255) / 256 * o.cost;
    if (least < 0 || cost < least) {
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
  if (t.hr == 128) hipLaunchKernelGGL((gemm_kernel<128, 128, USE>), grid, block, 0, s, a);
  else if (t.bn == 128) hipLaunchKernelGGL((gemm_kernel<256, 128, USE>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((gemm_kernel<256, 256, USE>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_turn(const uint16_t* from, int64_t ld_from, int rows, int cols, uint16_t* to, int64_t ld_to, int rows_pad,
                       const int32_t* marks, hipStream_t s) {
  if (rows_pad == 0) return hipSuccess;
  hipLaunchKernelGGL(turn_kernel, dim3((rows_pad + kTurn - 1) / kTurn, (cols + kTurn - 1) / kTurn), dim3(256), 0, s, from, ld_from, rows, cols, to,
                     ld_to, rows_pad, marks);
  return hipGetLastError();
}

// What the backward pass keeps in the workspace.
struct Plan {
  int piece;                 // columns of a piece
  int parts;                 // of k in dh's product
  int64_t mpad, vpad;
  size_t ht, wt, dz, dzt, sums, total;
};
constexpr int64_t kPieceBytes = 400 << 20;
Plan make_plan(int rows, int n, int d, bool f32) {
  Plan p{};
  p.mpad = up(rows, 64);
  const int64_t per_column = 2 * (rows + p.mpad * (f32 ? 2 : 1) + d);
  int64_t piece = kPieceBytes / per_column / 256 * 256;
  if (piece < 256) piece = 256;
  if (piece > 16384) piece = 16384;
  // pieces of one size
  const int64_t count = (n + piece - 1) / piece;
  piece = up((n + count - 1) / count, 256);
  p.piece = static_cast<int>(piece < n ? piece : n);
  p.vpad = up(p.piece, 64);
  const Shape t = choose(rows, d);
  const int64_t tiles = up(rows, t.hr) / t.hr * (up(d, t.bn) / t.bn);
  p.parts = 1;
  while (tiles * p.parts * 2 <= 256 && p.vpad / 64 / (p.parts * 2) >= 8) p.parts *= 2;
  p.ht = up256(2 * d * p.mpad);
  p.wt = up256(2 * d * p.vpad);
  p.dz = up256(2 * rows * p.vpad);
  p.dzt = up256(2 * p.piece * p.mpad * (f32 ? 2 : 1));
  p.sums = p.piece < n || p.parts > 1 ? up256(sizeof(float) * p.parts * static_cast<size_t>(rows) * d) : 0;
  p.total = p.ht + p.wt + p.dz + p.dzt + p.sums + 256;
  return p;
}

}  // namespace

size_t cross_entropy_bytes(int rows, int n, int) {
  const size_t tiles = (static_cast<size_t>(n) + 127) / 128;         // the narrowest tile's
  return up256(sizeof(float2) * tiles * rows) + up256(sizeof(float) * rows) + 256;
}

hipError_t launch_cross_entropy(const CrossEntropyArgs& c, hipStream_t s) {
  if (c.rows == 0) return hipSuccess;
  GemmArgs a{};
  a.A = c.h; a.B = c.W; a.lda = a.ldb = c.d;
  a.M = c.rows; a.N = c.n; a.KT = c.d / 64; a.tail = c.d % 64; a.wrapB = 0x7FFFFFFF; a.KS = 1;
  a.targets = c.targets;
  a.inv_tau = 1.f / c.tau; a.scale2 = kLog2e / c.tau;
  a.zt = static_cast<float*>(c.ws);
  a.part = reinterpret_cast<float2*>(static_cast<char*>(c.ws) + up256(sizeof(float) * c.rows));
  if (hipError_t e = launch_gemm<kLoss>(a, s); e != hipSuccess) return e;
  const int bn = choose(c.rows, c.n).bn;
  hipLaunchKernelGGL(finish_kernel, dim3((c.rows + 3) / 4), dim3(256), 0, s, a.part, a.zt, c.targets, c.rows, c.n, (c.n + bn - 1) / bn,
                     c.loss, c.lse);
  return hipGetLastError();
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
  hipError_t e = hipSuccess;
  if (c.dW && (e = launch_turn(c.h, c.d, c.rows, c.d, hT, p.mpad, static_cast<int>(p.mpad), c.targets, s)) != hipSuccess) return e;
  const int terms = c.f32 ? 2 : 1;
  for (int v0 = 0; v0 < c.n; v0 += p.piece) {
    const int v = c.n - v0 < p.piece ? c.n - v0 : p.piece;
    const int64_t vpad = up(v, 64);
    const uint16_t* const W = c.W + static_cast<int64_t>(v0) * c.d;
    if (c.rows > 0) {
      GemmArgs a{};
      a.A = c.h; a.B = W; a.lda = a.ldb = c.d;
      a.M = c.rows; a.N = v; a.KT = c.d / 64; a.tail = c.d % 64; a.wrapB = 0x7FFFFFFF; a.KS = 1;
      a.targets = c.targets; a.col0 = v0;
      a.inv_tau = 1.f / c.tau; a.scale2 = kLog2e / c.tau;
      a.lse = c.lse; a.weight = c.weight;
      a.dz = c.dh ? dz : nullptr; a.ldz = vpad;
      a.dzT = c.dW ? dzT : nullptr; a.ldT = p.mpad * terms; a.lo = static_cast<int>(p.mpad); a.two_terms = c.f32;
      if ((e = launch_gemm<kGradient>(a, s)) != hipSuccess) return e;
    }
    if (c.dh && c.rows > 0) {
      if ((e = launch_turn(W, c.d, v, c.d, WT, vpad, static_cast<int>(vpad), nullptr, s)) != hipSuccess) return e;
      GemmArgs a{};
      a.A = dz; a.B = WT; a.lda = a.ldb = vpad;
      a.M = c.rows; a.N = c.d; a.KT = static_cast<int>(vpad / 64); a.wrapB = 0x7FFFFFFF; a.KS = p.parts;
      a.sums = sums; a.first = v0 == 0; a.last = p.parts == 1 && v0 + v == c.n;
      a.out = c.dh;
      if ((e = launch_gemm<kRows>(a, s)) != hipSuccess) return e;
    }
    if (c.dW) {
      GemmArgs a{};
      a.A = dzT; a.B = hT; a.lda = p.mpad * terms; a.ldb = p.mpad;
      a.M = v; a.N = c.d; a.KT = static_cast<int>(p.mpad / 64) * terms; a.wrapB = static_cast<int>(p.mpad / 64); a.KS = 1;
      if (a.wrapB == 0) a.wrapB = 0x7FFFFFFF;
      a.out = c.f32 ? static_cast<void*>(static_cast<float*>(c.dW) + static_cast<int64_t>(v0) * c.d)
                    : static_cast<void*>(static_cast<uint16_t*>(c.dW) + static_cast<int64_t>(v0) * c.d);
      a.f32 = c.f32; a.accumulate = c.accumulate;
      if ((e = launch_gemm<kTable>(a, s)) != hipSuccess) return e;
    }
  }
  if (c.dh && c.rows > 0 && p.parts > 1) {
    const int64_t count = static_cast<int64_t>(c.rows) * c.d;
    hipLaunchKernelGGL(join_rows_kernel, dim3(static_cast<uint32_t>((count / 4 + 255) / 256)), dim3(256), 0, s, sums, p.parts, count, c.dh);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace scd
