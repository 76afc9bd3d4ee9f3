// Root-mean-square norm of hidden rows with the residual's addition, and its gradient:
//   s = x + r,   inv = 1 / sqrt(mean(s^2) + eps),   y = s * inv * g
//   a = g * dy,  dx = inv * (a - s * inv^2 * mean(a * s)) + ds,   dg = sum over the rows of dy * s * inv
// Everything in fp32 (s is normed before it is rounded to the stream's type), each result rounded once.  The normed rows are stored as
// bf16, or as e4m3 codes with a scale for each 128 of a row, which is what the LM head over 8-bit rows reads.  All of it moves
// memory and computes little: a row is read once and kept in registers until it is written.
//   Bound by memory: 25600 x 4096 rows in bf16 take 146 us (839 MB: 5.75 TB/s; a large copy reaches 5.1), 2304 x 4096 into 8 bits 12.8 us (66 MB), their
// gradient 152 us (839 MB and 17 MB of the workgroups' sums: 5.6 TB/s), with dx and ds in fp32 225 (1.26 GB: 5.6).  Small calls are a launch: one row of 1280
// takes 2.4 us on the card, 515 rows of the gradient 5.2 and 3.8 us for the gains.  Rows of more than 8192 columns are read twice: 4096 x 16384 take 111 us,
// 98 into 8 bits, the gradient 151, 194 with fp32 (4.8, 4.8, 3.6 and 4.2 TB/s of what has to move).
//   A row has a wavefront up to 1024 columns (no barrier; four rows to a workgroup), a workgroup beyond.
#include <algorithm>

#include "eights.h"
#include "scd_device.h"
#include "scd_kernels.h"

namespace scd {
namespace {

enum { kNoStream = 0, kStreamBf16 = 1, kStreamF32 = 2 };

template <int STREAM>
struct Pair {            // eight elements of x and of the residual
  Eight<false> x;
  Eight<STREAM == kStreamF32> r;
  __device__ __forceinline__ f32x8 sum() const {
    f32x8 s = x.wide();
    if constexpr (STREAM != kNoStream) s += r.wide();
    return s;
  }
};
template <int STREAM>
__device__ __forceinline__ Pair<STREAM> load_pair(const NormArgs& a, int64_t at) {
  Pair<STREAM> p;
  p.x = load_eight<false>(a.x, at);
  if constexpr (STREAM != kNoStream) p.r = load_eight<STREAM == kStreamF32>(a.residual, at);
  return p;
}
__device__ __forceinline__ float squares(f32x8 v) {
  const f32x8 q = v * v;
  return ((q[0] + q[1]) + (q[2] + q[3])) + ((q[4] + q[5]) + (q[6] + q[7]));
}
__device__ __forceinline__ float products(f32x8 v, f32x8 w) {
  const f32x8 q = v * w;
  return ((q[0] + q[1]) + (q[2] + q[3])) + ((q[4] + q[5]) + (q[6] + q[7]));
}
__device__ __forceinline__ float inverse_root(float sum, int d, float eps) {
  return __fdiv_rn(1.f, __fsqrt_rn(__fdiv_rn(sum, static_cast<float>(d)) + eps));
}
// Sum over the workgroup's wavefronts of one value each, in every thread; `ex`: a word per wavefront, not in use by an earlier fold.
template <int W>
__device__ __forceinline__ float block_sum(float v, float* ex) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) ex[wave_index()] = v;
  __syncthreads();
  return fold_sum<W>(ex);
}

// The normed piece `p` (of d / 8) of a row: stored as bf16, or as codes with their scales.  All lanes of a wavefront call it together, on
// neighbouring pieces (lane l: a piece that is l modulo 16), those with p >= pieces have none.
template <bool EIGHT_BITS>
__device__ __forceinline__ void store_normed(const NormArgs& a, int64_t row, int p, int pieces, f32x8 y) {
  if constexpr (EIGHT_BITS) {
    uint32_t most = p < pieces ? largest_bits(y) : 0u;             // over the 16 lanes that share a scale
    most = max(most, dpp_u32<kDppXor1>(most));
    most = max(most, dpp_u32<kDppXor2>(most));
    most = max(most, dpp_u32<kDppHalfMirror>(most));
    most = max(most, dpp_u32<kDppMirror>(most));
    const E4M3Scale s = e4m3_scale(most);
    if (p < pieces) {
      static_cast<uint2*>(a.y)[row * pieces + p] = to_e4m3(y, s);
      if (p % 16 == 0) a.scales[row * ((pieces + 15) / 16) + p / 16] = s.scale;
    }
  } else {
    if (p < pieces) store_eight<false>(a.y, row * pieces + p, y);
  }
}

// T threads (a wavefront, or the workgroup of four) per row, up to NV pieces of eight elements each, held in registers.
template <int STREAM, bool EIGHT_BITS, int T, int NV>
__global__ __launch_bounds__(256) void norm_kernel(const NormArgs a) {
  __shared__ float ex[2][4];
  const int t = threadIdx.x % T, pieces = a.d / 8;
  int turn = 0;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / T) + (T == 64 ? wave_index() : 0); row < a.rows;
       row += static_cast<int64_t>(gridDim.x) * (256 / T), turn ^= 1) {
    const int64_t first = row * pieces;
    Pair<STREAM> in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) in[i] = load_pair<STREAM>(a, first + min(i * T + t, pieces - 1));
    f32x8 s[NV];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      s[i] = in[i].sum();
      if (i * T + t < pieces) {
        sum += squares(s[i]);
        if (STREAM != kNoStream && a.sum) store_eight<STREAM == kStreamF32>(a.sum, first + i * T + t, s[i]);
      }
    }
    sum = T == 64 ? wave_sum(sum) : block_sum<4>(sum, ex[turn]);
    const float inv = inverse_root(sum, a.d, a.eps);
    if (a.inv && t == 0) a.inv[row] = inv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int p = i * T + t;
      if (NV > 1 && p - t % 64 >= pieces) break;                 // none of the wavefront's lanes has a piece
      store_normed<EIGHT_BITS>(a, row, p, pieces, s[i] * inv * eight_of(a.gain_f32, a.gain, min(p, pieces - 1)));
    }
  }
}

// Rows of any length: x and the residual are read a second time.
template <int STREAM, bool EIGHT_BITS>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs a) {
  __shared__ float ex[2][16];
  const int pieces = a.d / 8;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const int64_t first = row * pieces;
    float sum = 0.f;
    for (int p = threadIdx.x; p < pieces; p += 1024) sum += squares(load_pair<STREAM>(a, first + p).sum());
    sum = block_sum<16>(sum, ex[turn]);
    const float inv = inverse_root(sum, a.d, a.eps);
    if (a.inv && threadIdx.x == 0) a.inv[row] = inv;
    for (int p = threadIdx.x; p - static_cast<int>(threadIdx.x % 64) < pieces; p += 1024) {
      const int q = min(p, pieces - 1);
      const f32x8 s = load_pair<STREAM>(a, first + q).sum();
      const f32x8 y = s * inv * eight_of(a.gain_f32, a.gain, q);
      if (STREAM != kNoStream && a.sum && p < pieces) store_eight<STREAM == kStreamF32>(a.sum, first + p, s);
      store_normed<EIGHT_BITS>(a, row, p, pieces, y);
    }
  }
}

constexpr int kMostGroups = 1 << 21;

template <int STREAM, bool EIGHT_BITS>
hipError_t launch_norm_of(const NormArgs& a, hipStream_t s) {
  const int pieces = a.d / 8;
  auto groups = [&](int per) { return dim3(static_cast<unsigned>(std::min<int64_t>((static_cast<int64_t>(a.rows) + per - 1) / per, kMostGroups))); };
  if (pieces <= 64) hipLaunchKernelGGL((norm_kernel<STREAM, EIGHT_BITS, 64, 1>), groups(4), dim3(256), 0, s, a);
  else if (pieces <= 128) hipLaunchKernelGGL((norm_kernel<STREAM, EIGHT_BITS, 64, 2>), groups(4), dim3(256), 0, s, a);
  else if (pieces <= 256) hipLaunchKernelGGL((norm_kernel<STREAM, EIGHT_BITS, 256, 1>), groups(1), dim3(256), 0, s, a);
  else if (pieces <= 512) hipLaunchKernelGGL((norm_kernel<STREAM, EIGHT_BITS, 256, 2>), groups(1), dim3(256), 0, s, a);
  else if (pieces <= 1024) hipLaunchKernelGGL((norm_kernel<STREAM, EIGHT_BITS, 256, 4>), groups(1), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((norm_long_kernel<STREAM, EIGHT_BITS>), groups(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------------------------
// A workgroup goes over its share of the rows, R at a time, and keeps the gains' gradient of the columns that its threads hold in
// registers; what the workgroups leave is added up, in order, by a second launch.
constexpr int kMostParts = 512;      // two workgroups on a compute unit (768 take 165 us for 25600 x 4096, 640 174, 256 173, 512 152)

template <bool STREAM_F32, bool GRAD_F32, int T, int NV, int R>
__global__ __launch_bounds__(256) void norm_backward_kernel(const NormBackwardArgs a) {
  constexpr int RW = 256 / T;          // rows side by side
  __shared__ float ex[2][R][4];
  __shared__ f32x4 whole[T == 64 ? 4 * 64 * 2 : 1];
  const int t = threadIdx.x % T, pieces = a.d / 8, side = T == 64 ? wave_index() : 0;
  f32x8 gain[NV], dgain[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    gain[i] = i * T + t < pieces ? eight_of(a.gain_f32, a.gain, i * T + t) : f32x8{};
    dgain[i] = f32x8{};
  }
  int turn = 0;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * (R * RW); at < a.rows; at += static_cast<int64_t>(gridDim.x) * (R * RW), turn ^= 1) {
    Eight<STREAM_F32> s[R][NV];
    Eight<false> dy[R][NV];
    Eight<GRAD_F32> ds[R][NV];
    float inv[R], dot[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = min(at + r * RW + side, static_cast<int64_t>(a.rows) - 1);
      inv[r] = a.inv[row];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int64_t p = row * pieces + min(i * T + t, pieces - 1);
        s[r][i] = load_eight<STREAM_F32>(a.sum, p);
        dy[r][i] = load_eight<false>(a.dy, p);
        if (a.dsum) ds[r][i] = load_eight<GRAD_F32>(a.dsum, p);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      dot[r] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i * T + t < pieces) dot[r] += products(gain[i] * dy[r][i].wide(), s[r][i].wide());
      dot[r] = wave_sum(dot[r]);
      if (T == 256 && (threadIdx.x & 63) == 0) ex[turn][r][wave_index()] = dot[r];
    }
    if (T == 256) __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = at + r * RW + side;
      if (row >= a.rows) break;
      const float c = __fdiv_rn(T == 256 ? fold_sum<4>(ex[turn][r]) : dot[r], static_cast<float>(a.d)) * inv[r] * inv[r];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int p = i * T + t;
        if (p >= pieces) continue;
        const f32x8 sw = s[r][i].wide(), dyw = dy[r][i].wide();
        f32x8 dx = (gain[i] * dyw - sw * c) * inv[r];
        if (a.dsum) dx += ds[r][i].wide();
        store_eight<GRAD_F32>(a.dx, row * pieces + p, dx);
        dgain[i] += dyw * sw * inv[r];
      }
    }
  }
  if (!a.dgain) return;
  float* const part = a.part + static_cast<int64_t>(blockIdx.x) * a.d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if constexpr (T == 64) {           // the wavefronts' own rows are joined first
      __syncthreads();
      store_eight<true>(whole, threadIdx.x, dgain[i]);
      __syncthreads();
      if (threadIdx.x < 64)
#pragma unroll
        for (int w = 1; w < 4; ++w) dgain[i] += load_eight<true>(whole, w * 64 + threadIdx.x).wide();
    }
    if (threadIdx.x < T && i * T + t < pieces) store_eight<true>(part, i * T + t, dgain[i]);
  }
}

// Rows of any length: first every row's mean of a * s, then dx and the gains' gradient by stripes of 2048 columns.
__global__ __launch_bounds__(1024) void norm_backward_mean_kernel(const NormBackwardArgs a) {
  __shared__ float ex[2][16];
  const int pieces = a.d / 8;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    float dot = 0.f;
    for (int p = threadIdx.x; p < pieces; p += 1024) {
      const f32x8 g = eight_of(a.gain_f32, a.gain, p) * load_eight<false>(a.dy, row * pieces + p).wide();
      dot += products(g, eight_of(a.stream_f32, a.sum, row * pieces + p));
    }
    dot = block_sum<16>(dot, ex[turn]);
    if (threadIdx.x == 0) a.mean[row] = __fdiv_rn(dot, static_cast<float>(a.d));
  }
}
__global__ __launch_bounds__(256) void norm_backward_long_kernel(const NormBackwardArgs a) {
  const int pieces = a.d / 8, p = blockIdx.x * 256 + threadIdx.x;
  if (p >= pieces) return;
  const f32x8 gain = eight_of(a.gain_f32, a.gain, p);
  f32x8 dgain{};
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const int64_t at = row * pieces + p;
    const float inv = a.inv[row], c = a.mean[row] * inv * inv;
    const f32x8 s = eight_of(a.stream_f32, a.sum, at), dy = load_eight<false>(a.dy, at).wide();
    f32x8 dx = (gain * dy - s * c) * inv;
    if (a.dsum) dx += eight_of(a.grad_f32, a.dsum, at);
    put_eight(a.grad_f32, a.dx, at, dx);
    dgain += dy * s * inv;
  }
  if (a.dgain) store_eight<true>(a.part + static_cast<int64_t>(blockIdx.y) * a.d, p, dgain);
}

// dg of 32 columns: eight lanes of four side by side, 32 of them along the parts.
__global__ __launch_bounds__(256) void norm_gain_kernel(const float* __restrict__ part, int parts, int d, void* dgain, bool f32, bool accumulate) {
  __shared__ f32x4 sums[256];
  const int x = threadIdx.x % 8, y = threadIdx.x / 8, col = blockIdx.x * 32 + x * 4;
  f32x4 v{};
  if (col < d)
    for (int k = y; k < parts; k += 32) v += *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(k) * d + col);
  sums[threadIdx.x] = v;
  __syncthreads();
#pragma unroll
  for (int half = 16; half > 0; half /= 2) {
    if (y < half) sums[threadIdx.x] += sums[threadIdx.x + half * 8];
    __syncthreads();
  }
  if (y != 0 || col >= d) return;
  v = sums[x];
  if (f32) {
    f32x4* const to = reinterpret_cast<f32x4*>(static_cast<float*>(dgain) + col);
    *to = accumulate ? *to + v : v;
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4* const to = reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(dgain) + col);
    if (accumulate) v += __builtin_convertvector(*to, f32x4);
    *to = __builtin_convertvector(v, bf16x4);
  }
}

struct BackwardPlan {
  int threads, pieces, rows, parts;       // threads per row (0: the long form), pieces of a thread, rows at a time, workgroups
};
BackwardPlan backward_plan(int rows, int d) {
  const int pieces = d / 8;
  BackwardPlan p = pieces <= 64 ? BackwardPlan{64, 1, 4, 0} : pieces <= 128 ? BackwardPlan{64, 2, 2, 0} : pieces <= 256 ? BackwardPlan{256, 1, 4, 0}
                 : pieces <= 512 ? BackwardPlan{256, 2, 2, 0} : pieces <= 1024 ? BackwardPlan{256, 4, 1, 0} : BackwardPlan{0, 0, 1, 0};
  const int64_t per = p.rows * (p.threads == 64 ? 4 : 1);
  // (the long form's stripes take shares of the rows such that as many workgroups run)
  const int64_t most = p.threads ? kMostParts : std::max<int64_t>(1, kMostParts * 2 / ((pieces + 255) / 256));
  p.parts = static_cast<int>(std::min((rows + per - 1) / per, most));
  return p;
}
inline size_t up256(size_t b) { return (b + 255) / 256 * 256; }

template <bool S, bool G>
hipError_t launch_backward_of(const NormBackwardArgs& a, const BackwardPlan& p, hipStream_t s) {
  const dim3 grid(p.parts), block(256);
  if (p.threads == 64 && p.pieces == 1) hipLaunchKernelGGL((norm_backward_kernel<S, G, 64, 1, 4>), grid, block, 0, s, a);
  else if (p.threads == 64) hipLaunchKernelGGL((norm_backward_kernel<S, G, 64, 2, 2>), grid, block, 0, s, a);
  else if (p.pieces == 1) hipLaunchKernelGGL((norm_backward_kernel<S, G, 256, 1, 4>), grid, block, 0, s, a);
  else if (p.pieces == 2) hipLaunchKernelGGL((norm_backward_kernel<S, G, 256, 2, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_backward_kernel<S, G, 256, 4, 1>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const bool e = a.scales != nullptr;
  if (!a.residual) return e ? launch_norm_of<kNoStream, true>(a, s) : launch_norm_of<kNoStream, false>(a, s);
  if (a.stream_f32) return e ? launch_norm_of<kStreamF32, true>(a, s) : launch_norm_of<kStreamF32, false>(a, s);
  return e ? launch_norm_of<kStreamBf16, true>(a, s) : launch_norm_of<kStreamBf16, false>(a, s);
}

// the workgroups' sums for the gains; for long rows, a word per row
size_t norm_backward_bytes(int rows, int d) {
  const BackwardPlan p = backward_plan(rows, d);
  return 256 + up256(sizeof(float) * p.parts * static_cast<size_t>(d)) + (p.threads ? 0 : up256(sizeof(float) * static_cast<size_t>(rows)));
}

hipError_t launch_norm_backward(const NormBackwardArgs& n, hipStream_t s) {
  NormBackwardArgs a = n;
  const BackwardPlan p = backward_plan(a.rows, a.d);
  a.part = static_cast<float*>(a.ws);
  a.mean = reinterpret_cast<float*>(static_cast<char*>(a.ws) + up256(sizeof(float) * p.parts * static_cast<size_t>(a.d)));
  hipError_t e = hipSuccess;
  if (a.rows > 0 && p.threads == 0) {
    hipLaunchKernelGGL(norm_backward_mean_kernel, dim3(std::min(a.rows, kMostGroups)), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(norm_backward_long_kernel, dim3((a.d / 8 + 255) / 256, p.parts), dim3(256), 0, s, a);
    e = hipGetLastError();
  } else if (a.rows > 0) {
    if (a.stream_f32) e = a.grad_f32 ? launch_backward_of<true, true>(a, p, s) : launch_backward_of<true, false>(a, p, s);
    else e = a.grad_f32 ? launch_backward_of<false, true>(a, p, s) : launch_backward_of<false, false>(a, p, s);
  }
  if (e != hipSuccess || !a.dgain || (a.rows == 0 && a.accumulate)) return e;
  hipLaunchKernelGGL(norm_gain_kernel, dim3((a.d + 31) / 32), dim3(256), 0, s, a.part, p.parts, a.d, a.dgain, a.dgain_f32, a.accumulate);
  return hipGetLastError();
}

}  // namespace scd
