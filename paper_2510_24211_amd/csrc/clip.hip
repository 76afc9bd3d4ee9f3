// Global norm of gradients and their clipping:
//   norm = sqrt(sum over all tensors of g^2),   out = g * min(1, most / norm)
// The tensors (their addresses, sizes and types) travel in the kernel's arguments, kTensors to a launch: nothing has to be copied to the
// card first, and a recorded graph holds them.  Chunks of kChunk elements are dealt to the workgroups; squares are added up in 64 bits
// (they are exact there: no range is lost, and the unit that adds them is idle otherwise), the workgroups' sums in order by a last one.
//   Bound by memory, each gradient being read twice: the norm has to be known first.  Clipping goes backwards, so that it begins with what the
// norm's pass has left in the last cache, and stores past the caches, so that what it writes does not drive that out.  805 million bf16
// gradients in 50 tensors into bf16: 841 us (4.83 GB: 5.7 TB/s) where forwards and through the caches took 940; in place 878, 297 with nothing
// to clip; 34 million fp32 ones into bf16 62 us, 67 before.  512 workgroups of 64 KB at a time are as fast as any number up to 2048 (841 to
// 860 us), 4096 with 16 KB take 880.
#include <algorithm>

#include "eights.h"
#include "scd_device.h"
#include "scd_kernels.h"

namespace scd {
namespace {

constexpr int kTensors = 100;                    // (the arguments of a launch end at 4 KB)
constexpr int kUnroll = 8, kChunk = 256 * 8 * kUnroll;
constexpr int kGroups = 512;                     // workgroups of a launch

struct Table {
  const void* in[kTensors];
  void* out[kTensors];
  int64_t n[kTensors];
  uint32_t first[kTensors + 1];                  // first chunk of a tensor, among all chunks of the launch
  uint8_t in_f32[kTensors], out_f32[kTensors];
  int32_t count;
};
static_assert(sizeof(Table) + 64 <= 4096, "kernel arguments");

// The tensor that holds a chunk: the last one that begins at it or before (empty tensors begin where the next one does).
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t chunk) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Tensors are views of larger buffers as often as not: their elements' own alignment is all that is asked of them.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
template <bool F32>
struct AnyEight;
template <>
struct AnyEight<false> {
  u32x4 v;
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    v = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(p) + at);
  }
  __device__ __forceinline__ f32x8 wide() const { return widen(v); }
};
template <>
struct AnyEight<true> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    a = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(p) + at);
    b = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(p) + at + 4);
  }
  __device__ __forceinline__ f32x8 wide() const { return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; }
};
template <bool F32>
__device__ __forceinline__ void put_any(void* p, int64_t at, f32x8 v) {
  if constexpr (F32) {
    float* const q = static_cast<float*>(p) + at;
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_any*>(q));
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_any*>(q + 4));
  } else {
    __builtin_nontemporal_store(narrow(v), reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(p) + at));
  }
}
template <bool F32>
__device__ __forceinline__ float one_of(const void* p, int64_t at) {
  if constexpr (F32) return static_cast<const float*>(p)[at];
  else return static_cast<float>(static_cast<const __bf16*>(p)[at]);
}
template <bool F32>
__device__ __forceinline__ void put_one(void* p, int64_t at, float v) {
  if constexpr (F32) static_cast<float*>(p)[at] = v;
  else static_cast<__bf16*>(p)[at] = static_cast<__bf16>(v);
}

// Calls eight(v, at) for every whole eight of the chunk that this thread has, one(v, at) for its single elements behind the last of them.
template <bool F32, class E, class O>
__device__ __forceinline__ void over_chunk(const void* in, int64_t n, int64_t begin, E&& eight, O&& one) {
  if (begin + kChunk <= n) {
    AnyEight<F32> v[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) v[j].load(in, begin + (j * 256 + threadIdx.x) * 8);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) eight(v[j].wide(), begin + (j * 256 + threadIdx.x) * 8);
    return;
  }
  const int64_t whole = n & ~static_cast<int64_t>(7);
  for (int64_t at = begin + threadIdx.x * 8; at < whole; at += 256 * 8) {
    AnyEight<F32> v;
    v.load(in, at);
    eight(v.wide(), at);
  }
  if (whole + threadIdx.x < n) one(one_of<F32>(in, whole + threadIdx.x), whole + threadIdx.x);
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int m = 32; m > 0; m /= 2) v += __shfl_xor(v, m);
  return v;
}

__global__ __launch_bounds__(256) void square_sum_kernel(const Table t, double* __restrict__ parts) {
  __shared__ double waves[4];
  double sum = 0.0;
  const uint32_t chunks = t.first[t.count];
  auto add = [&](float x) { sum = __builtin_fma(static_cast<double>(x), static_cast<double>(x), sum); };
  auto eight = [&](f32x8 v, int64_t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) add(v[j]);
  };
  auto one = [&](float v, int64_t) { add(v); };
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int k = tensor_of(t, c);
    const int64_t begin = static_cast<int64_t>(c - t.first[k]) * kChunk;
    if (t.in_f32[k]) over_chunk<true>(t.in[k], t.n[k], begin, eight, one);
    else over_chunk<false>(t.in[k], t.n[k], begin, eight, one);
  }
  sum = wave_sum_f64(sum);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

__global__ __launch_bounds__(1024) void norm_of_parts_kernel(const double* __restrict__ parts, int64_t count, float* __restrict__ norm) {
  __shared__ double waves[16];
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += 1024) sum += parts[i];
  sum = wave_sum_f64(sum);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += waves[w];
  norm[0] = static_cast<float>(__builtin_sqrt(sum));
}

__global__ __launch_bounds__(256) void clip_kernel(const Table t, float most, const float* __restrict__ norm) {
  const float have = norm[0];
  // 0 under an infinite norm, whatever max_norm is; a NaN for a NaN.  Factors near or below the end of fp32's normal numbers, which would lose
  // digits, are kept 2^128 times as large, with 2^-64 on either side of the product.
  const bool whole = have <= most && have < __builtin_inff(), far = most < have * 0x1p-96f;
  const float by = whole ? 1.f : have == __builtin_inff() ? 0.f : far ? __fdiv_rn(most * 0x1p64f, have * 0x1p-64f) : __fdiv_rn(most, have);
  const float side = far ? 0x1p-64f : 1.f;
  const uint32_t chunks = t.first[t.count];
  for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
    const uint32_t c = chunks - 1 - i;
    const int k = tensor_of(t, c);
    const bool in_f32 = t.in_f32[k], out_f32 = t.out_f32[k];
    void* const out = t.out[k];
    if (whole && out == t.in[k]) continue;           // (of one type then: nothing changes)
    const int64_t begin = static_cast<int64_t>(c - t.first[k]) * kChunk;
    auto go = [&](auto in_type, auto out_type) {
      constexpr bool IN = decltype(in_type)::value, OUT = decltype(out_type)::value;
      over_chunk<IN>(t.in[k], t.n[k], begin, [&](f32x8 v, int64_t at) { put_any<OUT>(out, at, v * side * by * side); },
                     [&](float v, int64_t at) { put_one<OUT>(out, at, v * side * by * side); });
    };
    if (in_f32) out_f32 ? go(TrueT{}, TrueT{}) : go(TrueT{}, FalseT{});
    else out_f32 ? go(FalseT{}, TrueT{}) : go(FalseT{}, FalseT{});
  }
}

// Tables of the tensors, kTensors or 2^31 chunks at most to each: go(table) for every one that has any elements.
template <class F>
hipError_t over_tables(const GradientTensor* g, int count, F&& go) {
  Table t;
  t.count = 0;
  t.first[0] = 0;
  auto flush = [&]() {
    const hipError_t e = t.first[t.count] != 0 ? go(t) : hipSuccess;
    t.count = 0;
    return e;
  };
  for (int i = 0; i < count; ++i) {
    const uint64_t chunks = (static_cast<uint64_t>(g[i].n) + kChunk - 1) / kChunk;
    if (t.count == kTensors || t.first[t.count] + chunks > 0x7FFFFFFFull)
      if (hipError_t e = flush(); e != hipSuccess) return e;
    t.in[t.count] = g[i].in;
    t.out[t.count] = g[i].out;
    t.n[t.count] = g[i].n;
    t.in_f32[t.count] = g[i].in_f32;
    t.out_f32[t.count] = g[i].out_f32;
    t.first[t.count + 1] = t.first[t.count] + static_cast<uint32_t>(chunks);
    ++t.count;
  }
  return flush();
}
inline int groups_of(const Table& t) { return static_cast<int>(std::min<uint32_t>(t.first[t.count], kGroups)); }

}  // namespace

size_t gradient_norm_bytes(const GradientTensor* g, int count) {
  size_t parts = 0;
  (void)over_tables(g, count, [&](const Table& t) {
    parts += groups_of(t);
    return hipSuccess;
  });
  return (sizeof(double) * parts + 256) / 256 * 256;
}

hipError_t launch_gradient_norm(const GradientTensor* g, int count, float* norm, void* ws, hipStream_t s) {
  double* const parts = static_cast<double*>(ws);
  int64_t made = 0;
  const hipError_t e = over_tables(g, count, [&](const Table& t) {
    hipLaunchKernelGGL(square_sum_kernel, dim3(groups_of(t)), dim3(256), 0, s, t, parts + made);
    made += groups_of(t);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(norm_of_parts_kernel, dim3(1), dim3(1024), 0, s, parts, made, norm);
  return hipGetLastError();
}

hipError_t launch_clip_gradients(const GradientTensor* g, int count, float most, const float* norm, hipStream_t s) {
  return over_tables(g, count, [&](const Table& t) {
    hipLaunchKernelGGL(clip_kernel, dim3(groups_of(t)), dim3(256), 0, s, t, most, norm);
    return hipGetLastError();
  });
}

}  // namespace scd
