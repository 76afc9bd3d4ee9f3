// What the kernels that multiply LDS-staged tiles share: operand types, loads from memory straight into LDS, the
// fences around them, loops unrolled at compile time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <utility>

namespace scd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
// 16-byte register value; a native vector (the HIP struct type is copied with memcpy,
// which keeps arrays of it in scratch memory)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct TrueT { static constexpr bool value = true; };
struct FalseT { static constexpr bool value = false; };
template <int N>
struct IntT { static constexpr int value = N; };

__device__ __forceinline__ void compiler_fence() { asm volatile("" ::: "memory"); }
// Also a boundary for the machine scheduler, which otherwise treats loads of never-written
// global memory as freely movable and may sink a prefetch down to its use.
__device__ __forceinline__ void hard_fence() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// 16 bytes per lane from base + off (per lane) to LDS byte address lds + ADD + 16 * lane (lds uniform).  The
// LDS address travels in m0, a reserved register: the compiler warns that it does not save what a statement
// clobbers there.  It has nothing to save, but has to see that whatever it sets m0 for itself is set again behind.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool NT, int ADD>
__device__ __forceinline__ void load_lds16(uint64_t base, uint32_t off, uint32_t lds) {
  if constexpr (NT)
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                 ::"s"(lds), "v"(off), "s"(base), "n"(ADD) : "memory", "m0", "scc");
  else
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 ::"s"(lds), "v"(off), "s"(base), "n"(ADD) : "memory", "m0", "scc");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void wait_loads() {       // until at most N of this wavefront's loads are in flight
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(IntT<I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

}  // namespace
}  // namespace scd
