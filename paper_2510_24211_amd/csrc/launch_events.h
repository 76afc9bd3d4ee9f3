// Launches of the LM heads, timed where the caller asks for it.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

namespace scd {
namespace {

// Optional timing of the launch: the runtime attaches the two events to the dispatch itself
// (start and stop time of the kernel), so no marker packets of their own enter the stream.
struct LaunchEvents {
  hipEvent_t start, stop;
};
template <class Kern, class... Args>
void launch_kernel(Kern kernel, dim3 grid, dim3 block, hipStream_t s, const LaunchEvents& ev, Args... args) {
  if (ev.start && ev.stop) hipExtLaunchKernelGGL(kernel, grid, block, 0, s, ev.start, ev.stop, 0, args...);
  else hipLaunchKernelGGL(kernel, grid, block, 0, s, args...);
}

}  // namespace
}  // namespace scd
