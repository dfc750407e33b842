// Stand-ins for the launches of pages.hip (the HIP calls are fake_hip.cpp's).
#include <hip/hip_runtime.h>

#include "cache.h"

namespace gr {
hipError_t launch_read(const ReadArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_fork(const RefArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_grow(const RefArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_release(const RefArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_compact(const RefArgs &, hipStream_t) { return hipSuccess; }
static CopyArgs last;
hipError_t launch_copy(const CopyArgs &a, hipStream_t) {
  last = a;
  return hipSuccess;
}
}  // namespace gr

extern "C" int fake_copy_flat() { return gr::last.flat; }
