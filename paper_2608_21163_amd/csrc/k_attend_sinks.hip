// k_attend_sinks.hip -- attention over 16-bit pages with first tokens that every row sees
// beside its window.
#include "attend.h"

namespace gr {

hipError_t launch_attend_sinks(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? attend_type<F16, Sinks>(tile_rows, a, st) : attend_type<Bf16, Sinks>(tile_rows, a, st);
}

hipError_t launch_weights_sinks(bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? weights_type<F16, Sinks>(a, st) : weights_type<Bf16, Sinks>(a, st);
}

}  // namespace gr
