// k_attend_packed.hip -- attention over packed pages.
#include "attend.h"

namespace gr {

hipError_t launch_attend_packed(uint32_t tile_rows, bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? attend_type<F16, Packed>(tile_rows, a, st) : attend_type<Bf16, Packed>(tile_rows, a, st);
}

hipError_t launch_weights_packed(bool f16, const AttendArgs &a, hipStream_t st) {
  return f16 ? weights_type<F16, Packed>(a, st) : weights_type<Bf16, Packed>(a, st);
}

}  // namespace gr
