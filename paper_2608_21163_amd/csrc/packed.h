// packed.h -- rows held in 4 bits: blocks of 32 elements, each 16 bytes of codes
// (sign, and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6; even elements in the
// low halves) and a scale byte s, a power of two: 2^(s - 127).  The conversions
// are the hardware's, two codes an instruction at the full rate (4.6 cycles a wave):
// exact to 16 bits for all scales that an append writes, nearest with
// ties to the even code on the way back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gr {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Scales that appends write, so that every value is a normal bf16 number, or an
// fp16 one without rounding.  A block with a larger scale counts as NaN.
struct PackBf16 {
  static constexpr int kMinScale = 2, kMaxScale = 252;
  template <int SEL> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, SEL));
  }
  template <int SEL> static __device__ __forceinline__ uint32_t code(uint32_t to, uint32_t two, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(to, __builtin_bit_cast(v2bf, two), s, SEL);
  }
};
struct PackF16 {
  static constexpr int kMinScale = 104, kMaxScale = 140;
  template <int SEL> static __device__ __forceinline__ uint32_t pair(uint32_t codes, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, SEL));
  }
  template <int SEL> static __device__ __forceinline__ uint32_t code(uint32_t to, uint32_t two, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(to, __builtin_bit_cast(v2h, two), s, SEL);
  }
};

// The factor of a scale byte: exponent bits, which is all that the conversions read
// (0 is 2^-127, as a test of every byte shows); 255 makes NaN of every code.
template <class P> __device__ __forceinline__ float pack_factor(uint32_t s) {
  return __uint_as_float((s > (uint32_t)P::kMaxScale ? 255u : s) << 23);
}

// Eight codes as eight 16-bit values.
template <class P>
__device__ __forceinline__ v4u unpack8(uint32_t codes, float factor) {
  return v4u{P::template pair<0>(codes, factor), P::template pair<1>(codes, factor), P::template pair<2>(codes, factor),
             P::template pair<3>(codes, factor)};
}

}  // namespace gr
