// Activations in 8 bits: the format's arithmetic, shared by the checkpoint kernels
// (checkpoint.hip) and the expert feed-forward kernels.  Not part of the public ABI.
//
// 32 consecutive values of a row share a step 2^(e - 6), 2^e <= max |v| < 2^(e + 1)
// (e at least -127), kept as the byte e + 127; 255 stands for a block that holds a NaN
// or an infinity.  A value is the whole number nearest to v / step (ties to even) in
// [-127, 127].  Scaling by a power of two is exact, so a code is off by at most half a
// step (a value in (127.5, 128) steps by less than one: max |v| / 127), a value that was
// a code comes back as it was, and every code is exact in bf16.
#pragma once

#include "gemm.h"

namespace trimmoe {

constexpr int kPackBlock = 32;

// the scale byte of a block from the bits of its largest magnitude
__device__ __forceinline__ uint32_t pack_scale(uint32_t max_bits) { return max_bits >> 23; }

// code of v (a block without NaN or infinity: scale < 255) in the lowest byte.  The step
// is 2^(scale - 133); adding 1.5 2^23 leaves the nearest whole number, ties to even, in
// the last bits (held to 127 before: that rounds to itself)
__device__ __forceinline__ uint32_t pack_code_bits(float v, uint32_t scale) {
  const float q = __builtin_amdgcn_fmed3f(__builtin_ldexpf(v, 133 - (int)scale), -127.f, 127.f);
  return __float_as_uint(q + 12582912.f);
}
__device__ __forceinline__ int8_t pack_code(float v, uint32_t scale) {
  return (int8_t)pack_code_bits(v, scale);
}
// a block's step; NaN where it stands for no number
__device__ __forceinline__ float pack_step(uint32_t scale) {
  return scale == 255 ? __builtin_nanf("") : __builtin_ldexpf(1.f, (int)scale - 133);
}
// what a code stands for (exact: a power of two times a whole number)
__device__ __forceinline__ float pack_value(int code, uint32_t scale) {
  return (float)code * pack_step(scale);
}

// the larger of two magnitudes as bits (NaN the largest of all)
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// checkpoint.hip: x [n, c] to codes [n, c] and scale [n, cdiv(c, 32)], and back
hipError_t launch_checkpoint_pack(bool bf16, int n, int c, const void* x, int8_t* codes,
                                  uint8_t* scale, hipStream_t st);
hipError_t launch_checkpoint_unpack(bool bf16, int n, int c, const int8_t* codes,
                                    const uint8_t* scale, void* x, hipStream_t st);

}  // namespace trimmoe
