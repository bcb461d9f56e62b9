// Activations in 8 bits: 32 consecutive features of a row share a scale 2^e, stored as the
// byte e + 127, with e = max(emin, floor(log2 max|x|) - 6); a feature is the nearest multiple
// n 2^e, |n| <= 127 (ties to even; beyond 127 steps 127, so the error is at most half a step,
// and at most one for the values within half a step of 128). n has seven bits and the scale is
// a power of two, so the values read back are exact in bf16, f16 and float: reading a
// checkpoint adds no rounding of its own. emin = -24 for f16, whose values are multiples of
// 2^-24, else -126 (the scale stays a normal float). The byte 255 marks a block that holds an
// infinity or a NaN; all of it reads back as NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace lp {

constexpr int CK_BLOCK = 32;

template <typename T>
constexpr uint32_t ck_min_byte() {
  return std::is_same<T, _Float16>::value ? 127 - 24 : 1;
}

// The scale byte of a block whose largest magnitude has these float bits (an infinity or a
// NaN has larger bits than every finite value).
template <typename T>
__device__ __forceinline__ uint32_t ck_byte(uint32_t absbits) {
  const uint32_t e = absbits >> 23;
  if (e == 255) return 255;
  return max((int)e - 6, (int)ck_min_byte<T>());
}

// 1 / scale of a byte (0 for a block that is not finite: all its n are 0)
__device__ __forceinline__ float ck_inv(uint32_t byte) {
  return byte == 255 ? 0.f : __builtin_bit_cast(float, (254u - byte) << 23);
}

__device__ __forceinline__ float ck_scale(uint32_t byte) {
  return byte == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
}

__device__ __forceinline__ int ck_round(float x, float inv) {
  if (inv == 0.f) return 0;
  return (int)fminf(fmaxf(rintf(x * inv), -127.f), 127.f);
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

}  // namespace lp
