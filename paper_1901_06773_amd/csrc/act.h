// The smooth activation of group norm and of the gated layer, and its slope.
#pragma once
#include <hip/hip_runtime.h>

namespace acc {

// 1 / (1 + e^-z) by the base-two exponential and the reciprocal of the hardware, a rounding or two each; the rounding of z * log2 e makes e^-z wrong by
// |z| / 1.4 of them more, which is little beside 1 where z is positive and where z is negative leaves a value of at most 1 / 4 of z's size (an exact expf
// and a division took the kernels from memory to arithmetic: 8 images of 56x56, 64 channels, bf16 forward 39 us)
__device__ __forceinline__ float sigmoid(float z) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
#else
  return z;
#endif
}
__device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid(z);
  return s * (1.f + z * (1.f - s));
}

}  // namespace acc
