// Device helpers of the training-side operators: element types, block sums and
// the codes of 8-bit optimiser states.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "train.h"

namespace bergson {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The sum over the CTA (whole warps, at most 32), in every thread; `red` holds a
// value per warp and may be reused after the call.
template <typename F>
__device__ __forceinline__ F block_sum(F v, F* red) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  F t = (threadIdx.x & 31) < (blockDim.x >> 5) ? red[threadIdx.x & 31] : F(0);
  t = warp_sum(t);
  __syncthreads();
  return t;
}

// Kahan-compensated running sum.
struct CompensatedSum {
  float s = 0.0f, c = 0.0f;
  __device__ __forceinline__ void add(float x) {
    const float y = x - c;
    const float t = s + y;
    c = (t - s) - y;
    s = t;
  }
};

// ---- 8-bit states.  A code is the top bits of a positive float below its sign,
// less those of the smallest magnitude held: truncating the bits and adding chance
// below the cut rounds up with a probability equal to the part cut off.
constexpr int kCodeShift = 20;                 // three bits of mantissa stay
constexpr int kFirstBase = 112 << 3;           // m: exponents 2^-15 .. 2^0 in 7 bits
constexpr int kSecondBase = 96 << 3;           // v: exponents 2^-31 .. 2^0 in 8 bits
constexpr float kTopInverse = static_cast<float>(1.0 / 1.875);   // 1.875: the largest code

__device__ __forceinline__ float decode_first(uint32_t code) {
  const uint32_t mag = code & 127u;
  const uint32_t bits = ((mag + kFirstBase) << kCodeShift) | ((code & 128u) << 24);
  return mag != 0 ? __uint_as_float(bits) : __uint_as_float((code & 128u) << 24);
}
__device__ __forceinline__ float decode_second(uint32_t code) {
  return code != 0 ? __uint_as_float((code + kSecondBase) << kCodeShift) : 0.0f;
}
// The scale of a block whose largest magnitude is `top`, and its inverse (0 for a block of zeros).
__device__ __forceinline__ float block_scale(float top) {
  return top > 0.0f ? fmaxf(__fmul_rn(top, kTopInverse), 1.17549435e-38f) : top;
}
__device__ __forceinline__ float block_inverse(float scale) {
  return scale > 0.0f ? __frcp_rn(scale) : 0.0f;
}
// `chance`: 16 random bits.
__device__ __forceinline__ uint32_t encode_first(float m, float inv, uint32_t chance) {
  const float y = __fmul_rn(fabsf(m), inv);
  int code = ((__float_as_int(y) + static_cast<int>(chance << 4)) >> kCodeShift) - kFirstBase;
  code = min(max(code, 0), 127);
  return static_cast<uint32_t>(code) | (m < 0.0f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_second(float v, float inv, uint32_t chance) {
  const float y = __fmul_rn(v, inv);
  int code = ((__float_as_int(y) + static_cast<int>(chance << 4)) >> kCodeShift) - kSecondBase;
  code = min(max(code, 1), 255);
  return v > 0.0f ? static_cast<uint32_t>(code) : 0u;
}

// The SplitMix64 finaliser (Steele, Lea and Flood 2014) and its sequence's increment.
constexpr uint64_t kSplitMixGamma = 0x9E3779B97F4A7C15ull;
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

}  // namespace bergson
