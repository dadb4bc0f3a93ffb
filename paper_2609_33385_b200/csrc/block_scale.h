// Rows of e4m3 codes with one fp32 scale per 128 columns (oled_norm_residual, oled_quantize_blocks): a value is
// code * scale of its block.  scale = amax / 448 and code = e4m3(v * (448 / amax)), each one IEEE operation, amax being
// the block's largest magnitude, at least 2^-100 (blocks of zeros, and reciprocals that stay finite).  An infinity gives
// its block the scale inf and a NaN the scale NaN, and codes that are NaN or zero: every value of the block reads as NaN.
#pragma once
#include <cstdint>

namespace oled {

constexpr int kScaleBlock = 128;
constexpr uint32_t kAmaxFloor = 0x0d800000u;  // 2^-100

// Sixteen lanes (a half-warp) hold a block, eight values each.  Magnitudes as bit patterns: they order like the values,
// and a NaN stands above every number, where fmaxf would drop it.
__device__ __forceinline__ uint32_t amax8(const float (&v)[8]) {
  uint32_t big = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint(v[j]) & 0x7fffffffu);
  return big;
}
__device__ __forceinline__ uint32_t amax_half_warp(uint32_t big) {
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, d));
  return max(big, kAmaxFloor);
}
__device__ __forceinline__ float block_scale(uint32_t amax) { return __fdiv_rn(__uint_as_float(amax), 448.0f); }
__device__ __forceinline__ float block_inverse(uint32_t amax) { return __fdiv_rn(448.0f, __uint_as_float(amax)); }
// (a product above 448 by its rounding is clamped by the conversion)
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inverse) {
  uint2 c;
  c.x = e4m3x2(__fmul_rn(v[0], inverse), __fmul_rn(v[1], inverse)) |
        e4m3x2(__fmul_rn(v[2], inverse), __fmul_rn(v[3], inverse)) << 16;
  c.y = e4m3x2(__fmul_rn(v[4], inverse), __fmul_rn(v[5], inverse)) |
        e4m3x2(__fmul_rn(v[6], inverse), __fmul_rn(v[7], inverse)) << 16;
  return c;
}

// Eight bf16 values of a 16-byte vector.
__device__ __forceinline__ void unpack8(const uint4& p, float (&v)[8]) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}

}  // namespace oled
