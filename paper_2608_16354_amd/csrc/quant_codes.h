// What rows, cache groups and e4m3 blocks share when they become codes: magnitudes, their maxima, scales and the quotients
// that are rounded to codes.
#pragma once

#include <hip/hip_runtime.h>

namespace dc {
namespace {

constexpr int kWave = 64;
constexpr uint32_t kInfBits = 0x7F800000u;

__device__ inline float from_bf16(uint16_t u) { return __uint_as_float(uint32_t(u) << 16); }

// |x| as an integer: ordered as the magnitudes are, infinities and then NaN above all numbers
__device__ inline uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ inline uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, uint32_t(__shfl_xor(int(v), o, kWave)));
  return v;
}
// maximum over the 16 lanes of a row of the wave (DPP rotations of 8, 4, 2 and 1)
__device__ inline uint32_t row16_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xF, 0xF, true)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xF, 0xF, true)));
}

// the scale of a row or group whose largest magnitude is `m` (as mag() gives it)
__device__ inline float scale_of(uint32_t m, float levels) {
  return m >= kInfBits ? __uint_as_float(0x7FC00000u) : __uint_as_float(m) / levels;
}
// Quotients under one scale.  The fp32 quotient x / s comes from y = 1 / s without a division per value: with
// y + z = 1 / s to about 2^-45, q0 = x (y + z) is off by less than a step, r = x - q0 s is exact and q0 + r y
// rounds to the quotient that a division gives (Markstein's theorem); for an integer code, adding 1.5 2^23 rounds it, ties
// to even, and the low byte is the code.  Five operations a value, a division takes eleven (bf16 rows of 1,920:
// 18.8 against 29.6 us for 17,776 of them).  Outside [2^-100, 2^100] the small terms can leave fp32's range:
// there a division is made (and its quotient bounded, as s may have lost bits), and s = 0 or NaN gives 0.
struct Coder {
  float s, y, z, levels;
  bool direct;
  __device__ Coder(float scale, float lv) : s(scale), levels(lv) {
    y = 1.0f / scale;
    z = fmaf(-scale, y, 1.0f) * y;
    direct = scale >= 0x1p-100f && scale <= 0x1p100f;
  }
  // x / s where `direct`
  __device__ float quotient(float x) const {
    const float q0 = fmaf(x, y, x * z);
    return fmaf(fmaf(-q0, s, x), y, q0);
  }
  // x / s elsewhere, bounded
  __device__ float divided(float x) const { return s > 0.f ? fminf(fmaxf(x / s, -levels), levels) : 0.f; }
  // low byte: the integer code
  __device__ uint32_t fast(float x) const { return __float_as_uint(quotient(x) + 12582912.0f); }
  __device__ uint32_t slow(float x) const {
    return s > 0.f ? uint32_t(int(fminf(fmaxf(rintf(x / s), -levels), levels))) : 0u;
  }
};
}  // namespace
}  // namespace dc
