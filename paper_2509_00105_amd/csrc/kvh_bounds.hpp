// What the bounds of keys and the selection by them share: codes of 127ths.
#pragma once

#include "kvh_cache.hpp"

namespace kvh {

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  return ((uint32_t)(int)a & 0xffu) | ((uint32_t)(int)b & 0xffu) << 8 | ((uint32_t)(int)c & 0xffu) << 16 | (uint32_t)(int)d << 24;
}

// 127 x / a for |x| <= a, rounded once: x has 11 bits at most, so 127/128 of it is exact, and a >= 2^-100.
struct Part127 {
  float by;
  __device__ __forceinline__ explicit Part127(float a) : by(a * (1.0f / 128.0f)) {}
  __device__ __forceinline__ float of(float x) const { return x * (127.0f / 128.0f) / by; }
};

// Its floor and ceiling without a division each: the nearest whole number n of a quotient that is off by 2^-16 at most is one of the two, or the quotient itself,
// and the sign of x - n a says which (the fused product and sum is rounded once, which leaves a sign as it is).
struct Around127 {
  float by, inv;
  __device__ __forceinline__ explicit Around127(float a) : by(a * (1.0f / 128.0f)), inv(1.0f / by) {}
  __device__ __forceinline__ float down(float x) const {
    const float y = x * (127.0f / 128.0f), n = __builtin_rintf(y * inv);
    return __builtin_fmaf(-n, by, y) < 0.0f ? n - 1.0f : n;
  }
  __device__ __forceinline__ float up(float x) const { return -down(-x); }
};

}  // namespace kvh
