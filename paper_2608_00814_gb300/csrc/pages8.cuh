// Pages of 8 bits: e4m3 codes with a power of two for each block of 16 positions and kv
// head, held as its exponent + 127 (heads8.cu, pages.cu, and the attention's kernels).
#pragma once

#include "batch.cuh"

namespace oos {

constexpr int kScaleBlock = OOS_SCALE_BLOCK;
constexpr int kScaleLow = -117, kScaleHigh = 119;   // 2^-117 2^-9 is normal in fp32, 448 2^119 finite

struct Pages8View {
  PagesView p;   // k, v: codes
  uint8_t* k_scale;
  uint8_t* v_scale;
};
inline bool pages8_ok(const oos_paged_cache8* c) {
  return c->n_kv_heads >= 1 && c->page_size >= 1 && c->page_size % kScaleBlock == 0 && c->n_pages >= 1 && c->k && c->v &&
         c->k_scale && c->v_scale;
}
inline Pages8View view_of(const oos_paged_cache8& c) {
  return {{(uint8_t*)c.k, (uint8_t*)c.v, c.page_size, c.n_pages, c.n_kv_heads, c.head_dim}, c.k_scale, c.v_scale};
}

// exponent of a scale's byte
OOS_DEV int scale_exp(int byte) { return max(kScaleLow, min(kScaleHigh, byte - 127)); }
// what a score may be multiplied by: past fp32's largest number a score of 0 would be NaN
constexpr float kMostFactor = 0x1.fffffep127f;
OOS_DEV float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Exponent of the least scale that holds the magnitude: m 2^e <= 448 2^(e - 8) for m <= 1.75.
OOS_DEV int needed_exp(float amax) {
  if (!(amax > 0.f)) return kScaleLow;
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return max(kScaleLow, min(kScaleHigh, e));
}

// an e4m3 code, whose values are binary16's too
struct E4M3 {
  uint8_t c;
};
OOS_DEV uint32_t e4m3x2_half2(uint16_t two) {   // the low byte first
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
  return h;
}
OOS_DEV float2 e4m3x2_f32(uint16_t two) {
  const uint32_t h = e4m3x2_half2(two);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
OOS_DEV float to_f32(E4M3 v) { return e4m3x2_f32(v.c).x; }
OOS_DEV uint16_t f32x2_e4m3(float lo, float hi) {   // nearest even, at most 448 in magnitude
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// what a cache of 8 bits can hold of a value: what is not finite is NaN
OOS_DEV float finite_or_nan(float v) { return fabsf(v) < INFINITY ? v : __int_as_float(0x7fffffff); }

// four codes times 2^d, d <= 0, rounded again
OOS_DEV uint32_t rescale_codes4(uint32_t w, int d) {
  const float f = pow2f(max(d, -126));
  const float2 a = e4m3x2_f32((uint16_t)w), b = e4m3x2_f32((uint16_t)(w >> 16));
  return (uint32_t)f32x2_e4m3(a.x * f, a.y * f) | (uint32_t)f32x2_e4m3(b.x * f, b.y * f) << 16;
}

}  // namespace oos
