// From e4m3 codes to 16-bit numbers, by moving bits (batch_pages8.cu, batch_tiles8.cu).
#pragma once

#include "pages8.cuh"

namespace oos {

OOS_DEV uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// bytes 0 and 2 (1 and 3) of a word of codes as bf16 of 2^-120 the value
OOS_DEV uint32_t even_codes(uint32_t w) { return ((w << 8) & 0x80008000u) | ((w << 4) & 0x07f007f0u); }
OOS_DEV uint32_t odd_codes(uint32_t w) { return (w & 0x80008000u) | ((w >> 4) & 0x07f007f0u); }
// the same as binary16 of 2^-8 the value
OOS_DEV uint32_t even_codes_half(uint32_t w) { return ((w << 8) & 0x80008000u) | ((w << 7) & 0x3f803f80u); }
OOS_DEV uint32_t odd_codes_half(uint32_t w) { return (w & 0x80008000u) | ((w >> 1) & 0x3f803f80u); }
OOS_DEV uint32_t mul_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// 2^e as binary16, e <= 0; 0 below 2^-24
OOS_DEV uint32_t half_power(int e) { return e >= -14 ? (uint32_t)(min(e, 0) + 15) << 10 : e >= -24 ? 1u << (e + 24) : 0u; }

}  // namespace oos
