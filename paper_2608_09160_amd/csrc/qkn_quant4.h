// The 4-bit format of qkn_cache4.h on the device: exponents of blocks, codes of values, values of codes.
#ifndef QKN_QUANT4_H
#define QKN_QUANT4_H

#include "qkn_block.h"

namespace quant4 {

using namespace qkn_block;

// Exponent bytes from here on make a block NaN: the quantiser writes 255; with 253 and 254 a value could be infinite.
constexpr uint32_t kNan = 253;

// x c + y s, each operation rounded by itself.
__device__ __forceinline__ float cross(float x, float c, float y, float s) {
#pragma clang fp contract(off)
  const float a = x * c, b = y * s;
  return a + b;
}

// The largest magnitude of a group as bits: as integers they are ordered like the values, infinity and NaN above.
__device__ __forceinline__ uint32_t magnitude(const float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f[e]) & 0x7fffffffu;
    m = u > m ? u : m;
  }
  return m;
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t m) {
  const uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), CTRL, 0xf, 0xf, true));
  return o > m ? o : m;
}
__device__ __forceinline__ uint32_t max_of_2(uint32_t m) { return max_with<0xB1>(m); }  // lanes 2 i, 2 i + 1
__device__ __forceinline__ uint32_t max_of_4(uint32_t m) { return max_with<0x4E>(m); }  // of four, after max_of_2

// The exponent byte of a block. With A = m 2^k, 1 <= m < 2: the least e with A < 7 2^e is k - 2 for m < 1.75, else
// k - 1, which is what carrying from the mantissa's second bit does.
__device__ __forceinline__ uint32_t exponent(uint32_t most) {
  int e = static_cast<int>((most + 0x200000u) >> 23) - 2;
  e = e < 2 ? 2 : e > 252 ? 252 : e;
  return most > 0x7f800000u ? 255u : static_cast<uint32_t>(e);
}

// Two values' codes, the first in the lower half; exponent byte 255: 0. The conversion divides by its scale, rounds to
// nearest even and takes magnitudes beyond 6 as 6.
__device__ __forceinline__ uint32_t encode2(float a, float b, uint32_t e) {
  const float scale = __builtin_bit_cast(float, e << 23);
  const uint32_t u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, a, b, scale, 0);
  return e == 255 ? 0 : u & 0xff;
}
__device__ __forceinline__ uint32_t encode(const float (&f)[8], uint32_t e) {
  const float scale = __builtin_bit_cast(float, e << 23);
  uint32_t u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, f[0], f[1], scale, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, f[2], f[3], scale, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, f[4], f[5], scale, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, f[6], f[7], scale, 3);
  return e == 255 ? 0 : u;
}

// Eight codes times 2^(e - 127) as bf16, exactly; e below kNan.
__device__ __forceinline__ bf16x8 decode(uint32_t w, uint32_t e) {
  const float scale = __builtin_bit_cast(float, e << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace quant4

#endif  // QKN_QUANT4_H
