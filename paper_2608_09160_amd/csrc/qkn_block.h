// Device and host pieces shared by the attention-block sources (rotary positions, paged attention, adapters):
// bf16 and FP8-E4M3 conversions, division by a launch constant, checks of the paged cache.
#ifndef QKN_BLOCK_H
#define QKN_BLOCK_H

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "qkn_cache.h"
#include "qkn_host.h"

namespace qkn_block {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kXcds = 8;              // MI355X: workgroup id mod 8 selects the XCD
constexpr int kCus = 256;             // MI355X
constexpr float kFp8Max = 448.0f;     // largest finite e4m3fn value

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __builtin_bit_cast(float, u & 0xffff0000u); }

// Two floats to bf16, nearest even.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// The cache's saturating quantiser: beyond +-448 to +-448, NaN as it is (comparisons are false for it).
__device__ __forceinline__ float clamp_fp8(float f) {
  return f > kFp8Max ? kFp8Max : (f < -kFp8Max ? -kFp8Max : f);
}

// Four floats to e4m3fn codes, nearest even.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_fp8(a), clamp_fp8(b), 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(clamp_fp8(c), clamp_fp8(d), w, true));
}

// n / d by a multiplication: with 2^s >= d > 2^(s - 1), n ceil(2^(32 + s) / d) >> (32 + s) is exact for n < 2^32. The
// factor has 33 bits; `mul` is the lower 32 of them.
struct FastDiv {
  uint32_t mul, shift, d;
};
inline FastDiv fast_div(uint32_t d) {  // 1 <= d < 2^31
  uint32_t s = 0;
  while ((uint64_t{1} << s) < d) ++s;
  const unsigned __int128 one = 1;
  const unsigned __int128 mul = ((one << (32 + s)) + d - 1) / d;
  return FastDiv{static_cast<uint32_t>(mul - (one << 32)), s, d};
}
__device__ __forceinline__ uint32_t div(uint32_t n, FastDiv f) {
  return static_cast<uint32_t>((static_cast<uint64_t>(__umulhi(n, f.mul)) + n) >> f.shift);
}

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// log2 of a power of two.
inline int log2_of(int64_t v) {
  int s = 0;
  while ((int64_t{1} << s) < v) ++s;
  return s;
}

// Elements from the first to the last of a pool.
inline __int128 pool_extent(const qkn_cache& c, int64_t page, int64_t head, int64_t token) {
  if (!c.num_pages) return 0;
  return static_cast<__int128>(c.num_pages - 1) * page + static_cast<__int128>(c.n_kv - 1) * head +
         static_cast<__int128>(c.page_size - 1) * token + c.head_dim;
}

// Sizes and strides of a cache; its pointers are checked where they are used.
inline bool cache_ok(const qkn_cache& c) {
  if (c.num_pages < 0 || c.num_pages > (int64_t{1} << 31) || c.page_size < 1 || c.page_size > 65536 ||
      (c.page_size & (c.page_size - 1)) || c.n_kv < 1 || c.head_dim < 1)
    return false;
  const int64_t most = int64_t{1} << 40, space = int64_t{1} << 46;  // no pool is larger: offsets in it stay in 64 bits
  for (int64_t s : {c.k_page, c.k_head, c.k_token, c.v_page, c.v_head, c.v_token})
    if (s < c.head_dim || s > most) return false;
  if (pool_extent(c, c.k_page, c.k_head, c.k_token) > space || pool_extent(c, c.v_page, c.v_head, c.v_token) > space)
    return false;
  return c.fp8 || (!c.k_scale && !c.v_scale);
}

// Extent of a pool as one byte region (its gaps included).
inline qkn_host::Span pool_span(const qkn_cache& c, const void* base, int64_t page, int64_t head, int64_t token) {
  const int64_t n = static_cast<int64_t>(pool_extent(c, page, head, token));
  return qkn_host::Span{reinterpret_cast<uintptr_t>(base), n ? 1 : 0, n, n, c.fp8 ? 1 : 2};
}
inline qkn_host::Span array_span(const void* p, int64_t n, int64_t esz) {
  return qkn_host::Span{reinterpret_cast<uintptr_t>(p), p && n ? 1 : 0, n, n, esz};
}

}  // namespace qkn_block

#endif  // QKN_BLOCK_H
