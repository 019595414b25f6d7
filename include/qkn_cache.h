/*
 * qkn_cache.h -- the paged KV cache that qkn_rope.h writes and qkn_attn.h
 * reads (AMD MI355X, gfx950).
 *
 * K and V live in pools of pages; a page holds page_size consecutive tokens of
 * one sequence. Element (page, head, row, c) of the K pool is at
 *   k[page * k_page + head * k_head + row * k_token + c],
 * and the V pool's likewise, so a pool may be laid out [pages, heads, rows, D]
 * (a page of one head contiguous: the fastest to read), [pages, rows, heads, D],
 * or K and V may share one allocation.
 *
 * FP8 pools hold e4m3fn codes of value / scale, one scale per KV head and pool:
 * code = e4m3fn(clamp(value * (1 / scale), -448, 448)), nearest even, the
 * saturating quantiser (an outlier must not turn a cached token into NaN; a
 * NaN stays NaN). Readers multiply by the scale in fp32. A bf16 pool has none.
 */
#ifndef QKN_CACHE_H
#define QKN_CACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 *   k, v        device pools: bf16 bits, or e4m3fn codes (fp8 != 0).
 *   k_scale     fp32 [n_kv] on the device, finite and > 0, or NULL for 1 (NULL
 *   v_scale     unless fp8).
 *   num_pages   pages of each pool (>= 0).
 *   page_size   tokens of a page: a power of two, 1 to 65536.
 *   n_kv        KV heads of this rank (>= 1).
 *   head_dim    D (>= 1).
 *   strides     in elements; each at least head_dim and at most 2^40, and from
 *               a pool's first element to its last at most 2^46. Pages of a
 *               pool must not share elements, nor may the two pools.
 */
typedef struct qkn_cache {
  void* k;
  void* v;
  const float* k_scale;
  const float* v_scale;
  int64_t num_pages;
  int32_t page_size;
  int32_t n_kv;
  int32_t head_dim;
  int32_t fp8;
  int64_t k_page, k_head, k_token;
  int64_t v_page, v_head, v_token;
} qkn_cache;

#ifdef __cplusplus
}
#endif

#endif /* QKN_CACHE_H */
