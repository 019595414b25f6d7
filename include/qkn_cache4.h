/*
 * qkn_cache4.h -- C ABI of libqkn, part 5: a paged KV cache held in 4 bits
 * (AMD MI355X, gfx950): its write behind the rotary positions, attention over
 * it, and its rows read back.
 *
 * Conventions are those of qkn.h (device pointers owned by the caller,
 * asynchronous on `stream`, validation before any HIP call, negative status
 * codes, T == 0 a no-op).
 *
 * An element is a 4-bit E2M1 code: a sign (bit 3) and one of the values 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 (bits 0 to 2, in this order). 32 consecutive elements of a
 * head's row share an exponent byte E: a code's value is multiplied by
 * 2^(E - 127); E from 253 on makes the elements NaN (the quantiser writes 255).
 * From E = 2, the least that the quantiser writes, to 252, the most, such values
 * are exact and normal in bf16 (below, so small that a reader may take 0). 17
 * bytes hold 32 elements.
 *
 * The quantiser, for a block whose largest magnitude is A: the exponent is
 *   e = the least with A < 7 * 2^e, within [-125, 125];   E = e + 127,
 * (7 is halfway from the last value, 6, to where the next would be, so only
 * magnitudes of 6 to 7 units are cut), and each element the nearest of the
 * values times 2^e, ties to the even code, magnitudes beyond the last value to
 * the last (infinities among them); signs are kept, those of zeros too. A NaN
 * anywhere makes the block's E 255 and its codes 0.
 */
#ifndef QKN_CACHE4_H
#define QKN_CACHE4_H

#include <stdint.h>

#include "qkn.h"
#include "qkn_attn.h"
#include "qkn_rope.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Pools of pages, as in qkn_cache.h, all strides in bytes. Element c of a row is
 * in byte c / 2 of it, the even element in the lower half, its exponent in byte
 * c / 32 of the row of exponents: byte i of (page, head, row) of the K codes is at
 *   k[page * k_page + head * k_head + row * k_token + i],
 * and the V codes' and the exponents' likewise.
 *   k, v          codes; rows of head_dim / 2 bytes.
 *   k_exp, v_exp  exponents; rows of head_dim / 32 bytes.
 *   num_pages     pages of each pool (>= 0).
 *   page_size     tokens of a page: a power of two, 1 to 65536.
 *   n_kv          KV heads of this rank (>= 1).
 *   head_dim      D, a multiple of 32.
 *   strides       each at least the row's bytes and at most 2^40, and from a
 *                 pool's first byte to its last at most 2^46. Pages of a pool
 *                 must not share bytes, nor may pools.
 */
typedef struct qkn_cache4 {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  int64_t num_pages;
  int32_t page_size;
  int32_t n_kv;
  int32_t head_dim;
  int64_t k_page, k_head, k_token;
  int64_t v_page, v_head, v_token;
  int64_t ke_page, ke_head, ke_token;
  int64_t ve_page, ve_head, ve_token;
} qkn_cache4;

/*
 * qkn_rope_cache into the 4-bit cache, which must be given, with K (k or v may
 * still be NULL). The values before the quantiser (and before Q's and K's rows
 * are rounded to bf16) are fp32, each operation rounded by itself: the row times
 * w, times qkn_rope_cache's factor, then the rotation's two products and their
 * sum. Codes and rows do not depend on the path that a call takes. Statuses as for qkn_rope_cache; QKN_EINVAL also for a
 * head_dim that is not a multiple of 32.
 * Fast path: K's and V's rows (and Q's, for Q) as for qkn_rope_cache, head_dim
 * and rot_dim multiples of 64 (neighbouring pairs: of 32), code pools and their
 * strides multiples of 4 bytes; anything else takes a wavefront's half for 32
 * elements, with the same values.
 */
int qkn_rope_cache4(const qkn_rope_seg* q, const qkn_rope_seg* k, const uint16_t* v, int64_t ldv, int64_t T,
                    int head_dim, int rot_dim, int interleaved, const float* table, int64_t n_pos, const int32_t* pos,
                    const int64_t* slots, const qkn_cache4* cache, int tp, float eps, void* stream);

/*
 * qkn_attn_sinks over the 4-bit cache: the same arguments, masks, arithmetic (a
 * code times its power of two is a bf16 value) and statuses. QKN_ENOTSUP also:
 * code pools or their strides not multiples of 16 bytes. A page number outside
 * [0, num_pages) reads as zeros.
 */
int64_t qkn_attn4_workspace_bytes(const qkn_attn_args* args, const qkn_cache4* cache);
int qkn_attn4(const qkn_attn_args* args, int32_t sinks, const qkn_cache4* cache, void* workspace,
              int64_t workspace_bytes, void* stream);

/*
 * Rows of the cache as bf16, exactly: k [T, ldk] and v [T, ldv] receive, n_kv *
 * head_dim columns each, what slots[t] % page_size of page slots[t] / page_size
 * holds (int64 [T]; a slot outside [0, num_pages * page_size): zeros). k or v may
 * be NULL, not both. QKN_EINVAL: NULL or malformed cache, NULL slots, NULL pools
 * where num_pages > 0, strides below the row width, T < 0. QKN_EOVERLAP: an
 * output overlapping an input or the other output. QKN_ENOTSUP: more work than
 * one grid holds.
 */
int qkn_cache4_load(const qkn_cache4* cache, const int64_t* slots, int64_t T, uint16_t* k, int64_t ldk, uint16_t* v,
                    int64_t ldv, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QKN_CACHE4_H */
