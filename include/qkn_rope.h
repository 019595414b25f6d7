/*
 * qkn_rope.h -- C ABI of libqkn, part 3: rotary positions of Q and K, with the
 * norm's Phases B+C in front and the write into the paged cache behind, in one
 * pass over the rows (AMD MI355X, gfx950).
 *
 * Conventions are those of qkn.h (device pointers owned by the caller, bf16 as
 * uint16_t bits, asynchronous on `stream`, validation before any HIP call,
 * negative status codes, T == 0 a no-op).
 */
#ifndef QKN_ROPE_H
#define QKN_ROPE_H

#include <stdint.h>

#include "qkn.h"
#include "qkn_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Frequencies of the rotated pairs, i in [0, rot_dim / 2):
 *   f_i = base^(-2 i / rot_dim)
 * and, for contexts longer than a model was trained on (factor > 1),
 *   f_i (g_i + (1 - g_i) / factor),  g_i = clamp((r_i - low) / (high - low), 0, 1),
 *   r_i = original * f_i / (2 pi)    turns of pair i over the original context:
 * pairs of few turns are stretched, those of many turns keep their frequency.
 * low == high == 0 stretches every pair (g = 0; `original` is not used).
 * cos and sin are multiplied by `magnitude`.
 */
typedef struct qkn_rope_scaling {
  double base;       /* > 0 */
  double factor;     /* >= 1; 1: not scaled */
  double low, high;  /* 0 <= low < high, or both 0 */
  double original;   /* > 0 where low < high */
  double magnitude;  /* finite */
} qkn_rope_scaling;

/*
 * table[p, i] = (cos(p f_i), sin(p f_i)) * magnitude for p in [0, n_pos): fp32
 * [n_pos, rot_dim / 2, 2], angles and functions in 64 bits, rounded once. Made
 * once and kept with the model. QKN_EINVAL: NULL pointers, n_pos < 0, rot_dim
 * odd or < 2, a scaling outside the ranges above. n_pos == 0 is a no-op.
 */
int qkn_rope_table(float* table, int64_t n_pos, int rot_dim, const qkn_rope_scaling* scaling, void* stream);

/*
 * Q or K of one rank: rows of heads * head_dim columns.
 *   x         bf16 [T, ldx].
 *   w         fp32 [heads * head_dim], the rank's gamma: the row is normalised
 *             first, z = (x * w) * (1 / sqrt(S / d_full + eps)), S the sum over
 *             ranks (ascending, fp32) of partials, exactly qkn_apply's factor.
 *             NULL: z = x (partials and d_full are not used).
 *   partials  fp32 [tp * T], every rank's statistic.
 *   y         bf16 [T, ldy] output; y == x with ldy == ldx runs in place. K's
 *             may be NULL: then its rows go to the cache only.
 */
typedef struct qkn_rope_seg {
  const uint16_t* x;
  int64_t ldx;
  const float* w;
  const float* partials;
  int64_t d_full;
  uint16_t* y;
  int64_t ldy;
  int32_t heads;
} qkn_rope_seg;

/*
 * One pass over Q, K and V of T new tokens:
 *   - Q and K rows are normalised (where w is given) and each head's first
 *     rot_dim elements rotated by the token's position p = pos[t]:
 *       (a, b) -> (a cos - b sin, b cos + a sin),  cos, sin = table[p, i],
 *     pairs i = (element i, element i + rot_dim / 2), or with `interleaved`
 *     (2 i, 2 i + 1); the rest of the head passes;
 *   - Q is written to q->y, K to k->y (if given), and K and V to row
 *     slots[t] % page_size of page slots[t] / page_size of the cache.
 * All arithmetic is fp32 with one rounding, to bf16 or to the FP8 code: a
 * normalised row is not rounded between the norm and the rotation.
 *   q      may be NULL (K and V only); k may be NULL (Q only).
 *   v      bf16 [T, ldv], cache->n_kv * head_dim columns, or NULL.
 *   table, pos   as qkn_rope_table writes it; int32 [T]. Not used (may be NULL)
 *          when rot_dim is 0.
 *   slots  int64 [T]; a slot outside [0, num_pages * page_size) -- a padding
 *          token's -1 -- is not written. Tokens of one call have different
 *          slots, else either may win.
 *   cache  NULL: nothing is cached (v must be NULL, k->y set).
 * A position outside [0, n_pos) makes the token's rotated elements NaN.
 * QKN_EINVAL: neither q nor k; NULL x, NULL y of q; w without partials, or
 * d_full < heads * head_dim; heads < 1, head_dim < 1, strides below the row
 * width; rot_dim odd or outside [0, head_dim]; NULL table, pos or slots where
 * they are used; tp < 1, eps < 0 or not finite; a malformed cache, or
 * k->heads != cache->n_kv, or cache->head_dim != head_dim; v without a cache;
 * k with neither y nor cache; T < 0.
 * QKN_EOVERLAP: an output (y, the cache's pools) overlapping an input or
 * another output, in-place y apart.
 * QKN_ENOTSUP: more than 2^30 columns, or more work than one grid holds.
 * Fast path: 16-byte accesses where head_dim and rot_dim are multiples of 16
 * and rows, gamma and pools are aligned to their vectors; anything else goes
 * element by element, with the same values.
 */
int qkn_rope_cache(const qkn_rope_seg* q, const qkn_rope_seg* k, const uint16_t* v, int64_t ldv, int64_t T,
                   int head_dim, int rot_dim, int interleaved, const float* table, int64_t n_pos, const int32_t* pos,
                   const int64_t* slots, const qkn_cache* cache, int tp, float eps, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QKN_ROPE_H */
