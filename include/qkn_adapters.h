/*
 * qkn_adapters.h -- C ABI of libqkn, part 5: low-rank adapters of many
 * requests beside the shared projection (AMD MI355X, gfx950).
 *
 * qkn_proj_partial computes base = x W^T with the weights that all requests
 * share. A request may have an adapter of its own, W + scale B A with A
 * [rank, hidden] and B [d, rank]; this entry point adds its part to the
 * projection's rows, before the norm:
 *
 *   y[t, :]     = bf16( base[t, :] + scale_i * B_i (A_i x[t, :]) ),  i = ids[t]
 *   partials[t] = sum_j y[t, j]^2       fp32, of the stored bf16 values
 *
 * for 1 to 3 outputs (Q, K, V) of the same tokens, each with matrices of its
 * own. A token with an id outside [0, count) has no adapter: y = base.
 * partials is the norm's Phase A statistic, which the projection took of rows
 * without the adapter.
 *
 * Arithmetic: A x of bf16 values summed in fp32; the products with B take the
 * fp32 value of scale * (A x), as the sum of three bf16 values, summed in
 * fp32; base added in fp32; one rounding. An infinite element of B makes NaN
 * of the values that it is part of (it meets the three in turn, which may be 0
 * or of either sign). A row without an adapter keeps base's bits. A request's
 * result does not depend on the other requests' values. Deterministic for
 * given sizes and ids: no atomics, fixed orders.
 *
 * Conventions are those of qkn.h.
 */
#ifndef QKN_ADAPTERS_H
#define QKN_ADAPTERS_H

#include <stdint.h>

#include "qkn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 *   a         bf16: adapter i's A at a + i * a_adapter, rows of lda elements.
 *   b         bf16: adapter i's B at b + i * b_adapter, d_local rows of ldb.
 *   base      bf16 [T, ldbase]; base == y with equal strides runs in place.
 *   y         bf16 [T, ldy].
 *   partials  fp32 [T], or NULL.
 */
typedef struct qkn_adapter_seg {
  const uint16_t* a;
  int64_t a_adapter, lda;
  const uint16_t* b;
  int64_t b_adapter, ldb;
  const uint16_t* base;
  int64_t ldbase;
  uint16_t* y;
  int64_t ldy;
  float* partials;
  int64_t d_local;
} qkn_adapter_seg;

/*
 * Bytes of device workspace for A x of every token, in parts of hidden;
 * negative status for T < 0, hidden, rank < 1, nseg not 1 to 3.
 */
int64_t qkn_adapters_workspace_bytes(int64_t T, int64_t hidden, int rank, int nseg);

/*
 *   x      bf16 [T, ldx], columns [0, hidden): the projection's input.
 *   ids    int32 [T], the tokens' adapters.
 *   scale  fp32 [count], or NULL for 1.
 *   count  adapters (>= 0; with 0 a, b and scale are not used).
 * QKN_EINVAL: x, ids, a segment's a, b, base or y NULL with T > 0 (a, b with
 * count > 0); T or count < 0, hidden, rank or d_local < 1; nseg not 1 to 3;
 * strides below the row width, a_adapter or b_adapter < 0; a workspace that is
 * NULL or too small.
 * QKN_ENOTSUP: hidden, d_local, rank, or a stride not a multiple of 8, a
 * tensor (the workspace) not 16-byte aligned; rank over 128; T over 2^24,
 * count over 2^24, hidden, d_local or ldb over 2^30, ldx of 2^21 or lda of
 * 2^27 or more, or an adapter's stride over 2^38.
 * QKN_EOVERLAP: an output (y, partials, workspace) overlapping an input or
 * another output, in-place y apart.
 */
int qkn_adapters_add(const uint16_t* x, int64_t ldx, int64_t T, int64_t hidden, const qkn_adapter_seg* segs, int nseg,
                     int rank, int64_t count, const int32_t* ids, const float* scale, void* workspace,
                     int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QKN_ADAPTERS_H */
