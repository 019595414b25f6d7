/*
 * qkn_attn.h -- C ABI of libqkn, part 4: attention of new tokens over the
 * paged cache (AMD MI355X, gfx950).
 *
 * A batch of sequences, each with some new tokens whose keys and values the
 * cache holds already (qkn_rope_cache writes them): whole prompts, chunks of
 * prompts behind a cached prefix, single tokens, in any mixture.
 *
 * For sequence b with n = q_start[b+1] - q_start[b] new tokens and m =
 * kv_len[b] cached ones (the new ones last), new token i is at position
 * m - n + i, and for every query head h with KV head g = h / (n_q / n_kv)
 *   x_j = scale * <q_i, k_j>     over the keys j that token i sees:
 *         j < m;  j <= m - n + i  where causal;  j > m - n + i - window  where
 *         window > 0,
 *   out_i = sum_j exp(x_j) v_j / sum_j exp(x_j),   lse_i = log sum_j exp(x_j).
 * A token that sees no key (m < n leaves such tokens) has out = 0 and lse =
 * -infinity, and so has a token of no sequence: q_start may begin above 0 and
 * end below T, as in a replayed batch of fixed T with padding behind it. Keys and values that a token does not see take no part, whatever
 * they hold (a NaN in a later token's value reaches no earlier token).
 *
 * Arithmetic: products of bf16 values (an FP8 code is one exactly) summed in
 * fp32 on the matrix cores; softmax in fp32, each row's maximum tracked to
 * within a factor 2^8 and its sum taken before any rounding; the weights are
 * rounded to bf16 as operands of the second product, whose sums are fp32; one
 * rounding of the result to bf16. An FP8 cache's scales are applied in fp32 to
 * the scores and to the result. For given inputs and launch options results
 * are deterministic: no atomics, fixed orders.
 *
 * Conventions are those of qkn.h.
 */
#ifndef QKN_ATTN_H
#define QKN_ATTN_H

#include <stdint.h>

#include "qkn.h"
#include "qkn_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 *   q, out       bf16 [T, ldq], [T, ldo]: n_q * head_dim columns, heads in a
 *                row; the tokens of all sequences, in order, among T.
 *                out == q is not allowed.
 *   lse          fp32 [T, n_q], or NULL.
 *   q_start      int32 [batch + 1], ascending, within 0 and T.
 *   kv_len       int32 [batch].
 *   block_table  int32 [batch, ld_table]: entry p of row b is the page that
 *                holds tokens [p * page_size, (p + 1) * page_size) of sequence
 *                b. Entries past the sequence's last page are not used.
 *   max_q, max_kv  the largest n and m of the batch, or more. They choose the
 *                kernel and how far the keys are split over workgroups, and
 *                never the result beyond its last bits; a decode loop that is
 *                replayed as a HIP graph gives the most it will reach.
 *   window       0: all; else each token sees at most so many keys, its own
 *                the last. Needs causal.
 *   scale        finite, > 0.
 * What the device arrays hold cannot be checked before the launch; the
 * kernels stay inside the buffers whatever they hold: q_start is clamped to
 * [0, T], kv_len to [0, ld_table * page_size], and a page number outside
 * [0, num_pages) reads as zeros. A q_start that is not ascending leaves what
 * the tokens that it names twice or not at all receive undefined.
 */
typedef struct qkn_attn_args {
  const uint16_t* q;
  int64_t ldq;
  uint16_t* out;
  int64_t ldo;
  float* lse;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* block_table;
  int64_t ld_table;
  int64_t T;
  int32_t batch;
  int32_t n_q;
  int32_t max_q;
  int32_t max_kv;
  int32_t causal;
  int32_t window;
  float scale;
} qkn_attn_args;

/*
 * Bytes of device workspace qkn_attn needs for these arguments (the partial
 * results of split keys; 0 where they are not split); negative status for
 * sizes that qkn_attn refuses. Depends on T, batch, n_q, max_q, max_kv and the
 * cache's sizes only: one workspace serves layers of different windows and
 * masks, one after the other.
 */
int64_t qkn_attn_workspace_bytes(const qkn_attn_args* args, const qkn_cache* cache);

/*
 * QKN_EINVAL: args or cache NULL or malformed; T, batch, max_q, max_kv < 0;
 * n_q < 1 or not a multiple of n_kv; strides below the row width; ld_table < 0;
 * window < 0, or > 0 without causal; scale not finite or <= 0; NULL arrays or
 * pools where T > 0; a workspace that is NULL or too small where one is needed.
 * QKN_ENOTSUP: head_dim over 256 or not a multiple of 8 (FP8: 16); page_size
 * below 16; q, out, pools, their strides not multiples of 16 bytes (q, out: 8
 * elements), workspace not 16-byte aligned; T * n_q, a page's bytes, or the
 * grid beyond 2^31.
 * QKN_EOVERLAP: an output (out, lse, workspace) overlapping an input or
 * another output.
 */
int qkn_attn(const qkn_attn_args* args, const qkn_cache* cache, void* workspace, int64_t workspace_bytes,
             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QKN_ATTN_H */
