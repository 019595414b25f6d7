// libqkn, part 4: attention of new tokens over the paged cache (AMD MI355X, gfx950): host side and the joining of
// split keys. The kernels are in qkn_attn_kernels.h.

#include <string.h>

#include "qkn_attn.h"
#include "qkn_attn_kernels.h"

namespace attn {

using qkn_host::Span;
using qkn_host::spans_overlap;

// A row's parts, added in ascending order of the keys: four elements a thread.
__global__ __launch_bounds__(256) void qkn_attn_join(const Params p, int64_t rows, FastDiv vecs) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = div(static_cast<uint32_t>(u), vecs);
  if (r >= rows) return;
  const int d = static_cast<int>(u - r * vecs.d) * 4;
  const int splits = static_cast<int>(p.splits.d);
  float top = neg_inf();
  for (int s = 0; s < splits; ++s) top = fmaxf(top, p.part_ml[s * rows + r][0]);
  const float base = top == neg_inf() ? 0.0f : top;
  float sum = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < splits; ++s) {
    const f32x2 ml = p.part_ml[s * rows + r];
    if (ml[1] == 0.0f) continue;  // a part without keys has no o
    const float f = __builtin_amdgcn_exp2f(ml[0] - base);
    sum += f * ml[1];
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + (s * rows + r) * p.D + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += f * v[e];
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  const u32x2 y = {pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
  const int64_t t = r / p.n_q;
  *reinterpret_cast<u32x2*>(p.out + t * p.ldo + (r - t * p.n_q) * p.D + d) = y;
  if (d == 0 && p.lse) p.lse[r] = sum == 0.0f ? neg_inf() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

constexpr int kMaxSplits = 64;

struct Plan {
  Variant v;
  int64_t tiles, splits, grid, ws_bytes;
};

// Sizes alone: QKN_OK, QKN_EINVAL or QKN_ENOTSUP.
int check_sizes(const qkn_attn_args* a, const qkn_cache* c) {
  if (!a || !c || !cache_ok(*c) || a->T < 0 || a->batch < 0 || a->max_q < 0 || a->max_kv < 0 || a->n_q < 1 ||
      a->n_q % c->n_kv || a->ld_table < 0 || a->window < 0 || (a->window && !a->causal) || !(a->scale > 0.0f) ||
      isinf(a->scale))
    return QKN_EINVAL;
  const int64_t width = static_cast<int64_t>(a->n_q) * c->head_dim;
  if (a->ldq < width || a->ldo < width) return QKN_EINVAL;
  const int64_t lim = int64_t{1} << 31, esz = c->fp8 ? 1 : 2, group = a->n_q / c->n_kv;
  if (c->head_dim > 256 || c->head_dim % (c->fp8 ? 16 : 8) || c->page_size < 16 || a->T >= lim || a->n_q >= lim / 8 ||
      a->T * a->n_q >= lim || a->T * group + int64_t{a->batch} * 512 >= lim || a->ld_table > lim ||
      a->ld_table * c->page_size > lim - (1 << 17) || c->k_token * esz * c->page_size >= lim ||
      c->v_token * esz * c->page_size >= lim)
    return QKN_ENOTSUP;
  return QKN_OK;
}

Plan plan_of(const qkn_attn_args& a, const qkn_cache& c) {
  Plan pl{};
  const int dt = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
  const int64_t group = a.n_q / c.n_kv, rows = (a.max_q < 1 ? 1 : a.max_q) * group;
  if (rows <= (dt == 256 ? 32 : 64)) pl.v = few_rows(dt, c.fp8 != 0, static_cast<int>(rows));
  else pl.v = many_rows(dt, c.fp8 != 0);
  pl.tiles = a.T * group / pl.v.rows + a.batch;  // the most that find_sequence hands out
  // workgroups with rows, about: every sequence ends in a part of a tile
  const int64_t busy = ((a.T * group + pl.v.rows - 1) / pl.v.rows > a.batch ? (a.T * group + pl.v.rows - 1) / pl.v.rows
                                                                            : a.batch) * c.n_kv;
  const int64_t seen = a.window && a.window + int64_t{a.max_q} < a.max_kv ? a.window + int64_t{a.max_q} : a.max_kv;
  const int64_t tiles_k = (seen + pl.v.keys - 1) / pl.v.keys;
  int64_t splits = (2 * kCus + busy - 1) / (busy ? busy : 1);
  if (splits > tiles_k / 2) splits = tiles_k / 2;
  if (splits > kMaxSplits) splits = kMaxSplits;
  pl.splits = splits < 1 ? 1 : splits;
  pl.grid = pl.tiles * c.n_kv * pl.splits;
  pl.ws_bytes = pl.splits > 1 ? pl.splits * a.T * a.n_q * (4 * int64_t{c.head_dim} + 8) : 0;
  return pl;
}

int attn_impl(const qkn_attn_args* args, const qkn_cache* cache, void* workspace, int64_t workspace_bytes,
              void* stream) {
  int rc = check_sizes(args, cache);
  if (rc != QKN_OK) return rc;
  const qkn_attn_args& a = *args;
  const qkn_cache& c = *cache;
  if (a.T == 0 || a.batch == 0) return QKN_OK;
  if (!a.q || !a.out || !a.q_start || !a.kv_len || (a.ld_table && !a.block_table) || (c.num_pages && (!c.k || !c.v)))
    return QKN_EINVAL;
  const Plan pl = plan_of(a, c);
  if (pl.ws_bytes && (!workspace || workspace_bytes < pl.ws_bytes)) return QKN_EINVAL;
  const int64_t esz = c.fp8 ? 1 : 2, per = 16 / esz;
  if (!aligned(a.q, 16) || !aligned(a.out, 16) || a.ldq % 8 || a.ldo % 8 || !aligned(c.k, 16) || !aligned(c.v, 16) ||
      (pl.ws_bytes && !aligned(workspace, 16)))
    return QKN_ENOTSUP;
  for (int64_t s : {c.k_page, c.k_head, c.k_token, c.v_page, c.v_head, c.v_token})
    if (s % per) return QKN_ENOTSUP;
  const int64_t rows = a.T * a.n_q, vecs = c.head_dim / 4;
  if (pl.grid >= (int64_t{1} << 31) || (pl.splits > 1 && rows * vecs >= (int64_t{1} << 32) - 256)) return QKN_ENOTSUP;

  const int64_t width = int64_t{a.n_q} * c.head_dim;
  const Span in[] = {Span{reinterpret_cast<uintptr_t>(a.q), a.T, a.ldq, width, 2},
                     array_span(a.q_start, int64_t{a.batch} + 1, 4),
                     array_span(a.kv_len, a.batch, 4),
                     array_span(a.block_table, a.batch * a.ld_table, 4),
                     pool_span(c, c.k, c.k_page, c.k_head, c.k_token),
                     pool_span(c, c.v, c.v_page, c.v_head, c.v_token),
                     array_span(c.k_scale, c.n_kv, 4),
                     array_span(c.v_scale, c.n_kv, 4)};
  const Span out[] = {Span{reinterpret_cast<uintptr_t>(a.out), a.T, a.ldo, width, 2}, array_span(a.lse, rows, 4),
                      array_span(pl.ws_bytes ? workspace : nullptr, pl.ws_bytes, 1)};
  for (int i = 0; i < 3; ++i) {
    for (const Span& s : in)
      if (spans_overlap(out[i], s)) return QKN_EOVERLAP;
    for (int j = 0; j < i; ++j)
      if (spans_overlap(out[i], out[j])) return QKN_EOVERLAP;
  }

  Params p;
  memset(&p, 0, sizeof(p));
  p.q = a.q;
  p.out = a.out;
  p.lse = a.lse;
  p.q_start = a.q_start;
  p.kv_len = a.kv_len;
  p.table = a.block_table;
  p.ldq = a.ldq;
  p.ldo = a.ldo;
  p.ld_table = a.ld_table;
  p.T = a.T;
  p.k = Pool{static_cast<const unsigned char*>(c.k), c.k_scale, c.k_page * esz, c.k_head * esz,
             static_cast<uint32_t>(c.k_token * esz)};
  p.v = Pool{static_cast<const unsigned char*>(c.v), c.v_scale, c.v_page * esz, c.v_head * esz,
             static_cast<uint32_t>(c.v_token * esz)};
  p.num_pages = c.num_pages;
  p.page_shift = log2_of(c.page_size);
  p.batch = a.batch;
  p.n_q = a.n_q;
  p.n_kv = c.n_kv;
  p.D = c.head_dim;
  p.tiles = static_cast<int32_t>(pl.tiles);
  p.causal = a.causal != 0;
  p.window = a.window;
  p.c = a.scale * 1.44269504088896340736f;
  p.group = fast_div(static_cast<uint32_t>(a.n_q / c.n_kv));
  p.kv_heads = fast_div(static_cast<uint32_t>(c.n_kv));
  p.splits = fast_div(static_cast<uint32_t>(pl.splits));
  p.min_tiles = 2;
  if (pl.ws_bytes) {
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<f32x2*>(p.part_o + pl.splits * rows * c.head_dim);
  }
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{pl.v.name, 0, 0, 0, pl.v.lds});
    return QKN_EDRYRUN;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  void* kargs[] = {&p};
  if (hipLaunchKernel(pl.v.fn, dim3(static_cast<unsigned>(pl.grid)), dim3(static_cast<unsigned>(pl.v.threads)), kargs, 0,
                      st) != hipSuccess)
    return QKN_EHIP;
  if (pl.splits > 1) {
    int64_t n = rows;
    FastDiv fd = fast_div(static_cast<uint32_t>(vecs));
    void* jargs[] = {&p, &n, &fd};
    if (hipLaunchKernel(reinterpret_cast<const void*>(qkn_attn_join), dim3(static_cast<unsigned>((rows * vecs + 255) / 256)),
                        dim3(256), jargs, 0, st) != hipSuccess)
      return QKN_EHIP;
  }
  qkn_host::record_launch(
      qkn_launch_info{pl.v.name, pl.grid, pl.v.threads, pl.grid * (pl.v.threads / 64), pl.v.lds});
  return QKN_OK;
}

}  // namespace attn

extern "C" {

int64_t qkn_attn_workspace_bytes(const qkn_attn_args* args, const qkn_cache* cache) {
  const int rc = attn::check_sizes(args, cache);
  if (rc != QKN_OK) return rc;
  return args->T == 0 || args->batch == 0 ? 0 : attn::plan_of(*args, *cache).ws_bytes;
}

int qkn_attn(const qkn_attn_args* args, const qkn_cache* cache, void* workspace, int64_t workspace_bytes,
             void* stream) {
  return attn::attn_impl(args, cache, workspace, workspace_bytes, stream);
}

}  // extern "C"
