// libqkn, part 4: attention of new tokens over the paged cache (AMD MI355X, gfx950): host side and the joining of
// split keys. The kernels are in qkn_attn_kernels.h.

#include <string.h>

#include "qkn_attn.h"
#include "qkn_attn_kernels.h"
#include "qkn_cache4.h"

namespace attn {

using qkn_host::Span;
using qkn_host::spans_overlap;

// A row's parts, added in a fixed order: four elements a thread, 128 elements of 8 / GROUPS rows a workgroup. The launch
// is a chain of latencies. GROUPS = 8, for few rows, which may have many parts: eight threads take every eighth part of
// a row and are added through LDS (16 sequences of up to 32768 keys, 256 rows of up to 60 parts: 4.8 against 13.2 us).
// GROUPS = 1, for many rows (12432 rows of 5 parts: 9.5 against 14.3 us). In between, whole calls with 8 and with 1, us: 64
// tokens of 16 heads behind 29936 keys, 1024 rows, 34.0 and 36.9; 128 behind 15872, 2048 rows, 34.8 and 37.2; 48 single
// tokens of 48 heads over 3000 keys, 2304 rows, 29.2 and 28.4; 256 behind 11744, 4096 rows, 46.3 and 44.7.
// parts_of has been written for every row, unless q_start is not ascending: then some rows have what the workspace held
// before, so it is held against the launch before it is an index.
constexpr int kJoinVecs = 32, kJoinThreads = 8 * kJoinVecs;
template <int GROUPS>
__global__ __launch_bounds__(kJoinThreads) void qkn_attn_join(const Params p, int32_t tile_rows) {
  __shared__ f32x4 os[8][kJoinVecs];
  __shared__ f32x2 mls[8];
  const int vec = static_cast<int>(threadIdx.x) % kJoinVecs, slot = static_cast<int>(threadIdx.x) / kJoinVecs;
  const int group = slot % GROUPS;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (8 / GROUPS) + slot / GROUPS;
  const int d = (static_cast<int>(blockIdx.y) * kJoinVecs + vec) * 4;
  if (GROUPS == 1 && r >= p.T * p.n_q) return;
  const int32_t first = p.parts_of[r][0], v = p.parts_of[r][1], parts = v >> 8, i = v & 255;
  const bool inside = (first < p.items * p.n_kv) & (int64_t{parts - 1} * p.n_kv <= first) & (i < tile_rows);
  if (!(inside & (parts > 1))) return;  // parts <= 1: written already (GROUPS = 8: the whole workgroup's row)
  float top = neg_inf(), sum = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kBatch = GROUPS == 1 ? 8 : 4;  // parts whose loads go out together
  for (int k0 = group; k0 < parts; k0 += kBatch * GROUPS) {
    f32x2 ml[kBatch];
    f32x4 x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int part = k0 + k * GROUPS < parts ? k0 + k * GROUPS : parts - 1;
      const int64_t at = static_cast<int64_t>(first - part * p.n_kv) * tile_rows + i;
      ml[k] = p.part_ml[at];
      if (d < p.D) x[k] = *reinterpret_cast<const f32x4*>(p.part_o + at * p.D + d);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (k0 + k * GROUPS >= parts || ml[k][1] == 0.0f) continue;  // a part without keys wrote no o
      const float up = fmaxf(top, ml[k][0]), base = up == neg_inf() ? 0.0f : up;
      const float old = __builtin_amdgcn_exp2f(top - base), f = __builtin_amdgcn_exp2f(ml[k][0] - base);
      top = up;
      sum = sum * old + f * ml[k][1];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] * old + f * x[k][e];
    }
  }
  if constexpr (GROUPS > 1) {
    os[slot][vec] = o;
    if (vec == 0) mls[slot] = f32x2{top, sum};
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) top = fmaxf(top, mls[slot + g][0]);
    const float base = top == neg_inf() ? 0.0f : top;
    sum = 0.0f;
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const float f = __builtin_amdgcn_exp2f(mls[slot + g][0] - base);
      sum += f * mls[slot + g][1];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += f * os[slot + g][vec][e];
    }
  }
  if (d < p.D) {
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    const u32x2 y = {pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
    const int64_t t = r / p.n_q;
    *reinterpret_cast<u32x2*>(p.out + t * p.ldo + (r - t * p.n_q) * p.D + d) = y;
  }
  if (d == 0 && p.lse) p.lse[r] = sum == 0.0f ? neg_inf() : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

constexpr int64_t kJoinFew = 2048;  // rows
// Key steps of a part, at least (few rows: 128 keys each, many: 64): a part costs a workgroup's start and a share of the
// join (4 single tokens over up to 500 keys, D 128: 9.4 us whole, 11.6 in parts of two steps).
constexpr int kMinPart = 4;
// Such parts of keys from which a 4-bit cache's are also split where that only makes sequences of unequal lengths even, or
// fills a chip that the whole tiles fill by half: as many workgroups as the chip holds (single tokens, heads of 128, us
// whole and split: 32 over up to 16384 keys, 32 + 8 heads 133 and 72.6, 48 162 and 98.9, over 16384 each 175 and 162; 64
// over up to 4096, 16 + 8 heads 47.4 and 43.0; 32 of 4 tokens over up to 8192, 64 + 8 heads 76.3 and 51.8). Equal lengths
// can lose (64 over 8192 each, 16 + 8 heads 104 and 110; heads of 256, 32 over 4096 each, 64 + 8 heads 60.9 and 65.0), and
// so do short ones (64 over 2048 each, 8 + 8 heads 31.6 and 36.1). First tokens beside a window are among the keys (over up to
// 16384, 32 + 8 heads: 32 with a window of 1024 and 6000 first tokens 58.6 and 47.8, of 256 and 12000 104 and 63.6; 64 of 16 + 8
// heads 91.3 and 93.7, 140 and 139).
constexpr int64_t kLongParts = 8;
// Pairs of 64 rows and 64 keys up to which many-row launches take 64 rows to a workgroup (16 + 4 heads of 128, us with 64
// and with 128 rows: prompts of 256 tokens 9.6 and 12.2, 1024 21.7 and 26.6, 2048 39.1 and 49.7, 8192 344 and 277; 128
// tokens behind 8064 24.9 and 26.7, 512 behind 7680 54.1 and 49.9; 16 + 2 heads of 64, 12 chunks of up to 512 tokens,
// window 1024, 26.0 and 29.6; FP8 heads of 128: 2048 44.1 and 57.1, 4096 102 and 111, 8192 339 and 315, 512 behind 7680 64.1
// and 55.6; FP8 heads of 64: 2048 31.5 and 40.9, 4096 69.8 and 77.9, 8192 215 and 195; heads of 256: 2048 73.0 and 85.9, 4096
// 248 and 179, 128 behind 8064 44.8 and 41.6, 512 behind 7680 221 and 95.5). They read more from LDS for the same products, but
// make more workgroups. No count of pairs suits all: FP8 prompts of 4096 tokens lose a tenth, heads of 256 with 128 tokens
// behind 8064 the same.
constexpr int64_t kSmallPairs = 12288;

struct Plan {
  Variant v;
  int64_t items, grid;              // workgroups of a KV head, of the launch
  int64_t o_bytes, ml_bytes, ws_bytes;
  bool split;
};

// A cache of any format.
struct Source {
  Format format;
  bool ok;                                      // its sizes and strides
  int64_t num_pages;
  int32_t page_size, n_kv, head_dim, multiple;  // of head_dim
  Pool k, v;                                    // strides in bytes
  Exponents ke, ve;
  Span spans[4];                                // the pools; scales or exponents

  explicit Source(const qkn_cache& c)
      : format(c.fp8 ? kFp8 : kBf16), ok(cache_ok(c)), num_pages(c.num_pages), page_size(c.page_size), n_kv(c.n_kv),
        head_dim(c.head_dim), multiple(c.fp8 ? 16 : 8), ke{}, ve{}, spans{} {
    if (!ok) return;
    const int64_t esz = c.fp8 ? 1 : 2;
    k = Pool{static_cast<const unsigned char*>(c.k), c.k_scale, c.k_page * esz, c.k_head * esz, static_cast<uint32_t>(c.k_token * esz)};
    v = Pool{static_cast<const unsigned char*>(c.v), c.v_scale, c.v_page * esz, c.v_head * esz, static_cast<uint32_t>(c.v_token * esz)};
    spans[0] = pool_span(c, c.k, c.k_page, c.k_head, c.k_token);
    spans[1] = pool_span(c, c.v, c.v_page, c.v_head, c.v_token);
    spans[2] = array_span(c.k_scale, c.n_kv, 4);
    spans[3] = array_span(c.v_scale, c.n_kv, 4);
    widest = (c.k_token > c.v_token ? c.k_token : c.v_token) * esz;
  }
  explicit Source(const qkn_cache4& c)
      : format(kFp4), ok(cache4_ok(c)), num_pages(c.num_pages), page_size(c.page_size), n_kv(c.n_kv), head_dim(c.head_dim),
        multiple(32), ke{}, ve{}, spans{} {
    if (!ok) return;
    k = Pool{c.k, nullptr, c.k_page, c.k_head, static_cast<uint32_t>(c.k_token)};
    v = Pool{c.v, nullptr, c.v_page, c.v_head, static_cast<uint32_t>(c.v_token)};
    ke = Exponents{c.k_exp, c.ke_page, c.ke_head, static_cast<uint32_t>(c.ke_token)};
    ve = Exponents{c.v_exp, c.ve_page, c.ve_head, static_cast<uint32_t>(c.ve_token)};
    for (int i = 0; i < 4; ++i) spans[i] = pool4_span(c, i);
    widest = 0;
    for (int64_t t : {c.k_token, c.v_token, c.ke_token, c.ve_token}) widest = t > widest ? t : widest;
  }
  int64_t widest;  // stride of a token, bytes
  bool pools_given() const { return k.base && v.base && (format != kFp4 || (ke.base && ve.base)); }
  bool vectors() const {  // exponents are read byte by byte
    for (const Pool* x : {&k, &v})
      if (!aligned(x->base, 16) || x->page % 16 || x->head % 16 || x->token % 16) return false;
    return true;
  }
};

// Sizes alone: QKN_OK, QKN_EINVAL or QKN_ENOTSUP.
int check_sizes(const qkn_attn_args* a, int32_t sinks, const Source* c) {
  if (!a || !c || !c->ok || sinks < 0 || a->T < 0 || a->batch < 0 || a->max_q < 0 || a->max_kv < 0 || a->n_q < 1 ||
      a->n_q % c->n_kv || a->ld_table < 0 || a->window < 0 || (a->window && !a->causal) || !(a->scale > 0.0f) ||
      isinf(a->scale))
    return QKN_EINVAL;
  const int64_t width = static_cast<int64_t>(a->n_q) * c->head_dim;
  if (a->ldq < width || a->ldo < width) return QKN_EINVAL;
  const int64_t lim = int64_t{1} << 31, group = a->n_q / c->n_kv;
  if (c->head_dim > 256 || c->head_dim % c->multiple || c->page_size < 16 || a->T >= lim || a->n_q >= lim / 8 ||
      a->T * a->n_q >= lim || a->T * group + int64_t{a->batch} * 512 >= lim || a->ld_table > lim ||
      a->ld_table * c->page_size > lim - (1 << 17) || c->widest * c->page_size >= lim)
    return QKN_ENOTSUP;
  return QKN_OK;
}

// The workgroups of kernel v, and their workspace.
Plan plan_with(const qkn_attn_args& a, int32_t sinks, const Source& c, const Variant& v) {
  Plan pl{};
  pl.v = v;
  const int64_t group = a.n_q / c.n_kv;
  pl.items = a.T * group / pl.v.rows + a.batch;  // the most row tiles that T tokens can make
  if (pl.items < 1) pl.items = 1;                // no sequence: tokens to clear
  const int64_t slots = int64_t{pl.v.slots} * kCus / c.n_kv;
  // Split keys to fill the chip once, not more (two rounds of half the parts: 40.4 against 34.6 us for 64 single tokens
  // over up to 4096 keys), and not for less than a doubling (12 chunks of up to 512 tokens, window 1024: 41.7 split,
  // 29.7 us whole).
  const int64_t part = int64_t{kMinPart} * pl.v.step;
  pl.split = a.batch && 2 * pl.items <= slots && a.max_kv > part;
  if (pl.split) {
    // the workgroups that take turns on the chip, or as many as the keys can use
    const int64_t most = pl.items * ((a.max_kv + part - 1) / part);
    pl.items = slots < most ? slots : most;
  } else if (c.format == kFp4 && a.batch) {
    const int64_t full = int64_t{pl.v.fit} * kCus / c.n_kv;
    int64_t keys = a.max_kv;
    if (a.window && int64_t{a.window} + sinks < keys) keys = int64_t{a.window} + sinks;
    // row tiles of max_q tokens a sequence; sequences may have more, which the workgroups have to suffice for
    const int64_t each = ((a.max_q < 1 ? 1 : a.max_q) * group + pl.v.rows - 1) / pl.v.rows * a.batch;
    pl.split = 2 * (each < pl.items ? each : pl.items) <= full && keys >= kLongParts * part;
    if (pl.split && pl.items < full) pl.items = full;
  }
  if (pl.split) {
    pl.ml_bytes = pl.items * c.n_kv * pl.v.rows * 8;
    pl.o_bytes = pl.items * c.n_kv * pl.v.rows * 4 * int64_t{c.head_dim};
    pl.ws_bytes = pl.o_bytes + pl.ml_bytes + a.T * a.n_q * 8;
  }
  pl.grid = pl.items * c.n_kv;
  return pl;
}

Variant few_rows_of(const Source& c, bool sinks, int dt, int rows) {
  if (c.format == kFp4) return few_rows4(dt, rows);
  return (sinks ? few_rows_sinks : few_rows)(dt, c.format == kFp8, rows);
}
Variant many_rows_of(const Source& c, bool sinks, int dt, bool small) {
  if (c.format == kFp4) return many_rows4(dt, small);
  return (sinks ? many_rows_sinks : many_rows)(dt, c.format == kFp8, small);
}

// The kernel, of two that may serve where rows are many: little work, or much.
Plan plan_of(const qkn_attn_args& a, int32_t sinks, const Source& c, int64_t* workspace_bytes = nullptr) {
  const int dt = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
  const int64_t group = a.n_q / c.n_kv, rows = (a.max_q < 1 ? 1 : a.max_q) * group;
  const bool few = rows <= (dt == 256 ? 32 : 64);
  // the mask chooses kernels and splits, not the workspace: one serves a model's layers with and without a window
  qkn_attn_args whole = a;
  whole.window = 0;
  if (few) {
    const Variant v = few_rows_of(c, sinks, dt, static_cast<int>(rows));
    if (workspace_bytes) *workspace_bytes = plan_with(whole, 0, c, v).ws_bytes;
    return plan_with(a, sinks, c, v);
  }
  // keys that a row sees, about, and pairs of 64 rows and 64 keys in all
  int64_t keys = a.max_kv - (a.causal ? (a.max_q < a.max_kv ? a.max_q : a.max_kv) / 2 : 0);
  if (a.window && int64_t{a.window} + sinks < keys) keys = int64_t{a.window} + sinks;
  const int64_t pairs = (a.T * group + 63) / 64 * c.n_kv * ((keys + 63) / 64);
  const Variant small = many_rows_of(c, sinks, dt, true), large = many_rows_of(c, sinks, dt, false);
  if (workspace_bytes) {
    const int64_t s = plan_with(whole, 0, c, small).ws_bytes, l = plan_with(whole, 0, c, large).ws_bytes;
    *workspace_bytes = s > l ? s : l;
  }
  return plan_with(a, sinks, c, pairs <= kSmallPairs ? small : large);
}

int attn_impl(const qkn_attn_args* args, int32_t sinks, const Source* cache, void* workspace, int64_t workspace_bytes,
              void* stream) {
  int rc = check_sizes(args, sinks, cache);
  if (rc != QKN_OK) return rc;
  const qkn_attn_args& a = *args;
  const Source& c = *cache;
  if (!a.window) sinks = 0;  // every token sees them
  if (a.T == 0) return QKN_OK;
  if (!a.q || !a.out || !a.q_start || (a.batch && (!a.kv_len || (a.ld_table && !a.block_table))) ||
      (c.num_pages && !c.pools_given()))
    return QKN_EINVAL;
  const Plan pl = plan_of(a, sinks, c);
  if (pl.ws_bytes && (!workspace || workspace_bytes < pl.ws_bytes)) return QKN_EINVAL;
  if (!aligned(a.q, 16) || !aligned(a.out, 16) || a.ldq % 8 || a.ldo % 8 || !c.vectors() ||
      (pl.ws_bytes && !aligned(workspace, 16)))
    return QKN_ENOTSUP;
  const int64_t rows = a.T * a.n_q;
  const bool join_few = rows <= kJoinFew;
  const int64_t join_grid = join_few ? rows : (rows + 7) / 8;
  if (!qkn_host::launchable(pl.grid, pl.v.threads) || (pl.split && !qkn_host::launchable(join_grid, kJoinThreads)))
    return QKN_ENOTSUP;

  const int64_t width = int64_t{a.n_q} * c.head_dim;
  const Span in[] = {Span{reinterpret_cast<uintptr_t>(a.q), a.T, a.ldq, width, 2},
                     array_span(a.q_start, int64_t{a.batch} + 1, 4),
                     array_span(a.kv_len, a.batch, 4),
                     array_span(a.block_table, a.batch * a.ld_table, 4),
                     c.spans[0], c.spans[1], c.spans[2], c.spans[3]};
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
  p.k = c.k;
  p.v = c.v;
  p.ke = c.ke;
  p.ve = c.ve;
  p.num_pages = static_cast<uint32_t>(c.num_pages);
  p.page_shift = log2_of(c.page_size);
  p.batch = a.batch;
  p.n_q = a.n_q;
  p.n_kv = c.n_kv;
  p.D = c.head_dim;
  p.items = static_cast<int32_t>(pl.items);
  p.causal = a.causal != 0;
  p.window = a.window;
  p.sinks = sinks;
  p.c = a.scale * 1.44269504088896340736f;
  p.group = fast_div(static_cast<uint32_t>(a.n_q / c.n_kv));
  p.kv_heads = fast_div(static_cast<uint32_t>(c.n_kv));
  p.min_part = kMinPart;
  if (pl.split) {
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_ml = reinterpret_cast<f32x2*>(ws + pl.o_bytes);
    p.parts_of = reinterpret_cast<int32_t(*)[2]>(ws + pl.o_bytes + pl.ml_bytes);
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
  if (pl.split) {
    int32_t tile_rows = pl.v.rows;
    void* jargs[] = {&p, &tile_rows};
    const dim3 jgrid(static_cast<unsigned>(join_grid), static_cast<unsigned>((c.head_dim + 4 * kJoinVecs - 1) / (4 * kJoinVecs)));
    const void* join = join_few ? reinterpret_cast<const void*>(qkn_attn_join<8>) : reinterpret_cast<const void*>(qkn_attn_join<1>);
    if (hipLaunchKernel(join, jgrid, dim3(kJoinThreads), jargs, 0, st) != hipSuccess)
      return QKN_EHIP;
  }
  qkn_host::record_launch(
      qkn_launch_info{pl.v.name, pl.grid, pl.v.threads, pl.grid * (pl.v.threads / 64), pl.v.lds});
  return QKN_OK;
}

int64_t workspace_bytes_of(const qkn_attn_args* args, const Source* cache) {
  const int rc = check_sizes(args, 0, cache);
  if (rc != QKN_OK) return rc;
  if (args->T == 0) return 0;
  int64_t bytes = 0;
  plan_of(*args, 0, *cache, &bytes);
  return bytes;
}

}  // namespace attn

extern "C" {

int64_t qkn_attn_workspace_bytes(const qkn_attn_args* args, const qkn_cache* cache) {
  if (!cache) return QKN_EINVAL;
  const attn::Source c(*cache);
  return attn::workspace_bytes_of(args, &c);
}

int qkn_attn(const qkn_attn_args* args, const qkn_cache* cache, void* workspace, int64_t workspace_bytes,
             void* stream) {
  return qkn_attn_sinks(args, 0, cache, workspace, workspace_bytes, stream);
}

int qkn_attn_sinks(const qkn_attn_args* args, int32_t sinks, const qkn_cache* cache, void* workspace,
                   int64_t workspace_bytes, void* stream) {
  if (!cache) return QKN_EINVAL;
  const attn::Source c(*cache);
  return attn::attn_impl(args, sinks, &c, workspace, workspace_bytes, stream);
}

int64_t qkn_attn4_workspace_bytes(const qkn_attn_args* args, const qkn_cache4* cache) {
  if (!cache) return QKN_EINVAL;
  const attn::Source c(*cache);
  return attn::workspace_bytes_of(args, &c);
}

int qkn_attn4(const qkn_attn_args* args, int32_t sinks, const qkn_cache4* cache, void* workspace,
              int64_t workspace_bytes, void* stream) {
  if (!cache) return QKN_EINVAL;
  const attn::Source c(*cache);
  return attn::attn_impl(args, sinks, &c, workspace, workspace_bytes, stream);
}

}  // extern "C"
