// libqkn, part 3: rotary positions of Q and K, with the norm's Phases B+C in front and the write into the paged
// cache behind (AMD MI355X, gfx950).
//
// Per element a handful of flops for 2 bytes read and 1 or 2 written: bytes bound it, so each row is read once,
// and everything that a row goes through between projection and cache happens in registers.
//
// A head is cut into units of two groups of V elements, one unit a lane: for the half layout the groups are V
// apart by rot / 2, so that a unit holds whole pairs and no value crosses lanes; for neighbouring pairs and for
// the elements that pass they follow each other. V = 8 is one 16-byte vector a group. A wavefront takes 64 units
// of one token (its statistics, position and slot are then scalars), Q's heads first, then K's, then V's.
// No loop: every wavefront asks for all its rows at once and ends. Its loads, scalars among them, all go out before the
// first of them is waited for, on every lane alike (in branches by kind of row, with the slot read behind the stores, the
// prompt below took 35.7 us and the FP8 one 109). A loop over tokens that asks for the next one's rows ahead and keeps
// gamma in registers was no faster than that: 35 to 48 us, 139 to 181.
//
// Measured: 8192 tokens of 16 + 4 + 4 heads of 128 with the norm, bf16 cache, 105 MB: 24.6 us, 4.3 TB/s; 32768 tokens of
// 16 + 2 + 2 heads into an FP8 cache, 337 MB: 71 us, 4.7 TB/s; a copy of as many bytes reaches 5 to 5.9. 64 tokens: 5.1 us, a
// launch and one chain of latencies (position -> angles). Element by element (V = 1) 8192 tokens of 16 + 4 + 4 heads of 50, 41
// MB, take 37.5 us; of 48, in vectors, 12.8.

#include <string.h>

#include "qkn_block.h"
#include "qkn_rope.h"

namespace {

using namespace qkn_block;
using qkn_host::Span;
using qkn_host::spans_overlap;

constexpr int kWaves = 4;  // wavefronts per workgroup

struct SegDev {
  const uint16_t* x;
  const float* w;
  const float* partials;
  uint16_t* y;
  int64_t ldx, ldy;
  float rcp_d;
};

struct PoolDev {
  void* base;
  const float* scale;
  int64_t page, head, token;
};

struct RopeParams {
  SegDev q, k;
  const uint16_t* v;
  int64_t ldv;
  const float* table;
  const int32_t* pos;
  const int64_t* slots;
  PoolDev kp, vp;
  int64_t n_slots, n_pos, T;
  int32_t page_shift, page_mask;
  int32_t D, half;             // half: pairs of a head
  int32_t turn_units;          // units of a head that rotate
  int32_t q_units, k_units, units;  // units of a token: Q's end, K's end, all
  int32_t interleaved, cached, tp;
  float eps;
  FastDiv per_head, parts;     // units of a head; wavefronts of a token
};

// A token's first statistics (past tp the last one's again). The address is the same on all lanes.
constexpr int kRanks = 4;
__device__ __forceinline__ void load_ranks(const float* __restrict__ partials, int64_t t, int64_t T, int tp, int r0,
                                           float (&v)[kRanks]) {
#pragma unroll
  for (int i = 0; i < kRanks; ++i) v[i] = partials[(r0 + i < tp ? r0 + i : tp - 1) * T + t];
}
// Sum over the ranks, ascending, as Phase B adds them; `v`: the first ones, asked for before.
__device__ __forceinline__ float rank_sum(const float* __restrict__ partials, int64_t t, int64_t T, int tp,
                                          float (&v)[kRanks]) {
  float S = v[0];
#pragma unroll
  for (int i = 1; i < kRanks; ++i) S = i < tp ? S + v[i] : S;
  for (int r = kRanks; r < tp; r += kRanks) {
    load_ranks(partials, t, T, tp, r, v);
#pragma unroll
    for (int i = 0; i < kRanks; ++i) S = r + i < tp ? S + v[i] : S;
  }
  return S;
}

template <int V>
__device__ __forceinline__ void load_group(const uint16_t* p, float (&f)[V]) {
  if constexpr (V == 8) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = bf16_lo(u[e]);
      f[2 * e + 1] = bf16_hi(u[e]);
    }
  } else {
    f[0] = bf16_lo(*p);
  }
}

template <int V>
__device__ __forceinline__ void store_bf16(uint16_t* p, const float (&f)[V]) {
  if constexpr (V == 8) {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    *reinterpret_cast<u32x4*>(p) = u;
  } else {
    *p = static_cast<uint16_t>(pack_bf16x2(f[0], 0.0f));
  }
}

template <int V>
__device__ __forceinline__ void store_fp8(uint8_t* p, const float (&f)[V], float rcp) {
  if constexpr (V == 8) {
    u32x2 u;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      u[e] = pack_fp8x4(f[4 * e] * rcp, f[4 * e + 1] * rcp, f[4 * e + 2] * rcp, f[4 * e + 3] * rcp);
    *reinterpret_cast<u32x2*>(p) = u;
  } else {
    *p = static_cast<uint8_t>(pack_fp8x4(f[0] * rcp, 0.0f, 0.0f, 0.0f));
  }
}

// One unit of one token into the cache.
template <int V, bool FP8>
__device__ __forceinline__ void store_cache(const PoolDev& pool, int64_t page, int64_t row, int head, int a, int b,
                                            bool has_b, float scale, const float (&fa)[V], const float (&fb)[V]) {
  const int64_t at = page * pool.page + head * pool.head + row * pool.token;
  if constexpr (FP8) {
    const float rcp = 1.0f / scale;
    uint8_t* p = static_cast<uint8_t*>(pool.base) + at;
    store_fp8<V>(p + a, fa, rcp);
    if (has_b) store_fp8<V>(p + b, fb, rcp);
  } else {
    uint16_t* p = static_cast<uint16_t*>(pool.base) + at;
    store_bf16<V>(p + a, fa);
    if (has_b) store_bf16<V>(p + b, fb);
  }
}

template <int V, bool FP8>
__global__ __launch_bounds__(64 * kWaves) void qkn_rope(const RopeParams p) {
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  const uint32_t t32 = div(wave, p.parts);
  const int64_t t = t32;
  if (t >= p.T) return;
  const int u = static_cast<int>((wave - t32 * p.parts.d) * 64 + (threadIdx.x & 63));

  const bool of_q = u < p.q_units, of_v = u >= p.k_units;
  const int in_seg = u - (of_q ? 0 : of_v ? p.k_units : p.q_units);
  const int head = static_cast<int>(div(static_cast<uint32_t>(in_seg), p.per_head));
  const int uh = in_seg - head * static_cast<int>(p.per_head.d);
  const bool turns = !of_v && uh < p.turn_units;
  const bool apart = turns && !p.interleaved;  // a pair's elements are rot / 2 apart
  const int a = apart ? uh * V : 2 * uh * V;
  const int b = apart ? a + p.half : a + V;
  const bool has_b = V > 1 || b < p.D;  // an odd head ends in half a unit
  if (u >= p.units) return;             // lanes share nothing from here on

  float fa[V], fb[V];
  const uint16_t* x = (of_q ? p.q.x + t * p.q.ldx : of_v ? p.v + t * p.ldv : p.k.x + t * p.k.ldx) + head * p.D;
  load_group<V>(x + a, fa);
  load_group<V>(x + (has_b ? b : a), fb);

  // What the wavefront has in common, and what every lane needs next: all of it asked for before any of it is used, by
  // all lanes alike (V's units, which need no gamma and no angle, read the first ones), so that the waits are one.
  int32_t at = 0;
  int64_t slot = -1;
  float scale = 1.0f;
  float ranks_q[kRanks] = {}, ranks_k[kRanks] = {};
  if (p.half) at = p.pos[t];
  if (p.cached) {
    slot = p.slots[t];
    if constexpr (FP8) {
      const float* sc = of_v ? p.vp.scale : p.kp.scale;
      if (sc && !of_q) scale = sc[head];
    }
  }
  if (p.q.w) load_ranks(p.q.partials, t, p.T, p.tp, 0, ranks_q);
  if (p.k.w) load_ranks(p.k.partials, t, p.T, p.tp, 0, ranks_k);
  const float* w = of_q ? p.q.w : of_v ? nullptr : p.k.w;
  float wa[V], wb[V], cs[V][2];
  if (p.q.w || p.k.w) {
    const float* any = p.q.w ? p.q.w : p.k.w;
    const float* w1 = w ? w + head * p.D + a : any;
    const float* w2 = w && has_b ? w + head * p.D + b : any;
#pragma unroll
    for (int e = 0; e < V; ++e) wa[e] = w1[e];
#pragma unroll
    for (int e = 0; e < V; ++e) wb[e] = w2[e];
  }
  const bool inside = at >= 0 && at < p.n_pos;  // or nothing turns
  if (p.half && inside) {
    const float* row = p.table + 2 * (static_cast<int64_t>(at) * p.half + (turns ? uh * V : 0));
#pragma unroll
    for (int e = 0; e < V; ++e) {
      cs[e][0] = row[2 * e];
      cs[e][1] = row[2 * e + 1];
    }
  }

  float inv_q = 1.0f, inv_k = 1.0f;
  if (p.q.w) inv_q = __builtin_amdgcn_rsqf(__builtin_fmaf(rank_sum(p.q.partials, t, p.T, p.tp, ranks_q), p.q.rcp_d, p.eps));
  if (p.k.w) inv_k = __builtin_amdgcn_rsqf(__builtin_fmaf(rank_sum(p.k.partials, t, p.T, p.tp, ranks_k), p.k.rcp_d, p.eps));

  if (w) {
    const float inv = of_q ? inv_q : inv_k;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      fa[e] = fa[e] * wa[e] * inv;
      fb[e] = fb[e] * wb[e] * inv;
    }
  }
  if (!inside) {
    if (turns) {
#pragma unroll
      for (int e = 0; e < V; ++e) fa[e] = fb[e] = __builtin_nanf("");
    }
  } else if (turns) {
    if (V > 1 && p.interleaved) {  // pairs (0, 1), (2, 3), ... of group a, then of group b
      if constexpr (V > 1) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float c0 = cs[e / 2][0], s0 = cs[e / 2][1], c1 = cs[V / 2 + e / 2][0], s1 = cs[V / 2 + e / 2][1];
          const float x0 = fa[e], x1 = fa[e + 1], y0 = fb[e], y1 = fb[e + 1];
          fa[e] = x0 * c0 - x1 * s0;
          fa[e + 1] = x1 * c0 + x0 * s0;
          fb[e] = y0 * c1 - y1 * s1;
          fb[e + 1] = y1 * c1 + y0 * s1;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xa = fa[e], xb = fb[e];
        fa[e] = xa * cs[e][0] - xb * cs[e][1];
        fb[e] = xb * cs[e][0] + xa * cs[e][1];
      }
    }
  }

  uint16_t* y = of_q ? p.q.y : of_v ? nullptr : p.k.y;
  if (y) {
    y += t * (of_q ? p.q.ldy : p.k.ldy) + head * p.D;
    store_bf16<V>(y + a, fa);
    if (has_b) store_bf16<V>(y + b, fb);
  }
  if (p.cached && !of_q) {
    if (slot >= 0 && slot < p.n_slots) {
      const int64_t page = slot >> p.page_shift, row = slot & p.page_mask;
      if (of_v) store_cache<V, FP8>(p.vp, page, row, head, a, b, has_b, scale, fa, fb);
      else store_cache<V, FP8>(p.kp, page, row, head, a, b, has_b, scale, fa, fb);
    }
  }
}

// Frequencies and angles in 64 bits: an angle of 10^6 radians in 32 bits is off by up to 0.03.
__global__ __launch_bounds__(256) void qkn_rope_angles(float* table, int64_t n_pos, int half, qkn_rope_scaling s) {
  const int i = static_cast<int>(blockIdx.y * 256 + threadIdx.x);
  if (i >= half) return;
  double f = pow(s.base, -static_cast<double>(i) / half);
  if (s.factor > 1.0) {
    double g = 0.0;
    if (s.high > s.low) {
      const double turns = s.original * f / 6.283185307179586476925;
      g = fmin(1.0, fmax(0.0, (turns - s.low) / (s.high - s.low)));
    }
    f *= g + (1.0 - g) / s.factor;
  }
  for (int64_t p = blockIdx.x; p < n_pos; p += gridDim.x) {
    double sn, cs;
    sincos(static_cast<double>(p) * f, &sn, &cs);
    table[2 * (p * half + i)] = static_cast<float>(cs * s.magnitude);
    table[2 * (p * half + i) + 1] = static_cast<float>(sn * s.magnitude);
  }
}

struct Regions {
  Span item[16];
  bool out[16];
  int n = 0;
  void add(const Span& s, bool is_out) {
    item[n] = s;
    out[n++] = is_out;
  }
};

// 1 / d_full, rounded to 32 bits once, as the norm's own entry points take it.
float rcp_d(const qkn_rope_seg& s) { return s.w ? static_cast<float>(1.0 / static_cast<double>(s.d_full)) : 0.0f; }

// A row tensor for the vector path.
bool vec_rows(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

int rope_impl(const qkn_rope_seg* q, const qkn_rope_seg* k, const uint16_t* v, int64_t ldv, int64_t T, int head_dim,
              int rot_dim, int interleaved, const float* table, int64_t n_pos, const int32_t* pos,
              const int64_t* slots, const qkn_cache* cache, int tp, float eps, void* stream) {
  if ((!q && !k) || head_dim < 1 || rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 || T < 0 || tp < 1 ||
      !(eps >= 0.0f) || isinf(eps) || (v && !cache) || (rot_dim && n_pos < 0))
    return QKN_EINVAL;
  const int64_t D = head_dim, most = int64_t{1} << 30;
  int64_t units[3] = {0, 0, 0};
  const qkn_rope_seg* segs[2] = {q, k};
  for (int i = 0; i < 2; ++i) {
    const qkn_rope_seg* s = segs[i];
    if (!s) continue;
    if (s->heads < 1) return QKN_EINVAL;
    const int64_t width = s->heads * D;
    if (s->ldx < width || (s->y && s->ldy < width) || (s->w && s->d_full < width)) return QKN_EINVAL;
    if (width > most) return QKN_ENOTSUP;
  }
  if (k && !k->y && !cache) return QKN_EINVAL;
  if (cache && (!cache_ok(*cache) || cache->head_dim != head_dim || (k && k->heads != cache->n_kv) || (!k && !v)))
    return QKN_EINVAL;
  if (v && (ldv < cache->n_kv * D)) return QKN_EINVAL;
  if (v && cache->n_kv * D > most) return QKN_ENOTSUP;
  if (T == 0) return QKN_OK;
  for (const qkn_rope_seg* s : segs)
    if (s && (!s->x || (s->w && !s->partials))) return QKN_EINVAL;
  if (q && !q->y) return QKN_EINVAL;
  if (rot_dim && (!table || !pos)) return QKN_EINVAL;
  if (cache && (!slots || (cache->num_pages && ((k && !cache->k) || (v && !cache->v))))) return QKN_EINVAL;

  Regions r;
  bool vec = D % 16 == 0 && rot_dim % 16 == 0;
  for (int i = 0; i < 2; ++i) {
    const qkn_rope_seg* s = segs[i];
    if (!s) continue;
    const int64_t width = s->heads * D;
    r.add(Span{reinterpret_cast<uintptr_t>(s->x), T, s->ldx, width, 2}, false);
    vec = vec && vec_rows(s->x, s->ldx);
    if (s->y && !(s->y == s->x && s->ldy == s->ldx)) r.add(Span{reinterpret_cast<uintptr_t>(s->y), T, s->ldy, width, 2}, true);
    else if (s->y) r.out[r.n - 1] = true;  // in place: the input is the output
    if (s->y) vec = vec && vec_rows(s->y, s->ldy);
    if (s->w) {
      r.add(array_span(s->w, width, 4), false);
      r.add(array_span(s->partials, tp * T, 4), false);
    }
  }
  if (v) {
    r.add(Span{reinterpret_cast<uintptr_t>(v), T, ldv, cache->n_kv * D, 2}, false);
    vec = vec && vec_rows(v, ldv);
  }
  if (rot_dim) {
    r.add(array_span(table, n_pos * rot_dim, 4), false);
    r.add(array_span(pos, T, 4), false);
  }
  if (cache) {
    r.add(array_span(slots, T, 8), false);
    const qkn_cache& c = *cache;
    const int64_t esz = c.fp8 ? 1 : 2;
    if (c.k_scale) r.add(array_span(c.k_scale, c.n_kv, 4), false);
    if (c.v_scale) r.add(array_span(c.v_scale, c.n_kv, 4), false);
    const uintptr_t to = static_cast<uintptr_t>(8 * esz);  // a group of 8 elements
    if (k) {
      r.add(pool_span(c, c.k, c.k_page, c.k_head, c.k_token), true);
      vec = vec && aligned(c.k, to) && c.k_page % 8 == 0 && c.k_head % 8 == 0 && c.k_token % 8 == 0;
    }
    if (v) {
      r.add(pool_span(c, c.v, c.v_page, c.v_head, c.v_token), true);
      vec = vec && aligned(c.v, to) && c.v_page % 8 == 0 && c.v_head % 8 == 0 && c.v_token % 8 == 0;
    }
    if (k && v && c.num_pages && c.k == c.v) return QKN_EOVERLAP;
  }
  const bool two_pools = cache && k && v;  // they may share an allocation, their rows in turn
  for (int a = 0; a < r.n; ++a)
    for (int b = a + 1; b < r.n; ++b) {
      if (two_pools && a == r.n - 2 && b == r.n - 1) continue;
      if ((r.out[a] || r.out[b]) && spans_overlap(r.item[a], r.item[b])) return QKN_EOVERLAP;
    }

  const int64_t V = vec ? 8 : 1, per_head = (D + 2 * V - 1) / (2 * V);
  if (q) units[0] = q->heads * per_head;
  if (k) units[1] = k->heads * per_head;
  if (v) units[2] = cache->n_kv * per_head;
  const int64_t all = units[0] + units[1] + units[2], parts = (all + 63) / 64;
  if (all > most || T > (int64_t{1} << 31) - 8 || T * parts > (int64_t{1} << 31) - 8) return QKN_ENOTSUP;

  RopeParams p;
  memset(&p, 0, sizeof(p));
  if (q) p.q = SegDev{q->x, q->w, q->partials, q->y, q->ldx, q->ldy, rcp_d(*q)};
  if (k) p.k = SegDev{k->x, k->w, k->partials, k->y, k->ldx, k->ldy, rcp_d(*k)};
  p.v = v;
  p.ldv = ldv;
  p.table = table;
  p.pos = pos;
  p.slots = slots;
  if (cache) {
    const qkn_cache& c = *cache;
    p.kp = PoolDev{c.k, c.k_scale, c.k_page, c.k_head, c.k_token};
    p.vp = PoolDev{c.v, c.v_scale, c.v_page, c.v_head, c.v_token};
    p.n_slots = c.num_pages * c.page_size;
    p.page_shift = log2_of(c.page_size);
    p.page_mask = c.page_size - 1;
    p.cached = 1;
  }
  p.n_pos = n_pos;
  p.T = T;
  p.D = head_dim;
  p.half = rot_dim / 2;
  p.turn_units = static_cast<int32_t>(rot_dim / (2 * V));
  p.q_units = static_cast<int32_t>(units[0]);
  p.k_units = static_cast<int32_t>(units[0] + units[1]);
  p.units = static_cast<int32_t>(all);
  p.interleaved = interleaved != 0;
  p.tp = tp;
  p.eps = eps;
  p.per_head = fast_div(static_cast<uint32_t>(per_head));
  p.parts = fast_div(static_cast<uint32_t>(parts));

  const bool fp8 = cache && cache->fp8;
  const int64_t grid = (T * parts + kWaves - 1) / kWaves;
  const char* name = vec ? (fp8 ? "rope<8>/fp8" : "rope<8>/bf16") : (fp8 ? "rope<1>/fp8" : "rope<1>/bf16");
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{name, 0, 0, 0, 0});
    return QKN_EDRYRUN;
  }
  const void* fn = vec ? (fp8 ? reinterpret_cast<const void*>(qkn_rope<8, true>)
                              : reinterpret_cast<const void*>(qkn_rope<8, false>))
                       : (fp8 ? reinterpret_cast<const void*>(qkn_rope<1, true>)
                              : reinterpret_cast<const void*>(qkn_rope<1, false>));
  void* args[] = {&p};
  if (hipLaunchKernel(fn, dim3(static_cast<unsigned>(grid)), dim3(64 * kWaves), args, 0,
                      static_cast<hipStream_t>(stream)) != hipSuccess)
    return QKN_EHIP;
  qkn_host::record_launch(qkn_launch_info{name, grid, 64 * kWaves, grid * kWaves, 0});
  return QKN_OK;
}

}  // namespace

extern "C" {

int qkn_rope_table(float* table, int64_t n_pos, int rot_dim, const qkn_rope_scaling* s, void* stream) {
  if (!s || n_pos < 0 || rot_dim < 2 || rot_dim % 2 || !(s->base > 0.0) || isinf(s->base) || !(s->factor >= 1.0) ||
      isinf(s->factor) || !isfinite(s->magnitude))
    return QKN_EINVAL;
  const bool ramp = s->low != 0.0 || s->high != 0.0;
  if (ramp && (!(s->low >= 0.0) || !(s->low < s->high) || isinf(s->high) || !(s->original > 0.0) || isinf(s->original)))
    return QKN_EINVAL;
  if (n_pos == 0) return QKN_OK;
  if (!table) return QKN_EINVAL;
  if (n_pos > (int64_t{1} << 31)) return QKN_ENOTSUP;
  const int half = rot_dim / 2;
  const int64_t gx = n_pos < 65536 ? n_pos : 65536, gy = (half + 255) / 256;
  if (gy > 65535) return QKN_ENOTSUP;
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{"rope_table", 0, 0, 0, 0});
    return QKN_EDRYRUN;
  }
  qkn_rope_scaling sc = *s;
  int h = half;
  void* args[] = {&table, &n_pos, &h, &sc};
  if (hipLaunchKernel(reinterpret_cast<const void*>(qkn_rope_angles),
                      dim3(static_cast<unsigned>(gx), static_cast<unsigned>(gy)), dim3(256), args, 0,
                      static_cast<hipStream_t>(stream)) != hipSuccess)
    return QKN_EHIP;
  qkn_host::record_launch(qkn_launch_info{"rope_table", gx * gy, 256, gx * gy * 4, 0});
  return QKN_OK;
}

int qkn_rope_cache(const qkn_rope_seg* q, const qkn_rope_seg* k, const uint16_t* v, int64_t ldv, int64_t T,
                   int head_dim, int rot_dim, int interleaved, const float* table, int64_t n_pos, const int32_t* pos,
                   const int64_t* slots, const qkn_cache* cache, int tp, float eps, void* stream) {
  return rope_impl(q, k, v, ldv, T, head_dim, rot_dim, interleaved, table, n_pos, pos, slots, cache, tp, eps, stream);
}

}  // extern "C"
