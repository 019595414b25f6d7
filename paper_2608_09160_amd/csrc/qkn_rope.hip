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
// A 4-bit cache's blocks are four lanes' groups (where pairs are apart) or two lanes' both groups: the largest magnitude
// crosses lanes by DPP, as integers, and the exponent is a carry from the mantissa. Rows that no vector fits take half a
// wavefront for a block of 32, and so do heads for whose rotation this is not written: pairs apart where head or rotation is
// no multiple of 64, neighbouring pairs where the rotation is no multiple of 32. (Of rotations of 16 and 32 elements, and of
// neighbouring pairs, blocks would be two lanes' both groups as well.) V goes with K there. 8192 tokens of 16 + 4 heads, 88 MB,
// 23.0 us with two ranks: 247 vector instructions a wavefront, issued for 10 of them; two tokens a wavefront, which share
// gamma, were slower (25.4 for 24.4 at that time). Element by element, 32 of each head rotated: 75.9 (vectors, 64 or all
// rotated, 19 in calls in a row); 16 + 8 heads of 32, 16 rotated, 27 MB, 36.1 (none rotated 9.4).
// Instructions count beside the bytes, so what would only move registers is not there: a kernel for each layout of pairs,
// rows and slots addressed for all lanes at once, and lanes without gamma multiplied by 1 (16 + 4 + 4 heads over 4 bits, 354 ->
// 247 vector instructions a wavefront, 24.4 -> 23.0 us; the cases below 24.5 -> 23.2, 70.7 -> 70.2, 5.4 -> 4.5).
// Measured: 8192 tokens of 16 + 4 + 4 heads of 128 with the norm, bf16 cache, 105 MB: 23.2 us, 4.5 TB/s; 32768 tokens of
// 16 + 2 + 2 heads into an FP8 cache, 337 MB: 70 us, 4.8 TB/s; a copy of as many bytes reaches 5 to 5.9. 64 tokens: 4.5 us, a
// launch and one chain of latencies (position -> angles). Element by element (V = 1) 8192 tokens of 16 + 4 + 4 heads of 50,
// 41 MB, take 34.7 us; of 48, in vectors, 11.8.

#include <string.h>

#include "qkn_block.h"
#include "qkn_cache4.h"
#include "qkn_quant4.h"
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
  PoolDev ke, ve;              // exponents of a 4-bit cache
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
  const float* at = partials + (r0 < tp ? r0 : tp - 1) * T + t;
#pragma unroll
  for (int i = 0; i < kRanks; ++i) {
    v[i] = *at;
    at += r0 + i + 1 < tp ? T : 0;
  }
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

// What the cache holds.
enum Format { kBf16, kFp8, kFp4 };

// One unit of one token into the cache.
template <int V, int F>
__device__ __forceinline__ void store_cache(const PoolDev& pool, int64_t page, int64_t row, int head, int a, int b,
                                            bool has_b, float scale, const float (&fa)[V], const float (&fb)[V]) {
  const int64_t at = page * pool.page + head * pool.head + row * pool.token;
  if constexpr (F == kFp8) {
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

// One unit into a 4-bit cache: a block's 32 elements are the groups a (and the groups b) of four lanes where pairs are
// apart, else both groups of two. Units begin at even lanes (of fours where pairs are apart: head and rotated part are
// multiples of 64 there), so the lanes of a block are neighbours in one wavefront, all of them running.
__device__ __forceinline__ void store_cache4(uint8_t* p, uint8_t* q, int a, int b, bool apart, bool keep, const float (&fa)[8],
                                             const float (&fb)[8]) {
  uint32_t ma = quant4::magnitude(fa), mb = quant4::magnitude(fb);
  if (!apart) ma = mb = ma > mb ? ma : mb;
  ma = quant4::max_of_2(ma);
  mb = quant4::max_of_2(mb);
  const uint32_t ma4 = quant4::max_of_4(ma), mb4 = quant4::max_of_4(mb);
  const uint32_t ea = quant4::exponent(apart ? ma4 : ma), eb = quant4::exponent(apart ? mb4 : mb);
  const uint32_t ca = quant4::encode(fa, ea), cb = quant4::encode(fb, eb);
  if (!keep) return;
  *reinterpret_cast<uint32_t*>(p + a / 2) = ca;
  *reinterpret_cast<uint32_t*>(p + b / 2) = cb;
  if (a % 32 == 0) q[a / 32] = static_cast<uint8_t>(ea);
  if (b % 32 == 0) q[b / 32] = static_cast<uint8_t>(eb);
}

// x c + y s. APART: each operation rounded by itself, as what the 4-bit quantiser gets must not depend on the path.
template <bool APART>
__device__ __forceinline__ float cross(float x, float c, float y, float s) {
  if constexpr (APART) {
    return quant4::cross(x, c, y, s);
  } else {
    return x * c + y * s;
  }
}

// What lanes without gamma multiply by, and what is read for angles where there are none.
__device__ const float kOnes[16] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f,
                                    1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};

// A pointer to global memory: chosen among parameters and kOnes it would be one to any memory, whose loads are slower.
typedef const __attribute__((address_space(1))) float* GlobalFloats;
__device__ __forceinline__ GlobalFloats in_global(const float* p) { return (GlobalFloats)p; }

// INTER: pairs are neighbours (V = 1: either, at run time).
template <int V, int F, bool INTER>
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
  const bool apart = turns && !(V > 1 ? INTER : p.interleaved != 0);  // a pair's elements are rot / 2 apart
  const int a = apart ? uh * V : 2 * uh * V;
  const int b = apart ? a + p.half : a + V;
  const bool has_b = V > 1 || b < p.D;  // an odd head ends in half a unit
  if (u >= p.units) return;             // lanes share nothing from here on

  // What the wavefront has in common, and what every lane needs next: all of it asked for before any of it is used, by
  // all lanes alike (lanes without gamma read ones, those that do not turn the first angles), so that the waits are one.
  int32_t at = 0;
  int64_t slot = -1;
  float scale = 1.0f;
  float ranks_q[kRanks] = {}, ranks_k[kRanks] = {};
  if (p.half) at = p.pos[t];
  if (p.cached) {
    slot = p.slots[t];
    if constexpr (F == kFp8) {
      const float* sc = of_v ? p.vp.scale : p.kp.scale;
      if (sc && !of_q) scale = sc[head];
    }
  }
  if (p.q.w) load_ranks(p.q.partials, t, p.T, p.tp, 0, ranks_q);
  if (p.k.w) load_ranks(p.k.partials, t, p.T, p.tp, 0, ranks_k);

  float fa[V], fb[V];
  // the token's rows are the same for all lanes
  const uint16_t *xq = p.q.x + t * p.q.ldx, *xk = p.k.x + t * p.k.ldx, *xv = p.v + t * p.ldv;
  const uint16_t* x = (of_q ? xq : of_v ? xv : xk) + head * p.D;
  load_group<V>(x + a, fa);
  load_group<V>(x + (has_b ? b : a), fb);
  const float* w = of_q ? p.q.w : of_v ? nullptr : p.k.w;
  float wa[V], wb[V], cs[V][2];
  const GlobalFloats w1 = in_global(w ? w + head * p.D + a : kOnes), w2 = in_global(w && has_b ? w + head * p.D + b : kOnes);
#pragma unroll
  for (int e = 0; e < V; ++e) wa[e] = w1[e];
#pragma unroll
  for (int e = 0; e < V; ++e) wb[e] = w2[e];
  const bool inside = at >= 0 && at < p.n_pos, angles = p.half && inside;  // or nothing turns
  const GlobalFloats row = in_global(angles ? p.table + 2 * (static_cast<int64_t>(at) * p.half) : kOnes) +
                           (angles && turns ? 2 * uh * V : 0);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    cs[e][0] = row[2 * e];
    cs[e][1] = row[2 * e + 1];
  }

  float inv_q = 1.0f, inv_k = 1.0f;
  if (p.q.w) inv_q = __builtin_amdgcn_rsqf(__builtin_fmaf(rank_sum(p.q.partials, t, p.T, p.tp, ranks_q), p.q.rcp_d, p.eps));
  if (p.k.w) inv_k = __builtin_amdgcn_rsqf(__builtin_fmaf(rank_sum(p.k.partials, t, p.T, p.tp, ranks_k), p.k.rcp_d, p.eps));

  const float inv = of_q ? inv_q : of_v ? 1.0f : inv_k;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    fa[e] = fa[e] * wa[e] * inv;
    fb[e] = fb[e] * wb[e] * inv;
  }
  if (turns) {
    if constexpr (V > 1 && INTER) {  // pairs (0, 1), (2, 3), ... of group a, then of group b
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float c0 = cs[e / 2][0], s0 = cs[e / 2][1], c1 = cs[V / 2 + e / 2][0], s1 = cs[V / 2 + e / 2][1];
        const float x0 = fa[e], x1 = fa[e + 1], y0 = fb[e], y1 = fb[e + 1];
        fa[e] = cross<F == kFp4>(x0, c0, -x1, s0);
        fa[e + 1] = cross<F == kFp4>(x1, c0, x0, s0);
        fb[e] = cross<F == kFp4>(y0, c1, -y1, s1);
        fb[e + 1] = cross<F == kFp4>(y1, c1, y0, s1);
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xa = fa[e], xb = fb[e];
        fa[e] = cross<F == kFp4>(xa, cs[e][0], -xb, cs[e][1]);
        fb[e] = cross<F == kFp4>(xb, cs[e][0], xa, cs[e][1]);
      }
    }
    if (__builtin_expect(!inside, 0)) {
#pragma unroll
      for (int e = 0; e < V; ++e) fa[e] = fb[e] = __builtin_nanf("");
    }
  }

  if (of_q ? p.q.y != nullptr : !of_v && p.k.y) {
    uint16_t *yq = p.q.y + t * p.q.ldy, *yk = p.k.y + t * p.k.ldy;
    uint16_t* y = (of_q ? yq : yk) + head * p.D;
    store_bf16<V>(y + a, fa);
    if (has_b) store_bf16<V>(y + b, fb);
  }
  const bool keep = !of_q && slot >= 0 && slot < p.n_slots;
  const int64_t page = slot >> p.page_shift, in_page = slot & p.page_mask;
  if constexpr (F == kFp4) {
    if constexpr (V == 8)
      if (__builtin_amdgcn_ballot_w64(keep)) {
        const auto at_row = [&](const PoolDev& pool) {
          return static_cast<uint8_t*>(pool.base) + page * pool.page + in_page * pool.token;
        };
        uint8_t *kc = at_row(p.kp), *vc = at_row(p.vp), *ke = at_row(p.ke), *ve = at_row(p.ve);
        store_cache4((of_v ? vc : kc) + head * (of_v ? p.vp.head : p.kp.head),
                     (of_v ? ve : ke) + head * (of_v ? p.ve.head : p.ke.head), a, b, apart, keep, fa, fb);
      }
  } else if (p.cached && keep) {
    if (of_v) store_cache<V, F>(p.vp, page, in_page, head, a, b, has_b, scale, fa, fb);
    else store_cache<V, F>(p.kp, page, in_page, head, a, b, has_b, scale, fa, fb);
  }
}

// K and V into a 4-bit cache where rows do not fit the vectors: half a wavefront for 32 elements, a lane each.
struct Elements4 {
  FastDiv blocks, per_head;  // blocks of a token (K's and V's); of a head
  int32_t k_blocks;
};
__global__ __launch_bounds__(64 * kWaves) void qkn_rope4_elements(const RopeParams p, const Elements4 x) {
  const uint32_t block = blockIdx.x * (2 * kWaves) + (threadIdx.x >> 5);
  const uint32_t t32 = div(block, x.blocks);
  const int64_t t = t32;
  if (t >= p.T) return;  // half a wavefront at a time
  const int lane = static_cast<int>(threadIdx.x) & 31, in_token = static_cast<int>(block - t32 * x.blocks.d);
  const bool of_v = in_token >= x.k_blocks;
  const int in_seg = in_token - (of_v ? x.k_blocks : 0);
  const int head = static_cast<int>(div(static_cast<uint32_t>(in_seg), x.per_head));
  const int c = 32 * (in_seg - head * static_cast<int>(x.per_head.d)) + lane;

  const uint16_t* row_x = (of_v ? p.v + t * p.ldv : p.k.x + t * p.k.ldx) + head * p.D;
  float f = bf16_lo(row_x[c]);
  if (!of_v) {
    const bool turns = c < 2 * p.half;
    const bool second = turns && (p.interleaved ? (c & 1) != 0 : c >= p.half);
    const int pair = p.interleaved ? c / 2 : second ? c - p.half : c;
    const int other = !turns ? c : p.interleaved ? (c ^ 1) : second ? c - p.half : c + p.half;
    float g = bf16_lo(row_x[other]);
    if (p.k.w) {
      float ranks[kRanks];
      load_ranks(p.k.partials, t, p.T, p.tp, 0, ranks);
      const float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(rank_sum(p.k.partials, t, p.T, p.tp, ranks), p.k.rcp_d, p.eps));
      const float* w = p.k.w + head * p.D;
      f = f * w[c] * inv;
      g = g * w[other] * inv;
    }
    if (turns) {
      const int32_t at = p.pos[t];
      if (at >= 0 && at < p.n_pos) {
        const float* cs = p.table + 2 * (static_cast<int64_t>(at) * p.half + pair);
        f = quant4::cross(f, cs[0], second ? g : -g, cs[1]);
      } else {
        f = __builtin_nanf("");
      }
    }
  }
  uint32_t most = __builtin_bit_cast(uint32_t, f) & 0x7fffffffu;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t m = static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), d));
    most = m > most ? m : most;
  }
  const uint32_t e = quant4::exponent(most);
  const float next = __shfl_xor(f, 1);
  const int64_t slot = p.slots[t];
  if (slot < 0 || slot >= p.n_slots) return;
  const int64_t page = slot >> p.page_shift, row = slot & p.page_mask;
  const PoolDev& codes = of_v ? p.vp : p.kp;
  const PoolDev& exps = of_v ? p.ve : p.ke;
  if (lane % 2 == 0)
    (static_cast<uint8_t*>(codes.base) + page * codes.page + head * codes.head + row * codes.token)[c / 2] =
        static_cast<uint8_t>(quant4::encode2(f, next, e));
  if (lane == 0)
    (static_cast<uint8_t*>(exps.base) + page * exps.page + head * exps.head + row * exps.token)[c / 32] =
        static_cast<uint8_t>(e);
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
              const int64_t* slots, const qkn_cache* cache, const qkn_cache4* cache4, int tp, float eps, void* stream) {
  const bool cached = cache || cache4;
  const int32_t n_kv = cache ? cache->n_kv : cache4 ? cache4->n_kv : 0;
  if ((!q && !k) || head_dim < 1 || rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 || T < 0 || tp < 1 ||
      !(eps >= 0.0f) || isinf(eps) || (v && !cached) || (rot_dim && n_pos < 0))
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
  if (k && !k->y && !cached) return QKN_EINVAL;
  if (cache && (!cache_ok(*cache) || cache->head_dim != head_dim || (k && k->heads != cache->n_kv) || (!k && !v)))
    return QKN_EINVAL;
  if (cache4 && (!cache4_ok(*cache4) || cache4->head_dim != head_dim || (k && k->heads != n_kv) || (!k && !v)))
    return QKN_EINVAL;
  if (v && ldv < n_kv * D) return QKN_EINVAL;
  if (v && n_kv * D > most) return QKN_ENOTSUP;
  if (T == 0) return QKN_OK;
  for (const qkn_rope_seg* s : segs)
    if (s && (!s->x || (s->w && !s->partials))) return QKN_EINVAL;
  if (q && !q->y) return QKN_EINVAL;
  if (rot_dim && (!table || !pos)) return QKN_EINVAL;
  if (cache && (!slots || (cache->num_pages && ((k && !cache->k) || (v && !cache->v))))) return QKN_EINVAL;
  if (cache4 && (!slots || (cache4->num_pages && ((k && (!cache4->k || !cache4->k_exp)) || (v && (!cache4->v || !cache4->v_exp))))))
    return QKN_EINVAL;

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
    r.add(Span{reinterpret_cast<uintptr_t>(v), T, ldv, n_kv * D, 2}, false);
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
  int pools = cache && k && v ? 2 : 0;  // at the end of the list: they may share an allocation, their rows in turn
  bool fit4 = true;
  if (cache4) {
    r.add(array_span(slots, T, 8), false);
    for (int i = 0; i < 4; ++i) {
      if (!(i % 2 ? v != nullptr : k != nullptr)) continue;
      for (int j = 0; j < i; ++j)
        if ((j % 2 ? v != nullptr : k != nullptr) && cache4->num_pages && pool4(*cache4, i).base == pool4(*cache4, j).base)
          return QKN_EOVERLAP;
      r.add(pool4_span(*cache4, i), true);
      ++pools;
      const Pool4 x = pool4(*cache4, i);
      if (i < 2) fit4 = fit4 && aligned(x.base, 4) && x.page % 4 == 0 && x.head % 4 == 0 && x.token % 4 == 0;
    }
    // a block's elements on neighbouring lanes
    fit4 = fit4 && rot_dim % 32 == 0 && (interleaved || rot_dim == 0 || (D % 64 == 0 && rot_dim % 64 == 0));
  }
  for (int a = 0; a < r.n; ++a)
    for (int b = a + 1; b < r.n; ++b) {
      if (a >= r.n - pools) continue;
      if ((r.out[a] || r.out[b]) && spans_overlap(r.item[a], r.item[b])) return QKN_EOVERLAP;
    }

  const int64_t V = vec ? 8 : 1, per_head = (D + 2 * V - 1) / (2 * V);
  if (q) units[0] = q->heads * per_head;
  if (k) units[1] = k->heads * per_head;
  if (v) units[2] = n_kv * per_head;
  // K and V of a 4-bit cache that do not fit the vectors go by themselves, before K's rows may be written in place
  const bool elements = cache4 && !(vec && fit4);
  const int64_t blocks = elements ? ((k ? n_kv : 0) + (v ? n_kv : 0)) * (D / 32) : 0;
  if (T >= int64_t{1} << 31) return QKN_ENOTSUP;
  const int64_t grid4 = (T * blocks + 2 * kWaves - 1) / (2 * kWaves);
  if (elements) {
    units[2] = 0;
    if (k && !k->y) units[1] = 0;
  }
  const int64_t all = units[0] + units[1] + units[2], parts = all ? (all + 63) / 64 : 1;
  const int64_t grid = (T * parts + kWaves - 1) / kWaves;
  // both launches, before either writes
  if (all > most || !qkn_host::launchable(grid4, 64 * kWaves) || (all && !qkn_host::launchable(grid, 64 * kWaves)))
    return QKN_ENOTSUP;

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

  if (cache4) {
    const qkn_cache4& c = *cache4;
    const auto dev = [&](int i) {
      const Pool4 x = pool4(c, i);
      return PoolDev{x.base, nullptr, x.page, x.head, x.token};
    };
    p.kp = dev(0);
    p.vp = dev(1);
    p.ke = dev(2);
    p.ve = dev(3);
    p.n_slots = c.num_pages * c.page_size;
    p.page_shift = log2_of(c.page_size);
    p.page_mask = c.page_size - 1;
    p.cached = 1;
  }

  const Format f = cache4 ? kFp4 : cache && cache->fp8 ? kFp8 : kBf16;
  const char* name = elements ? "rope4/elements" : f == kFp4 ? "rope<8>/fp4"
                     : vec    ? (f == kFp8 ? "rope<8>/fp8" : "rope<8>/bf16")
                              : (f == kFp8 ? "rope<1>/fp8" : "rope<1>/bf16");
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{name, 0, 0, 0, 0});
    return QKN_EDRYRUN;
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (elements) {
    Elements4 x{fast_div(static_cast<uint32_t>(blocks)), fast_div(static_cast<uint32_t>(D / 32)),
                static_cast<int32_t>(k ? n_kv * (D / 32) : 0)};
    void* args[] = {&p, &x};
    if (hipLaunchKernel(reinterpret_cast<const void*>(qkn_rope4_elements), dim3(static_cast<unsigned>(grid4)),
                        dim3(64 * kWaves), args, 0, st) != hipSuccess)
      return QKN_EHIP;
    p.cached = 0;  // the rest writes rows only
  }
  const auto kernel = !vec            ? (f == kFp4   ? qkn_rope<1, kFp4, false>
                                         : f == kFp8 ? qkn_rope<1, kFp8, false>
                                                     : qkn_rope<1, kBf16, false>)
                      : p.interleaved ? (f == kFp4   ? qkn_rope<8, kFp4, true>
                                         : f == kFp8 ? qkn_rope<8, kFp8, true>
                                                     : qkn_rope<8, kBf16, true>)
                                      : (f == kFp4   ? qkn_rope<8, kFp4, false>
                                         : f == kFp8 ? qkn_rope<8, kFp8, false>
                                                     : qkn_rope<8, kBf16, false>);
  const void* fn = reinterpret_cast<const void*>(kernel);
  void* args[] = {&p};
  if (all && hipLaunchKernel(fn, dim3(static_cast<unsigned>(grid)), dim3(64 * kWaves), args, 0, st) != hipSuccess)
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
  return rope_impl(q, k, v, ldv, T, head_dim, rot_dim, interleaved, table, n_pos, pos, slots, cache, nullptr, tp, eps, stream);
}

int qkn_rope_cache4(const qkn_rope_seg* q, const qkn_rope_seg* k, const uint16_t* v, int64_t ldv, int64_t T,
                    int head_dim, int rot_dim, int interleaved, const float* table, int64_t n_pos, const int32_t* pos,
                    const int64_t* slots, const qkn_cache4* cache, int tp, float eps, void* stream) {
  if (!cache) return QKN_EINVAL;
  return rope_impl(q, k, v, ldv, T, head_dim, rot_dim, interleaved, table, n_pos, pos, slots, nullptr, cache, tp, eps, stream);
}

}  // extern "C"
