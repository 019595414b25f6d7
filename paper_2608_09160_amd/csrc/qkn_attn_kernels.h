// Attention over the paged cache: the kernels (templates; instantiated in qkn_attn_*.hip).
//
// Rows. The query heads of one KV head see the same keys, so a sequence's rows for KV head g are its (token, head of
// the group) pairs, row r = token r / G, head g G + r % G: a tile of rows uses each key tile for all of them.
//
// Products (v_mfma_f32_16x16x32_bf16: A 16 x 32, B 32 x 16, lane l holds row (column) l mod 16, k 8 (l / 16) .. + 7;
// result column l mod 16, rows 4 (l / 16) .. + 3). Scores are formed transposed, S^T = K Q^T: a lane then holds 4
// keys of each 16 for one query row, its softmax needs no other lane, and its weights are, packed to bf16, already
// the B operand of O^T = V^T P^T, with keys 16 a + 4 (l / 16) + r as the product's k (any order of keys serves, as
// long as V's is the same). O^T also has one row per lane, so a row's rescaling is one factor per lane.
// V^T is read from the row-major V tile by the transposing LDS read: 16 lanes fetch 4 rows (8 for FP8) of 16 columns
// and lane i receives column i.
//
// Softmax. m is a bound on the row's scores that is raised only where a score exceeds it by 2^8 in weight
// (`kSlack`): most tiles then need no maximum across lanes and no rescaling. Weights are at most 2^8, which changes
// nothing in their relative rounding. The sum l is of the unrounded fp32 weights.
//
// Tiles. KT keys at a time, rows straight from the cache's pages into LDS (buffer_load ... lds, 16 bytes a lane), two
// buffers, the next tile in flight while one is computed. A wavefront fetches 16 rows at a time: they lie in one page,
// whose descriptor ends at the sequence's last token (or has no bytes for a bad page number), so rows past it read
// zeros. 16-byte chunks of a row are stored at chunk ^ f(row), f such that the rows of one LDS read fall on different
// banks.
//
// Two ways to share the work of a workgroup:
//   SHARED  every wavefront has its own 16 CB rows, all take the same key tiles (many rows: products bound it);
//   !SHARED every wavefront takes its own key tiles for the same 16 CB rows, with no barrier in the loop, and the
//           wavefronts' results are joined at the end (few rows: bytes bound it). No other wavefront wants its K rows,
//           and a row is an operand as it is: they go to registers, LDS has V only, and with half the LDS a CU holds
//           twice the wavefronts, so twice the bytes are on their way.
// Over workgroups the keys are split further where rows alone do not fill the chip (`schedule`); qkn_attn_join adds the
// parts in a fixed order.
//
// What bounds it (times of calls in a row; the first ones after a pause take up to a sixth longer). Few rows: the cache's bytes.
// 64 single tokens over up to 4096 keys of 8 + 2 heads of 128, 139 MB, 34.3 us, 4.1 TB/s (4.7 the join);
// 16 over up to 32768 FP8 keys of 16 + 2 heads, 158 MB, 39.7 us, 4.0 TB/s; 4 over up to 500 keys 9.7 us, latencies. Many rows:
// instruction issue. A prompt of 8192 tokens of 16 + 4 heads, 275 Gflop, takes 274 to 286 us, 1.0 Pflop/s. By its counters
// a SIMD's matrix core is busy for 264 k of the 523 k cycles (128 products of 16 cycles for 64 rows x 64 keys of 128), and
// the 372 other vector instructions of such a block (the softmax's fma, exp and conversions, most of them) are issued for
// 1800 cycles, 227 k in all: products and softmax take turns more than they overlap. The LDS is no bound: its reads, 4
// cycles for 16 bytes a lane and 2 for a transposing one of 8, take 133 k. Windowed chunks (12 of up to 512 tokens, window
// 1024, 16 + 2 heads of 64, 25.8 us) too: a wavefront's 16 rows and 64 keys take 256 cycles of products and 620 of
// other vector instructions; 560 workgroups make three wavefronts on some SIMDs, whose up to 3 x 18 such steps are the
// call's 49 k cycles.
// Slower: the wavefronts in two groups that take turns at products and softmax (288 to 309 us), 64 rows a wavefront with
// one tile's softmax between another's products (322), wave priorities by phase and operands fetched 1 to 10 products ahead
// (within 4 %).
#ifndef QKN_ATTN_KERNELS_H
#define QKN_ATTN_KERNELS_H

#include "qkn_block.h"

namespace attn {

using namespace qkn_block;

typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef __attribute__((address_space(3))) unsigned char LdsByte;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Pool {
  const unsigned char* base;
  const float* scale;
  int64_t page, head;   // strides in bytes
  uint32_t token;
};

struct Params {
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* table;
  int64_t ldq, ldo, ld_table, T;
  Pool k, v;
  uint32_t num_pages;
  int32_t page_shift;
  int32_t batch, n_q, n_kv, D;
  int32_t items;                       // workgroups of a KV head
  int32_t causal, window;
  float c;                             // scale * log2(e)
  FastDiv group, kv_heads;
  // split keys (NULL: not split): what each workgroup has of its row tile, and which workgroups have a row's parts
  float* part_o;                       // [workgroups, BM, D]
  f32x2* part_ml;                      // [workgroups, BM]: bound (log2 units) and sum; sum 0: nothing
  int32_t (*parts_of)[2];              // [T * n_q]: workgroup of the first part; parts * 256 + row of the tile, or 0
  int32_t min_part;                    // key steps of a part, at least
};

// A kernel and what its launch has to know.
struct Variant {
  const void* fn;
  int rows, step, threads, lds, slots;  // rows of a workgroup; keys that it takes at a time; workgroups of a CU
  const char* name;
};

constexpr float kSlack = 8.0f;  // log2
constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

__device__ __forceinline__ Rsrc rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0), static_cast<int>(bytes),
                                           0x00020000);
}
// Lane l's 16 bytes at byte `off` of the buffer go to dst + 16 l.
__device__ __forceinline__ void load_to_lds(Rsrc r, unsigned char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsByte*)dst, 16, off, 0, 0, 0);
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the N youngest
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void group_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// DT: head size, rounded up (the rest reads as zeros); OCC: wavefronts per SIMD that the registers must allow.
template <int DT_, bool FP8_, int CB_, int WAVES_, bool SHARED_, int KT_, int OCC_>
struct Cfg {
  static constexpr int DT = DT_, CB = CB_, WAVES = WAVES_, KT = KT_, OCC = OCC_;
  static constexpr bool FP8 = FP8_, SHARED = SHARED_;
  static constexpr int AHEAD = 4;                 // LDS reads ahead of their products
  static constexpr int ES = FP8 ? 1 : 2;
  static constexpr int RB = DT * ES;              // bytes of an LDS row
  static constexpr int CH = RB / 16;              // its 16-byte chunks
  static constexpr int RPL = 64 / CH;             // rows of one load instruction
  static constexpr int PER256 = RB >= 256 ? 1 : 256 / RB;  // rows of one pass over the banks
  static constexpr int BM = 16 * CB * (SHARED ? WAVES : 1);  // rows of a workgroup
  static constexpr int TILE = KT * RB;            // bytes of a K (V) tile
  static constexpr int BUF = (SHARED ? 2 : 1) * TILE;  // a buffer: K and V, or V
  static constexpr int V_AT = SHARED ? TILE : 0;  // V in it
  static constexpr int STEP = KT * (SHARED ? 1 : WAVES);  // keys that a workgroup takes at a time
  static constexpr int KL = DT * ES / 64;         // 16-byte loads of 16 K rows into registers (!SHARED)
  static constexpr int BR = SHARED ? KT / WAVES : 16;  // rows that a wavefront loads together, of one page
  static constexpr int BLOCKS = SHARED ? 1 : KT / 16;  // how often for a tile
  static constexpr int V_LOADS = BLOCKS * BR / RPL;    // load instructions of a wavefront for a V tile
  static constexpr int STAGES = SHARED ? 1 : WAVES;    // key streams of a workgroup
  static constexpr int JOIN_ROW = DT + 4;         // floats of a row while wavefronts are joined
  static constexpr int JOIN = SHARED ? 0 : WAVES * 16 * CB * (JOIN_ROW + 2) * 4;
  static constexpr int LDS = 2 * BUF * STAGES > JOIN ? 2 * BUF * STAGES : JOIN;
  static_assert(BR % RPL == 0, "whole load instructions");
  static_assert(WAVES == 4, "a wavefront of a workgroup on each SIMD");
  static constexpr int SLOTS = OCC < 160 * 1024 / LDS ? OCC : 160 * 1024 / LDS;  // workgroups that a CU holds
  static_assert(LDS <= 160 * 1024, "LDS");
  static_assert(CH <= 64 && V_LOADS < 64, "loads");
  // Chunk c of row r is stored at c ^ swizzle(r). K: 16 lanes read the same chunk of 16 rows.
  __device__ static constexpr int swizzle_k(int r) { return (r / PER256) & ((CH < 16 ? CH : 16) - 1); }
  // V, bf16: 32 lanes read 2 chunks of 8 rows. FP8: one chunk of rows 0 to 7 and 16 to 23.
  __device__ static constexpr int swizzle_v(int r) {
    if constexpr (FP8) return ((r & 7) / PER256) | (((r >> 4) & 1) * (8 / PER256));
    else return (((r & 7) / PER256) * 2) & (CH - 1);
  }
};

// The keys that the workgroup's (wavefront's) rows see.
struct Range {
  int32_t lo, hi;
};

// The transposing LDS reads. `filling` is the buffer that loads in flight write, which the read does not touch: without
// being told, the compiler waits for all of them before each of these reads (unlike before plain ones).
__device__ __forceinline__ s16x4 read_tr16(unsigned char* src, const unsigned char* __restrict filling) {
  if (filling == src) __builtin_unreachable();
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(src));
}
__device__ __forceinline__ i32x2 read_tr8(unsigned char* src, const unsigned char* __restrict filling) {
  if (filling == src) __builtin_unreachable();
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(src));
}

template <bool FP8>
struct RawOf {
  using T = u32x4;
};
template <>
struct RawOf<true> {
  using T = i32x2;
};

template <class C>
struct Tiles {
  // One wavefront's view of the key tiles: which lane fetches and reads what.
  unsigned char* buf;       // its stream's two buffers
  int lane, wave;
  const Params& p;
  const unsigned char* base_k;  // the head's rows of page 0
  const unsigned char* base_v;
  int32_t kv_len;
  const int32_t* table;     // the sequence's pages
  int32_t last_page;        // last entry in use
  int32_t page0;            // pages held: lane i has the bytes to page entry page0 + i (lower, upper half; < 0: none)
  int32_t k_lo, k_hi, v_lo, v_hi;
  int32_t next;             // and entry page0 + 64 + i

  __device__ __forceinline__ Tiles(const Params& pp, unsigned char* b, int l, int w) : buf(b), lane(l), wave(w), p(pp) {}

  __device__ __forceinline__ int32_t entry(int32_t i) const {
    i = i < last_page ? i : last_page;
    return table[i < 0 ? 0 : i];
  }
  // Takes 64 pages' places at once, a lane each: the address of a tile is then a few scalar instructions.
  __device__ __forceinline__ void hold(int32_t page) {
    const bool none = static_cast<uint32_t>(page) >= p.num_pages;
    const int64_t k = none ? -1 : page * p.k.page, v = none ? -1 : page * p.v.page;
    k_lo = static_cast<int32_t>(k);
    k_hi = static_cast<int32_t>(k >> 32);
    v_lo = static_cast<int32_t>(v);
    v_hi = static_cast<int32_t>(v >> 32);
  }
  __device__ __forceinline__ void open(int b, int head, int32_t m, int32_t first_key) {
    base_k = p.k.base + head * p.k.head;
    base_v = p.v.base + head * p.v.head;
    kv_len = m;
    table = p.table + b * p.ld_table;
    last_page = (m - 1) >> p.page_shift;
    page0 = first_key >> p.page_shift;
    const int32_t first = entry(page0 + lane);
    next = entry(page0 + 64 + lane);
    hold(first);
  }
  // The BR rows of K (V) from key j on, which are in one page: a descriptor of those that the sequence has.
  template <bool V>
  __device__ __forceinline__ Rsrc rows_of(int32_t j) {
    const int32_t pi = j >> p.page_shift;
    while (pi - page0 >= 64) {  // pages are taken in ascending order
      hold(next);
      page0 += 64;
      next = entry(page0 + 64 + lane);
    }
    const int32_t lo = __builtin_amdgcn_readlane(V ? v_lo : k_lo, pi - page0);
    const int32_t hi = __builtin_amdgcn_readlane(V ? v_hi : k_hi, pi - page0);
    const uint32_t token = V ? p.v.token : p.k.token, row0 = j & ((1 << p.page_shift) - 1);
    const int32_t left = kv_len - j, rows = left < C::BR ? left : C::BR;
    const bool none = left <= 0 || hi < 0;
    const uint64_t off = (static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo)) +
                         static_cast<uint64_t>(row0 * token);
    // a scalar, as it is the same on all lanes: a descriptor in vector registers costs a loop around every load
    const uint32_t bytes = __builtin_amdgcn_readfirstlane(none ? 0 : rows * token - (token - p.D * C::ES));
    return rsrc((V ? base_v : base_k) + (none ? 0 : off), bytes);
  }
  __device__ __forceinline__ int first_row(int bl) const { return C::BR * (C::SHARED ? wave : bl); }
  // Requests this wavefront's rows of the K (V) tile at key j0 into buffer `at`.
  template <bool V>
  __device__ __forceinline__ void request(int32_t j0, int at) {
#pragma unroll
    for (int bl = 0; bl < C::BLOCKS; ++bl) {
      const int row0 = first_row(bl);
      const Rsrc rs = rows_of<V>(j0 + row0);
      const uint32_t token = V ? p.v.token : p.k.token;
      unsigned char* dst = buf + at * C::BUF + (V ? C::V_AT : 0) + row0 * C::RB;
#pragma unroll
      for (int i = 0; i < C::BR / C::RPL; ++i) {
        const int r = i * C::RPL + lane / C::CH;
        const int chunk = (lane % C::CH) ^ (V ? C::swizzle_v(row0 + r) : C::swizzle_k(row0 + r));
        load_to_lds(rs, dst + i * C::RPL * C::RB, chunk * 16 < p.D * C::ES ? r * token + chunk * 16 : 0x7fffffffu);
      }
    }
  }
  // Requests the K rows [j0, j0 + KT) into registers: lane l has 16 bytes from 64 x + 16 (l / 16) on of row l mod 16 of
  // each block. FP8: they are 16 elements, half for one product step and half for the next (q is laid out alike).
  __device__ __forceinline__ void request_k(int32_t j0, u32x4 (&k)[C::KT / 16][C::KL]) {
#pragma unroll
    for (int bl = 0; bl < C::KT / 16; ++bl) {
      const Rsrc r = rows_of<false>(j0 + 16 * bl);
#pragma unroll
      for (int x = 0; x < C::KL; ++x) {
        const uint32_t at = 64 * x + 16 * (lane >> 4);
        k[bl][x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                 r, at < p.D * C::ES ? (lane & 15) * p.k.token + at : 0x7fffffffu, 0, 0));
      }
    }
  }
  // A weight of 0 times an infinite or NaN value is NaN, which a row that does not see the key must not get. In a
  // tile that some rows see in part the product takes 0 in the place of such values (add_infinities gives them to the
  // rows that see them): puts it there in the V rows that this wavefront fetched; true if it found any.
  __device__ __forceinline__ bool make_finite(int at) {
    bool any = false;
#pragma unroll
    for (int bl = 0; bl < C::BLOCKS; ++bl)
#pragma unroll
      for (int i = 0; i < C::BR / C::RPL; ++i) {
        u32x4* src =
            reinterpret_cast<u32x4*>(buf + at * C::BUF + C::V_AT + (first_row(bl) + i * C::RPL) * C::RB + lane * 16);
        u32x4 u = *src;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t field = C::FP8 ? 0x7fu : 0x7f80u;  // all ones: NaN; infinite or NaN
#pragma unroll
          for (int h = 0; h < 32; h += C::FP8 ? 8 : 16)
            if (((u[e] >> h) & field) == field) {
              u[e] &= ~((C::FP8 ? 0xffu : 0xffffu) << h);
              bad = true;
            }
        }
        if (__builtin_amdgcn_ballot_w64(bad)) {
          *src = u;
          any = true;
        }
      }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): written before the barrier
    return any;
  }
  // What a lane reads for an operand; FP8 codes are widened where the operand is used, not where it is read.
  using Raw = typename RawOf<C::FP8>::T;
  __device__ static __forceinline__ bf16x8 operand(Raw w) {
    if constexpr (C::FP8) return widen(w);
    else return __builtin_bit_cast(bf16x8, w);
  }
  // A operand of S^T: 16 keys from row 16 kb, elements 32 step .. + 31.
  __device__ __forceinline__ Raw k_frag(int at, int kb, int step) const {
    const int r = lane & 15, g = lane >> 4;
    const unsigned char* row = buf + at * C::BUF + (16 * kb + r) * C::RB;
    if constexpr (C::FP8) {
      const int c = 2 * step + (g >> 1);
      return *reinterpret_cast<const i32x2*>(row + ((c ^ C::swizzle_k(r)) * 16) + (g & 1) * 8);
    } else {
      const int c = 4 * step + g;
      return *reinterpret_cast<const u32x4*>(row + (c ^ C::swizzle_k(r)) * 16);
    }
  }
  // A operand of O^T: elements 16 db .. + 15 of 32 keys from row 32 kc; k slot 8 g + e is key 4 g + e (e < 4), or
  // 16 + 4 g + e - 4.
  __device__ __forceinline__ Raw v_frag(int at, int kc, int db) const {
    const int i = lane & 15, g = lane >> 4;
    unsigned char* tile = buf + at * C::BUF + C::V_AT + 32 * kc * C::RB;
    const unsigned char* filling = buf + (at ^ 1) * C::BUF;
    if constexpr (C::FP8) {
      const int j = i >> 1, r = j < 4 ? 4 * g + j : 12 + 4 * g + j;
      unsigned char* src = tile + r * C::RB + (db ^ C::swizzle_v(r)) * 16 + (i & 1) * 8;
      return read_tr8(src, filling);
    } else {
      const int r = 4 * g + (i >> 2);
      unsigned char* src = tile + r * C::RB + ((2 * db + ((i >> 1) & 1)) ^ C::swizzle_v(r)) * 16 + (i & 1) * 8;
      const s16x4 a = read_tr16(src, filling), b = read_tr16(src + 16 * C::RB, filling);
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  // Eight e4m3fn codes as bf16, exactly.
  __device__ static __forceinline__ bf16x8 widen(i32x2 w) {
    bf16x8 f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], 1.0f, false);
      const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], 1.0f, true);
      f[4 * e] = lo[0];
      f[4 * e + 1] = lo[1];
      f[4 * e + 2] = hi[0];
      f[4 * e + 3] = hi[1];
    }
    return f;
  }
};

// Running state of a wavefront's 16 CB rows: column block cb, this lane's row 16 cb + lane % 16.
template <class C>
struct Rows {
  bf16x8 q[C::DT / 32][C::CB];
  f32x4 o[C::DT / 16][C::CB];   // O^T, this lane's elements 16 db + 4 (lane / 16) .. + 3
  float m[C::CB], l[C::CB];     // bound (of raw scores); sum over this lane's keys
  int32_t lo[C::CB], hi[C::CB]; // the keys that the row sees
};

template <class C>
using Scores = f32x4[C::KT / 16][C::CB];
template <class C>
using Weights = bf16x8[C::KT / 32][C::CB];

// S^T = K Q^T of the tile in buffer `at` (!SHARED: of the K rows in kr).
template <class C>
__device__ __forceinline__ void scores(const Tiles<C>& t, const Rows<C>& w, const u32x4 (&kr)[C::KT / 16][C::KL], int at,
                                       Scores<C>& s) {
  constexpr int KB = C::KT / 16, NS = C::DT / 32;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb) s[kb][cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // AHEAD operands ahead of the products, no more: left to itself the compiler reads them all first and runs out of
  // registers
  constexpr int AHEAD = C::AHEAD, RING = AHEAD + 1;
  typename Tiles<C>::Raw a[RING];
  if constexpr (C::SHARED) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = t.k_frag(at, i % KB, i / KB);
  }
#pragma unroll
  for (int i = 0; i < NS * KB; ++i) {
    const int step = i / KB, kb = i % KB, n = i + AHEAD;
    bf16x8 f;
    if constexpr (C::SHARED) {
      if (n < NS * KB) a[n % RING] = t.k_frag(at, n % KB, n / KB);
      f = Tiles<C>::operand(a[i % RING]);
    } else if constexpr (C::FP8) {
      const u32x4 u = kr[kb][step / 2];
      f = Tiles<C>::widen(i32x2{static_cast<int>(u[2 * (step % 2)]), static_cast<int>(u[2 * (step % 2) + 1])});
    } else {
      f = __builtin_bit_cast(bf16x8, kr[kb][step]);
    }
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb)
      s[kb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, w.q[step][cb], s[kb][cb], 0, 0, 0);
    if constexpr (C::SHARED) __builtin_amdgcn_sched_barrier(0);
  }
}

// The scores of keys j0 .. j0 + KT - 1 to weights, with the rows' bounds and sums. masked: some row does not see some
// of the keys.
template <class C>
__device__ __forceinline__ void softmax(Rows<C>& w, Scores<C>& s, Weights<C>& pf, int lane, int32_t j0, float c,
                                        bool masked) {
  constexpr int KB = C::KT / 16, KC = C::KT / 32, ND = C::DT / 16;
  const int g = lane >> 4;
  if (masked) {
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb) {
      const uint32_t seen = static_cast<uint32_t>(w.hi[cb] - w.lo[cb]);
      const int32_t first = j0 + 4 * g - w.lo[cb];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[kb][cb][r] = static_cast<uint32_t>(first + 16 * kb + r) < seen ? s[kb][cb][r] : neg_inf();
    }
  }
  // the largest score of this lane's keys against the row's bound
  bool raise = false;
  float top[C::CB];
#pragma unroll
  for (int cb = 0; cb < C::CB; ++cb) {
    float x = s[0][cb][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) x = fmaxf(x, s[kb][cb][r]);
    top[cb] = x;
    raise |= (x - w.m[cb]) * c > kSlack;  // m = -infinity: any score (+infinity), or none (NaN: false)
  }
  if (__builtin_amdgcn_ballot_w64(raise)) {
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb) {
      float x = fmaxf(top[cb], w.m[cb]);
      x = fmaxf(x, __shfl_xor(x, 16));
      x = fmaxf(x, __shfl_xor(x, 32));
      // each row for itself, so that a row's result does not depend on what else is in the wavefront
      const bool raised = (x - w.m[cb]) * c > kSlack;
      const float f = raised ? __builtin_amdgcn_exp2f((w.m[cb] - x) * c) : 1.0f;
      w.m[cb] = raised ? x : w.m[cb];
      w.l[cb] *= f;
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) w.o[db][cb][r] *= f;
    }
  }

  // weights, their sums, and the operand of the second product
#pragma unroll
  for (int cb = 0; cb < C::CB; ++cb) {
    const float shift = w.m[cb] == neg_inf() ? 0.0f : -w.m[cb] * c;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * kc + e / 4][cb][e % 4], c, shift));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * kc + e / 4][cb][e % 4 + 1], c, shift));
        w.l[cb] += p0;
        w.l[cb] += p1;
        const bf16x2 pk = __builtin_convertvector(f32x2{p0, p1}, bf16x2);
        pf[kc][cb][e] = pk[0];
        pf[kc][cb][e + 1] = pk[1];
      }
  }

}

// O^T += V^T P^T of the tile in buffer `at`.
template <class C>
__device__ __forceinline__ void product(const Tiles<C>& t, Rows<C>& w, const Weights<C>& pf, int at) {
  constexpr int ND = C::DT / 16, N = C::KT / 32 * ND, AHEAD = C::AHEAD, RING = AHEAD + 1;
  typename Tiles<C>::Raw a[RING];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) a[i] = t.v_frag(at, i / ND, i % ND);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int n = i + AHEAD;
    if (n < N) a[n % RING] = t.v_frag(at, n / ND, n % ND);
    const bf16x8 f = Tiles<C>::operand(a[i % RING]);
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb)
      w.o[i % ND][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[i / ND][cb], w.o[i % ND][cb], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The infinite and NaN values of a masked tile, which its product left out, for the rows that see them.
template <class C>
__device__ __forceinline__ void add_infinities(const Tiles<C>& t, Rows<C>& w, int32_t j0) {
#pragma unroll 1
  for (int32_t j = j0; j < j0 + C::KT && j < t.kv_len; ++j) {
    const int64_t page = t.table[j >> t.p.page_shift];
    if (page < 0 || page >= t.p.num_pages) continue;
    const unsigned char* row =
        t.base_v + page * t.p.v.page + (j & ((1 << t.p.page_shift) - 1)) * static_cast<int64_t>(t.p.v.token);
#pragma unroll
    for (int db = 0; db < C::DT / 16; ++db) {
      const int d = 16 * db + 4 * (t.lane >> 4);
      if (d >= t.p.D) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v;
        if constexpr (C::FP8) v = (row[d + r] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
        else v = bf16_lo(reinterpret_cast<const uint16_t*>(row)[d + r]);
        if (__builtin_isfinite(v)) continue;
#pragma unroll
        for (int cb = 0; cb < C::CB; ++cb)
          if (j >= w.lo[cb] && j < w.hi[cb]) w.o[db][cb][r] += v;
      }
    }
  }
}

// x plus what another lane has (lanes without a source: plus 0).
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T add_from(T x) {
  return x + __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}
// Inclusive sums over the lanes.
template <class T>
__device__ __forceinline__ T lane_sums(T x) {
  x = add_from<0x111, 0xf>(x);  // 1, 2, 4, 8 lanes back in the row of 16
  x = add_from<0x112, 0xf>(x);
  x = add_from<0x114, 0xf>(x);
  x = add_from<0x118, 0xf>(x);
  x = add_from<0x142, 0xa>(x);     // the end of row 0 (2) into row 1 (3)
  return add_from<0x143, 0xc>(x);  // the end of row 1 into rows 2 and 3
}
template <class T>
__device__ __forceinline__ T last_lane(T x) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// A sequence as the kernels see it, whatever its arrays hold.
struct Sequence {
  int32_t q0, n, m;  // first token, new tokens, cached tokens
};
__device__ __forceinline__ Sequence sequence(const Params& p, int b) {
  const int32_t T = static_cast<int32_t>(p.T);
  int32_t q0 = p.q_start[b], q1 = p.q_start[b + 1], m = p.kv_len[b];
  q0 = q0 < 0 ? 0 : q0 > T ? T : q0;
  q1 = q1 < q0 ? q0 : q1 > T ? T : q1;
  const int64_t most = p.ld_table << p.page_shift;
  m = m < 0 ? 0 : m > most ? static_cast<int32_t>(most) : m;
  return Sequence{q0, q1 - q0, m};
}

// What a workgroup does: a row tile of a sequence and a part of its keys.
struct Item {
  int32_t b, tile, part, parts, per;  // per: key steps of a part
  Sequence s;
  int32_t first, end;                 // the first sequence's first token, the last one's end
};

// Deals the sequences' row tiles and parts to the p.items workgroups of a KV head. A part has `per` key steps, the
// same for all sequences, the least with which the parts are no more than the workgroups: workgroups take equally
// long whatever the sequences' lengths. Every wavefront finds the same from q_start and kv_len, a lane for a sequence.
// False: nothing left for workgroup `idx`; it.first and it.end are set all the same.
template <class C>
__device__ __forceinline__ bool schedule(const Params& p, int lane, int32_t idx, Item& it) {
  const int32_t G = static_cast<int32_t>(p.group.d);
  struct Need {
    int32_t tiles, steps;
  };
  Sequence mine{0, 0, 0};
  const auto need = [&](int base) {
    mine = base + lane < p.batch ? sequence(p, base + lane) : Sequence{0, 0, 0};
    int32_t keys = mine.m;
    if (p.window) {  // a row tile's rows see a window and the tokens that they span
      const int32_t span = (C::BM + G - 2) / G + 1, most = p.window < 0x7fffffff - span ? p.window + span : 0x7fffffff;
      keys = keys < most ? keys : most;
    }
    return Need{(mine.n * G + C::BM - 1) / C::BM, (keys + C::STEP - 1) / C::STEP + (p.window ? 1 : 0)};
  };
  const auto parts = [](const Need& x, int32_t per) { return x.steps > per ? (x.steps + per - 1) / per : 1; };
  Need x = need(0);
  it.first = __builtin_amdgcn_readlane(mine.q0, 0);
  it.end = 0;
  int32_t per = 0x7fffffff, count = 0;  // not split
  if (p.part_o) {
    float work = 0.0f;
    for (int base = 0; base < p.batch; base += 64) {
      if (base) x = need(base);
      work += last_lane(lane_sums(static_cast<float>(x.tiles) * static_cast<float>(x.steps)));
    }
    per = static_cast<int32_t>(work / static_cast<float>(p.items));
    per = per < p.min_part ? p.min_part : per;
    if (p.batch > 64) x = need(0);
  }
  while (true) {
    count = 0;
    for (int base = 0; base < p.batch; base += 64) {
      if (base) x = need(base);
      count += last_lane(lane_sums(x.tiles * parts(x, per)));
      const int32_t last = p.batch - 1 - base;
      it.end = __builtin_amdgcn_readlane(mine.q0 + mine.n, last < 63 ? last : 63);
    }
    if (p.batch > 64) x = need(0);
    // with one part each the tiles of any ascending q_start are no more than the workgroups
    if (count <= p.items || per >= 1 << 30) break;
    const int32_t more = per / 16;
    per += more < 1 ? 1 : more;
  }
  // later tiles, which see more keys where causal, come first
  int32_t left = count - 1 - idx;
  if (left < 0) return false;
  for (int base = 0; base < p.batch; base += 64) {
    if (base) x = need(base);
    const int32_t own = x.tiles * parts(x, per), upto = lane_sums(own);
    const uint64_t after = __builtin_amdgcn_ballot_w64(upto > left);
    if (after) {
      const int at = __builtin_ctzll(after);
      const auto of = [&](int32_t v) { return __builtin_amdgcn_readlane(v, at); };
      it.b = base + at;
      it.parts = of(parts(x, per));
      it.per = per;
      const int32_t in = left - (of(upto) - of(own));
      it.tile = in / it.parts;
      it.part = in - it.tile * it.parts;
      it.s = Sequence{of(mine.q0), of(mine.n), of(mine.m)};
      return true;
    }
    left -= last_lane(upto);
  }
  return false;  // not reached
}

// The tokens that no sequence has, before the first one's and behind the last one's (the padding of a batch whose T is
// fixed): zeros and a log-sum-exp of -infinity, as for a token that sees no key. The workgroups of a KV head take the
// tokens in turn. Nothing to do is the rule, and costs no load: `schedule` has q_start. Where keys are split the rows
// have no parts, which the joining reads for every row.
__device__ __forceinline__ void clear_rest(const Params& p, int head, int32_t idx, int32_t first, int32_t end) {
  if (end < first) end = first;
  const int64_t G = p.group.d, rest = first + p.T - end;
  for (int64_t i = idx; i < rest; i += p.items) {
    const int64_t t = i < first ? i : end + (i - first);
    uint16_t* row = p.out + t * p.ldo + head * G * p.D;
    for (int64_t e = 8 * threadIdx.x; e < G * p.D; e += 8 * blockDim.x)
      *reinterpret_cast<u32x4*>(row + e) = u32x4{0u, 0u, 0u, 0u};
    for (int64_t h = threadIdx.x; h < G; h += blockDim.x) {
      const int64_t r = t * p.n_q + head * G + h;
      if (p.lse) p.lse[r] = neg_inf();
      if (p.part_o) p.parts_of[r][0] = p.parts_of[r][1] = 0;
    }
  }
}

template <class C>
__global__ __launch_bounds__(64 * C::WAVES, C::OCC) void qkn_attn_kernel(const Params p) {
  __shared__ __align__(16) unsigned char lds[C::LDS];
  __shared__ int any_infinite;
  constexpr int ND = C::DT / 16, NS = C::DT / 32;
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);

  // consecutive workgroups take the KV heads in turn: on 8 XCDs a head's keys then stay in few L2s
  const uint32_t bid = blockIdx.x, idx = div(bid, p.kv_heads);
  const int head = static_cast<int>(bid - idx * p.kv_heads.d);
  Item it;
  const bool any_left = schedule<C>(p, lane, static_cast<int32_t>(idx), it);
  clear_rest(p, head, static_cast<int32_t>(idx), it.first, it.end);
  if (!any_left) return;
  const int b = it.b;
  const int32_t q0 = it.s.q0, n = it.s.n, m = it.s.m, G = static_cast<int32_t>(p.group.d), R = n * G;
  const int32_t row0 = it.tile * C::BM;

  // keys that the rows first .. last see
  const int32_t ahead = m - n;  // position of the first new token
  const auto range = [&](int32_t first, int32_t last) {
    Range x;
    x.lo = 0;
    x.hi = m;
    if (p.causal) {
      const int32_t end = ahead + static_cast<int32_t>(div(last, p.group)) + 1;
      x.hi = end < m ? end : m;
      const int32_t from = ahead + static_cast<int32_t>(div(first, p.group)) + 1;
      if (p.window && from > p.window) x.lo = from - p.window;
    }
    if (x.hi < 0) x.hi = 0;
    if (x.lo > x.hi) x.lo = x.hi;
    return x;
  };
  const int32_t row_end = row0 + C::BM < R ? row0 + C::BM : R;
  const Range all = range(row0, row_end - 1);
  // key steps of the row tile and of this part
  const int32_t step0 = all.lo / C::STEP, steps = all.hi > all.lo ? (all.hi + C::STEP - 1) / C::STEP - step0 : 0;
  const int32_t first = it.part * it.per;  // one part: 0
  const int32_t rest = steps - first, mine = rest < 0 ? 0 : it.part == it.parts - 1 || rest < it.per ? rest : it.per;
  const int32_t j_begin = (step0 + first) * C::STEP, count = mine * (C::STEP / C::KT);

  // rows of this wavefront
  const int32_t w0 = row0 + (C::SHARED ? wave * 16 * C::CB : 0);
  const int32_t w1 = w0 + 16 * C::CB < R ? w0 + 16 * C::CB : R;
  const bool busy = w0 < R;
  Rows<C> w;
  int32_t row[C::CB];
  int64_t at_t[C::CB];  // token
  int32_t at_h[C::CB];  // query head
#pragma unroll
  for (int cb = 0; cb < C::CB; ++cb) {
    row[cb] = w0 + 16 * cb + (lane & 15);
    const bool live = row[cb] < R;
    const int32_t r = live ? row[cb] : R - 1;
    const int32_t tok = static_cast<int32_t>(div(r, p.group));
    at_t[cb] = q0 + tok;
    at_h[cb] = head * G + r - tok * G;
    const Range x = range(r, r);
    w.lo[cb] = x.lo;
    w.hi[cb] = x.hi;
    w.m[cb] = neg_inf();
    w.l[cb] = 0.0f;
    const uint16_t* src = p.q + at_t[cb] * p.ldq + static_cast<int64_t>(at_h[cb]) * p.D;
#pragma unroll
    for (int step = 0; step < NS; ++step) {
      // the elements that K's operand has there (request_k)
      const int d = !C::SHARED && C::FP8 ? 64 * (step / 2) + 16 * (lane >> 4) + 8 * (step % 2) : 32 * step + 8 * (lane >> 4);
      u32x4 u = {0u, 0u, 0u, 0u};
      if (d < p.D) u = *reinterpret_cast<const u32x4*>(src + d);
      w.q[step][cb] = __builtin_bit_cast(bf16x8, u);
    }
#pragma unroll
    for (int db = 0; db < ND; ++db) w.o[db][cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // every row of the wavefront (workgroup) sees the keys full.lo .. full.hi - 1 (inner); some row those of any
  const int32_t wf = busy ? w0 : R - 1, wl = busy ? w1 - 1 : R - 1;
  const Range full{range(wl, wl).lo, range(wf, wf).hi}, any = range(wf, wl);
  const Range inner{range(row_end - 1, row_end - 1).lo, range(row0, row0).hi};

  const float k_scale = p.k.scale ? p.k.scale[head] : 1.0f, v_scale = p.v.scale ? p.v.scale[head] : 1.0f;
  const float c = p.c * k_scale;
  const auto in_part = [&](int32_t j0) { return j0 < inner.lo || j0 + C::KT > inner.hi; };
  u32x4 kr[C::KT / 16][C::KL];
  Scores<C> sc;
  Weights<C> pf;
  const auto sees = [&](int32_t j0) { return !C::SHARED || (busy && j0 < any.hi && j0 + C::KT > any.lo); };
  const auto masked = [&](int32_t j0) { return j0 < full.lo || j0 + C::KT > full.hi; };

  if (threadIdx.x == 0) any_infinite = 0;
  __syncthreads();
  if (count > 0) {
    Tiles<C> t(p, lds + (C::SHARED ? 0 : wave * 2 * C::BUF), lane, wave);
    t.open(b, head, m, j_begin);
    if constexpr (C::SHARED) {
      t.template request<false>(j_begin, 0);
      t.template request<true>(j_begin, 0);
      for (int32_t i = 0; i < count; ++i) {
        const int32_t j0 = j_begin + i * C::KT;
        wait_loads<0>();   // this wavefront's rows of tile i are there,
        if (in_part(j0) && t.make_finite(i & 1)) any_infinite = 1;
        group_barrier();   // every wavefront's are, and all have read tile i - 1
        if (i + 1 < count) {
          t.template request<false>(j0 + C::KT, (i + 1) & 1);
          t.template request<true>(j0 + C::KT, (i + 1) & 1);
        }
        if (sees(j0)) {
          scores(t, w, kr, i & 1, sc);
          softmax(w, sc, pf, lane, j0, c, masked(j0));
          product(t, w, pf, i & 1);
        }
      }
    } else {
      if (wave < count) {
        t.template request<true>(j_begin + wave * C::KT, 0);
        t.request_k(j_begin + wave * C::KT, kr);
      }
      int at = 0;
      for (int32_t i = wave; i < count; i += C::WAVES, at ^= 1) {
        const int32_t j0 = j_begin + i * C::KT, j1 = j0 + C::WAVES * C::KT;
        const bool more = i + C::WAVES < count;
        if (more) {
          t.template request<true>(j1, at ^ 1);
          wait_loads<C::V_LOADS>();  // all but those: this tile's
        } else {
          wait_loads<0>();
        }
        if (in_part(j0) && t.make_finite(at)) any_infinite = 1;
        scores(t, w, kr, at, sc);
        if (more) t.request_k(j1, kr);  // the registers are free
        softmax(w, sc, pf, lane, j0, c, masked(j0));
        product(t, w, pf, at);
        asm volatile("" ::: "memory");  // the next request writes where this tile was read
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
    if (any_infinite) {
      for (int32_t i = C::SHARED ? 0 : wave; i < count; i += C::SHARED ? 1 : C::WAVES)
        if (in_part(j_begin + i * C::KT)) add_infinities(t, w, j_begin + i * C::KT);
    }
  }

  // a row's sum over the lanes that share it
#pragma unroll
  for (int cb = 0; cb < C::CB; ++cb) {
    w.l[cb] += __shfl_xor(w.l[cb], 16);
    w.l[cb] += __shfl_xor(w.l[cb], 32);
  }
  const bool whole = it.parts == 1;
  const auto put = [&](int32_t i, int64_t tok, int32_t h, int d, f32x4 o, float bound, float sum, bool first_lane) {
    // row i of the tile; bound in log2 units; o, sum relative to it
    const int64_t r = tok * p.n_q + h;
    if (first_lane && p.part_o && it.part == 0) {  // the next part is p.n_kv workgroups before this one
      p.parts_of[r][0] = static_cast<int32_t>(bid);
      p.parts_of[r][1] = it.parts * 256 + i;
    }
    if (whole) {
      const float f = sum == 0.0f ? 0.0f : v_scale / sum;
      if (d < p.D) {
        const u32x2 u = {pack_bf16x2(o[0] * f, o[1] * f), pack_bf16x2(o[2] * f, o[3] * f)};
        *reinterpret_cast<u32x2*>(p.out + tok * p.ldo + static_cast<int64_t>(h) * p.D + d) = u;
      }
      if (first_lane && p.lse) p.lse[r] = sum == 0.0f ? neg_inf() : (bound + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
      const int64_t at = static_cast<int64_t>(bid) * C::BM + i;
      if (d < p.D && sum != 0.0f) {
        const f32x4 x = {o[0] * v_scale, o[1] * v_scale, o[2] * v_scale, o[3] * v_scale};
        *reinterpret_cast<f32x4*>(p.part_o + at * p.D + d) = x;
      }
      if (first_lane) p.part_ml[at] = f32x2{bound, sum};
    }
  };
  if constexpr (C::SHARED) {
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb)
      if (row[cb] < R)
#pragma unroll
        for (int db = 0; db < ND; ++db)
          put(row[cb] - row0, at_t[cb], at_h[cb], 16 * db + 4 * (lane >> 4), w.o[db][cb], w.m[cb] * c, w.l[cb], db == 0 && lane < 16);
  } else {
    // join the wavefronts, in ascending order: rows of (DT + 4) floats, then bounds, then sums
    float* rows = reinterpret_cast<float*>(lds);
    float* bounds = rows + C::WAVES * 16 * C::CB * C::JOIN_ROW;
    float* sums = bounds + C::WAVES * 16 * C::CB;
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < C::CB; ++cb) {
      const int i = (wave * C::CB + cb) * 16 + (lane & 15);
      if (lane < 16) {
        bounds[i] = w.m[cb] * c;
        sums[i] = w.l[cb];
      }
#pragma unroll
      for (int db = 0; db < ND; ++db)
        *reinterpret_cast<f32x4*>(rows + i * C::JOIN_ROW + 16 * db + 4 * (lane >> 4)) = w.o[db][cb];
    }
    __syncthreads();
    constexpr int kVecs = C::DT / 4, kAll = 16 * C::CB * kVecs, kThreads = 64 * C::WAVES;
    for (int u = static_cast<int>(threadIdx.x); u < kAll; u += kThreads) {
      const int i = u / kVecs, d = (u % kVecs) * 4;
      const int32_t r = row0 + i;
      if (r >= R) break;
      float top = neg_inf();
#pragma unroll
      for (int x = 0; x < C::WAVES; ++x) top = fmaxf(top, bounds[x * 16 * C::CB + i]);
      float sum = 0.0f;
      f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int x = 0; x < C::WAVES; ++x) {
        const float f = __builtin_amdgcn_exp2f(bounds[x * 16 * C::CB + i] - (top == neg_inf() ? 0.0f : top));
        sum += f * sums[x * 16 * C::CB + i];
        const f32x4 v = *reinterpret_cast<const f32x4*>(rows + (x * 16 * C::CB + i) * C::JOIN_ROW + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f * v[e];
      }
      const int32_t tok = static_cast<int32_t>(div(r, p.group));
      put(i, q0 + tok, head * G + r - tok * G, d, o, top, sum, d == 0);
    }
  }
}

template <class C>
Variant variant(const char* name) {
  return Variant{reinterpret_cast<const void*>(&qkn_attn_kernel<C>), C::BM, C::STEP, 64 * C::WAVES, C::LDS, C::SLOTS, name};
}

// A kernel for sequences of up to `rows` rows, and one for more. dt: 64, 128 or 256.
__attribute__((visibility("hidden"))) Variant few_rows(int dt, bool fp8, int rows);
__attribute__((visibility("hidden"))) Variant many_rows(int dt, bool fp8, bool small);

}  // namespace attn

#endif  // QKN_ATTN_KERNELS_H
