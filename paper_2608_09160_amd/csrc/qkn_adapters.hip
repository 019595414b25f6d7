// libqkn, part 5: low-rank adapters of many requests beside the shared projection (AMD MI355X, gfx950).
//
// Two launches. The first takes u = A_i x for every token into the workspace (fp32, in `ks` parts of hidden); the
// second adds the parts, multiplies by B_i, adds base, rounds, and takes the statistic of the whole row.
//
// Both products run on the matrix cores (v_mfma_f32_16x16x32_bf16: A 16 x 32, B 32 x 16, lane l holds row (column)
// l mod 16, k 8 (l / 16) .. + 7; result column l mod 16, rows 4 (l / 16) .. + 3). A product's rows belong to one adapter:
// tokens are listed by adapter first, x is read through the list. Bytes bound both launches (x, base and y, and in
// decode the adapters): 64 tokens of 32 adapters of rank 16 (hidden 4096, 1024 + 256 columns, 10.6 MB) 11.8 us; 8192
// tokens in runs of 8 adapters of rank 64 (2048 + 512 columns, 162 MB) 90 us, 43 of them the first launch, whose LDS
// receives 201 MB, x once and A's rows once for 64 tokens, and which writes 34 MB of A x in 8 parts of hidden; the second
// reads those, base and, once for 16 tokens, B: 300 MB with what the caches give twice, by its counters.
// Above 512 tokens a product's tokens are of 64 consecutive ones, whose adapters take turns: made for prompts in runs. Ids
// that change from token to token cost more there (hidden 4096, 1024 + 256 columns, rank 16, us in runs and mixed: 512
// tokens of 64 adapters 23.6 and 22.7, 1024 of 8 16.4 and 31.0, of 64 27.7 and 106, 4096 of 64 27.2 and 137).

#include <string.h>

#include "qkn_adapters.h"
#include "qkn_block.h"

namespace {

using namespace qkn_block;
using qkn_host::Span;
using qkn_host::spans_overlap;

constexpr int kWavesB = 8;      // wavefronts of a workgroup of the second launch
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef __attribute__((address_space(3))) unsigned char LdsByte;

constexpr int kList = 64;        // tokens of a product
constexpr int kGather = 512;     // calls of up to so many tokens look for an adapter's tokens in all of them
constexpr int kMaxRank = 128;
constexpr int kParts = 3;        // bf16 values that hold an fp32 one

struct SegDev {
  const uint16_t* a;
  const uint16_t* b;
  const uint16_t* base;
  uint16_t* y;
  float* partials;
  int64_t a_adapter, lda, b_adapter, ldb, ldbase, ldy;
  int32_t d;
};

struct Params {
  const uint16_t* x;
  int64_t ldx;
  const int32_t* ids;
  const float* scale;
  float* u;               // [ks, T, n]: seg s's row j of A at column s * rank + j
  int32_t T, hidden, count, rank, n, kper, nt;
  FastDiv ks, by_rank;
  SegDev seg[3];
};

__device__ __forceinline__ Rsrc rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0), static_cast<int>(bytes),
                                           0x00020000);
}
// Lane l's 16 bytes at byte `off` of the buffer go to dst + 16 l.
__device__ __forceinline__ void load_to_lds(Rsrc r, unsigned char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsByte*)dst, 16, off, 0, 0, 0);
}
// Until at most n (0 to 6) loads of this wavefront are on their way.
__device__ __forceinline__ void wait_loads(int n) {
  switch (n) {
    case 1: __builtin_amdgcn_s_waitcnt(0x0F71); break;
    case 2: __builtin_amdgcn_s_waitcnt(0x0F72); break;
    case 3: __builtin_amdgcn_s_waitcnt(0x0F73); break;
    case 4: __builtin_amdgcn_s_waitcnt(0x0F74); break;
    case 5: __builtin_amdgcn_s_waitcnt(0x0F75); break;
    case 6: __builtin_amdgcn_s_waitcnt(0x0F76); break;
    default: __builtin_amdgcn_s_waitcnt(0x0F70); break;
  }
}

__device__ __forceinline__ bool has_adapter(const Params& p, int32_t id) { return id >= 0 && id < p.count; }

__device__ __forceinline__ SegDev pick_seg(const Params& p, int i) {
  SegDev s = p.seg[0];
  if (i == 1) s = p.seg[1];
  if (i == 2) s = p.seg[2];
  return s;
}

// Tiles of the first launch: ROWS tokens (16 or 64) x 16 NBT columns, 64 of hidden a stage. Both operands' rows go
// straight into LDS (buffer_load ... lds: whole 128-byte lines of 8 rows an instruction; fetched as operands, 64 bytes of
// 16 rows at a time, 64 tokens x 128 columns took 60 against 43 us), three stages, two on their way during the products of one. Chunk c of
// row r is stored at c ^ (r / 2 mod 8): 16 rows' chunks are then on different banks.
template <int NBT>
struct StageA {
  static constexpr int kRowBytes = 128;
  static constexpr int kX = kList * kRowBytes, kBytes = kX + 16 * NBT * kRowBytes, kStages = 3;
  static constexpr int kAcross = NBT < 4 ? NBT : 4;  // wavefronts over the columns
  static constexpr int NB = NBT / kAcross;           // a wavefront's blocks of 16 columns
};

// u[slice, token, col0 ..] for the n <= ROWS tokens of `list`, which have the same adapter; rows of x from `x` on.
template <int ROWS, int NBT>
__device__ __forceinline__ void product_a(const Params& p, const uint16_t* x, const int32_t* list, int n, int32_t t0,
                                          int64_t adapter, int slice, int col0, unsigned char* lds) {
  using C = StageA<NBT>;
  constexpr int kDown = ROWS == 16 ? 1 : 4 / C::kAcross, MB = ROWS / 16 / kDown, NB = C::NB;
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int g = lane >> 4, i16 = lane & 15;
  const int k0 = slice * p.kper, k1 = k0 + p.kper < p.hidden ? k0 + p.kper : p.hidden;
  const int stages = (k1 - k0 + 63) / 64;
  const bool works = wave < C::kAcross * kDown;
  const int across = wave % C::kAcross, down = works ? wave / C::kAcross : 0;

  // loads of this wavefront: 8 rows each, of x, then of A; the same ones every stage
  constexpr int kLoadsX = (ROWS / 8 + kWaves - 1) / kWaves, kLoadsA = (2 * NBT + kWaves - 1) / kWaves;
  const int r8 = lane >> 3;
  uint32_t off_x[kLoadsX], off_a[kLoadsA];
  Rsrc rs_a[kLoadsA];
  int loads = 0;
  const Rsrc rs_x = rsrc(x, 0x7ffffff0u);  // rows of the list: offsets below 2^31 (checked on the host)
#pragma unroll
  for (int i = 0; i < kLoadsX; ++i) {
    const int row = 8 * (wave + kWaves * i) + r8;
    off_x[i] = static_cast<uint32_t>((list[row < n ? row : n - 1] - t0) * p.ldx * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
    loads += wave + kWaves * i < ROWS / 8;
  }
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) {
    const int c8 = col0 + 8 * (wave + kWaves * i), row = 8 * (wave + kWaves * i) + r8;  // rank is a multiple of 8
    const int sg = static_cast<int>(div(static_cast<uint32_t>(c8 < p.n ? c8 : 0), p.by_rank));
    const uint16_t* a = sg == 0 ? p.seg[0].a : sg == 1 ? p.seg[1].a : p.seg[2].a;
    const int64_t per = sg == 0 ? p.seg[0].a_adapter : sg == 1 ? p.seg[1].a_adapter : p.seg[2].a_adapter;
    const int64_t ld = sg == 0 ? p.seg[0].lda : sg == 1 ? p.seg[1].lda : p.seg[2].lda;
    rs_a[i] = rsrc(a + adapter * per + (c8 - sg * p.rank) * ld, __builtin_amdgcn_readfirstlane(c8 < p.n ? 0x7ffffff0 : 0));
    off_a[i] = static_cast<uint32_t>(r8 * ld * 2) + 16 * ((lane & 7) ^ ((row >> 1) & 7));
    loads += wave + kWaves * i < 2 * NBT;
  }
  const auto request = [&](int s) {
    unsigned char* buf = lds + s % C::kStages * C::kBytes;
    const uint32_t k = static_cast<uint32_t>(k0 + 64 * s);
#pragma unroll
    for (int i = 0; i < kLoadsX; ++i) {
      const int at = wave + kWaves * i, row = 8 * at + r8, c = (lane & 7) ^ ((row >> 1) & 7);
      if (at < ROWS / 8) load_to_lds(rs_x, buf + at * 1024, static_cast<int>(k) + 8 * c < k1 ? off_x[i] + 2 * k : 0x7fffffffu);
    }
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) {
      const int at = wave + kWaves * i, row = 8 * at + r8, c = (lane & 7) ^ ((row >> 1) & 7);
      if (at < 2 * NBT)
        load_to_lds(rs_a[i], buf + C::kX + at * 1024, static_cast<int>(k) + 8 * c < k1 ? off_a[i] + 2 * k : 0x7fffffffu);
    }
  };

  f32x4 acc[MB][NB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < C::kStages - 1 && s < stages; ++s) request(s);
  for (int s = 0; s < stages; ++s) {
    wait_loads(s + 1 < stages ? loads : 0);  // all but the next stage's
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // everyone's are there, and everyone has read the stage before
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (s + C::kStages - 1 < stages) request(s + C::kStages - 1);
    const unsigned char* buf = lds + s % C::kStages * C::kBytes;
    if (works) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 xf[MB], af[NB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const int row = 16 * (down * MB + mb) + i16;
          xf[mb] = *reinterpret_cast<const bf16x8*>(buf + row * C::kRowBytes + 16 * ((4 * h + g) ^ ((row >> 1) & 7)));
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int row = 16 * (across * NB + nb) + i16;
          af[nb] = *reinterpret_cast<const bf16x8*>(buf + C::kX + row * C::kRowBytes + 16 * ((4 * h + g) ^ ((row >> 1) & 7)));
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            acc[mb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[mb], af[nb], acc[mb][nb], 0, 0, 0);
      }
    }
  }
  if (works) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * (down * MB + mb) + 4 * g + r;
        if (i >= n) continue;
        float* dst = p.u + (static_cast<int64_t>(slice) * p.T + list[i]) * p.n + col0;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int c = 16 * (across * NB + nb) + i16;
          if (col0 + c < p.n) dst[c] = acc[mb][nb][r];
        }
      }
  }
}
template <int NBT>
__device__ __forceinline__ void product_a(const Params& p, const int32_t* list, int n, int32_t t0, int64_t adapter,
                                          int slice, int col0, unsigned char* lds) {
  const uint16_t* x = p.x + t0 * p.ldx;
  if (n <= 16) product_a<16, NBT>(p, x, list, n, t0, adapter, slice, col0, lds);
  else product_a<kList, NBT>(p, x, list, n, t0, adapter, slice, col0, lds);
}

// GATHER (few tokens): a workgroup for every token, which goes on if it is the first, 65th, ... of its adapter and
// takes the adapter's tokens from there on: each adapter is read once for 64 of its tokens, wherever they are. Else:
// a workgroup for every 64 consecutive tokens, their adapters in turn (in a prompt they are mostly one).
template <int NBT, bool GATHER>
__global__ __launch_bounds__(kThreads) void qkn_adapters_a(const Params p) {
  __shared__ __align__(16) unsigned char lds[StageA<NBT>::kStages * StageA<NBT>::kBytes];
  __shared__ int32_t list[kList];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const bool first_wave = threadIdx.x < 64;
  const int item = static_cast<int>(div(blockIdx.x, p.ks));
  const int slice = static_cast<int>(blockIdx.x - item * p.ks.d);
  const int col0 = static_cast<int>(blockIdx.y) * 16 * NBT;
  const uint64_t below = (uint64_t{1} << lane) - 1;
  if constexpr (GATHER) {
    const int32_t id = p.ids[item];
    if (!has_adapter(p, id)) return;
    int before = 0, n = 0;
    int32_t v[kGather / 64];
#pragma unroll
    for (int c = 0; c < kGather / 64; ++c) v[c] = 64 * c + lane < p.T ? p.ids[64 * c + lane] : -1;
#pragma unroll
    for (int c = 0; c < kGather / 64; ++c) {
      const uint64_t same = __builtin_amdgcn_ballot_w64(v[c] == id);
      const uint64_t earlier = __builtin_amdgcn_ballot_w64(64 * c + lane < item);
      before += __builtin_popcountll(same & earlier);
      const uint64_t later = same & ~earlier;
      const int at = n + __builtin_popcountll(later & below);
      if (first_wave && ((later >> lane) & 1) && at < kList) list[at] = 64 * c + lane;
      n += __builtin_popcountll(later);
    }
    if (before % kList) return;
    __syncthreads();
    product_a<NBT>(p, list, n < kList ? n : kList, 0, id, slice, col0, lds);
  } else {
    const int32_t t = item * kList + lane;
    const int32_t id = t < p.T ? p.ids[t] : -1;
    uint64_t left = __builtin_amdgcn_ballot_w64(has_adapter(p, id));
    while (left) {
      const int32_t cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
      const uint64_t same = __builtin_amdgcn_ballot_w64(id == cur);
      left &= ~same;
      if (first_wave && ((same >> lane) & 1)) list[__builtin_popcountll(same & below)] = t;
      __syncthreads();
      product_a<NBT>(p, list, __builtin_popcountll(same), item * kList, cur, slice, col0, lds);
      __syncthreads();
    }
  }
}

// The rows of p.nt tokens and one segment; RS: steps of 32 over the rank. The 24 bits of scale u are kept as three bf16
// parts in LDS, and B's values meet each of them: the product is of the fp32 value. (Two parts, 16 bits, left the
// rows' statistic with 3 times the error of fp32 sums, from stored values that round the other way.) Transposed,
// Y^T = B U^T: a lane has one token, and rows of B are dealt to the product's so that two of its blocks leave each
// lane 8 consecutive elements, and four lanes a row's 32. 16 tokens and eight wavefronts (both launches of 8192 tokens: 89.8
// us; 32 tokens 89.3, four wavefronts 97.3, sixteen 93.4): B comes from the caches, 16 tokens' base and y from memory.
template <int WAVES, int RS>
__global__ __launch_bounds__(64 * WAVES) void qkn_adapters_b(const Params p) {
  // rows of 16 bytes more than 64 RS, a multiple of all banks' width from RS 4 on: conflicts are left (4.5e5 of 1.1e6 cycles
  // of LDS reads at 8192 tokens of rank 64), about 2 % of the launch
  constexpr int MT = 1, kTok = 16 * MT, kRow = 32 * RS + 8;
  __shared__ __align__(16) uint16_t parts[kParts][kTok][kRow];
  __shared__ float sums[WAVES][kTok];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, i16 = lane & 15;
  const int seg = static_cast<int>(blockIdx.y);
  const SegDev s = pick_seg(p, seg);
  const int32_t t0 = static_cast<int32_t>(blockIdx.x) * p.nt;
  const int32_t n = p.T - t0 < p.nt ? p.T - t0 : p.nt;

  for (int e = tid; e < kTok * 32 * RS; e += 64 * WAVES) {
    const int i = e / (32 * RS), j = e % (32 * RS);
    float v = 0.0f;
    if (i < n && j < p.rank) {
      const int32_t id = p.ids[t0 + i];
      if (has_adapter(p, id)) {
        const float* src = p.u + static_cast<int64_t>(t0 + i) * p.n + seg * p.rank + j;
        const int64_t part = static_cast<int64_t>(p.T) * p.n;
        const int ks = static_cast<int>(p.ks.d);
        for (int k0 = 0; k0 < ks; k0 += 8) {  // eight at a time on their way
          float w[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) w[k] = src[(k0 + k < ks ? k0 + k : ks - 1) * part];
#pragma unroll
          for (int k = 0; k < 8; ++k) v += k0 + k < ks ? w[k] : 0.0f;
        }
        if (p.scale) v *= p.scale[id];
      }
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const uint32_t part = pack_bf16x2(v, 0.0f) & 0xffffu;
      parts[k][i][j] = static_cast<uint16_t>(part);
      v -= bf16_lo(part);
      if (!__builtin_isfinite(v)) v = 0.0f;  // an infinity or NaN has no rest
    }
  }
  __syncthreads();

  // ids of the tile: lane i has token i's; this lane's tokens' own
  int32_t id_of = -1, own[MT];
  if (lane < n) id_of = p.ids[t0 + lane];
  const uint64_t adapted = __builtin_amdgcn_ballot_w64(lane < kTok && has_adapter(p, id_of));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) own[mt] = __shfl(id_of, 16 * mt + i16);

  float sum[MT] = {};
  for (int d0 = 64 * wave; d0 < s.d; d0 += 64 * WAVES) {
    // base first: its loads are in flight during the products
    u32x4 base[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int d = d0 + 32 * h + 8 * g;
        base[mt][h] = u32x4{0u, 0u, 0u, 0u};
        if (16 * mt + i16 < n && d < s.d)
          base[mt][h] = *reinterpret_cast<const u32x4*>(s.base + (t0 + 16 * mt + i16) * s.ldbase + d);
      }
    f32x4 y[4][MT];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) y[b][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    uint64_t left = adapted;
    while (left) {
      const int32_t cur = __builtin_amdgcn_readlane(id_of, __builtin_ctzll(left));
      left &= ~__builtin_amdgcn_ballot_w64(id_of == cur);
      const uint16_t* mat = s.b + cur * s.b_adapter;
      bf16x8 bf[RS][4];
#pragma unroll
      for (int k = 0; k < RS; ++k)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int d = d0 + 32 * (b >> 1) + 8 * (i16 >> 2) + 4 * (b & 1) + (i16 & 3), c = 32 * k + 8 * g;
          u32x4 v = {0u, 0u, 0u, 0u};
          if (d < s.d && c < p.rank) v = *reinterpret_cast<const u32x4*>(mat + d * s.ldb + c);
          bf[k][b] = __builtin_bit_cast(bf16x8, v);
        }
      f32x4 part[4][MT];
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) part[b][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < RS; ++k)
#pragma unroll
        for (int q = kParts - 1; q >= 0; --q)  // the smallest first
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const bf16x8 uf =
                __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&parts[q][16 * mt + i16][32 * k + 8 * g]));
#pragma unroll
            for (int b = 0; b < 4; ++b)
              part[b][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[k][b], uf, part[b][mt], 0, 0, 0);
          }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        if (own[mt] == cur) {
#pragma unroll
          for (int b = 0; b < 4; ++b) y[b][mt] = part[b][mt];
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int d = d0 + 32 * h + 8 * g;
        u32x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4& v = y[2 * h + e / 2][mt];
          out[e] = pack_bf16x2(bf16_lo(base[mt][h][e]) + v[2 * (e % 2)], bf16_hi(base[mt][h][e]) + v[2 * (e % 2) + 1]);
          // a row without an adapter as it is: + 0 would turn -0 into 0 and change a NaN's bits
          if (!has_adapter(p, own[mt])) out[e] = base[mt][h][e];
        }
        if (16 * mt + i16 < n && d < s.d) {
          *reinterpret_cast<u32x4*>(s.y + (t0 + 16 * mt + i16) * s.ldy + d) = out;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float lo = bf16_lo(out[e]), hi = bf16_hi(out[e]);
            sum[mt] = __builtin_fmaf(lo, lo, sum[mt]);
            sum[mt] = __builtin_fmaf(hi, hi, sum[mt]);
          }
        }
      }
  }
  if (!s.partials) return;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    sum[mt] += __shfl_xor(sum[mt], 16);
    sum[mt] += __shfl_xor(sum[mt], 32);
    if (lane < 16) sums[wave][16 * mt + lane] = sum[mt];
  }
  __syncthreads();
  if (tid < n) {
    float all = sums[0][tid];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all += sums[w][tid];
    s.partials[t0 + tid] = all;
  }
}

// How hidden is cut: `ks` parts of `kper`.
struct Plan {
  int64_t tiles, ks, kper;
  bool gather;
};

Plan plan_of(int64_t T, int64_t hidden) {
  Plan pl{};
  pl.gather = T <= kGather;
  pl.tiles = pl.gather ? T : (T + kList - 1) / kList;
  // few tokens: about 2048 workgroups, most of which find that they are not their adapter's first (hidden 4096, 1024 + 256
  // columns, us with 1024, 2048 and 4096: 64 tokens 11.8, 12.5 and 11.7; 128 of rank 64 21.4, 24.7 and 24.7; 256 20.9, 18.2 and
  // 19.8; 512 of rank 64 59.4, 45.8 and 48.5); else about four a CU (8192 tokens, rank 64: 43 us, 47 with two, 83 with one)
  int64_t ks = pl.gather ? 2048 / (T < 1 ? 1 : T) : 4 * kCus / pl.tiles;
  const int64_t most = (hidden + 255) / 256 < 16 ? (hidden + 255) / 256 : 16;
  if (ks > most) ks = most;
  if (ks < 1) ks = 1;
  pl.kper = ((hidden + ks - 1) / ks + 63) / 64 * 64;
  pl.ks = (hidden + pl.kper - 1) / pl.kper;
  return pl;
}

bool sizes_ok(int64_t T, int64_t hidden, int rank, int nseg) {
  return T >= 0 && hidden >= 1 && rank >= 1 && nseg >= 1 && nseg <= 3;
}

template <int WAVES>
const void* kernel_b(int rank) {
  return rank <= 32 ? reinterpret_cast<const void*>(qkn_adapters_b<WAVES, 1>)
         : rank <= 64 ? reinterpret_cast<const void*>(qkn_adapters_b<WAVES, 2>)
                      : reinterpret_cast<const void*>(qkn_adapters_b<WAVES, 4>);
}

template <int NBT>
const void* kernel_a(bool gather) {
  return gather ? reinterpret_cast<const void*>(qkn_adapters_a<NBT, true>)
                : reinterpret_cast<const void*>(qkn_adapters_a<NBT, false>);
}
template <int NBT>
int lds_a() {
  return StageA<NBT>::kStages * StageA<NBT>::kBytes + kList * 4;
}

int adapters_impl(const uint16_t* x, int64_t ldx, int64_t T, int64_t hidden, const qkn_adapter_seg* segs, int nseg,
                  int rank, int64_t count, const int32_t* ids, const float* scale, void* workspace,
                  int64_t workspace_bytes, void* stream) {
  if (!segs || !sizes_ok(T, hidden, rank, nseg) || count < 0 || ldx < hidden) return QKN_EINVAL;
  for (int i = 0; i < nseg; ++i) {
    const qkn_adapter_seg& s = segs[i];
    if (s.d_local < 1 || s.ldbase < s.d_local || s.ldy < s.d_local || s.lda < hidden || s.ldb < rank ||
        s.a_adapter < 0 || s.b_adapter < 0)
      return QKN_EINVAL;
  }
  if (T == 0) return QKN_OK;
  if (!x || !ids) return QKN_EINVAL;
  const int64_t lim = int64_t{1} << 30;
  bool fits = aligned(x, 16) && ldx % 8 == 0 && hidden % 8 == 0 && rank % 8 == 0 && rank <= kMaxRank &&
              T <= (int64_t{1} << 24) && hidden <= lim && count <= (int64_t{1} << 24) && kGather * ldx * 2 < 2 * lim - 16;
  for (int i = 0; i < nseg; ++i) {
    const qkn_adapter_seg& s = segs[i];
    if (!s.base || !s.y || (count && (!s.a || !s.b))) return QKN_EINVAL;
    fits = fits && s.d_local % 8 == 0 && s.d_local <= lim && s.ldbase % 8 == 0 && s.ldy % 8 == 0 && aligned(s.base, 16) &&
           aligned(s.y, 16);
    if (count)
      fits = fits && s.a_adapter % 8 == 0 && s.lda % 8 == 0 && s.b_adapter % 8 == 0 && s.ldb % 8 == 0 &&
             aligned(s.a, 16) && aligned(s.b, 16) && s.a_adapter <= lim * 256 && s.b_adapter <= lim * 256 &&
             s.ldb <= lim && 8 * s.lda * 2 < 2 * lim - 16;
  }
  if (!fits) return QKN_ENOTSUP;
  const int64_t need = qkn_adapters_workspace_bytes(T, hidden, rank, nseg);
  if (!workspace || workspace_bytes < need) return QKN_EINVAL;
  if (!aligned(workspace, 16)) return QKN_ENOTSUP;

  Span item[24];
  bool out[24];
  int n = 0;
  const auto add = [&](const Span& s, bool is_out) {
    item[n] = s;
    out[n++] = is_out;
  };
  const auto rows = [](const void* ptr, int64_t r, int64_t ld, int64_t width) {
    return Span{reinterpret_cast<uintptr_t>(ptr), r, ld, width, 2};
  };
  add(rows(x, T, ldx, hidden), false);
  add(array_span(ids, T, 4), false);
  add(array_span(scale, count, 4), false);
  add(array_span(workspace, need, 1), true);
  for (int i = 0; i < nseg; ++i) {
    const qkn_adapter_seg& s = segs[i];
    if (count) {
      const int64_t na = (count - 1) * s.a_adapter + (rank - 1) * s.lda + hidden;
      const int64_t nb = (count - 1) * s.b_adapter + (s.d_local - 1) * s.ldb + rank;
      add(array_span(s.a, na, 2), false);
      add(array_span(s.b, nb, 2), false);
    }
    if (!(s.base == s.y && s.ldbase == s.ldy)) add(rows(s.base, T, s.ldbase, s.d_local), false);
    add(rows(s.y, T, s.ldy, s.d_local), true);
    add(array_span(s.partials, T, 4), true);
  }
  for (int a = 0; a < n; ++a)
    for (int b = a + 1; b < n; ++b)
      if ((out[a] || out[b]) && spans_overlap(item[a], item[b])) return QKN_EOVERLAP;

  const Plan pl = plan_of(T, hidden);
  Params p;
  memset(&p, 0, sizeof(p));
  p.x = x;
  p.ldx = ldx;
  p.ids = ids;
  p.scale = scale;
  p.u = static_cast<float*>(workspace);
  p.T = static_cast<int32_t>(T);
  p.hidden = static_cast<int32_t>(hidden);
  p.count = static_cast<int32_t>(count);
  p.rank = rank;
  p.n = nseg * rank;
  p.kper = static_cast<int32_t>(pl.kper);
  p.ks = fast_div(static_cast<uint32_t>(pl.ks));
  p.by_rank = fast_div(static_cast<uint32_t>(rank));
  for (int i = 0; i < nseg; ++i) {
    const qkn_adapter_seg& s = segs[i];
    p.seg[i] = SegDev{s.a,  s.b,     s.base, s.y,      s.partials, s.a_adapter,
                      s.lda, s.b_adapter, s.ldb, s.ldbase, s.ldy,      static_cast<int32_t>(s.d_local)};
  }
  // tokens of a workgroup of the second launch, which reads B once for them all: one while workgroups are few (hidden
  // 4096, 2048 + 512 columns, both launches, us with 1 and with 4 tokens: 32 adapters of rank 16, 64 tokens 14.7 and 21.7,
  // 160 17.0 and 23.6, 256 17.6 and 24.3, 384 23.1 and 26.4; runs of 8 of rank 64, 256 31.9 and 37.3, 384 45.2 and 43.3, 512
  // 52.4 and 46.8, 768 53.3 and 36.5), then four, sixteen from where those are many (4 and 16 tokens: 768 36.5 and 37.6,
  // 1024 38.5 and 38.1, 1536 44.3 and 39.5, 4096 87.1 and 60.9)
  p.nt = T <= 256 ? 1 : T <= 1024 ? 4 : 16;
  const int nb = p.n <= 32 ? 2 : p.n <= 64 ? 4 : 8;
  const char* name = pl.gather ? "adapters<gather>" : "adapters<tiles>";
  const int lds = nb == 2 ? lds_a<2>() : nb == 4 ? lds_a<4>() : lds_a<8>();
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{name, 0, 0, 0, lds});
    return QKN_EDRYRUN;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  void* args[] = {&p};
  const int64_t grid = pl.tiles * pl.ks, cols = (p.n + 16 * nb - 1) / (16 * nb);
  if (count) {
    const void* fn = nb == 2 ? kernel_a<2>(pl.gather) : nb == 4 ? kernel_a<4>(pl.gather) : kernel_a<8>(pl.gather);
    if (hipLaunchKernel(fn, dim3(static_cast<unsigned>(grid), static_cast<unsigned>(cols)), dim3(kThreads), args, 0, st) !=
        hipSuccess)
      return QKN_EHIP;
  }
  const void* fb = kernel_b<kWavesB>(rank);
  const dim3 gb(static_cast<unsigned>((T + p.nt - 1) / p.nt), static_cast<unsigned>(nseg));
  if (hipLaunchKernel(fb, gb, dim3(64 * kWavesB), args, 0, st) != hipSuccess) return QKN_EHIP;
  qkn_host::record_launch(qkn_launch_info{name, grid * cols, kThreads, grid * cols * kWaves, lds});
  return QKN_OK;
}

}  // namespace

extern "C" {

int64_t qkn_adapters_workspace_bytes(int64_t T, int64_t hidden, int rank, int nseg) {
  if (!sizes_ok(T, hidden, rank, nseg)) return QKN_EINVAL;
  return T == 0 ? 0 : 4 * plan_of(T, hidden).ks * T * nseg * rank;
}

int qkn_adapters_add(const uint16_t* x, int64_t ldx, int64_t T, int64_t hidden, const qkn_adapter_seg* segs, int nseg,
                     int rank, int64_t count, const int32_t* ids, const float* scale, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  return adapters_impl(x, ldx, T, hidden, segs, nseg, rank, count, ids, scale, workspace, workspace_bytes, stream);
}

}  // extern "C"
