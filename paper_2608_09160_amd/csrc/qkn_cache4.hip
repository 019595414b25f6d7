// libqkn, part 5: rows of the 4-bit cache read back as bf16 (AMD MI355X, gfx950). The write is in qkn_rope.hip,
// attention in qkn_attn*.
//
// Bytes bound it: 17/32 of a byte in and 2 out for an element. A lane takes 8 elements, one word of codes, and stores
// one 16-byte vector; four lanes share an exponent. 8192 tokens of 4 + 4 heads of 128, 21 MB, 7.1 us, 64 tokens 2.7: a launch
// and two trips to memory, slot and codes. Four such units a lane were no faster (7.4 and 3.7 us).

#include <string.h>

#include "qkn_cache4.h"
#include "qkn_quant4.h"

namespace {

using namespace qkn_block;
using qkn_host::Span;
using qkn_host::spans_overlap;

constexpr int kThreads = 256;

struct LoadParams {
  Pool4 codes[2], exps[2];  // K's and V's
  uint16_t* y[2];
  int64_t ld[2];
  const int64_t* slots;
  int64_t T, n_slots;
  int32_t page_shift, page_mask;
  int32_t k_units;          // of a token
  FastDiv units, per_head;  // of a token, of a head
};

// VEC: words of codes and 16-byte stores; else bytes and single values.
template <bool VEC>
__global__ __launch_bounds__(kThreads) void qkn_cache4_rows(const LoadParams p) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x, t = div(i, p.units);
  if (t >= p.T) return;
  const int in_token = static_cast<int>(i - t * p.units.d);
  const int s = in_token >= p.k_units;  // K or V
  const int in_seg = in_token - (s ? p.k_units : 0);
  const int head = static_cast<int>(div(static_cast<uint32_t>(in_seg), p.per_head));
  const int c = 8 * (in_seg - head * static_cast<int>(p.per_head.d)), D = 8 * static_cast<int>(p.per_head.d);
  const int64_t slot = p.slots[t];
  uint32_t w = 0, e = 0;
  if (slot >= 0 && slot < p.n_slots) {
    const int64_t page = slot >> p.page_shift, row = slot & p.page_mask;
    const Pool4& codes = s ? p.codes[1] : p.codes[0];
    const Pool4& exps = s ? p.exps[1] : p.exps[0];
    const uint8_t* from = codes.base + page * codes.page + head * codes.head + row * codes.token + c / 2;
    e = exps.base[page * exps.page + head * exps.head + row * exps.token + c / 32];
    if constexpr (VEC) w = *reinterpret_cast<const uint32_t*>(from);
    else w = from[0] | from[1] << 8 | from[2] << 16 | static_cast<uint32_t>(from[3]) << 24;
  }
  u32x4 u = __builtin_bit_cast(u32x4, quant4::decode(w, e));
  if (e >= quant4::kNan) u = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
  uint16_t* y = (s ? p.y[1] : p.y[0]) + t * (s ? p.ld[1] : p.ld[0]) + static_cast<int64_t>(head) * D + c;
  if constexpr (VEC) {
    *reinterpret_cast<u32x4*>(y) = u;
  } else {
#pragma unroll
    for (int x = 0; x < 8; ++x) y[x] = static_cast<uint16_t>(u[x / 2] >> (16 * (x % 2)));
  }
}

}  // namespace

extern "C" int qkn_cache4_load(const qkn_cache4* cache, const int64_t* slots, int64_t T, uint16_t* k, int64_t ldk,
                               uint16_t* v, int64_t ldv, void* stream) {
  if (!cache || !cache4_ok(*cache) || T < 0 || (T && !k && !v)) return QKN_EINVAL;
  const qkn_cache4& c = *cache;
  const int64_t width = int64_t{c.n_kv} * c.head_dim, most = int64_t{1} << 30;
  if ((k && ldk < width) || (v && ldv < width)) return QKN_EINVAL;
  if (T == 0) return QKN_OK;
  if (!slots || (c.num_pages && ((k && (!c.k || !c.k_exp)) || (v && (!c.v || !c.v_exp))))) return QKN_EINVAL;
  const int64_t units = (k ? width / 8 : 0) + (v ? width / 8 : 0);
  if (width > most || T > most || T * units > (int64_t{1} << 31) - kThreads) return QKN_ENOTSUP;

  Span in[5], out[2];
  int n_in = 0, n_out = 0;
  in[n_in++] = array_span(slots, T, 8);
  for (int i = 0; i < 4; ++i)
    if (i % 2 ? v != nullptr : k != nullptr) in[n_in++] = pool4_span(c, i);
  if (k) out[n_out++] = Span{reinterpret_cast<uintptr_t>(k), T, ldk, width, 2};
  if (v) out[n_out++] = Span{reinterpret_cast<uintptr_t>(v), T, ldv, width, 2};
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (spans_overlap(out[i], in[j])) return QKN_EOVERLAP;
    for (int j = 0; j < i; ++j)
      if (spans_overlap(out[i], out[j])) return QKN_EOVERLAP;
  }

  LoadParams p;
  memset(&p, 0, sizeof(p));
  bool vec = true;
  for (int s = 0; s < 2; ++s) {
    p.codes[s] = pool4(c, s);
    p.exps[s] = pool4(c, 2 + s);
    p.y[s] = s ? v : k;
    p.ld[s] = s ? ldv : ldk;
    if (!p.y[s]) continue;
    const Pool4& x = p.codes[s];
    vec = vec && aligned(x.base, 4) && x.page % 4 == 0 && x.head % 4 == 0 && x.token % 4 == 0 && aligned(p.y[s], 16) &&
          p.ld[s] % 8 == 0;
  }
  p.slots = slots;
  p.T = T;
  p.n_slots = c.num_pages * c.page_size;
  p.page_shift = log2_of(c.page_size);
  p.page_mask = c.page_size - 1;
  p.k_units = static_cast<int32_t>(k ? width / 8 : 0);
  p.units = fast_div(static_cast<uint32_t>(units));
  p.per_head = fast_div(static_cast<uint32_t>(c.head_dim / 8));
  const int64_t grid = (T * units + kThreads - 1) / kThreads;
  const char* name = vec ? "cache4_load<8>" : "cache4_load<1>";
  if (qkn_host::validate_only()) {
    qkn_host::record_launch(qkn_launch_info{name, 0, 0, 0, 0});
    return QKN_EDRYRUN;
  }
  void* args[] = {&p};
  const void* fn = vec ? reinterpret_cast<const void*>(qkn_cache4_rows<true>) : reinterpret_cast<const void*>(qkn_cache4_rows<false>);
  if (hipLaunchKernel(fn, dim3(static_cast<unsigned>(grid)), dim3(kThreads), args, 0, static_cast<hipStream_t>(stream)) !=
      hipSuccess)
    return QKN_EHIP;
  qkn_host::record_launch(qkn_launch_info{name, grid, kThreads, grid * (kThreads / 64), 0});
  return QKN_OK;
}
