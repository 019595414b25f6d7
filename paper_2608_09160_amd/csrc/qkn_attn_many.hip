// Attention over the paged cache, many rows: every wavefront has its own rows, all take the same key tiles.
#include "qkn_attn_kernels.h"

namespace attn {

template <int DT, bool FP8>
using Many = Cfg<DT, FP8, 2, 4, true, 64, DT == 256 ? 1 : 2>;

Variant many_rows(int dt, bool fp8) {
  if (fp8)
    return dt == 64 ? variant<Many<64, true>>("attn<64,128,shared>/fp8")
                    : dt == 128 ? variant<Many<128, true>>("attn<128,128,shared>/fp8")
                                : variant<Many<256, true>>("attn<256,128,shared>/fp8");
  return dt == 64 ? variant<Many<64, false>>("attn<64,128,shared>/bf16")
                  : dt == 128 ? variant<Many<128, false>>("attn<128,128,shared>/bf16")
                              : variant<Many<256, false>>("attn<256,128,shared>/bf16");
}

}  // namespace attn
