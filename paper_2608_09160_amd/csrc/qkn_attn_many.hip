// Attention over the paged cache, many rows: every wavefront has its own rows, all take the same key tiles.
#include "qkn_attn_many.h"

namespace attn {

Variant many_rows(int dt, bool fp8, bool small) {
  return fp8 ? QKN_PICK_DT(kFp8, false, "fp8") : QKN_PICK_DT(kBf16, false, "bf16");
}

}  // namespace attn
