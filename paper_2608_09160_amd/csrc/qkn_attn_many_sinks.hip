// Attention over the paged cache, many rows, which see first keys besides their window.
#include "qkn_attn_many.h"

namespace attn {

Variant many_rows_sinks(int dt, bool fp8, bool small) {
  return fp8 ? QKN_PICK_DT(kFp8, true, "fp8+sinks") : QKN_PICK_DT(kBf16, true, "bf16+sinks");
}

}  // namespace attn
