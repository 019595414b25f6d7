// Attention over the paged cache, few rows, which see first keys besides their window.
#include "qkn_attn_few.h"

namespace attn {

Variant few_rows_sinks(int dt, bool fp8, int rows) {
  return fp8 ? QKN_PICK_DT(kFp8, true, "fp8+sinks") : QKN_PICK_DT(kBf16, true, "bf16+sinks");
}

}  // namespace attn
