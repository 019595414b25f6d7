// Attention over the paged cache, few rows: every wavefront takes its own key tiles.
#include "qkn_attn_few.h"

namespace attn {

Variant few_rows(int dt, bool fp8, int rows) {
  return fp8 ? QKN_PICK_DT(kFp8, false, "fp8") : QKN_PICK_DT(kBf16, false, "bf16");
}

}  // namespace attn
