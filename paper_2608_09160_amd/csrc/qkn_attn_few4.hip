// Attention over the paged cache, few rows, the 4-bit cache.
#include "qkn_attn_few.h"

namespace attn {

Variant few_rows4(int dt, int rows) { return QKN_PICK_DT(kFp4, true, "fp4"); }

}  // namespace attn
