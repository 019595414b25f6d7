// Attention over the paged cache, many rows, the 4-bit cache.
#include "qkn_attn_many.h"

namespace attn {

Variant many_rows4(int dt, bool small) { return QKN_PICK_DT(kFp4, true, "fp4"); }

}  // namespace attn
