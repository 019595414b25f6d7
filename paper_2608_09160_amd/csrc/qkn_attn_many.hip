// Attention over the paged cache, many rows: every wavefront has its own rows, all take the same key tiles.
#include "qkn_attn_kernels.h"

namespace attn {

// Much work: 128 rows to a workgroup, two wavefronts on a SIMD where the registers allow it. Little: 64 rows, for more
// workgroups.
template <int DT, bool FP8>
using Large = Cfg<DT, FP8, 2, 4, true, 64, DT == 256 ? 1 : 2>;
template <int DT, bool FP8>
using Small = Cfg<DT, FP8, 1, 4, true, 64, DT == 256 ? 1 : 2>;

#define QKN_PICK(DT, FP8, F)                                             \
  (small ? variant<Small<DT, FP8>>("attn<" #DT ",64,shared>/" F)        \
         : variant<Large<DT, FP8>>("attn<" #DT ",128,shared>/" F))

Variant many_rows(int dt, bool fp8, bool small) {
  if (fp8) return dt == 64 ? QKN_PICK(64, true, "fp8") : dt == 128 ? QKN_PICK(128, true, "fp8") : QKN_PICK(256, true, "fp8");
  return dt == 64 ? QKN_PICK(64, false, "bf16") : dt == 128 ? QKN_PICK(128, false, "bf16") : QKN_PICK(256, false, "bf16");
}

}  // namespace attn
