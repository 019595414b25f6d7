// Attention over the paged cache, many rows: the kernels' choice, for the units that instantiate them.
#ifndef QKN_ATTN_MANY_H
#define QKN_ATTN_MANY_H

#include "qkn_attn_kernels.h"

namespace attn {

// Much work: 128 rows to a workgroup, two wavefronts on a SIMD where the registers allow it. Little: 64 rows, for more
// workgroups.
template <int DT, int F, bool SINKS>
using Large = Cfg<DT, F, 2, 4, true, 64, DT == 256 ? 1 : 2, SINKS>;
template <int DT, int F, bool SINKS>
using Small = Cfg<DT, F, 1, 4, true, 64, DT == 256 ? 1 : 2, SINKS>;

}  // namespace attn

#define QKN_PICK(DT, F, SINKS, NAME)                                     \
  (small ? variant<Small<DT, F, SINKS>>("attn<" #DT ",64,shared>/" NAME) \
         : variant<Large<DT, F, SINKS>>("attn<" #DT ",128,shared>/" NAME))
#define QKN_PICK_DT(F, SINKS, NAME) \
  (dt == 64 ? QKN_PICK(64, F, SINKS, NAME) : dt == 128 ? QKN_PICK(128, F, SINKS, NAME) : QKN_PICK(256, F, SINKS, NAME))

#endif  // QKN_ATTN_MANY_H
