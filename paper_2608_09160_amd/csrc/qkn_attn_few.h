// Attention over the paged cache, few rows: the kernels' choice, for the units that instantiate them.
#ifndef QKN_ATTN_FEW_H
#define QKN_ATTN_FEW_H

#include "qkn_attn_kernels.h"

namespace attn {

// 32 keys a tile; as many workgroups on a CU as registers and LDS have room for.
constexpr int occupancy(int dt, int format, int cb) {
  return cb == 1 ? (dt == 64 || (dt == 128 && format != kBf16) ? 4 : dt == 128 || format == kFp4 ? 2 : 1)
                 : dt == 64 || (dt == 128 && cb == 2) ? 2 : 1;
}
template <int DT, int F, int CB, bool SINKS>
using Few = Cfg<DT, F, CB, 4, false, 32, occupancy(DT, F, CB), SINKS>;

template <int DT, int F, bool SINKS>
static Variant pick(int rows, const char* n1, const char* n2, const char* n4) {
  if constexpr (DT < 256)  // 64 rows of 256 do not fit the registers
    if (rows > 32) return variant<Few<DT, F, 4, SINKS>>(n4);
  return rows > 16 ? variant<Few<DT, F, 2, SINKS>>(n2) : variant<Few<DT, F, 1, SINKS>>(n1);
}

}  // namespace attn

#define QKN_PICK(DT, F, SINKS, NAME) \
  pick<DT, F, SINKS>(rows, "attn<" #DT ",16>/" NAME, "attn<" #DT ",32>/" NAME, "attn<" #DT ",64>/" NAME)
#define QKN_PICK_DT(F, SINKS, NAME) \
  (dt == 64 ? QKN_PICK(64, F, SINKS, NAME) : dt == 128 ? QKN_PICK(128, F, SINKS, NAME) : QKN_PICK(256, F, SINKS, NAME))

#endif  // QKN_ATTN_FEW_H
