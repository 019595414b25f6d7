// Attention over the paged cache, few rows: every wavefront takes its own key tiles.
#include "qkn_attn_kernels.h"

namespace attn {

// 32 keys a tile; as many workgroups on a CU as registers and LDS have room for.
constexpr int occupancy(int dt, bool fp8, int cb) {
  return cb == 1 ? (dt == 64 || (dt == 128 && fp8) ? 4 : dt == 128 ? 2 : 1) : dt == 64 || (dt == 128 && cb == 2) ? 2 : 1;
}
template <int DT, bool FP8, int CB>
using Few = Cfg<DT, FP8, CB, 4, false, 32, occupancy(DT, FP8, CB)>;

template <int DT, bool FP8>
static Variant pick(int rows, const char* n1, const char* n2, const char* n4) {
  if constexpr (DT < 256)  // 64 rows of 256 do not fit the registers
    if (rows > 32) return variant<Few<DT, FP8, 4>>(n4);
  return rows > 16 ? variant<Few<DT, FP8, 2>>(n2) : variant<Few<DT, FP8, 1>>(n1);
}

#define QKN_PICK(DT, FP8, F) pick<DT, FP8>(rows, "attn<" #DT ",16>/" F, "attn<" #DT ",32>/" F, "attn<" #DT ",64>/" F)

Variant few_rows(int dt, bool fp8, int rows) {
  if (fp8) return dt == 64 ? QKN_PICK(64, true, "fp8") : dt == 128 ? QKN_PICK(128, true, "fp8") : QKN_PICK(256, true, "fp8");
  return dt == 64 ? QKN_PICK(64, false, "bf16") : dt == 128 ? QKN_PICK(128, false, "bf16") : QKN_PICK(256, false, "bf16");
}

}  // namespace attn
