// Attention of many query rows over the same keys (rows_attention.h), f32.
#include "rows_attention.h"

namespace ckv {

int launch_cross_f32(int head_dim, const CrossArgs &a, hipStream_t s) {
  return head_dim == 128 ? launch_rows_cross<CHUNKKV_F32, 128>(a, s) : launch_rows_cross<CHUNKKV_F32, 64>(a, s);
}
int launch_shared_f32(int head_dim, const SharedArgs &a, hipStream_t s) {
  return head_dim == 128 ? launch_rows<CHUNKKV_F32, 128, true, false>(a, s) : launch_rows<CHUNKKV_F32, 64, true, false>(a, s);
}

}  // namespace ckv
