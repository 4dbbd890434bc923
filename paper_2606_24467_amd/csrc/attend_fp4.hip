// Attention over 4-bit rows (attend_kernels.h).
#include "attend_kernels.h"

namespace ckv {

void launch_attend_fp4(const AttendArgs &a, bool f32, int head_dim, dim3 grid, hipStream_t stream) {
  auto go = [&]<int D, int QP, bool MASKS>() {   // a row tile per workgroup
    a.one ? launch_attend_as<kOverCache, kCacheFp4, D, 1, QP, MASKS, true>(a, grid, stream)
          : launch_attend_as<kOverCache, kCacheFp4, D, 1, QP, MASKS, false>(a, grid, stream);
  };
  auto kind = [&]<int D>() {
    if (f32) a.masks ? go.template operator()<D, 3, true>() : go.template operator()<D, 3, false>();
    else a.masks ? go.template operator()<D, 1, true>() : go.template operator()<D, 1, false>();
  };
  head_dim == 64 ? kind.template operator()<64>() : kind.template operator()<128>();
}

}  // namespace ckv
