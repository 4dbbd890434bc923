// Attention over 4-bit rows (attend_kernels.h).
#include "attend_kernels.h"

namespace ckv {

void launch_attend_fp4(const AttendArgs &a, bool f32, int head_dim, dim3 grid, hipStream_t stream) {
  auto go = [&]<int D, int RT, int QP, bool MASKS, bool ONE>() {
    launch_attend_as<kOverCache, kCacheFp4, D, RT, QP, MASKS, ONE>(a, grid, stream);
  };
  auto tiles = [&]<int D, int QP, bool MASKS>() {
    if (a.one) go.template operator()<D, 1, QP, MASKS, true>();
    else if (a.rt == 1) go.template operator()<D, 1, QP, MASKS, false>();
    else if (a.rt == 2) go.template operator()<D, 2, QP, MASKS, false>();
    else if constexpr (QP == 1) go.template operator()<D, 4, QP, MASKS, false>();
  };
  auto kind = [&]<int D>() {
    if (f32) a.masks ? tiles.template operator()<D, 3, true>() : tiles.template operator()<D, 3, false>();
    else a.masks ? tiles.template operator()<D, 1, true>() : tiles.template operator()<D, 1, false>();
  };
  head_dim == 64 ? kind.template operator()<64>() : kind.template operator()<128>();
}

}  // namespace ckv
