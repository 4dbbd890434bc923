// Attention over f32 rows, of a cache or packed (attend_kernels.h).
#include "attend_kernels.h"

namespace ckv {

void launch_attend_f32(const AttendArgs &a, AttendSource source, int head_dim, dim3 grid,
                      hipStream_t stream) {
  auto go = [&]<AttendSource SRC, int D, int RT, bool MASKS, bool ONE>() {
    launch_attend_as<SRC, kCacheF32, D, RT, 1, MASKS, ONE>(a, grid, stream);
  };
  auto tiles = [&]<AttendSource SRC, int D, bool MASKS>() {
    if (a.one) go.template operator()<SRC, D, 1, MASKS, true>();
    else if (a.rt == 1) go.template operator()<SRC, D, 1, MASKS, false>();
    else go.template operator()<SRC, D, 2, MASKS, false>();
  };
  auto dim = [&]<AttendSource SRC, bool MASKS>() {
    head_dim == 64 ? tiles.template operator()<SRC, 64, MASKS>()
                   : tiles.template operator()<SRC, 128, MASKS>();
  };
  if (source == kOverCache)
    a.masks ? dim.template operator()<kOverCache, true>() : dim.template operator()<kOverCache, false>();
  else
    a.masks ? dim.template operator()<kOverWindow, true>() : dim.template operator()<kOverWindow, false>();
}

}  // namespace ckv
