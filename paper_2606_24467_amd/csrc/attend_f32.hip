// Attention over f32 rows, of a cache or packed (attend_kernels.h).
#include "attend_kernels.h"

namespace ckv {

void launch_attend_f32(const AttendArgs &a, AttendSource source, int head_dim, dim3 grid,
                      hipStream_t stream) {
  auto go = [&]<AttendSource SRC, int D, int RT>() {
    hipLaunchKernelGGL((attend_kernel<SRC, kCacheF32, D, RT, 1>), grid, dim3(64 * kAttendWaves), 0,
                       stream, a);
  };
  auto tiles = [&]<AttendSource SRC, int D>() {
    if (a.rt == 1) go.template operator()<SRC, D, 1>();
    else if (a.rt == 2) go.template operator()<SRC, D, 2>();
    else go.template operator()<SRC, D, 4>();
  };
  auto dim = [&]<AttendSource SRC>() {
    head_dim == 64 ? tiles.template operator()<SRC, 64>() : tiles.template operator()<SRC, 128>();
  };
  source == kOverCache ? dim.template operator()<kOverCache>() : dim.template operator()<kOverWindow>();
}

}  // namespace ckv
