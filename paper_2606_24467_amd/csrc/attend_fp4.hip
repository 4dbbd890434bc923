// Attention over 4-bit rows (attend_kernels.h).
#include "attend_kernels.h"

namespace ckv {

void launch_attend_fp4(const AttendArgs &a, bool f32, int head_dim, dim3 grid, hipStream_t stream) {
  auto go = [&]<int D, int RT, int QP>() {
    hipLaunchKernelGGL((attend_kernel<kOverCache, kCacheFp4, D, RT, QP>), grid, dim3(64 * kAttendWaves),
                       0, stream, a);
  };
  auto tiles = [&]<int D>() {
    if (f32) a.rt == 1 ? go.template operator()<D, 1, 3>() : go.template operator()<D, 2, 3>();
    else if (a.rt == 1) go.template operator()<D, 1, 1>();
    else if (a.rt == 2) go.template operator()<D, 2, 1>();
    else go.template operator()<D, 4, 1>();
  };
  head_dim == 64 ? tiles.template operator()<64>() : tiles.template operator()<128>();
}

}  // namespace ckv
