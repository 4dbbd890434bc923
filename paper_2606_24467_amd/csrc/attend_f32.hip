// Attention over f32 rows, of a cache or packed (attend_kernels.h).
//
// Windowed prompts and chunks run here too, 32 rows per workgroup.  They share no tile: each
// wave reads its own K and V rows from the caches, a key again for every 32 rows (6.4 GB and
// 8.8 GB in the first and the last call below).  32 / 8
// heads, D = 128, against the fp32 products alone (a library product reaches 153
// TFLOP/s): 4 prompts of 2048 tokens, 1024 keys, 1112 us against 676; a chunk of 1024 over
// 8192 keys 190 against 113; a prompt of 32768 tokens, 256 keys, 1990 against 909.
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
