// Windowed attention of prompts and their chunks in bf16: many query rows per
// key, bound by the matrix and vector pipes.
//
// A workgroup takes 32 query rows per wave (row = query token, head of the
// group, so that the heads of a group share every key) and walks the keys that
// any of them sees, 64 at a time, through two LDS buffers: while one is worked
// on, the next tile's loads are in flight to the other.  Products are transposed
// (S^T = K Q^T, O^T = V^T P^T) on the 32x32x16 instruction: lane 32 h + c holds
// query row c against the keys 8 (i / 4) + 4 h + i % 4 (element i), which is the
// order of the reduction slots that P^T goes into the second product with, if V
// comes in the same order.  The transposing LDS read gives it so: four
// consecutive keys of one head dimension per lane.  So P never leaves the
// registers, and the sums of a row belong to the lanes of its column.
// P is rounded to bf16 once (2^-8 of each probability, as the output itself);
// its sum is taken before that, in fp32.
//
// 32 / 8 heads, D = 128 (medians): a prompt of 32768 tokens under a window of 4096 keys 2.22 ms,
// 930 TFLOP/s of the products that its visible pairs need, where a library product of
// 8192^3 reaches 1240; 8 prompts of 4096 to 16384 tokens under 1024 keys 1.69 ms,
// 797 TFLOP/s (the tiles at both ends of a window of 1024 are a tenth more).  Narrow windows
// leave few tiles to a row block, and its first load, masks and output uncovered: 8 prompts of
// 4096 tokens under 1024, 512, 256, 128, 32 keys 631, 405, 284, 220, 187 us, where the
// products and the bytes take 389, 209, 116, 116, 116.  The matrix
// pipe is busy for 45% of the cycles and the vector one for 45%: two waves per SIMD
// overlap the softmax of one with the products of the other by chance alone.  (One wave that
// works on the softmax of a tile between the products of its neighbours took 2480 us:
// its registers did not hold both.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend.h"
#include "row_blocks.h"
#include "score_common.h"

namespace ckv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kPromptWaves = 4;
static_assert(kPromptRows == 32 * kPromptWaves, "32 rows per wave");
constexpr int kPromptKeys = 64;                  // keys per tile

// The 32-row form of add_unbounded (attend_kernels.h), with the values of V that
// are not finite replaced by zeros: one kind of value at a time.
__device__ __forceinline__ void add_unbounded32(f32x16 &acc, bf16x8 &v, bf16x8 sees) {
#pragma unroll
  for (int kind = 0; kind < 3; ++kind) {
    bf16x8 is;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = (float)v[e];
      is[e] = (__bf16)((kind == 0 ? f == INFINITY : kind == 1 ? f == -INFINITY : f != f) ? 1.f : 0.f);
    }
    const f32x16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is, sees, f32x16{}, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (n[i] > 0.f) acc[i] = kind == 2 ? NAN : acc[i] + (kind == 0 ? INFINITY : -INFINITY);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)(fabsf((float)v[e]) < INFINITY ? (float)v[e] : 0.f);
}

template <int D>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void window_prompt_kernel(const AttendArgs a, int run) {
  constexpr int NF = D / 16, DB = D / 32;        // K fragments, blocks of 32 head dimensions
  constexpr int U = D / 8;                       // 16-byte units per row
  constexpr int LD = kPromptKeys * U / (64 * kPromptWaves);   // loads of K (of V) per wave and tile
  constexpr int RB = D * 2;                      // bytes of a row in LDS
  // Two buffers, each K then V.  They are two arrays, which the loop's two copies
  // name: the compiler then sees that reads of one need not wait for the loads that
  // are under way to the other.
  constexpr int KB = kPromptKeys * RB;
  __shared__ __align__(16) char even_s[2 * KB], odd_s[2 * KB];
  static_assert(kPromptRows / 2 * (D + 8) * 2 <= 2 * KB, "half of the outputs fits a buffer");
  __shared__ int wild_s[2][kPromptWaves];        // a wave's loads held V values that are not finite
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, h = lane >> 5;

  // Consecutive row blocks share their keys, so runs of them go to
  // one XCD (workgroups go round the XCDs in turn) and the runs go round the XCDs, the
  // latest rows of a group first.  Each wave finds its sequence.  (8 prompts of 4k to
  // 16k tokens: 1810 us with a grid over the longest one's blocks for each, most XCDs
  // waiting for the one with the most rows, 1700 so.)
  const int in_xcd = (int)blockIdx.x >> 3;
  const int id = (in_xcd / run * 8 + ((int)blockIdx.x & 7)) * run + in_xcd % run;
  if (id >= a.blocks) return;                     // uniform
  RowBlock at;
  if (!find_row_block<true>(a, id, kPromptRows, at)) return;   // uniform
  const int g = at.g, rb = at.rb, q0 = at.q0, lq = at.lq, k0 = at.k0, lk = at.lk;
  const int rows = lq * a.G, r0 = rb * kPromptRows;
  const int t0 = lk - lq;                        // position of query token 0
  const int t_first = t0 + r0 / a.G, t_last = t0 + (min(rows, r0 + kPromptRows) - 1) / a.G;
  // the keys that any row sees, counted from 0 ("virtual"): the sinks outside the
  // window first, then the window's
  const int lo = max(0, t_first - a.window + 1), sinks = min(a.sinks, lo), shift = lo - sinks;
  const int n = t_last < 0 ? 0 : t_last - shift + 1;
  const int all_tiles = (n + kPromptKeys - 1) / kPromptKeys;
  const int per = (all_tiles + a.splits - 1) / a.splits, split = blockIdx.y;
  const int tile0 = min(all_tiles, split * per), tile1 = min(all_tiles, tile0 + per);

  // this wave's rows, the last one in the place of those past the end
  const int w0 = min(rows - 1, r0 + 32 * wave), w1 = min(rows - 1, w0 + 31);
  const int wt_first = t0 + w0 / a.G, wt_last = t0 + w1 / a.G;
  const int r = r0 + 32 * wave + c;
  const bool in = r < rows;
  const int tok = min(r, rows - 1) / a.G, head = g * a.G + (min(r, rows - 1) - tok * a.G);
  const int t = t0 + tok;
  bf16x8 q[NF];
  {
    const gptr<const char> p = to_global(a.q) + (int64_t)(q0 + tok) * a.q_tok + head * a.q_head;
#pragma unroll
    for (int f = 0; f < NF; ++f) q[f] = __builtin_bit_cast(bf16x8, load16(p + (16 * f + 8 * h) * 2));
  }

  // A tile goes from memory to LDS without passing registers, each wave 1 KB at a
  // time: lane i of a load fills the i-th 16-byte unit.  Rows are not padded then;
  // instead the unit u of row r lies at unit u ^ swizzle(r), so that the reads of
  // K (16 rows, one unit each) and the transposing ones of V (4 rows, four units
  // each) fall on banks of their own.
  auto swizzle_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto swizzle_v = [](int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; };
  // A tile is a run of rows: a base that every lane shares and offsets in 32 bits
  // (the host sends longer strides elsewhere), but for the tile that the sinks end
  // in and the last one, whose keys past the end read the last one.
  const int k_row = (int)a.k_tok, v_row = (int)a.v_tok;
  const char *kg = a.k + (k0 + shift) * a.k_tok + g * a.k_head;   // virtual key 0 behind the sinks
  const char *vg = a.v + (k0 + shift) * a.v_tok + g * a.v_head;
  int k_off[LD], v_off[LD];
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    const int unit = 64 * (wave + kPromptWaves * i) + lane, row = unit / U, u = unit % U;
    k_off[i] = row * k_row + 16 * (u ^ swizzle_k(row));
    v_off[i] = row * v_row + 16 * (u ^ swizzle_v(row));
  }
  typedef __attribute__((address_space(3))) void *lds_ptr;
  typedef const __attribute__((address_space(1))) void *global_ptr;
  auto load = [&]<int BUF>(int tile) {
    char *to = BUF ? odd_s : even_s;
    const int x0 = tile * kPromptKeys;
    const char *kt = kg + (int64_t)x0 * k_row, *vt = vg + (int64_t)x0 * v_row;
    if (x0 >= sinks && x0 + kPromptKeys <= n) {  // uniform
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int at = 64 * (wave + kPromptWaves * i) * 16;
        __builtin_amdgcn_global_load_lds((global_ptr)(kt + (uint32_t)k_off[i]), (lds_ptr)(to + at), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_ptr)(vt + (uint32_t)v_off[i]), (lds_ptr)(to + KB + at), 16, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int at = 64 * (wave + kPromptWaves * i) * 16;
        const int row = (64 * (wave + kPromptWaves * i) + lane) / U, x = min(x0 + row, n - 1);
        const int64_t back = x < sinks ? x - shift : x, over = x0 + row;   // its row, and the run's
        __builtin_amdgcn_global_load_lds((global_ptr)(kt + (back - over) * k_row + k_off[i]),
                                         (lds_ptr)(to + at), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_ptr)(vt + (back - over) * v_row + v_off[i]),
                                         (lds_ptr)(to + KB + at), 16, 0, 0);
      }
    }
  };
  // Virtual keys that every row of this wave, and of the workgroup, sees: a tile
  // within them needs no mask.
  const int w_from = max(sinks, wt_last - a.window - shift + 1), w_to = min(n - 1, wt_first - shift);
  const int g_from = max(sinks, t_last - a.window - shift + 1), g_to = min(n - 1, t_first - shift);
  auto within = [](int tile, int from, int to) {
    return tile * kPromptKeys >= from && tile * kPromptKeys + kPromptKeys - 1 <= to;
  };
  // Waits for this wave's loads of a tile; where some row sees a part of it only,
  // looks for V values that are not finite among them.
  auto arrive = [&]<int BUF>(int tile) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (within(tile, g_from, g_to)) return;
    uint32_t wild = 0;                           // a carry out of an exponent of all ones
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const uint4 x = *reinterpret_cast<const uint4 *>(
          (BUF ? odd_s : even_s) + KB + (64 * (wave + kPromptWaves * i) + lane) * 16);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) wild |= ((w[e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
    }
    const bool any = __any(wild != 0);
    if (lane == 0) wild_s[BUF][wave] = any;
  };
  // this lane's places in a tile: of K fragment f in row c, of V block d in row
  // 4 h + (lane & 15) / 4 (rows 8 and 16 further on are swizzled alike)
  int k_at[NF], v_at[DB];
#pragma unroll
  for (int f = 0; f < NF; ++f) k_at[f] = c * RB + 16 * ((2 * f + h) ^ swizzle_k(c));
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    const int row = 4 * h + ((lane & 15) >> 2);
    const int u = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    v_at[d] = row * RB + 16 * (u ^ swizzle_v(row)) + 8 * (lane & 1);
  }

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  float m = -INFINITY, l = 0.f;

  // the virtual keys that this lane's row sees: first_x .. last_x and those before a.sinks
  const int last_x = min(t - shift, n - 1) - 4 * h, first_x = t - shift - a.window + 1 - 4 * h;

  // One tile.  UNBOUNDED: with care for V values that are not finite.
  auto work = [&]<bool UNBOUNDED, int BUF>(int tile) {
    const char *kt = BUF ? odd_s : even_s, *vt = kt + KB;
    f32x16 s[2] = {f32x16{}, f32x16{}};
    __builtin_amdgcn_s_setprio(1);   // the logits' products before another wave's softmax (32k: 2189 -> 2155 us)
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int f = 0; f < NF; ++f)
        s[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8 *>(kt + k_at[f] + 32 * k * RB), q[f], s[k], 0, 0, 0);
    if constexpr (!UNBOUNDED) {                  // half 0's fragments, then each product with one of half 1
      __builtin_amdgcn_sched_group_barrier(0x100, NF, 0);
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, NF, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    if (UNBOUNDED || !within(tile, w_from, w_to)) {
      // the keys of the tile that this lane's row sees, a bit each; two instructions a logit
      const int from = tile * kPromptKeys, last = last_x - from, first = first_x - from;
      const int sink = min(a.sinks - 4 * h - from, last + 1);
      auto below = [](int x) { return x >= 64 ? ~0ull : x <= 0 ? 0ull : ~0ull >> (64 - x); };
      const uint64_t seen = (below(last + 1) & ~below(first)) | below(sink);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t word = (uint32_t)(seen >> (32 * k));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t all = __builtin_amdgcn_sbfe(word, 8 * (i >> 2) + (i & 3), 1);
          s[k][i] = __uint_as_float((__float_as_uint(s[k][i]) & all) | (0xFF800000u & ~all));
        }
      }
    }
    // (the maximum that returns a NaN needs no quieting of its operands)
    float top = __builtin_elementwise_maximum(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i)
      top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[0][i], s[1][i]), top);
    top *= a.c1;
    if (__any(top > m + 8.f)) {                  // the reference follows in steps of 2^8
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      const float next = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
      const float shrink = m == next ? 1.f : fast_exp2(m - next);
      l *= shrink;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= shrink;
      m = next;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      bf16x8 p[2], sees[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (UNBOUNDED) sees[i >> 3][i & 7] = (__bf16)(s[k][i] != -INFINITY ? 1.f : 0.f);
        const float x = fast_exp2(__builtin_fmaf(s[k][i], a.c1, -ref));
        l += x;
        p[i >> 3][i & 7] = (__bf16)x;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          // 16 lanes read four rows, 16 head dimensions of each; lane i gets column i
          typedef __attribute__((address_space(3))) i16x4 *lptr;
          const char *at = vt + v_at[d] + (32 * k + 16 * half) * RB;
          const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)at);
          const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(at + 8 * RB));
          bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          if constexpr (UNBOUNDED) add_unbounded32(acc[d], vf, sees[half]);
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[half], acc[d], 0, 0, 0);
        }
    }
    if constexpr (!UNBOUNDED) {
      // fragments of V four products ahead; the softmax of half 1 between the
      // products of half 0
      __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
      __builtin_amdgcn_sched_group_barrier(0x402, 60, 1);
#pragma unroll
      for (int e = 0; e < 2 * DB; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        __builtin_amdgcn_sched_group_barrier(0x402, 56 / (2 * DB), 1);
      }
#pragma unroll
      for (int e = 0; e < 2 * DB; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
      }
    }
  };

  // One step of the loop: the next tile's loads, this tile's work, the wait for the
  // loads.  False: the tile has such values in keys that some row does not see.
  auto step = [&]<int BUF>(int tile) {
    if (!within(tile, g_from, g_to)) {           // uniform over the workgroup
      int any = 0;
#pragma unroll
      for (int w = 0; w < kPromptWaves; ++w) any |= wild_s[BUF][w];
      if (__any(any != 0)) return false;
    }
    if (tile + 1 < tile1) load.template operator()<1 - BUF>(tile + 1);
    work.template operator()<false, BUF>(tile);
    if (tile + 1 < tile1) arrive.template operator()<1 - BUF>(tile + 1);
    __syncthreads();
    return true;
  };

  bool wild = false;
  if (tile0 < tile1) {
    load.template operator()<0>(tile0);
    arrive.template operator()<0>(tile0);
  }
  __syncthreads();
  for (int tile = tile0; tile < tile1; tile += 2) {
    if (!step.template operator()<0>(tile) ||
        (tile + 1 < tile1 && !step.template operator()<1>(tile + 1))) {
      wild = true;
      break;
    }
  }
  if (wild) {
    // Some rows see a part only of a tile with V values that are not finite: all of
    // it again, with care for them, one tile after the other.
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
    m = -INFINITY;
    l = 0.f;
    for (int tile = tile0; tile < tile1; ++tile) {
      __syncthreads();
      load.template operator()<0>(tile);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      work.template operator()<true, 0>(tile);
    }
  }
  __syncthreads();                               // the buffers are done with

  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if (a.splits > 1) {                            // joined by attend_join_kernel
    const int64_t slot = (int64_t)at.part * a.splits + split;
    const int64_t row = slot * kPromptRows + 32 * wave + c;
    if (in) {
      if (h == 0) a.part_ml[row] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4 *>(a.part_o + row * D + 32 * d + 8 * (i >> 2) + 4 * h) =
              f32x4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  // each wave's 32 rows through LDS, so that whole rows go out in 16-byte lanes
  constexpr int OS = D + 8;
  __bf16(*o_s)[OS] = reinterpret_cast<__bf16(*)[OS]>(wave < kPromptWaves / 2 ? even_s : odd_s) +
                     32 * (wave % (kPromptWaves / 2));
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<bf16x4 *>(&o_s[c][32 * d + 8 * (i >> 2) + 4 * h]) =
          bf16x4{(__bf16)(acc[d][i] * inv), (__bf16)(acc[d][i + 1] * inv),
                 (__bf16)(acc[d][i + 2] * inv), (__bf16)(acc[d][i + 3] * inv)};
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32 * U / 64; ++i) {
    const int e = lane + 64 * i, row = e / U, u = e % U, rr = r0 + 32 * wave + row;
    if (rr < rows) {
      const int tk = rr / a.G, hd = g * a.G + (rr - tk * a.G);
      store16(to_global(a.out) + (((int64_t)(q0 + tk) * ((int64_t)a.Hkv * a.G) + hd) * D + 8 * u) * 2,
              *reinterpret_cast<const uint4 *>(&o_s[row][8 * u]));
    }
  }
}

void launch_window_prompt(const AttendArgs &a, int head_dim, int max_rows, hipStream_t stream) {
  // 32 row blocks (half of what an XCD holds at a time) in a run, fewer where that
  // would leave an XCD with less than about 16 runs
  const int run = std::clamp(a.blocks / 128, 1, 32);
  const dim3 grid((unsigned)(((int64_t)a.blocks + 8 * run - 1) / (8 * run) * (8 * run)), a.splits);
  if (head_dim == 64)
    hipLaunchKernelGGL((window_prompt_kernel<64>), grid, dim3(64 * kPromptWaves), 0, stream, a, run);
  else
    hipLaunchKernelGGL((window_prompt_kernel<128>), grid, dim3(64 * kPromptWaves), 0, stream, a, run);
  launch_attend_join(a, kOverWindow, false, head_dim, max_rows, stream);
}

}  // namespace ckv
