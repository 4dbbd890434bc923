// Attention of chunks of prompts over the pages of a cache, for bf16 queries (pages_attend.h): many
// query rows per key, bound by the matrix and vector pipes.
//
// A workgroup takes 32 query rows per wave (row = new token, head of the group, so that the heads
// of a group share every key) and walks its split of the keys that any of them sees, in tiles of
// 64 through LDS.  Products are transposed (S^T = K Q^T, O^T = V^T P^T) on the 32x32x16
// instruction: lane 32 h + c holds query row c against the keys 8 (i / 4) + 4 h + i % 4 of 32
// (element i), which is the order of the reduction slots that P^T goes into the second product
// with, if V comes in the same order; the transposing LDS read gives it so.  P never leaves the
// registers.  It is rounded to bf16 once, and its sum is taken before that, in fp32: a second part
// of it would be a third product beside two on the pipe that bounds the kernel, where the output is rounded
// to bf16 as well (it is off by 0.0023 of exact arithmetic, where rounding the exact one gives 0.0017).
//
// A wave's matrix and vector work overlap: in one step it takes the logits of the 32 keys to come,
// the exponentials of 32 and the second product of the 32 before, none of which needs another, and
// the compiler is told to put the vector instructions between the products.  So there is no time
// for a maximum of the logits before the exponentials: the reference m of a row stays where it is
// as long as the sum of its exponentials shows that none is above 2^12 (fp32 and bf16 hold them to
// the same relative precision, and the sums with V have that much less room below 2^128), and only
// else it follows the maximum and the step's exponentials are taken again.
//
// Bound by the matrix and vector pipes, half of the cycles each, at the clock that their power leaves
// (about 2 GHz): 2048 tokens of 32 heads over 32768 keys of 8 groups of 128 bf16 values take 960 to
// 1060 us on different cards, 1.0 to 1.11 PFLOP/s, where a large library product reaches 1.25.  256 rows a workgroup
// (128: 1107 us in an earlier form, more LDS writes and barriers per product) where a sequence has
// more than 128; 8 waves then fill a CU, and what is not overlapped is the start and end of a
// block, about 13 us of CU time, and its tiles with masks.
//
// Rows of 16 keys lie in one page.  Their numbers are looked up 64 at a time, a lane each, one
// such window ahead of the tiles.  bf16 rows go from memory to LDS without passing registers;
// 8-bit ones are loaded into registers, a block of 32 values a thread, while others are worked on,
// and widened to bf16 (exactly) on their way to LDS.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pages_attend.h"
#include "score_common.h"

namespace ckv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

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

// NW: waves of a workgroup, 32 rows each.
template <int D, bool FP8, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void pages_prompt_kernel(const PagesArgs a, int run) {
  constexpr int NF = D / 16, DB = D / 32;        // K fragments, blocks of 32 head dimensions
  constexpr int U = D / 8;                       // 16-byte units per row in LDS
  constexpr int LD = kPromptKeys * U / (64 * NW);   // loads of K (of V) per wave and tile
  constexpr int RB = D * 2;                      // bytes of a row in LDS
  constexpr int PB = FP8 ? D : 2 * D;            // ... in a page
  constexpr int SEGS = kPromptKeys / 16;         // 16-key segments of a tile
  // Two buffers of K and of V, as arrays that the loop's copies name: the compiler then sees that
  // reads of one need not wait for the loads that are under way to another.
  constexpr int KB = kPromptKeys * RB;
  __shared__ __align__(16) char k0_s[KB], k1_s[KB], v0_s[KB], v1_s[KB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, h = lane >> 5;

  // Neighbouring units share their keys, so runs of them go to one XCD (workgroups go round the
  // XCDs in turn) and the runs go round the XCDs, the latest rows of a group first.
  const int in_xcd = (int)blockIdx.x >> 3;
  const int id = (in_xcd / run * 8 + ((int)blockIdx.x & 7)) * run + in_xcd % run;
  if (id >= a.grid) return;                      // uniform
  PageUnit at;
  if (!find_page_unit<true, false>(a, id, at)) return;   // uniform
  const int g = at.g, q0 = at.q0, rows = at.lq * a.G, r0 = at.rb * (32 * NW);
  const int t0 = at.len - at.lq, n = at.n;       // position of new token 0
  const int split = at.split, splits = at.splits;
  const int all_tiles = (n + kPromptKeys - 1) / kPromptKeys, per = at.split_keys / kPromptKeys;
  const int tile0 = split * per, tile1 = min(all_tiles, tile0 + per);

  // this wave's rows, the last one in the place of those past the end
  const bool working = r0 + 32 * wave < rows;    // uniform
  const int r = r0 + 32 * wave + c;
  const bool in = r < rows;
  const int tok = min(r, rows - 1) / a.G, head = g * a.G + (min(r, rows - 1) - tok * a.G);
  const int t = t0 + tok;
  bf16x8 q[NF];
  auto load_q = [&]() __attribute__((always_inline)) {
    const gptr<const char> p = to_global(a.q) + (int64_t)(q0 + tok) * a.q_tok + head * a.q_head;
#pragma unroll
    for (int f = 0; f < NF; ++f) q[f] = __builtin_bit_cast(bf16x8, load16(p + (16 * f + 8 * h) * 2));
  };

  // The pages of 64 segments, of those before and of those after them, in LDS: window w holds the
  // segments tile0 SEGS + 64 w .., and is loaded 16 tiles ahead.  (In registers they would make the first look
  // at them wait for the rows that are under way.)  The wave that loads one waits for it before the next
  // tile's barrier (arrive), the others read it behind that.
  constexpr int kWindow = 64 / SEGS;             // tiles of a window
  __shared__ __align__(16) int page_s[4][64];
  const int segments = (n + 15) / 16;
  typedef __attribute__((address_space(3))) void *lds_ptr;
  typedef const __attribute__((address_space(1))) void *global_ptr;
  const int32_t *table = a.c.table + (int64_t)at.b * a.c.max_pages;
  auto look_up = [&](int window) __attribute__((always_inline)) {
    if (wave != window % NW) return;             // uniform
    const int seg = min(tile0 * SEGS + 64 * window + lane, segments - 1);
    __builtin_amdgcn_global_load_lds((global_ptr)(table + (seg * 16 >> a.c.shift)), (lds_ptr)page_s[window & 3], 4, 0, 0);
  };

  // In LDS rows are not padded; instead the unit u of row r lies at unit u ^ swizzle(r), so that
  // the reads of K (16 rows, one unit each) and the transposing ones of V (4 rows, four units
  // each) fall on banks of their own.
  auto swizzle_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto swizzle_v = [](int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; };
  // Rows of a group: page p's begin p * page_rows rows behind the first page's.
  const int in_page = (1 << a.c.shift) - 1;
  const uint32_t page_rows = (uint32_t)a.c.Hkv << a.c.shift;
  const char *k_pool = a.c.k + ((int64_t)g << a.c.shift) * PB, *v_pool = a.c.v + ((int64_t)g << a.c.shift) * PB;
  // bf16: each wave 1 KB at a time, lane i of a load fills the i-th 16-byte unit.  A load's rows lie in
  // one segment: a base that all lanes share.
  uint32_t k_off[FP8 ? 1 : LD], v_off[FP8 ? 1 : LD];
  if constexpr (!FP8) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int unit = 64 * (wave + NW * i) + lane, row = unit / U, u = unit % U;
      k_off[i] = row % 16 * RB + 16 * (u ^ swizzle_k(row));
      v_off[i] = row % 16 * RB + 16 * (u ^ swizzle_v(row));
    }
  }
  uint64_t row0[FP8 ? 1 : LD];                   // the rows that a tile's loads begin with
  // 8-bit: a thread's block of 32 values of K, or of V (or of each, where the threads are too few)
  constexpr int RW = D / 32, BLOCKS = kPromptKeys * RW;   // blocks of a row, of a tile
  constexpr bool BOTH = 2 * BLOCKS > 64 * NW;
  const int block = tid % BLOCKS, b_row = block / RW, b_of = block % RW;
  const bool is_v = !BOTH && tid >= BLOCKS, has = BOTH || tid < 2 * BLOCKS;
  uint4 raw[BOTH ? 2 : 1][2];
  uint32_t raw_scale[BOTH ? 2 : 1];
  uint64_t raw_row = 0;                          // of the block: K's now, V's a tile later

  // A tile's pages, asked for before they are needed, and what follows from them before its K and then its
  // V are loaded.  Segments without a page are read in some page, and seen by no row; so are rows past
  // the end, in the last segment's page.
  int4 pages;
  int last_gap = tile0 - 1;                      // the last tile seen so far with such a segment
  auto pages_of = [&](int tile) __attribute__((always_inline)) {
    const int w = tile - tile0;
    return *reinterpret_cast<const int4 *>(&page_s[w / kWindow & 3][w % kWindow * SEGS]);
  };
  const uint32_t n_pages = (uint32_t)a.c.n_pages;
  auto gap = [&](int4 p) __attribute__((always_inline)) {
    return __any(max(max((uint32_t)p.x, (uint32_t)p.y), max((uint32_t)p.z, (uint32_t)p.w)) >= n_pages);
  };
  auto find = [&](int tile) __attribute__((always_inline)) {
    if (gap(pages)) last_gap = tile;
    const int x0 = tile * kPromptKeys;
    auto first_row = [&](int seg) __attribute__((always_inline)) {   // of a segment's page
      const int p = seg == 0 ? pages.x : seg == 1 ? pages.y : seg == 2 ? pages.z : pages.w;
      return (uint64_t)min((uint32_t)p, n_pages - 1) * page_rows;
    };
    if constexpr (FP8) {
      raw_row = first_row(b_row / 16) + (uint32_t)((x0 + b_row) & in_page);
    } else {
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int seg = 64 * (wave + NW * i) / (16 * U);       // uniform
        row0[i] = first_row(seg) + (uint32_t)((x0 + 16 * seg) & in_page);
      }
    }
  };
  // A tile's segments without a page, a bit each (of the last two tiles found).
  auto gone_of = [&](int tile) __attribute__((always_inline)) {
    if (tile > last_gap) return 0u;              // uniform
    const int4 p = pages_of(tile);
    const bool none[SEGS] = {(uint32_t)p.x >= n_pages, (uint32_t)p.y >= n_pages, (uint32_t)p.z >= n_pages,
                             (uint32_t)p.w >= n_pages};
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < SEGS; ++e) bits |= __any(none[e]) ? 1u << e : 0u;
    return bits;
  };
  // Starts the loads of a tile's K or V (8-bit: of the threads that load it).
  auto load = [&](const char *pool, char *to, const uint32_t (&off)[FP8 ? 1 : LD]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < (FP8 ? 0 : LD); ++i)
      __builtin_amdgcn_global_load_lds((global_ptr)(pool + row0[i] * RB + off[i]),
                                       (lds_ptr)(to + 64 * (wave + NW * i) * 16), 16, 0, 0);
  };
  auto load8 = [&](const char *pool, const uint8_t *scales, int b) __attribute__((always_inline)) {
    const gptr<const char> p = to_global(pool) + raw_row * PB + 32 * b_of;
    raw[b][0] = load16(p);
    raw[b][1] = load16(p + 16);
    raw_scale[b] = to_global(scales)[(((uint64_t)(uint32_t)g << a.c.shift) + raw_row) * RW + b_of];
  };
  auto load_k = [&]<int BUF>() __attribute__((always_inline)) {
    if constexpr (!FP8) load(k_pool, BUF ? k1_s : k0_s, k_off);
    else if (has && !is_v) load8(k_pool, a.c.k_scale, 0);
  };
  auto load_v = [&]<int BUF>() __attribute__((always_inline)) {
    if constexpr (!FP8) load(v_pool, BUF ? v1_s : v0_s, v_off);
    else if (has && (BOTH || is_v)) load8(v_pool, a.c.v_scale, BOTH);
  };
  // The last key that every row of the workgroup sees: keys up to there need no mask.
  const int g_to = min(n - 1, t0 + r0 / a.G);
  // 8-bit: widens a thread's block into row b_row of a buffer.
  auto widen = [&](char *to, int b, int swizzle) __attribute__((always_inline)) {
    const float sc = fp4_scale(raw_scale[b]);
    const uint32_t w[8] = {raw[b][0].x, raw[b][0].y, raw[b][0].z, raw[b][0].w,
                           raw[b][1].x, raw[b][1].y, raw[b][1].z, raw[b][1].w};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint2 lo = fp8_values(w[2 * u], sc), hi = fp8_values(w[2 * u + 1], sc);
      const uint4 x = make_uint4(lo.x, lo.y, hi.x, hi.y);
      *reinterpret_cast<uint4 *>(to + b_row * RB + 16 * ((4 * b_of + u) ^ swizzle)) = x;
    }
  };
  // Waits for this wave's loads, of K to k (if `more`) and of V to v (8-bit: widens them), and of page
  // numbers.  Every wave waits, those too that have no rows of 8 bits to widen: the barrier behind this
  // does not order their loads to LDS before the other waves' reads.
  auto arrive = [&](char *k, char *v, bool more) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    if constexpr (FP8 && BOTH) {
      if (more) widen(k, 0, swizzle_k(b_row));
      widen(v, 1, swizzle_v(b_row));
    } else if constexpr (FP8) {
      if (has && (is_v || more)) widen(is_v ? v : k, 0, is_v ? swizzle_v(b_row) : swizzle_k(b_row));
    }
  };

  // This lane's places in a tile: of K fragment f in row c at k_at ^ 32 f, of V block d in row
  // 4 h + (lane & 15) / 4 at v_at ^ 64 d (rows 8 and 16 further on are swizzled alike).
  int k_at, v_at;
  {
    const int row = 4 * h + ((lane & 15) >> 2), u = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    k_at = c * RB + 16 * (h ^ swizzle_k(c));
    v_at = row * RB + 16 * (u ^ swizzle_v(row)) + 8 * (lane & 1);
  }

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  float m = -INFINITY, l = 0.f;
  const int last_x = min(t, n - 1) - 4 * h;      // the last key that this lane's row sees

  // The parts of a step: fragments of K (half of a tile, 32 keys) and V (16 keys of it), the logits that
  // a row does not see, the exponentials under the reference and their sum.
  auto k_frag = [&](const char *kt, int half, int f) __attribute__((always_inline)) {
    return *reinterpret_cast<const bf16x8 *>(kt + (k_at ^ 32 * f) + 32 * half * RB);
  };
  auto v_frag = [&](const char *vt, int sixteen, int d) __attribute__((always_inline)) {
    // 16 lanes read four rows, 16 head dimensions of each; lane i gets column i
    typedef __attribute__((address_space(3))) i16x4 *lptr;
    const char *at = vt + (v_at ^ 64 * d) + 16 * sixteen * RB;
    const i16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)at);
    const i16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(at + 8 * RB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // The keys of half `half` of a tile that this lane's row sees, a bit each: element i's is 8 (i / 4) + i % 4.
  auto sees = [&](int tile, int half, uint32_t gone) __attribute__((always_inline)) {
    const int seen = last_x - tile * kPromptKeys - 32 * half + 1;
    uint32_t word = seen >= 32 ? ~0u : seen <= 0 ? 0u : ~0u >> (32 - seen);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (gone >> (2 * half + e) & 1) word &= ~(0xFFFFu << 16 * e >> 4 * h);
    return word;
  };
  auto mask = [&](f32x16 &s, uint32_t word) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t all = __builtin_amdgcn_sbfe(word, 8 * (i >> 2) + (i & 3), 1);
      s[i] = __uint_as_float((__float_as_uint(s[i]) & all) | (0xFF800000u & ~all));
    }
  };
  auto exponentials = [&](const f32x16 &s, float ref, bf16x8 (&p)[2]) __attribute__((always_inline)) {
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = fast_exp2(__builtin_fmaf(s[i], a.c1, -ref));
      sum[i & 1] += x;
      p[i >> 3][i & 7] = (__bf16)x;
    }
    return sum[0] + sum[1];
  };
  // The reference moves to the maximum (with m = -infinity every sum is NaN or infinite).
  auto move_reference = [&](const f32x16 &s) __attribute__((always_inline)) {
    // (the maximum that returns a NaN needs no quieting of its operands)
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[i]);
    top *= a.c1;
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    const float next = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
    const float shrink = m == next ? 1.f : fast_exp2(m - next);
    l *= shrink;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] *= shrink;
    m = next;
  };
  auto settle = [&](const f32x16 &s, float sum, bf16x8 (&p)[2]) __attribute__((always_inline)) {
    if (__any(!(sum <= 0x1p12f))) {              // seldom
      move_reference(s);
      sum = exponentials(s, m == -INFINITY ? 0.f : m, p);
    }
    l += sum;
  };

  // A step: `next` gets the logits of half NEXT of the tile in kt, p (the last step's) goes into the
  // second product with half LAST of the tile in vt and is replaced by the exponentials of s.  In
  // this order: with each product the vector instructions of one exponential, and with every fourth
  // the reads of the four fragments that the next four take, which arrive meanwhile.  (The compiler
  // waits for all reads wherever it needs one.)  k_next: K0 .. 3, read by the step before (READ: by
  // this one); LAST = 0: for the step behind it, which reads the same tile's other half.
  bf16x8 k_next[4];
  auto step = [&]<int NEXT, int LAST, bool READ>(const char *kt, const char *vt, f32x16 &s, f32x16 &next,
                                                 bf16x8 (&p)[2]) __attribute__((always_inline)) {
    bf16x8 fresh[2], even[4], odd[4];
    float sum[2] = {0.f, 0.f}, last = 0.f;
    asm volatile("" : "+v"(k_at), "+v"(v_at));   // (the places take a register each, not one per fragment)
    auto exponential = [&](int i) __attribute__((always_inline)) {
      const float x = fast_exp2(__builtin_fmaf(s[i], a.c1, -m));
      sum[i & 1] += x;
      if (i & 1) fresh[i >> 3][(i & 7) - 1] = (__bf16)last, fresh[i >> 3][i & 7] = (__bf16)x;
      last = x;
    };
    constexpr int SLOTS = 2 * NF;                // products
    constexpr int FIRST = READ ? 4 : 0;          // exponentials before them, while the first K arrives
    auto exponentials_at = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int i = FIRST + slot * (16 - FIRST) / SLOTS; i < FIRST + (slot + 1) * (16 - FIRST) / SLOTS; ++i) exponential(i);
    };
    next = f32x16{};
    if constexpr (READ) {
#pragma unroll
      for (int e = 0; e < 4; ++e) k_next[e] = k_frag(kt, NEXT, e);
#pragma unroll
      for (int i = 0; i < FIRST; ++i) exponential(i);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) even[e] = k_next[e];
#pragma unroll
    for (int slot = 0; slot < SLOTS; ++slot) {
      auto &mine = slot & 4 ? odd : even, &other = slot & 4 ? even : odd;
      if (slot < NF) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mine[slot & 3], q[slot], next, 0, 0, 0);
      else acc[slot % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mine[slot & 3], p[(slot - NF) / DB], acc[slot % DB], 0, 0, 0);
      if (slot % 4 == 0) {
        __builtin_amdgcn_sched_barrier(0);       // (behind the wait for what this product takes)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int to = slot + 4 + e;           // its product
          if (to < NF) other[e] = k_frag(kt, NEXT, to);
          else if (to < SLOTS) other[e] = v_frag(vt, 2 * LAST + (to - NF) / DB, to % DB);
          else if (LAST == 0) k_next[e] = k_frag(kt, 1 - NEXT, e);
        }
      }
      exponentials_at(slot);
      __builtin_amdgcn_sched_barrier(0);
    }
    p[0] = fresh[0], p[1] = fresh[1];
    settle(s, sum[0] + sum[1], p);
  };

  // The walk.  A segment without a page ends the fast loop: the split's tiles from there on go through the
  // one with masks (2048 tokens over 32768 bf16 keys 1007 us, with a page missing in the middle 1313, with the
  // first one missing 1641; 8-bit keys 1049 and, the first one, 1817).
  // When a tile's turn comes, p holds the exponentials of its first half and `next` the
  // logits of its second; afterwards they hold the next tile's.
  f32x16 s, next;
  bf16x8 p[2];
  uint32_t p_sees = 0;                           // what p's row sees (known where not all rows see all)

  auto turn = [&]<bool WORK, int BUF>(int tile) __attribute__((always_inline)) {
    char *ko = BUF ? k0_s : k1_s, *vt = BUF ? v1_s : v0_s;     // the next tile's K, this one's V
    arrive(ko, vt, true);
    __syncthreads();
    load_v.template operator()<1 - BUF>();
    find(tile + 2);
    load_k.template operator()<BUF>();
    pages = pages_of(tile + 3);
    const int w = tile + 3 - tile0;
    if (w % kWindow == 0) look_up(w / kWindow + 1);            // uniform
    if constexpr (WORK) {
      step.template operator()<0, 0, true>(ko, vt, next, s, p);
      step.template operator()<1, 1, false>(ko, vt, s, next, p);
    }
  };
  // Two tiles with one more behind them in the split, all of whose keys and of the first half of that
  // one's every row of the workgroup sees (`pages` are that one's).
  int plain_to = tile1 - 2;
  asm volatile("" : "+s"(plain_to));             // (else the code behind the loop is compiled once per way out of it)
  auto plain = [&](int tile) __attribute__((always_inline)) {
    return tile < plain_to && (tile + 2) * kPromptKeys + 31 <= g_to && tile > last_gap && !gap(pages);
  };
  // The other tiles, one product after the other.  A V value that is not finite must reach the rows that
  // see it only, but 0 times it is NaN: it takes a product of its own.
  auto second_product = [&](const char *vt, int half, bool all) __attribute__((always_inline)) {
    bf16x8 vf[2][DB];
    uint32_t wild = 0;                           // a carry out of an exponent of all ones
#pragma unroll
    for (int sixteen = 0; sixteen < 2; ++sixteen)
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        vf[sixteen][d] = v_frag(vt, 2 * half + sixteen, d);
        const uint4 w = __builtin_bit_cast(uint4, vf[sixteen][d]);
        auto out_of = [](uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; };
        wild |= out_of(w.x) | out_of(w.y) | out_of(w.z) | out_of(w.w);
      }
    if (!all && __any(wild != 0)) {              // uniform
#pragma unroll
      for (int sixteen = 0; sixteen < 2; ++sixteen) {
        bf16x8 seen;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          seen[i] = (__bf16)(p_sees >> (16 * sixteen + 8 * (i >> 2) + (i & 3)) & 1 ? 1.f : 0.f);
#pragma unroll
        for (int d = 0; d < DB; ++d) add_unbounded32(acc[d], vf[sixteen][d], seen);
      }
    }
#pragma unroll
    for (int sixteen = 0; sixteen < 2; ++sixteen)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[sixteen][d], p[sixteen], acc[d], 0, 0, 0);
  };
  auto logits = [&](const char *kt, int half) __attribute__((always_inline)) {
    f32x16 x = f32x16{};
#pragma unroll
    for (int f = 0; f < NF; ++f) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(kt, half, f), q[f], x, 0, 0, 0);
    return x;
  };
  auto masked = [&](const f32x16 &x, int tile, int half, uint32_t gone) __attribute__((always_inline)) {
    s = x;
    p_sees = sees(tile, half, gone);
    mask(s, p_sees);
    settle(s, INFINITY, p);
  };
  auto other = [&]<bool WORK>(int tile) __attribute__((always_inline)) {
    const bool odd = (tile - tile0) & 1;
    char *ko = odd ? k0_s : k1_s, *vt = odd ? v1_s : v0_s;
    const bool more = tile + 1 < tile1;          // uniform
    arrive(ko, vt, more);
    __syncthreads();
    if (more) odd ? load_v.template operator()<0>() : load_v.template operator()<1>();
    if (tile + 2 < tile1) {
      find(tile + 2);
      odd ? load_k.template operator()<1>() : load_k.template operator()<0>();
      pages = pages_of(tile + 3);                // (past the last tile: not used)
      const int w = tile + 3 - tile0;
      if (w % kWindow == 0) look_up(w / kWindow + 1);
    }
    if constexpr (WORK) {
      const bool all = (tile + 1) * kPromptKeys - 1 <= g_to && tile > last_gap;   // uniform
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        second_product(vt, half, all);
        if (half && !more) break;                // uniform
        masked(next, tile + half, 1 - half, gone_of(tile + half));
        if (more) next = logits(ko, half);
      }
    }
  };
  auto walk = [&]<bool WORK>() __attribute__((always_inline)) {
    look_up(0);
    look_up(1);
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    __syncthreads();
    pages = pages_of(tile0);
    find(tile0);
    load_k.template operator()<0>();
    load_v.template operator()<0>();
    if constexpr (WORK) load_q();                // (behind the first rows, which wait for their pages)
    if constexpr (FP8) {
      if (has && !is_v) widen(k0_s, 0, swizzle_k(b_row));
    } else {
      __builtin_amdgcn_s_waitcnt(0x0F70);
    }
    __syncthreads();                             // (it waits for all loads to LDS that are under way)
    if (tile0 + 1 < tile1) {
      pages = pages_of(tile0 + 1);
      find(tile0 + 1);
      load_k.template operator()<1>();
      pages = pages_of(tile0 + 2);
    }
    if constexpr (WORK) {
      masked(logits(k0_s, 0), tile0, 0, gone_of(tile0));
      next = logits(k0_s, 1);
    }
    int tile = tile0;
    while (plain(tile)) {                        // uniform
      turn.template operator()<WORK, 0>(tile++);
      turn.template operator()<WORK, 1>(tile++);
    }
    for (; tile < tile1; ++tile) other.template operator()<WORK>(tile);
  };
  // (waves without rows take part in the loads, and pass the same barriers)
  if (tile0 < tile1) working ? walk.template operator()<true>() : walk.template operator()<false>();   // uniform
  __syncthreads();                               // the buffers are done with

  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if (splits > 1) {                              // joined by pages_join_kernel
    const int64_t row = ((int64_t)at.slot + split) * a.part_rows + 32 * wave + c;
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
  // Each wave's 32 rows through LDS, so that whole rows go out in 16-byte lanes: the unit u of row r at
  // u ^ r.
  char *o_s = (wave / 2 == 0 ? k0_s : wave / 2 == 1 ? k1_s : wave / 2 == 2 ? v0_s : v1_s) + wave % 2 * 32 * RB;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<bf16x4 *>(o_s + c * RB + 16 * ((4 * d + (i >> 2)) ^ (c & (U - 1))) + 8 * h) =
          bf16x4{(__bf16)(acc[d][i] * inv), (__bf16)(acc[d][i + 1] * inv),
                 (__bf16)(acc[d][i + 2] * inv), (__bf16)(acc[d][i + 3] * inv)};
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32 * U / 64; ++i) {
    const int e = lane + 64 * i, row = e / U, u = e % U, rr = r0 + 32 * wave + row;
    if (rr < rows) {
      const int tk = rr / a.G, hd = g * a.G + (rr - tk * a.G);
      store16(to_global(a.out) + (((int64_t)(q0 + tk) * ((int64_t)a.c.Hkv * a.G) + hd) * D + 8 * u) * 2,
              *reinterpret_cast<const uint4 *>(o_s + row * RB + 16 * (u ^ (row & (U - 1)))));
    }
  }
}

void launch_pages_prompt(const PagesArgs &a, bool fp8, int head_dim, hipStream_t stream) {
  // Units in a run: half of what an XCD holds at a time, fewer where that would leave an XCD with
  // less than about 16 runs of unsplit blocks.
  const bool wide = a.rm_log2 == 8;
  const int run = std::clamp(a.blocks / 128, 1, wide ? 16 : 32);
  const dim3 grid((unsigned)(((int64_t)a.grid + 8 * run - 1) / (8 * run) * (8 * run)));
  auto go = [&]<int D, bool FP8, int NW>() {
    hipLaunchKernelGGL((pages_prompt_kernel<D, FP8, NW>), grid, dim3(64 * NW), 0, stream, a, run);
  };
  auto rows = [&]<int D, bool FP8>() {
    wide ? go.template operator()<D, FP8, 8>() : go.template operator()<D, FP8, 4>();
  };
  if (fp8) head_dim == 64 ? rows.template operator()<64, true>() : rows.template operator()<128, true>();
  else head_dim == 64 ? rows.template operator()<64, false>() : rows.template operator()<128, false>();
}

}  // namespace ckv
