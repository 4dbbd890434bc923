// The kernel behind launch_attend (attend.h).
//
//   z_s = c1 q . k_s,  P = 2^(z - m),  o = sum_s P_s v_s / sum_s P_s
//
// with m a running reference of the row.  Everything stays in the registers of
// one wave: a wave takes 32 keys (16 of fp32) at a time and works on the
// transposed products, so that what one matrix instruction leaves is what the
// next one reads:
//   S^T = K Q^T    lane 16 quad + c holds query row c against keys 4 quad + i of a
//                  16-key tile (element i): the operand P^T of
//   O^T = V^T P^T  whose reduction slots quad, 4 t + i are the keys 16 t + 4 quad + i; a lane
//                  supplies its eight keys' values of the head dimensions
//                  (D / 16) c + j for the j-th product, which is one short run of
//                  each V row, and its sums all belong to query row c, so that
//                  the softmax rescales them lane by lane.
// No shared memory is used in the loop and no wave waits for another; the
// waves of a workgroup, and the workgroups a row is split over, join their
// (reference, sum, output) at the end.
//
// 4-bit rows are widened by the conversion instructions to bf16, exactly, two
// values an instruction; bf16 products then run on the 16x16x32 instruction.
// fp32 rows run on the 16x16x4 fp32 instruction; fp32 queries over 4-bit rows
// are split into three bf16 parts (24 bits), which loses nothing.
// P goes into bf16 products, for bf16 queries, as two parts (16 bits): the loop
// waits for memory, so the second product costs nothing and the output is rounded
// once, at its end.
//
// Bound by memory where the rows are many: 8 caches of up to 131072 4-bit slots, D = 128,
// 28 / 4 heads, 98 us for 496 MB (5.0 TB/s; a copy reaches 4.9, a read 5.8), the CUs busy for
// 80% of the cycles, the vector pipe (which widens the rows) for 46%, the matrix pipe for
// 18%; single tokens in windows of 1028 keys, 256 groups of bf16, 24 us for 134 MB (5.6
// TB/s); four tokens over 16 caches of up to 3936 bf16 slots 29 us for 114 MB of rows and
// 24 MB of logits.  Shorter calls wait: for the chain of a few dependent loads
// (length, rows, the waves' join), and for the longest group, as every group has the same
// number of splits.  16 caches of up to 4096 4-bit slots, 32 / 8 heads, 17.3 us for 50 MB (2.9
// TB/s): CUs busy for 49%, vector pipe 22%, matrix pipe 7%.  The whole call with as many
// slots in all, uneven (a third of 4096 to all) and even: 16 caches 21.8 and 18.9 us,
// 64 caches 43.3 and 33.3 us.  One cache of 1001 slots 9.2 us.
#pragma once

#include "attend.h"
#include "row_blocks.h"
#include "score_common.h"

namespace ckv {

// A probability as two parts for bf16 products, off by 2^-16 of it at most: its upper
// bits, and the rest rounded.  Both are positive, so that neither makes a NaN of an
// infinite V value.
__device__ __forceinline__ void split_probability(float p, __bf16 (&part)[2]) {
  const uint32_t upper = __float_as_uint(p) & 0xFFFF0000u;
  part[0] = __builtin_bit_cast(__bf16, (uint16_t)(upper >> 16));
  part[1] = (__bf16)fmaxf(p - __uint_as_float(upper), p * 0x1p-24f);
}

// The parts that a value is split into before a bf16 product: 1 exact, 2 (16
// bits of mantissa) or 3 (24 bits).
template <int PARTS>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&p)[PARTS]) {
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    p[i] = (__bf16)x;
    x -= (float)p[i];
  }
}

// A key that some rows of a tile see and others do not may hold anything in its
// V row, but 0 * infinity in a product would give the others NaN.  Where such a
// key holds a value that is not finite, the product takes a zero in its place,
// and what the rows that see it get is added here: how many visible +infinities,
// -infinities and NaN stand in the place of each output.
__device__ __forceinline__ void add_unbounded(f32x4 &acc, f32x4 up, f32x4 down, f32x4 none) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (up[i] > 0.f) acc[i] += INFINITY;
    if (down[i] > 0.f) acc[i] -= INFINITY;
    if (none[i] > 0.f) acc[i] = NAN;
  }
}

constexpr int64_t kNearStride = 1 << 24;   // bytes between rows: 64 of them stay within 32 bits

template <CacheType CT, int D>
struct AttendShape {
  static constexpr int NT = CT == kCacheF32 ? 1 : 2;     // 16-key tiles per step
  static constexpr int KS = 16 * NT;                     // keys per step
  static constexpr int NK = CT == kCacheF32 ? D / 16 : D / 32;   // K fragments per row
  static constexpr int DL = D / 16;                      // head dimensions per lane in V
  static constexpr int VW = CT == kCacheFp4 ? 1 : DL * (CT == kCacheF32 ? 4 : 2) / 4;   // dwords
};

// What a lane loads for one step.
template <CacheType CT, int D>
struct AttendRaw {
  using S = AttendShape<CT, D>;
  uint4 k[S::NT][CT == kCacheFp4 ? 1 : S::NK];
  uint32_t v[S::NT][4][S::VW];
  uint32_t ks[S::NT];                 // 4-bit: the scale byte of the lane's K values
  uint32_t vs[S::NT][4];              // 4-bit: the scale bytes of its four V rows
  int4 pos[S::NT];                    // several query tokens: positions of its four keys
};

// Q fragments as the products take them.
template <CacheType CT, int D, int RT, int QP>
struct AttendQ {
  bf16x8 h[CT == kCacheF32 ? 1 : RT][QP][CT == kCacheF32 ? 1 : AttendShape<CT, D>::NK];
  f32x4 f[CT == kCacheF32 ? RT : 1][CT == kCacheF32 ? AttendShape<CT, D>::NK : 1];
};

// QP: parts of a query (1: bf16 queries, or fp32 ones over fp32 rows; 3: fp32
// queries over 4-bit rows).  MASKS: rows of a workgroup may see different keys.
// ONE: a workgroup of eight waves takes all keys of its rows and, over a cache,
// adds to the weights itself, from logits held in LDS: one launch and no
// workspace, for few keys.
template <AttendSource SRC, CacheType CT, int D, int RT, int QP, bool MASKS, bool ONE>
__global__ __launch_bounds__(64 * (ONE ? 2 : 1) * kAttendWaves) void attend_kernel(const AttendArgs a) {
  constexpr int NW = (ONE ? 2 : 1) * kAttendWaves, NTH = 64 * NW;
  // steps whose rows are in registers or under way, as many as the registers hold (16
  // caches of up to 4096 4-bit slots with one step, then two: 27.2, 23.6 us a call)
  constexpr int DEPTH = (ONE && MASKS) || (CT != kCacheFp4 && RT >= 2) ? 1
                        : 2;
  using S = AttendShape<CT, D>;
  constexpr bool F32Q = CT == kCacheF32 || QP == 3;
  constexpr int NT = S::NT, KS = S::KS, NK = S::NK, DL = S::DL, VW = S::VW;
  constexpr int PP = QP == 3 ? 3 : 2;           // parts of P
  constexpr int RM = 16 * RT;
  extern __shared__ __align__(16) float logit_s[];  // ONE: [rows][logit_stride]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, quad = lane >> 4;
  const int split = blockIdx.z;
  int rb = blockIdx.x, b = (int)blockIdx.y / a.Hkv, g = (int)blockIdx.y - b * a.Hkv;
  int part = (int)blockIdx.y * a.row_blocks + rb;   // the row block's number
  if constexpr (SRC == kOverWindow && MASKS && !ONE) {
    if (a.packed) {
      RowBlock found;
      if (!find_row_block<false>(a, rb, RM, found)) return;   // uniform
      rb = found.rb, b = found.b, g = found.g, part = found.part;
    }
  }
  const int bg = b * a.Hkv + g;

  // the rows of this workgroup and the keys that any of them sees
  int rows, n, t_first = 0, t_last = 0, lo = 0, sinks = 0;
  int q0 = 0, k0 = 0;
  if constexpr (SRC == kOverCache) {
    rows = a.rows;
    n = live_slots(a.c, bg);
    t_first = (int)((uint32_t)a.c.seen[bg] - (uint32_t)a.n_q);   // position of query token 0
  } else {
    q0 = a.cu_q[b];
    k0 = a.cu_k[b];
    const int lq = a.cu_q[b + 1] - q0, lk = a.cu_k[b + 1] - k0;
    rows = lq * a.G;
    if (rb * RM >= rows) return;                // uniform
    t_first = lk - lq + rb * RM / a.G;
    t_last = lk - lq + (min(rows, rb * RM + RM) - 1) / a.G;
    lo = max(0, t_first - a.window + 1);
    sinks = min(a.sinks, lo);                   // sinks outside the window come first
    n = t_last < 0 ? 0 : sinks + t_last - lo + 1;
  }
  // virtual key x in [0, n) -> its row
  auto key_of = [&](int x) {
    if constexpr (SRC == kOverCache) return x;
    else return x < sinks ? x : x - sinks + lo;
  };
  const int steps = (n + KS - 1) / KS, per = (steps + a.splits - 1) / a.splits;
  const int st0 = min(steps, split * per), st1 = min(steps, st0 + per);

  // address of query row r (row tile rt, column c); rows past the end are zero
  auto row_ptr = [&](const char *base, int r, bool dense) {
    const int i = r / a.G, h = g * a.G + (r - i * a.G);
    constexpr int64_t size = F32Q ? 4 : 2;
    if constexpr (SRC == kOverCache)
      return base + (((int64_t)b * a.n_q + i) * ((int64_t)a.Hkv * a.G) + h) * (D * size);
    else if (dense)
      return base + ((int64_t)(q0 + i) * ((int64_t)a.Hkv * a.G) + h) * (D * size);
    else
      return base + (int64_t)(q0 + i) * a.q_tok + h * a.q_head;
  };

  // positions of the lane's rows (row tile rt, column c); rows past the end as the last
  int t_row[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(rb * RM + 16 * rt + c, rows - 1);
    if constexpr (SRC == kOverCache) t_row[rt] = t_first + r / a.G;
    else t_row[rt] = t_first - rb * RM / a.G + r / a.G;
  }

  // row bases
  const char *kb, *vb;
  int64_t k_row, v_row;
  if constexpr (SRC == kOverCache) {
    k_row = v_row = CT == kCacheFp4 ? D / 2 : D * (CT == kCacheF32 ? 4 : 2);
    kb = a.c.k + (int64_t)bg * a.c.capacity * k_row;
    vb = a.c.v + (int64_t)bg * a.c.capacity * v_row;
  } else {
    k_row = a.k_tok;
    v_row = a.v_tok;
    kb = a.k + k0 * a.k_tok + g * a.k_head;
    vb = a.v + k0 * a.v_tok + g * a.v_head;
  }
  // Bytes that a lane takes of a K row (16 each) and of a V row, and its places in
  // the first tile of a step: offsets in 32 bits, to a base that all lanes share.
  constexpr int VB = CT == kCacheFp4 ? DL / 2 : DL * (CT == kCacheF32 ? 4 : 2);
  constexpr int KB = CT == kCacheFp4 ? D / 8 : 16;
  const bool near = SRC == kOverCache || (k_row <= kNearStride && v_row <= kNearStride);
  const uint32_t k_off = near ? (uint32_t)(c * (int)k_row + KB * quad) : 0;
  const uint32_t v_off = near ? (uint32_t)(4 * quad * (int)v_row + VB * c) : 0;
  auto load_k = [&](gptr<const char> p, uint4 (&k)[CT == kCacheFp4 ? 1 : NK]) {
    if constexpr (CT == kCacheFp4 && D == 64) {
      const uint64_t h = *reinterpret_cast<gptr<const uint64_t>>(p);
      k[0] = make_uint4((uint32_t)h, (uint32_t)(h >> 32), 0, 0);
    } else if constexpr (CT == kCacheFp4) {
      k[0] = load16(p);
    } else {
#pragma unroll
      for (int s = 0; s < NK; ++s) k[s] = load16(p + 64 * s);
    }
  };
  auto load_v = [&](gptr<const char> p, uint32_t (&v)[VW]) {
    if constexpr (VB == 2) {
      v[0] = *reinterpret_cast<gptr<const uint16_t>>(p);
    } else if constexpr (VB == 4) {
      v[0] = *reinterpret_cast<gptr<const uint32_t>>(p);
    } else if constexpr (VB == 8) {
      const uint64_t h = *reinterpret_cast<gptr<const uint64_t>>(p);
      v[0] = (uint32_t)h, v[VW - 1] = (uint32_t)(h >> 32);
    } else {
#pragma unroll
      for (int u = 0; u < VB / 16; ++u) {
        const uint4 h = load16(p + 16 * u);
        v[4 * u] = h.x, v[4 * u + 1] = h.y, v[4 * u + 2] = h.z, v[4 * u + 3] = h.w;
      }
    }
  };

  // Loads of step st (uniform).  Of a cache any slot can be read, dead ones too; past
  // the last one, and past the last key of a window, the last one is.
  const int end = SRC == kOverCache ? a.c.capacity : n;
  auto load = [&](int st, AttendRaw<CT, D> &w) {
    const int base = st * KS;
    if (CT == kCacheFp4 || (near && base + KS <= end && base >= sinks)) {   // uniform: a run of rows
      const char *kt = kb + (int64_t)(base - sinks + lo) * k_row, *vt = vb + (int64_t)(base - sinks + lo) * v_row;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        load_k(to_global(kt + 16 * t * k_row) + k_off, w.k[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_v(to_global(vt + (16 * t + i) * v_row) + v_off, w.v[t][i]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        load_k(to_global(kb) + key_of(min(base + 16 * t + c, end - 1)) * k_row + KB * quad, w.k[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          load_v(to_global(vb) + key_of(min(base + 16 * t + 4 * quad + i, end - 1)) * v_row + VB * c, w.v[t][i]);
      }
    }
    if constexpr (CT == kCacheFp4) {
      const int64_t slot0 = (int64_t)bg * a.c.capacity + base;
      const uint8_t *ks = a.c.k_scale + slot0 * (D / 32), *vs = a.c.v_scale + slot0 * (D / 32);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        w.ks[t] = (to_global(ks + 16 * t * (D / 32)))[(uint32_t)(c * (D / 32) + (D == 128 ? quad : quad >> 1))];
        const gptr<const char> p = to_global(reinterpret_cast<const char *>(vs) + 16 * t * (D / 32)) +
                                   (uint32_t)(4 * quad * (D / 32));
        if constexpr (D == 128) {
          const uint4 h = load16(p);
          w.vs[t][0] = h.x, w.vs[t][1] = h.y, w.vs[t][2] = h.z, w.vs[t][3] = h.w;
        } else {
          const uint64_t h = *reinterpret_cast<gptr<const uint64_t>>(p);
#pragma unroll
          for (int i = 0; i < 4; ++i) w.vs[t][i] = (uint32_t)(h >> (16 * i)) & 0xFFFFu;
        }
      }
    }
    if constexpr (MASKS && SRC == kOverCache) {
      const gptr<const int32_t> p = to_global(a.c.pos + (int64_t)bg * a.c.capacity);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int s = base + 16 * t + 4 * quad;
        w.pos[t] = make_int4(p[min(s, end - 1)], p[min(s + 1, end - 1)], p[min(s + 2, end - 1)],
                             p[min(s + 3, end - 1)]);
      }
    }
  };

  // the first steps' loads, before everything else that waits for memory; in one
  // workgroup they do not depend on the length
  AttendRaw<CT, D> w[DEPTH];
  {
    const int first = ONE && SRC == kOverCache ? wave : st0 + wave;
    const int stop = ONE && SRC == kOverCache ? (a.c.capacity + KS - 1) / KS : st1;
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (first + i * NW < stop) load(first + i * NW, w[i]);
  }

  AttendQ<CT, D, RT, QP> q;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rb * RM + 16 * rt + c;
    const bool in = r < rows;
    const gptr<const char> p = to_global(row_ptr(a.q, in ? r : rb * RM, false));
    if constexpr (CT == kCacheF32) {
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        const uint4 w = load16(p + (16 * s + 4 * quad) * 4);
        q.f[rt][s] = in ? __builtin_bit_cast(f32x4, w) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    } else {
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        const int d = CT == kCacheFp4 ? (D / 4) * quad + 8 * s : 32 * s + 8 * quad;
        if constexpr (QP == 1) {
          const uint4 w = load16(p + d * 2);
          q.h[rt][0][s] = __builtin_bit_cast(bf16x8, in ? w : make_uint4(0, 0, 0, 0));
        } else {
          const f32x4 x0 = __builtin_bit_cast(f32x4, load16(p + d * 4));
          const f32x4 x1 = __builtin_bit_cast(f32x4, load16(p + d * 4 + 16));
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 part[QP];
            split_bf16<QP>(in ? (e < 4 ? x0[e & 3] : x1[e & 3]) : 0.f, part);
#pragma unroll
            for (int w = 0; w < QP; ++w) q.h[rt][w][s][e] = part[w];
          }
        }
      }
    }
  }
  float m[RT], l[RT];
  f32x4 acc[RT][DL];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int j = 0; j < DL; ++j) acc[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  auto compute = [&](int st, AttendRaw<CT, D> &w) {
    const int base = st * KS;
    // ---- logits
    f32x4 s[RT][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (CT == kCacheF32) {
#pragma unroll
        for (int f = 0; f < NK; ++f) {
          const f32x4 kf = __builtin_bit_cast(f32x4, w.k[t][f]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q.f[rt][f][e], s[rt][t], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int f = 0; f < NK; ++f) {
          bf16x8 kf;
          if constexpr (CT == kCacheFp4) {
            const uint32_t word = f == 0 ? w.k[t][0].x : f == 1 ? w.k[t][0].y
                                  : f == 2 ? w.k[t][0].z : w.k[t][0].w;
            kf = __builtin_bit_cast(bf16x8, fp4_values(word, fp4_scale(w.ks[t])));
          } else {
            kf = __builtin_bit_cast(bf16x8, w.k[t][f]);
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int part = 0; part < QP; ++part)
              s[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q.h[rt][part][f], s[rt][t], 0, 0, 0);
        }
      }
    }
    // ---- masks (uniform: none in most steps)
    const bool tail = base + KS > n;
    bool partial = false;                          // some key is seen by some rows only
    if constexpr (MASKS && SRC == kOverCache) {
      partial = true;
    } else if constexpr (MASKS) {
      const int j0 = key_of(base), j1 = key_of(min(base + KS, n) - 1);
      partial = !(j1 <= t_first && (j0 > t_last - a.window || j1 < a.sinks));
    }
    if (tail || partial) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int x = base + 16 * t + 4 * quad + i;
          const bool live = x < n;
          int j;
          if constexpr (!MASKS) {
            j = 0;
          } else if constexpr (SRC == kOverCache) {
            const int p4[4] = {w.pos[t].x, w.pos[t].y, w.pos[t].z, w.pos[t].w};
            j = p4[i];
          } else {
            j = key_of(x);
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            bool sees = live;
            if (MASKS && partial) {
              sees = sees && j <= t_row[rt];
              if constexpr (SRC == kOverWindow)
                sees = sees && (j > t_row[rt] - a.window || j < a.sinks);
            }
            s[rt][t][i] = sees ? s[rt][t][i] : -INFINITY;
          }
          if (!live) {                             // such a V row counts as zeros
#pragma unroll
            for (int u = 0; u < VW; ++u) w.v[t][i][u] = 0;
            if constexpr (CT == kCacheFp4) w.vs[t][i] = 0x7F7F7F7Fu;
          }
        }
    }
    if constexpr (SRC == kOverCache) {
      if (a.accumulate) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const int r = rb * RM + 16 * rt + c;
          if (r < rows) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              float *z;
              if constexpr (ONE) z = logit_s + r * (int)a.logit_stride;
              else z = a.logits + ((int64_t)bg * rows + r) * a.logit_stride;
              *reinterpret_cast<f32x4 *>(z + base + 16 * t + 4 * quad) = s[rt][t];
            }
          }
        }
      }
    }
    // ---- softmax: the reference moves only when a logit passes it by 2^8
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = s[rt][0][0];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[rt][t][i]);
      top *= a.c1;
      if (__any(top > m[rt] + 8.f)) {
        const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top),
                                                          false, false);
        top = fmaxf(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
        const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top),
                                                          false, false);
        top = fmaxf(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
        const float next = fmaxf(m[rt], top);
        const float shrink = m[rt] == next ? 1.f : fast_exp2(m[rt] - next);
        l[rt] *= shrink;
#pragma unroll
        for (int j = 0; j < DL; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[rt][j][i] *= shrink;
        m[rt] = next;
      }
    }
    f32x4 p[RT][NT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float ref = m[rt] == -INFINITY ? 0.f : m[rt];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[rt][t][i] = fast_exp2(__builtin_fmaf(s[rt][t][i], a.c1, -ref));
          l[rt] += p[rt][t][i];
        }
    }
    // ---- P V
    if constexpr (CT == kCacheF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DL; ++j) {
          float vv = __uint_as_float(w.v[0][i][j]);
          if (MASKS && partial && __any(!(fabsf(vv) < INFINITY))) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              const float sees = s[rt][0][i] != -INFINITY ? 1.f : 0.f;
              const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
              add_unbounded(acc[rt][j],
                            __builtin_amdgcn_mfma_f32_16x16x4f32(vv == INFINITY ? 1.f : 0.f, sees, zero, 0, 0, 0),
                            __builtin_amdgcn_mfma_f32_16x16x4f32(vv == -INFINITY ? 1.f : 0.f, sees, zero, 0, 0, 0),
                            __builtin_amdgcn_mfma_f32_16x16x4f32(vv != vv ? 1.f : 0.f, sees, zero, 0, 0, 0));
            }
            vv = fabsf(vv) < INFINITY ? vv : 0.f;
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            acc[rt][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv, p[rt][0][i], acc[rt][j], 0, 0, 0);
        }
    } else {
      // the V rows as pairs of bf16
      uint32_t u[8][DL / 2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (CT == kCacheFp4) {
            const int block = D == 128 ? c >> 2 : c >> 3;
            const float sc = fp4_scale(__builtin_amdgcn_ubfe(w.vs[t][i], 8 * block, 8));
            const uint4 x = fp4_values(w.v[t][i][0], sc);
            u[4 * t + i][0] = x.x, u[4 * t + i][1] = x.y;
            if constexpr (DL == 8) u[4 * t + i][DL / 2 - 2] = x.z, u[4 * t + i][DL / 2 - 1] = x.w;
          } else {
#pragma unroll
            for (int h = 0; h < VW; ++h) u[4 * t + i][h] = w.v[t][i][h];
          }
        }
      bf16x8 pf[RT][PP];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          __bf16 part[PP];
          if constexpr (PP == 2) split_probability(p[rt][e >> 2][e & 3], part);
          else split_bf16<PP>(p[rt][e >> 2][e & 3], part);
#pragma unroll
          for (int x = 0; x < PP; ++x) pf[rt][x][e] = part[x];
        }
      // the j-th value of the eight rows
      auto v_frag = [&](int j) {
        uint4 x;
        const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
        x.x = __builtin_amdgcn_perm(u[1][j / 2], u[0][j / 2], sel);
        x.y = __builtin_amdgcn_perm(u[3][j / 2], u[2][j / 2], sel);
        x.z = __builtin_amdgcn_perm(u[5][j / 2], u[4][j / 2], sel);
        x.w = __builtin_amdgcn_perm(u[7][j / 2], u[6][j / 2], sel);
        return __builtin_bit_cast(bf16x8, x);
      };
      if (MASKS && partial) {
        uint32_t wild = 0;                         // a carry out of an exponent of all ones
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int h = 0; h < DL / 2; ++h) wild |= ((u[e][h] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
        if (__any(wild != 0)) {
#pragma unroll
          for (int j = 0; j < DL; ++j) {
            const bf16x8 vf = v_frag(j);
            bf16x8 up, down, none;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float f = (float)vf[e];
              up[e] = (__bf16)(f == INFINITY ? 1.f : 0.f);
              down[e] = (__bf16)(f == -INFINITY ? 1.f : 0.f);
              none[e] = (__bf16)(f != f ? 1.f : 0.f);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              bf16x8 sees;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                sees[e] = (__bf16)(s[rt][e >> 2][e & 3] != -INFINITY ? 1.f : 0.f);
              const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
              add_unbounded(acc[rt][j], __builtin_amdgcn_mfma_f32_16x16x32_bf16(up, sees, zero, 0, 0, 0),
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(down, sees, zero, 0, 0, 0),
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(none, sees, zero, 0, 0, 0));
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int h = 0; h < DL / 2; ++h) {
              if ((u[e][h] & 0x7F80u) == 0x7F80u) u[e][h] &= 0xFFFF0000u;
              if ((u[e][h] & 0x7F800000u) == 0x7F800000u) u[e][h] &= 0xFFFFu;
            }
        }
      }
#pragma unroll
      for (int j = 0; j < DL; ++j) {
        const bf16x8 vf = v_frag(j);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int part = 0; part < PP; ++part)
            acc[rt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rt][part], acc[rt][j], 0, 0, 0);
      }
    }
  };

  // ---- the wave's steps: each one's registers are loaded again as soon as it is done
  {
    int st = st0 + wave;
    while (st < st1) {
      bool done = false;
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        if (done) continue;
        compute(st, w[i]);
        if (st + DEPTH * NW < st1) load(st + DEPTH * NW, w[i]);
        st += NW;
        done = st >= st1;
      }
    }
  }

  // ---- join the waves: of every lane's output, four runs of DL head dimensions, one
  // after the other (in one workgroup, which waits for this, all at once)
  constexpr int RUNS = ONE ? 4 : 1;
  constexpr int OS = 4 * DL * RUNS + 4;            // padded row of RUNS runs of the four quads
  __shared__ __align__(16) float o_s[NW][16][OS];
  __shared__ float2 ml_s[NW][RM];
  __shared__ float2 row_s[RM];                     // (reference, 1 / sum) of the joined rows
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = quad_sum(l[rt]);
    if (quad == 0) ml_s[wave][16 * rt + c] = make_float2(m[rt], l[rt]);
  }
  __syncthreads();
  const int64_t slot = (int64_t)part * a.splits + split;
  if (tid < RM) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ml_s[w][tid].x);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(ml_s[w][tid].x - ref);
      sum += ml_s[w][tid].y * f;
      ml_s[w][tid].x = f;                          // the wave's share from here on
    }
    row_s[tid] = make_float2(ref, sum == 0.f ? 0.f : 1.f / sum);
    if (!ONE && (a.splits > 1 || a.accumulate) && rb * RM + tid < rows)
      a.part_ml[slot * RM + tid] = make_float2(top, sum);
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int i0 = 0; i0 < 4; i0 += RUNS) {
      if (rt || i0) __syncthreads();
#pragma unroll
      for (int i = i0; i < i0 + RUNS; ++i)
#pragma unroll
        for (int j = 0; j < DL; j += 4)
          *reinterpret_cast<f32x4 *>(&o_s[wave][c][DL * (4 * (i - i0) + quad) + j]) =
              f32x4{acc[rt][j][i], acc[rt][j + 1][i], acc[rt][j + 2][i], acc[rt][j + 3][i]};
      __syncthreads();
      // 16 rows of 4 DL RUNS values, four to a thread: value DL (4 i + quad) + j of a run is
      // head dimension DL (4 quad + i) + j
      for (int e = tid; e < 16 * DL * RUNS; e += NTH) {
        const int row = e / (DL * RUNS), x = 4 * (e % (DL * RUNS)), part = x / DL;
        const int d = DL * (4 * (part % 4) + i0 + part / 4) + x % DL;
        const int r = rb * RM + 16 * rt + row;
        if (r >= rows) break;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float f = ml_s[w][16 * rt + row].x;
          const f32x4 v = *reinterpret_cast<const f32x4 *>(&o_s[w][row][x]);
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] += v[k] * f;
        }
        if (!ONE && a.splits > 1) {
          *reinterpret_cast<f32x4 *>(a.part_o + (slot * RM + 16 * rt + row) * D + d) = o;
        } else {
          const float inv = row_s[16 * rt + row].y;
          char *to = const_cast<char *>(row_ptr(a.out, r, true)) + d * (F32Q ? 4 : 2);
          if constexpr (F32Q) {
            *reinterpret_cast<f32x4 *>(to) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
          } else {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4 *>(to) = bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv),
                                                     (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
          }
        }
      }
    }
  if constexpr (ONE && SRC == kOverCache) {        // (one row block)
    if (a.accumulate)
      for (int x = tid; x < n; x += NTH) {
        // (a row whose sum is a NaN gives nothing to a slot that it does not see)
        const int32_t pos = MASKS ? a.c.pos[(int64_t)bg * a.c.capacity + x] : INT32_MIN;
        float got = 0.f;
        int t = t_first, h = 0;
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
          const float p = fast_exp2(__builtin_fmaf(logit_s[r * (int)a.logit_stride + x], a.c1, -row_s[r].x)) *
                          row_s[r].y;
          got += pos <= t ? p : 0.f;
          if (++h == a.G) h = 0, ++t;
        }
        a.c.weight[(int64_t)bg * a.c.capacity + x] += got;
      }
  }
}

template <AttendSource SRC, CacheType CT, int D, int RT, int QP, bool MASKS, bool ONE>
void launch_attend_as(const AttendArgs &a, dim3 grid, hipStream_t stream) {
  const size_t lds = ONE && a.accumulate ? (size_t)a.rows * a.logit_stride * sizeof(float) : 0;
  hipLaunchKernelGGL((attend_kernel<SRC, CT, D, RT, QP, MASKS, ONE>), grid,
                     dim3(64 * (ONE ? 2 : 1) * kAttendWaves), lds, stream, a);
}

}  // namespace ckv
