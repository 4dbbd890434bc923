// The bounded cache's store (include/compresskv_cache.h): rows in (from a
// compressed prompt, or a decoding step's tokens), rows out, and the eviction
// of the slots of least accumulated weight.
//
//   cache_load_kernel     kept rows of a prompt into slots 0 ..
//   cache_append_kernel   new tokens' rows behind the live slots
//   cache_len_kernel      ... and the lengths, where several workgroups append
//   cache_read_kernel     rows as bf16 or fp32 values
//   evict_kernel          which slots go, which kept slots take their place, and
//                         the moves, where they can only be few
//   evict_move_kernel     the moves alone
#include <hip/hip_runtime.h>

#include <algorithm>

#include "api_common.h"
#include "cache_api.h"
#include "cache_device.h"

namespace ckv {

// Eight consecutive values of a row, as loaded.
template <typename T>
__device__ __forceinline__ void load8(gptr<const char> p, uint4 (&raw)[sizeof(T) / 2]) {
  raw[0] = load16(p);
  if constexpr (sizeof(T) == 4) raw[1] = load16(p + 16);
}

template <typename T>
__device__ __forceinline__ void values8(const uint4 (&raw)[sizeof(T) / 2], float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    x[0] = __uint_as_float(raw[0].x), x[1] = __uint_as_float(raw[0].y);
    x[2] = __uint_as_float(raw[0].z), x[3] = __uint_as_float(raw[0].w);
    x[4] = __uint_as_float(raw[1].x), x[5] = __uint_as_float(raw[1].y);
    x[6] = __uint_as_float(raw[1].z), x[7] = __uint_as_float(raw[1].w);
  } else {
    const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

// Values 8u .. 8u + 7 of a row into slot `slot` (over all groups) of rows / scales.  The
// four lanes of a 4-bit block stand next to each other and call this together.
template <typename T, int D, bool FP4>
__device__ __forceinline__ void store8(char *rows, uint8_t *scales, int64_t slot, int u,
                                       const uint4 (&raw)[sizeof(T) / 2]) {
  if constexpr (!FP4) {
    const gptr<char> to = to_global(rows) + (slot * D + 8 * u) * (int64_t)sizeof(T);
    store16(to, raw[0]);
    if constexpr (sizeof(T) == 4) store16(to + 16, raw[1]);
  } else {
    float x[8];
    values8<T>(raw, x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t byte = fp4_scale_byte(top);
    reinterpret_cast<uint32_t *>(rows)[slot * (D / 8) + u] = fp4_codes(x, byte);
    if ((u & 3) == 0) scales[slot * (D / 32) + (u >> 2)] = (uint8_t)byte;
  }
}

struct LoadArgs {
  CacheView c;
  const char *k, *v;
  const int32_t *idx, *cu;
  int64_t rows_per_b;           // source rows per sequence
  int32_t n_rows;               // per group (0: ragged)
  int32_t off[kMaxKvHeads + 1]; // ragged: first row of a group within its sequence
};

constexpr int kUnits = 4;           // 8-value units that a lane of a load or read takes

// Grid (blocks, groups, 3), 256 threads.  z = 0, 1: the group's K, V rows, a lane per 8
// values and kUnits of these, so that a wave reads 1 KB (bf16) in a row; all
// positions are asked for before the rows, and rows that were not kept are not
// read.  z = 2: the first workgroup counts the kept rows.  Bound by HBM: 2 D values
// read, a 4-bit row written: 64 groups of 2048 rows of bf16, D = 128, 16.0 us (5.3 TB/s), of
// 16384 rows 126 us.  (2, 4, 8 units a lane: 16.3, 16.0, 15.0 and 136, 126, 132 us.  A grid
// over the groups: 64-bit divisions of a flat index took longer than the rows.)
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void cache_load_kernel(const LoadArgs a) {
  const int tid = threadIdx.x, bg = blockIdx.y;
  const int b = bg / a.c.Hkv, g = bg - b * a.c.Hkv;
  constexpr int U = D / 8;                       // lanes per row
  const int n = a.n_rows ? a.n_rows : a.off[g + 1] - a.off[g];
  const int64_t row0 = (int64_t)b * a.rows_per_b + (a.n_rows ? (int64_t)g * a.n_rows : (int64_t)a.off[g]);
  const int32_t *idx = a.idx + row0;
  if (blockIdx.z == 2) {
    if (blockIdx.x) return;                      // uniform
    int kept = 0;
#pragma unroll 4
    for (int j = tid; j < n; j += 256) kept += idx[j] >= 0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) kept += __shfl_xor(kept, o);
    __shared__ int part[4];
    if ((tid & 63) == 0) part[tid >> 6] = kept;
    __syncthreads();
    if (tid == 0) {
      a.c.len[bg] = part[0] + part[1] + part[2] + part[3];
      a.c.seen[bg] = a.cu[b + 1] - a.cu[b];
    }
    return;
  }
  const bool is_v = blockIdx.z == 1;
  const gptr<const char> src = to_global(is_v ? a.v : a.k) + row0 * (D * (int64_t)sizeof(T));
  const int u = tid % U, j0 = (int)blockIdx.x * (256 / U * kUnits) + tid / U;
  int32_t position[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int j = j0 + 256 / U * i;
    position[i] = j < n ? idx[j] : -1;
  }
  uint4 raw[kUnits][sizeof(T) / 2];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
    if (position[i] >= 0)
      load8<T>(src + ((int64_t)(j0 + 256 / U * i) * U + u) * (8 * (int64_t)sizeof(T)), raw[i]);
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (position[i] < 0) continue;               // the four lanes of a block agree
    const int64_t slot = (int64_t)bg * a.c.capacity + j0 + 256 / U * i;
    store8<T, D, FP4>(is_v ? a.c.v : a.c.k, is_v ? a.c.v_scale : a.c.k_scale, slot, u, raw[i]);
    if (!is_v && u == 0) {
      a.c.pos[slot] = position[i];
      a.c.weight[slot] = 0.f;
    }
  }
}

struct AppendArgs {
  CacheView c;
  const char *k, *v;
  int64_t ks[3], vs[3];         // byte strides: sequence, token, head
  int32_t n_new;
  int32_t own_len;              // the group's one workgroup updates len and seen
};

// Grid (groups, blocks per group), 256 or 1024 threads: a lane per 8 values of a K or
// V row.  Bound by latency at a decoding step's one token: 2.2 us for 2 groups, 3.1 us
// for 512.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(1024) void cache_append_kernel(const AppendArgs a) {
  constexpr int U = D / 8;
  const int ROWS = (int)blockDim.x / (2 * U);      // tokens per workgroup and trip
  const int tid = threadIdx.x, bg = blockIdx.x;
  const int b = bg / a.c.Hkv, g = bg - b * a.c.Hkv;
  const int len = live_slots(a.c, bg);
  const int32_t seen = a.c.seen[bg];
  const bool is_v = (tid / U) & 1;
  const int u = tid % U;
  const int64_t *st = is_v ? a.vs : a.ks;
  const char *src = (is_v ? a.v : a.k) + b * st[0] + g * st[2] + u * (8 * (int64_t)sizeof(T));
  const int n = min(a.n_new, a.c.capacity - len);   // rows that fit
  for (int i = (int)blockIdx.y * ROWS + tid / (2 * U); i < n; i += (int)gridDim.y * ROWS) {
    uint4 raw[sizeof(T) / 2];
    load8<T>(to_global(src) + i * st[1], raw);
    const int64_t slot = (int64_t)bg * a.c.capacity + len + i;
    store8<T, D, FP4>(is_v ? a.c.v : a.c.k, is_v ? a.c.v_scale : a.c.k_scale, slot, u, raw);
    if (!is_v && u == 0) {
      a.c.pos[slot] = (int32_t)((uint32_t)seen + (uint32_t)i);
      a.c.weight[slot] = 0.f;
    }
  }
  if (a.own_len) {
    __syncthreads();             // every thread has read len and seen
    if (tid == 0) {
      a.c.len[bg] = len + n;
      a.c.seen[bg] = (int32_t)((uint32_t)seen + (uint32_t)a.n_new);
    }
  }
}

__global__ __launch_bounds__(256) void cache_len_kernel(const CacheView c, int n_new) {
  const int bg = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (bg >= c.groups) return;
  const int len = live_slots(c, bg);
  c.len[bg] = len + min(n_new, c.capacity - len);
  c.seen[bg] = (int32_t)((uint32_t)c.seen[bg] + (uint32_t)n_new);
}

// Grid (blocks, groups, 2), 256 threads: K (z = 0) or V, a lane per 8 values and kUnits
// of these.  Bound by HBM: 64 groups of 2048 4-bit rows to bf16 13.8 us (6.1 TB/s, partly
// out of the caches), of 16384 rows 114 us.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheView c, char *k_out,
                                                         char *v_out) {
  constexpr int U = D / 8;
  const bool is_v = blockIdx.z == 1;
  const int bg = blockIdx.y, live = live_slots(c, bg), u = threadIdx.x % U;
  const int j0 = (int)blockIdx.x * (256 / U * kUnits) + (int)threadIdx.x / U;
  const char *rows = is_v ? c.v : c.k;
  const uint8_t *scales = is_v ? c.v_scale : c.k_scale;
  const int64_t slot0 = (int64_t)bg * c.capacity + j0;
  uint4 raw[kUnits][sizeof(T) / 2] = {};
  uint32_t code[kUnits] = {}, byte[kUnits] = {};
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int64_t slot = slot0 + 256 / U * i;
    if (j0 + 256 / U * i >= live) continue;
    if constexpr (FP4) {
      code[i] = to_global(reinterpret_cast<const uint32_t *>(rows))[slot * U + u];
      byte[i] = to_global(scales)[slot * (D / 32) + (u >> 2)];
    } else {
      load8<T>(to_global(rows) + (slot * U + u) * (8 * (int64_t)sizeof(T)), raw[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int64_t slot = slot0 + 256 / U * i;
    if (j0 + 256 / U * i >= c.capacity) break;
    if constexpr (FP4) {
      const uint4 w = fp4_values(code[i], fp4_scale(byte[i]));
      if constexpr (sizeof(T) == 2) {
        raw[i][0] = w;
      } else {
        raw[i][0] = make_uint4(w.x << 16, w.x & 0xFFFF0000u, w.y << 16, w.y & 0xFFFF0000u);
        raw[i][sizeof(T) / 2 - 1] = make_uint4(w.z << 16, w.z & 0xFFFF0000u, w.w << 16, w.w & 0xFFFF0000u);
      }
    }
    const gptr<char> to = to_global(is_v ? v_out : k_out) + (slot * U + u) * (8 * (int64_t)sizeof(T));
    store16(to, raw[i][0]);
    if constexpr (sizeof(T) == 4) store16(to + 16, raw[i][sizeof(T) / 2 - 1]);
  }
}

// ---------------------------------------------------------------- eviction
struct EvictArgs {
  CacheView c;
  int32_t *count;               // [groups] moves
  int32_t *to, *from;           // [groups][stride] slots, ascending each
  int64_t stride;
  int32_t budget, n_sinks, n_recent;
  int32_t row_bytes, scale_bytes;
};

// Order of a slot for eviction: as its weight (NaN below all), held slots last.
__device__ __forceinline__ uint32_t evict_key(float w, int32_t pos, int32_t n_sinks,
                                              int64_t recent_from) {
  if (pos < n_sinks || pos >= recent_from) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);   // -0 as 0
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The sum of one int per wave over the waves before this one, and over all.
template <int NW>
__device__ __forceinline__ int wave_prefix(int mine, int wave, int lane, int *lds, int &total) {
  __syncthreads();
  if (lane == 0) lds[wave] = mine;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    before += w < wave ? lds[w] : 0;
    total += lds[w];
  }
  return before;
}

// A move: the lanes of a wave copy 16 bytes each of the K and the V row (at most
// 512 bytes each), four of them the rest.  No slot is both read and written (from
// >= budget > to).
__device__ __forceinline__ void move_slot(const EvictArgs &a, int64_t to, int64_t from, int lane) {
  const int units = a.row_bytes / 16;
  if (lane < 2 * units) {
    char *rows = lane < units ? a.c.k : a.c.v;
    const int u = lane < units ? lane : lane - units;
    store16(to_global(rows) + to * a.row_bytes + 16 * u,
            load16(to_global(rows) + from * a.row_bytes + 16 * u));
  }
  if (lane < a.scale_bytes) {
    a.c.k_scale[to * a.scale_bytes + lane] = a.c.k_scale[from * a.scale_bytes + lane];
    a.c.v_scale[to * a.scale_bytes + lane] = a.c.v_scale[from * a.scale_bytes + lane];
  }
  if (lane == 0) a.c.pos[to] = a.c.pos[from];
  if (lane == 1) a.c.weight[to] = a.c.weight[from];
}

constexpr int kFusedMoves = 256;    // moves that evict_kernel makes itself, at most
constexpr int kEvictList = 512;     // keys that it ranks against each other, at most

// The key of the last of the `drop` slots that go, and how many keys lie below it: two
// bits at a time from the top, by counting the keys below three candidates (each
// wave's by ballots, then one LDS counter each).  No histogram: the weights have
// few exponents, and all of them would meet in a few bins.  count(t1, t2, t3, n): the
// wave's keys below each.  counters [16][4] are zero.  STEPS < 16: the top 2 STEPS bits
// alone.  FEW > 0: ends before, with `bits` bits to go, where at most FEW keys are left in t's
// range.
template <int STEPS, int FEW, typename F>
__device__ __forceinline__ uint32_t search_key(F &&count, int (*counters)[4], int drop, int lane, int &less,
                                               int &bits) {
  uint32_t t = 0;
  less = 0;
  int upto = INT32_MAX;          // keys below the range's end
#pragma unroll 1
  for (int step = 0; step < STEPS && (FEW == 0 || upto - less > FEW); ++step) {
    const int bit = 30 - 2 * step;
    int n[3] = {0, 0, 0};
    count(t | 1u << bit, t | 2u << bit, t | 3u << bit, n);
    if (lane < 3) atomicAdd(&counters[step][lane], lane == 0 ? n[0] : lane == 1 ? n[1] : n[2]);
    __syncthreads();
    const int c1 = counters[step][0], c2 = counters[step][1], c3 = counters[step][2];
    bits = bit;
    if (c3 < drop) t |= 3u << bit, less = c3;
    else if (c2 < drop) t |= 2u << bit, less = c2, upto = c3;
    else if (c1 < drop) t |= 1u << bit, less = c1, upto = c2;
    else upto = c1;
  }
  return t;
}

// One workgroup of NT threads per group, each wave on a consecutive run of its slots.
// One slot to drop, the case of a decoding step: one look at the weights, the
// smallest (key, highest slot) by butterflies, and at most one move.
// Up to 256: the threads' smallest keys bound the drop-th smallest of all (its top
// 14 bits are searched for: a float to 3%), and the few (key, slot) below the bound
// are ranked against each other in LDS; so are the freed slots, for their order.
// Else, or where too many keys are alike: search_key over all keys (in LDS, up to
// LKEYS of them; else read anew each time), until those left are few enough to be
// ranked, then the freed slots below the budget
// and the kept ones from it on, both ascending, by ballots and prefix sums.
// FUSED: the moves too; else their lists go to the workspace.
// Bound by the latency of its phases, one workgroup a group: 512 groups of 4001 slots, one
// to drop, 6.6 us (16 MB, 2.5 TB/s); 32 groups of 32832 slots, 64 to drop, 17.2 us; 32 of
// 32768 with 600 to drop, or 64 among many equal ones, 57 and 75 us (72 and 73 us without
// ranking the last ones); 8 of 131072, all but 4072 to drop, 364 us (462 us).
// Loops stay loops: unrolled over a thread's keys in registers, the code that each
// workgroup runs once took longer to fetch than to run.
template <int NT, int LKEYS, bool FUSED>
__global__ __launch_bounds__(NT) void evict_kernel(const EvictArgs a) {
  constexpr int NW = NT / 64;
  static_assert(LKEYS % (4 * NT) == 0, "a thread's keys come in fours");
  __shared__ int count_s[2][16][4];
  __shared__ uint64_t least_s[NW];
  __shared__ int sums[NW];
  __shared__ int2 pairs[NW];
  __shared__ int to_s[FUSED ? kFusedMoves : 1], from_s[FUSED ? kFusedMoves : 1];
  __shared__ uint64_t list_s[kEvictList];   // key << 32 | ~slot: the first ones go first
  __shared__ int freed_s[kEvictList];       // of each, its slot if it is freed below the budget
  __shared__ uint8_t tail_gone_s[kFusedMoves];
  __shared__ __align__(16) uint32_t keys_s[LKEYS ? LKEYS : 1];   // of the slots
  __shared__ int listed_s, moves_s, less_s;
  __shared__ uint32_t last_s;
  const int tid = threadIdx.x, lane = tid & 63, bg = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = live_slots(a.c, bg);
  if (n <= a.budget) {           // uniform
    if (!FUSED && tid == 0) a.count[bg] = 0;
    return;
  }
  const int64_t base = (int64_t)bg * a.c.capacity;
  const float *weight = a.c.weight + base;
  const int32_t *pos = a.c.pos + base;
  const int64_t recent_from = (int64_t)a.c.seen[bg] - a.n_recent;
  const int nj = (n + 4 * NT - 1) / (4 * NT) * 4;           // keys of a thread, in fours
  const int first = wave * 64 * nj + lane;                  // its slots: first + 64 j
  auto read_key = [&](int slot) {                           // past the end: below no candidate
    const int s = min(slot, n - 1);
    const uint32_t k = evict_key(weight[s], pos[s], a.n_sinks, recent_from);
    return slot < n ? k : 0xFFFFFFFFu;
  };
  // f(slot, keys of slot .. slot + 3) for all of the wave's slots: 16-byte loads of four
  // slots a lane (to 4 bytes aligned, as a group begins anywhere), several under way
  auto each_four = [&](auto &&f) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef int32_t i4 __attribute__((ext_vector_type(4), aligned(4)));
    const int begin = wave * 64 * nj;
    const int whole = min(max(a.c.capacity - begin, 0) / 256, nj / 4);
    for (int i = 0; i < whole; i += 4) {
      f4 w[4];
      i4 p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int slot = begin + 4 * lane + 256 * min(i + u, whole - 1);
        w[u] = *reinterpret_cast<const f4 *>(weight + slot);
        p[u] = *reinterpret_cast<const i4 *>(pos + slot);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i + u >= whole) break;               // uniform
        const int slot = begin + 4 * lane + 256 * (i + u);
        uint32_t k[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k[e] = evict_key(w[u][e], p[u][e], a.n_sinks, recent_from);
          k[e] = slot + e < n ? k[e] : 0xFFFFFFFFu;
        }
        f(slot, k);
      }
    }
    for (int i = whole; i < nj / 4; ++i) {       // past the capacity
      const int slot = begin + 4 * lane + 256 * i;
      uint32_t k[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = read_key(slot + e);
      f(slot, k);
    }
  };
  const int drop = n - a.budget;
  int moves = 0;
  if (drop == 1) {
    uint64_t least = ~0ull;
    each_four([&](int slot, const uint32_t (&k)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (slot + e < n) least = min(least, (uint64_t)k[e] << 32 | (uint32_t)~(slot + e));
    });
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, o));
    if (lane == 0) least_s[wave] = least;
    __syncthreads();
    if (wave) return;            // uniform; no barrier follows on this path
#pragma unroll
    for (int w = 0; w < NW; ++w) least = min(least, least_s[w]);
    const int gone = (int)~(uint32_t)least;
    if (lane == 0) {
      if constexpr (!FUSED) {
        a.count[bg] = gone < a.budget ? 1 : 0;
        a.to[bg * a.stride] = gone;
        a.from[bg * a.stride] = a.budget;
      }
      a.c.len[bg] = a.budget;
    }
    // by the one slot from the budget on
    if (FUSED && gone < a.budget) move_slot(a, base + gone, base + a.budget, lane);
    return;
  }
  uint32_t least = 0xFFFFFFFFu;
  each_four([&](int slot, const uint32_t (&k)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) least = min(least, k[e]);
    if (LKEYS) *reinterpret_cast<uint4 *>(&keys_s[slot]) = make_uint4(k[0], k[1], k[2], k[3]);   // for this wave
  });
  // keys j .. j + 3, together
  auto keys_at = [&](int j, uint32_t (&k)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) k[e] = LKEYS ? keys_s[first + 64 * (j + e)] : read_key(first + 64 * (j + e));
  };
  // f(slot, key) for all of the wave's slots, in any order
  auto each_key = [&](auto &&f) {
    if constexpr (LKEYS > 0) {
      for (int j = 0; j < nj; j += 4) {
        uint32_t k[4];
        keys_at(j, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) f(first + 64 * (j + e), k[e]);
      }
    } else {
      each_four([&](int slot, const uint32_t (&k)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f(slot + e, k[e]);
      });
    }
  };
  if (tid < 128) reinterpret_cast<int *>(count_s)[tid] = 0;
  if (tid == 0) listed_s = 0;
  __syncthreads();
  uint32_t t = 0;                // the key of the last slot that goes
  int less = 0, bits = 0;        // keys below it; lower bits of it not searched for
  if (drop <= kFusedMoves && drop <= NT / 2) {
    auto count_least = [&](uint32_t t1, uint32_t t2, uint32_t t3, int (&c)[3]) {
      c[0] = __popcll(__ballot(least < t1));
      c[1] = __popcll(__ballot(least < t2));
      c[2] = __popcll(__ballot(least < t3));
    };
    uint32_t bound = 0xFFFFFFFFu;                // (all keys but the held slots')
    if (n > kEvictList) {
      bound = search_key<7, 0>(count_least, count_s[0], drop, lane, less, bits) + (1u << 18);
      if (bound == 0u) bound = 0xFFFFFFFFu;
    }
    each_key([&](int slot, uint32_t k) {
      if (k < bound) {
        const int i = atomicAdd(&listed_s, 1);
        if (i < kEvictList) list_s[i] = (uint64_t)k << 32 | (uint32_t)~slot;
      }
    });
    if (tid < kFusedMoves) tail_gone_s[tid] = 0;
    __syncthreads();
    const int listed = listed_s;
    if (listed >= drop && listed <= kEvictList) {   // uniform
      for (int i = tid; i < listed; i += NT) {
        const uint64_t mine = list_s[i];
        int rank = 0;
#pragma unroll 8
        for (int o = 0; o < listed; ++o) rank += list_s[o] < mine;
        const int slot = (int)~(uint32_t)mine;
        const bool gone = rank < drop;
        freed_s[i] = gone && slot < a.budget ? slot : INT32_MAX;
        if (gone && slot >= a.budget) tail_gone_s[slot - a.budget] = 1;
      }
      __syncthreads();
      int32_t *to = FUSED ? to_s : a.to + bg * a.stride, *from = FUSED ? from_s : a.from + bg * a.stride;
      for (int i = tid; i < listed; i += NT) {
        const int mine = freed_s[i];
        int rank = 0;
#pragma unroll 8
        for (int o = 0; o < listed; ++o) rank += freed_s[o] < mine;
        if (mine != INT32_MAX) to[rank] = mine;
      }
      if (wave == 0) {
        int kept = 0;
        for (int x = 0; x < drop; x += 64) {
          const bool tail = x + lane < drop && !tail_gone_s[x + lane];
          const uint64_t m = __ballot(tail);
          if (tail) from[kept + __popcll(m & ((1ull << lane) - 1))] = a.budget + x + lane;
          kept += __popcll(m);
        }
        if (lane == 0) {
          moves_s = kept;        // as many as freed slots: drop of n - budget slots stay behind
          if constexpr (!FUSED) a.count[bg] = kept;
          a.c.len[bg] = a.budget;
        }
      }
      if constexpr (FUSED) {
        __syncthreads();
        for (int m = wave; m < moves_s; m += NW) move_slot(a, base + to_s[m], base + from_s[m], lane);
      }
      return;
    }
  }
  auto count_all = [&](uint32_t t1, uint32_t t2, uint32_t t3, int (&c)[3]) {
    each_key([&](int, uint32_t k) {
      c[0] += __popcll(__ballot(k < t1));
      c[1] += __popcll(__ballot(k < t2));
      c[2] += __popcll(__ballot(k < t3));
    });
  };
  t = search_key<16, kEvictList>(count_all, count_s[1], drop, lane, less, bits);
  if (bits > 0) {                // uniform: the few keys left are ranked
    if (tid == 0) listed_s = less_s = 0;
    __syncthreads();
    each_key([&](int slot, uint32_t k) {
      if (slot < n && k >= t && (k - t) >> bits == 0) {
        const int i = atomicAdd(&listed_s, 1);
        if (i < kEvictList) list_s[i] = (uint64_t)k << 32 | (uint32_t)~slot;
      }
    });
    __syncthreads();
    const int alike = min(listed_s, kEvictList);
    for (int i = tid; i < alike; i += NT) {
      const uint64_t mine = list_s[i];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < alike; ++o) rank += list_s[o] < mine;
      if (rank == drop - less - 1) last_s = (uint32_t)(mine >> 32);
    }
    __syncthreads();
    t = last_s;
    for (int i = tid; i < alike; i += NT)
      if ((uint32_t)(list_s[i] >> 32) < t) atomicAdd(&less_s, 1);
    __syncthreads();
    less += less_s;
  }
  // keys below t go, and the highest slots of those equal to it
  int equal = 0;
  each_key([&](int slot, uint32_t k) { equal += __popcll(__ballot(k == t && slot < n)); });
  int all_equal;
  const int equal_before = wave_prefix<NW>(equal, wave, lane, sums, all_equal);
  const int keep_equal = all_equal - (drop - less);
  const uint64_t below = (1ull << lane) - 1;
  int2 at = make_int2(0, 0);     // freed slots and kept tails before this wave's
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {         // count, then write
    int eq = equal_before, nh = 0, nt = 0;
#pragma unroll 1
    for (int j = 0; j < nj; j += 4) {
      uint32_t k[4];
      keys_at(j, k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int slot = first + 64 * (j + e);
        const bool in = slot < n;
        const uint64_t eq_m = __ballot(in && k[e] == t);
        const bool gone = k[e] < t || (k[e] == t && eq + __popcll(eq_m & below) >= keep_equal);
        eq += __popcll(eq_m);
        const bool hole = in && gone && slot < a.budget, tail = in && !gone && slot >= a.budget;
        const uint64_t h_m = __ballot(hole), t_m = __ballot(tail);
        if (pass == 1) {
          const int h = at.x + nh + __popcll(h_m & below), l = at.y + nt + __popcll(t_m & below);
          if constexpr (FUSED) {
            if (hole) to_s[h] = slot;
            if (tail) from_s[l] = slot;
          } else {
            if (hole) a.to[bg * a.stride + h] = slot;
            if (tail) a.from[bg * a.stride + l] = slot;
          }
        }
        nh += __popcll(h_m);
        nt += __popcll(t_m);
      }
    }
    if (pass == 0) {
      if (lane == 0) pairs[wave] = make_int2(nh, nt);
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int2 x = pairs[w];
        if (w < wave) at.x += x.x, at.y += x.y;
        moves += x.x;
      }
    }
  }
  if (tid == 0) {
    if constexpr (!FUSED) a.count[bg] = moves;
    a.c.len[bg] = a.budget;
  }
  if constexpr (FUSED) {
    __syncthreads();
    for (int m = wave; m < moves; m += NW) move_slot(a, base + to_s[m], base + from_s[m], lane);
  }
}

// Grid (groups, blocks), a wave per move.
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a) {
  const int lane = threadIdx.x & 63, bg = blockIdx.x, n = a.count[bg];
  const int64_t base = (int64_t)bg * a.c.capacity;
  for (int m = (int)blockIdx.y * 4 + ((int)threadIdx.x >> 6); m < n; m += 4 * (int)gridDim.y)
    move_slot(a, base + a.to[bg * a.stride + m], base + a.from[bg * a.stride + m], lane);
}

}  // namespace ckv

using ckv_api::cache_view;
using ckv_api::check_cache;
using ckv_api::check_rows_dtype;
using ckv_api::fail;
using ckv_api::launched;
using ckv_api::ok;
using ckv_api::round_up;

namespace {

// Calls f.operator()<T, D, FP4>() for rows of `dtype` in and out of the cache.
template <typename F>
void with_rows(const ckv_cache *c, int dtype, F &&f) {
  const bool fp4 = c->dtype == CKV_FP4;
  if (dtype == CKV_BF16) {
    if (c->head_dim == 64)
      fp4 ? f.template operator()<__bf16, 64, true>() : f.template operator()<__bf16, 64, false>();
    else
      fp4 ? f.template operator()<__bf16, 128, true>() : f.template operator()<__bf16, 128, false>();
  } else {
    if (c->head_dim == 64)
      fp4 ? f.template operator()<float, 64, true>() : f.template operator()<float, 64, false>();
    else
      fp4 ? f.template operator()<float, 128, true>() : f.template operator()<float, 128, false>();
  }
}

int check_pointer(const void *p, const char *name, size_t align) {
  if (!p) return fail(CKV_INVALID_ARGUMENT, "%s is NULL", name);
  if (!ckv_api::aligned(p, align))
    return fail(CKV_UNSUPPORTED, "%s must be %zu-byte aligned", name, align);
  return CKV_OK;
}

// Moves of one group at most, and the workspace's parts.
int64_t evict_stride(const ckv_cache *c, int budget) {
  return std::max(1, std::min(budget, c->capacity - budget));
}

size_t evict_bytes(const ckv_cache *c, int budget) {
  const size_t groups = (size_t)c->batch * c->n_kv_heads;
  return round_up(groups * 4, 256) + 2 * round_up(groups * evict_stride(c, budget) * 4, 256);
}

int check_budget(const ckv_cache *c, int budget) {
  if (budget < 1 || budget > c->capacity)
    return fail(CKV_INVALID_ARGUMENT, "budget must be in [1, capacity] (got %d)", budget);
  return CKV_OK;
}

}  // namespace

extern "C" {

int compresskv_cache_load(const ckv_cache *c, int32_t dtype, int32_t n_rows, const void *k_rows,
                          const void *v_rows, const int32_t *idx, const int32_t *group_rows_host,
                          const int32_t *cu_seqlens, void *stream) {
  int st;
  if ((st = check_cache(c))) return st;
  if ((st = check_rows_dtype(c, dtype))) return st;
  ckv::LoadArgs a{};
  int64_t per_b = 0;
  if (group_rows_host) {
    for (int g = 0; g < c->n_kv_heads; ++g) {
      if (group_rows_host[g] < 1 || group_rows_host[g] > c->capacity)
        return fail(CKV_INVALID_ARGUMENT, "group %d: rows must be in [1, capacity] (got %d)", g,
                    group_rows_host[g]);
      a.off[g] = (int32_t)per_b;
      per_b += group_rows_host[g];
      if (per_b > INT32_MAX)
        return fail(CKV_UNSUPPORTED, "the groups' rows sum to 2^31 or more");
    }
    a.off[c->n_kv_heads] = (int32_t)per_b;
  } else {
    if (n_rows < 1 || n_rows > c->capacity)
      return fail(CKV_INVALID_ARGUMENT, "n_rows must be in [1, capacity] (got %d)", n_rows);
    per_b = (int64_t)n_rows * c->n_kv_heads;
    a.n_rows = n_rows;
    if (per_b > INT32_MAX) return fail(CKV_UNSUPPORTED, "n_rows * n_kv_heads is 2^31 or more");
  }
  if ((st = check_pointer(k_rows, "k_rows", 16))) return st;
  if ((st = check_pointer(v_rows, "v_rows", 16))) return st;
  if ((st = check_pointer(idx, "idx", 4))) return st;
  if ((st = check_pointer(cu_seqlens, "cu_seqlens", 4))) return st;
  a.c = cache_view(c);
  a.k = static_cast<const char *>(k_rows);
  a.v = static_cast<const char *>(v_rows);
  a.idx = idx;
  a.cu = cu_seqlens;
  a.rows_per_b = per_b;
  const int rows_per_block = 256 / (c->head_dim / 8) * ckv::kUnits;
  int most = n_rows;
  if (group_rows_host) most = *std::max_element(group_rows_host, group_rows_host + c->n_kv_heads);
  const dim3 grid((most + rows_per_block - 1) / rows_per_block, a.c.groups, 3);
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_load_kernel<T, D, FP4>), grid, dim3(256), 0, (hipStream_t)stream, a);
  });
  return launched("cache load");
}

int compresskv_cache_append(const ckv_cache *c, int32_t dtype, int32_t n_new, const void *k_new,
                            const int64_t *k_strides_host, const void *v_new,
                            const int64_t *v_strides_host, void *stream) {
  int st;
  if ((st = check_cache(c))) return st;
  if ((st = check_rows_dtype(c, dtype))) return st;
  if (n_new < 1) return fail(CKV_INVALID_ARGUMENT, "n_new must be >= 1 (got %d)", n_new);
  if ((st = check_pointer(k_new, "k_new", 16))) return st;
  if ((st = check_pointer(v_new, "v_new", 16))) return st;
  if (!k_strides_host || !v_strides_host)
    return fail(CKV_INVALID_ARGUMENT, "k_strides_host and v_strides_host are required");
  ckv::AppendArgs a{};
  const int64_t size = dtype == CKV_BF16 ? 2 : 4;
  for (int i = 0; i < 3; ++i) {
    const int64_t s[2] = {k_strides_host[i], v_strides_host[i]};
    for (int w = 0; w < 2; ++w) {
      if (s[w] < 0 || s[w] > (int64_t)1 << 40)
        return fail(CKV_INVALID_ARGUMENT, "strides must be in [0, 2^40]");
      if (s[w] * size % 16)
        return fail(CKV_UNSUPPORTED, "strides must be multiples of 16 bytes");
    }
    a.ks[i] = s[0] * size;
    a.vs[i] = s[1] * size;
  }
  a.c = cache_view(c);
  a.k = static_cast<const char *>(k_new);
  a.v = static_cast<const char *>(v_new);
  a.n_new = n_new;
  // one workgroup per group takes up to eight trips, and the lengths with them (8 groups,
  // 64, 256, 1024 tokens of bf16, D = 128: 4.6, 6.5, 13.8 us in one workgroup; 6.2, 8.0,
  // 8.4 us in several and a launch for the lengths)
  const int threads = n_new * 2 * (c->head_dim / 8) <= 256 ? 256 : 1024;
  const int64_t rows = threads / (2 * (c->head_dim / 8)), trips = (n_new + rows - 1) / rows;
  a.own_len = trips <= 8;
  const unsigned per_group = a.own_len ? 1u : (unsigned)std::min<int64_t>((trips + 7) / 8, 1024);
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_append_kernel<T, D, FP4>), dim3(a.c.groups, per_group), dim3(threads),
                       0, (hipStream_t)stream, a);
  });
  if (!a.own_len) {
    if ((st = launched("cache append"))) return st;
    hipLaunchKernelGGL(ckv::cache_len_kernel, dim3((a.c.groups + 255) / 256), dim3(256), 0,
                       (hipStream_t)stream, a.c, n_new);
  }
  return launched("cache append");
}

int compresskv_cache_read(const ckv_cache *c, int32_t dtype, void *k_out, void *v_out,
                          void *stream) {
  int st;
  if ((st = check_cache(c))) return st;
  if ((st = check_rows_dtype(c, dtype))) return st;
  if ((st = check_pointer(k_out, "k_out", 16))) return st;
  if ((st = check_pointer(v_out, "v_out", 16))) return st;
  const ckv::CacheView v = cache_view(c);
  const int rows_per_block = 256 / (c->head_dim / 8) * ckv::kUnits;
  const dim3 grid((c->capacity + rows_per_block - 1) / rows_per_block, v.groups, 2);
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_read_kernel<T, D, FP4>), grid, dim3(256), 0, (hipStream_t)stream, v,
                       static_cast<char *>(k_out), static_cast<char *>(v_out));
  });
  return launched("cache read");
}

size_t compresskv_cache_evict_workspace_bytes(const ckv_cache *c, int32_t budget) {
  if (check_cache(c) || check_budget(c, budget)) return 0;
  ok();
  return evict_bytes(c, budget);
}

int compresskv_cache_evict(const ckv_cache *c, int32_t budget, int32_t n_sinks, int32_t n_recent,
                           void *ws, size_t ws_bytes, void *stream) {
  int st;
  if ((st = check_cache(c))) return st;
  if ((st = check_budget(c, budget))) return st;
  if (n_sinks < 0 || n_recent < 0)
    return fail(CKV_INVALID_ARGUMENT, "n_sinks and n_recent must be >= 0");
  if ((st = check_pointer(ws, "ws", 256))) return st;
  if (ws_bytes < evict_bytes(c, budget))
    return fail(CKV_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given",
                evict_bytes(c, budget), ws_bytes);
  if (budget == c->capacity) return ok();   // no group can hold more
  ckv::EvictArgs a{};
  a.c = cache_view(c);
  a.stride = evict_stride(c, budget);
  char *w = static_cast<char *>(ws);
  a.count = reinterpret_cast<int32_t *>(w);
  w += round_up((size_t)a.c.groups * 4, 256);
  a.to = reinterpret_cast<int32_t *>(w);
  w += round_up((size_t)a.c.groups * a.stride * 4, 256);
  a.from = reinterpret_cast<int32_t *>(w);
  a.budget = budget;
  a.n_sinks = n_sinks;
  a.n_recent = n_recent;
  a.row_bytes = ckv_api::row_bytes(c);
  a.scale_bytes = c->dtype == CKV_FP4 ? c->head_dim / 32 : 0;
  const bool fused = a.stride <= ckv::kFusedMoves;
  auto go = [&]<int NT, int LKEYS>() {
    if (fused)
      hipLaunchKernelGGL((ckv::evict_kernel<NT, LKEYS, true>), dim3(a.c.groups), dim3(NT), 0,
                         (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL((ckv::evict_kernel<NT, LKEYS, false>), dim3(a.c.groups), dim3(NT), 0,
                         (hipStream_t)stream, a);
  };
  // Few keys, or more groups than CUs (a workgroup of 1024 threads has one to itself): 256
  // threads.  64 of 2048, 4096, 8192 slots evicted, 256 / 1024 threads: of 8 groups 15.8/18.3,
  // 23.1/18.5, 37.5/23.2 us, of 512 groups 18.3/34.0, 27.2/34.5, 45.4/48.0 us.
  if (c->capacity <= (a.c.groups > 256 ? 8192 : 2048)) go.template operator()<256, 8192>();
  else if (c->capacity <= 36864) go.template operator()<1024, 36864>();
  else go.template operator()<1024, 0>();
  if (fused) return launched("cache evict");
  if ((st = launched("cache evict"))) return st;
  const unsigned per_group = (unsigned)std::min<int64_t>((a.stride + 31) / 32, 64);
  hipLaunchKernelGGL(ckv::evict_move_kernel, dim3(a.c.groups, per_group), dim3(256), 0,
                     (hipStream_t)stream, a);
  return launched("cache evict");
}

}  // extern "C"
