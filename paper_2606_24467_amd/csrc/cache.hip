// The bounded cache's store (include/compresskv_cache.h): rows in (from a
// compressed prompt, or a decoding step's tokens), rows out, and the eviction
// of the slots of least accumulated weight.
//
//   cache_load_kernel     kept rows of a prompt into slots 0 ..
//   cache_append_kernel   new tokens' rows behind the live slots
//   cache_len_kernel      ... and the lengths, where several workgroups append
//   cache_read_kernel     rows as bf16 or fp32 values
//   evict_select_kernel   which slots go, and which kept slots take their place
//   evict_move_kernel     the moves
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
  int32_t batch;
  int32_t off[kMaxKvHeads + 1]; // ragged: first row of a group within its sequence
};

// Grid (blocks, 3), 256 threads.  y = 0, 1: K, V rows, a lane per 8 values, so
// that a wave reads 1 KB (bf16) in a row; y = 2: one workgroup per group counts
// its kept rows.  Bound by HBM: 2 D values read, a 4-bit row written.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void cache_load_kernel(const LoadArgs a) {
  const int tid = threadIdx.x;
  constexpr int U = D / 8;                       // lanes per row
  if (blockIdx.y == 2) {
    const int bg = blockIdx.x;
    if (bg >= a.c.groups) return;                // uniform
    const int b = bg / a.c.Hkv, g = bg - b * a.c.Hkv;
    const int n = a.n_rows ? a.n_rows : a.off[g + 1] - a.off[g];
    const int32_t *id = a.idx + (int64_t)b * a.rows_per_b +
                        (a.n_rows ? (int64_t)g * a.n_rows : (int64_t)a.off[g]);
    int kept = 0;
    for (int j = tid; j < n; j += 256) kept += id[j] >= 0;
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
  const int64_t unit = (int64_t)blockIdx.x * 256 + tid, row = unit / U;
  const int u = (int)(unit % U);
  if (row >= a.batch * a.rows_per_b) return;     // whole rows, so whole 4-lane blocks
  const int b = (int)(row / a.rows_per_b);
  const int r = (int)(row - b * a.rows_per_b);
  int g, j;
  if (a.n_rows) {
    g = r / a.n_rows;
    j = r - g * a.n_rows;
  } else {
    int lo = 0, hi = a.c.Hkv;                    // off[lo] <= r < off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.off[mid] <= r) lo = mid; else hi = mid;
    }
    g = lo;
    j = r - a.off[g];
  }
  const int32_t position = a.idx[row];
  uint4 raw[sizeof(T) / 2];
  const bool is_v = blockIdx.y == 1;
  load8<T>(to_global(is_v ? a.v : a.k) + unit * (8 * (int64_t)sizeof(T)), raw);
  if (position < 0) return;                      // the four lanes of a block agree
  const int64_t slot = ((int64_t)b * a.c.Hkv + g) * a.c.capacity + j;
  store8<T, D, FP4>(is_v ? a.c.v : a.c.k, is_v ? a.c.v_scale : a.c.k_scale, slot, u, raw);
  if (!is_v && u == 0) {
    a.c.pos[slot] = position;
    a.c.weight[slot] = 0.f;
  }
}

struct AppendArgs {
  CacheView c;
  const char *k, *v;
  int64_t ks[3], vs[3];         // byte strides: sequence, token, head
  int32_t n_new;
  int32_t own_len;              // the group's one workgroup updates len and seen
};

// Grid (groups, blocks per group), 256 threads: a lane per 8 values of a K or
// V row.  Bound by latency at a decoding step's one token.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs a) {
  constexpr int U = D / 8, ROWS = 256 / (2 * U);   // tokens per workgroup and trip
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

// Grid (blocks, 2), 256 threads: 8 values of a K (y = 0) or V row per lane.
template <typename T, int D, bool FP4>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheView c, char *k_out,
                                                         char *v_out) {
  constexpr int U = D / 8;
  const bool is_v = blockIdx.y == 1;
  const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x, slot = unit / U;
  if (slot >= (int64_t)c.groups * c.capacity) return;
  const int u = (int)(unit % U), bg = (int)(slot / c.capacity);
  uint4 raw[sizeof(T) / 2] = {};
  if ((int)(slot - (int64_t)bg * c.capacity) < live_slots(c, bg)) {
    const char *rows = is_v ? c.v : c.k;
    if constexpr (FP4) {
      const uint8_t *scales = is_v ? c.v_scale : c.k_scale;
      const uint4 w = fp4_values(reinterpret_cast<const uint32_t *>(rows)[unit],
                                 fp4_scale(scales[slot * (D / 32) + (u >> 2)]));
      if constexpr (sizeof(T) == 2) {
        raw[0] = w;
      } else {
        raw[0] = make_uint4(w.x << 16, w.x & 0xFFFF0000u, w.y << 16, w.y & 0xFFFF0000u);
        raw[sizeof(T) / 2 - 1] = make_uint4(w.z << 16, w.z & 0xFFFF0000u, w.w << 16, w.w & 0xFFFF0000u);
      }
    } else {
      load8<T>(to_global(rows) + unit * (8 * (int64_t)sizeof(T)), raw);
    }
  }
  const gptr<char> to = to_global(is_v ? v_out : k_out) + unit * (8 * (int64_t)sizeof(T));
  store16(to, raw[0]);
  if constexpr (sizeof(T) == 4) store16(to + 16, raw[1]);
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

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// The sum of one int per wave over the waves before this one, and over all.
__device__ __forceinline__ int wave_prefix(int mine, int wave, int lane, int *lds, int &total) {
  __syncthreads();
  if (lane == 0) lds[wave] = mine;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    before += w < wave ? lds[w] : 0;
    total += lds[w];
  }
  return before;
}

// One workgroup per group: the key of the (len - budget)-th smallest slot by
// radix select (11 + 11 + 10 bits, histograms in LDS), then, every wave on a
// consecutive run of slots, the freed slots below the budget and the kept ones
// from it on, both in ascending order by ballots and prefix sums.
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ int hist[2048];
  __shared__ int sums[kEvictWaves];
  __shared__ int pick[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bg = blockIdx.x;
  const int n = live_slots(a.c, bg);
  if (n <= a.budget) {           // uniform
    if (tid == 0) a.count[bg] = 0;
    return;
  }
  const int64_t base = (int64_t)bg * a.c.capacity;
  const float *weight = a.c.weight + base;
  const int32_t *pos = a.c.pos + base;
  const int64_t recent_from = (int64_t)a.c.seen[bg] - a.n_recent;
  auto key_of = [&](int s) { return evict_key(weight[s], pos[s], a.n_sinks, recent_from); };
  int left = n - a.budget;       // to drop among the keys that share `prefix`
  uint32_t prefix = 0, mask = 0;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < 2048; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    for (int s = tid; s < n; s += kEvictThreads) {
      const uint32_t key = key_of(s);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    if (wave == 0) {             // the digit at which the running count reaches `left`
      int mine = 0;
      for (int i = 0; i < 32; ++i) mine += hist[32 * lane + i];
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(upto, o);
        if (lane >= o) upto += t;
      }
      if (upto >= left && upto - mine < left) {   // one lane
        int run = upto - mine, d = 32 * lane;
        while (run + hist[d] < left) run += hist[d++];
        pick[0] = d;
        pick[1] = run;
      }
    }
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    mask |= ((1u << bits) - 1) << shift;
    left -= pick[1];
  }
  // keys below `prefix` go, and the `left` highest slots of those equal to it
  const int run = ((n + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  const int s0 = min(n, wave * run), s1 = min(n, s0 + run);
  int equal = 0;
  for (int s = s0; s < s1; s += 64)
    equal += __popcll(__ballot(s + lane < s1 && key_of(min(s + lane, n - 1)) == prefix));
  int all_equal;
  const int equal_before = wave_prefix(equal, wave, lane, sums, all_equal);
  const int keep_equal = all_equal - left;
  const uint64_t below = (1ull << lane) - 1;
  int holes = 0, tails = 0, hole0 = 0, tail0 = 0, unused;
  for (int pass = 0; pass < 2; ++pass) {          // count, then write
    int eq = equal_before, nh = 0, nt = 0;
    for (int s = s0; s < s1; s += 64) {
      const int slot = s + lane;
      const bool in = slot < s1;
      const uint32_t key = key_of(min(slot, n - 1));
      const uint64_t eq_m = __ballot(in && key == prefix);
      const bool gone = key < prefix || (key == prefix && eq + __popcll(eq_m & below) >= keep_equal);
      eq += __popcll(eq_m);
      const bool hole = in && gone && slot < a.budget, tail = in && !gone && slot >= a.budget;
      const uint64_t h_m = __ballot(hole), t_m = __ballot(tail);
      if (pass == 1) {
        if (hole) a.to[bg * a.stride + hole0 + nh + __popcll(h_m & below)] = slot;
        if (tail) a.from[bg * a.stride + tail0 + nt + __popcll(t_m & below)] = slot;
      }
      nh += __popcll(h_m);
      nt += __popcll(t_m);
    }
    if (pass == 0) {
      hole0 = wave_prefix(nh, wave, lane, sums, holes);
      tail0 = wave_prefix(nt, wave, lane, sums, unused);
      tails = unused;
    }
  }
  (void)tails;                   // as many as holes: n - drop = budget slots stay
  if (tid == 0) {
    a.count[bg] = holes;
    a.c.len[bg] = a.budget;
  }
}

// Grid (groups, blocks), a wave per move: the lanes copy 16 bytes each of the
// K and the V row (at most 512 bytes each), four of them the rest.  No slot is
// both read and written (from >= budget > to).
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a) {
  const int lane = threadIdx.x & 63, bg = blockIdx.x;
  const int n = a.count[bg], units = a.row_bytes / 16;
  const int64_t base = (int64_t)bg * a.c.capacity;
  for (int m = (int)blockIdx.y * 4 + ((int)threadIdx.x >> 6); m < n; m += 4 * (int)gridDim.y) {
    const int64_t to = base + a.to[bg * a.stride + m], from = base + a.from[bg * a.stride + m];
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
  a.batch = c->batch;
  const int64_t blocks = std::max<int64_t>(
      a.c.groups, ((int64_t)c->batch * per_b * (c->head_dim / 8) + 255) / 256);
  if (blocks > INT32_MAX / 256)
    return fail(CKV_UNSUPPORTED, "batch * rows is too large for one launch");
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_load_kernel<T, D, FP4>), dim3((unsigned)blocks, 3), dim3(256), 0,
                       (hipStream_t)stream, a);
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
  // one workgroup per group takes up to four trips, and the lengths with them
  const int rows = 256 / (2 * c->head_dim / 8);
  const int64_t trips = ((int64_t)n_new + rows - 1) / rows;
  a.own_len = trips <= 4;
  const unsigned per_group = a.own_len ? 1u : (unsigned)std::min<int64_t>((trips + 3) / 4, 1024);
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_append_kernel<T, D, FP4>), dim3(a.c.groups, per_group), dim3(256),
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
  const int64_t blocks = ((int64_t)v.groups * c->capacity * (c->head_dim / 8) + 255) / 256;
  if (blocks > INT32_MAX / 256)
    return fail(CKV_UNSUPPORTED, "batch * capacity is too large for one launch");
  with_rows(c, dtype, [&]<typename T, int D, bool FP4>() {
    hipLaunchKernelGGL((ckv::cache_read_kernel<T, D, FP4>), dim3((unsigned)blocks, 2), dim3(256), 0,
                       (hipStream_t)stream, v, static_cast<char *>(k_out),
                       static_cast<char *>(v_out));
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
  hipLaunchKernelGGL(ckv::evict_select_kernel, dim3(a.c.groups), dim3(ckv::kEvictThreads), 0,
                     (hipStream_t)stream, a);
  if ((st = launched("cache evict"))) return st;
  const unsigned per_group = (unsigned)std::min<int64_t>((a.stride + 31) / 32, 64);
  hipLaunchKernelGGL(ckv::evict_move_kernel, dim3(a.c.groups, per_group), dim3(256), 0,
                     (hipStream_t)stream, a);
  return launched("cache evict");
}

}  // extern "C"
