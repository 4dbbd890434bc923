// Attention over a bounded cache (include/compresskv_cache.h): the entry point,
// the join of split rows with the accumulation of the slots' weights, and the
// dispatch of the attention kernel (attend_kernels.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attend.h"
#include "cache_api.h"
#include "row_blocks.h"
#include "score_common.h"

namespace ckv {

// References and 1 / sum (0: it saw nothing) over the splits of `rows` rows, the first at
// global row r0 of the group, into row_s: 2^k lanes per row (at least one per
// split, up to 64), all rows' loads under way together.
__device__ __forceinline__ void join_rows(const AttendArgs &a, int64_t slot0, int r0, int rows, float2 *row_s) {
  const int RM = 16 * a.rt;
  int lanes = 1;
  while (lanes < a.splits && lanes < 64) lanes *= 2;
  const int sub = (int)threadIdx.x & (lanes - 1);
  for (int base = 0; base < rows; base += 256 / lanes) {   // uniform: every lane takes part in the butterflies
    const int r = base + (int)threadIdx.x / lanes;
    const int row = r0 + min(r, rows - 1), rb = row / RM;
    const float2 *ml = a.part_ml + (slot0 + (int64_t)rb * a.splits) * RM + (row - rb * RM);
    float2 x[kAttendMaxSplits / 64];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kAttendMaxSplits / 64; ++i) {
      const int s = sub + lanes * i;
      x[i] = s < a.splits ? ml[(int64_t)s * RM] : make_float2(-INFINITY, 0.f);
      top = fmaxf(top, x[i].x);
    }
    for (int o = lanes / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kAttendMaxSplits / 64; ++i) sum += x[i].y * fast_exp2(x[i].x - ref);
    for (int o = lanes / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    if (sub == 0 && r < rows) row_s[r] = make_float2(ref, sum == 0.f ? 0.f : 1.f / sum);
  }
}

constexpr int kJoinSlots = 1024;   // slots whose weights one workgroup adds to

// Grid (out_blocks + weight blocks, groups), or where the row blocks are packed (row
// blocks * workgroups of each, 1), 256 threads.  The first out_blocks
// join the splits' outputs, up to 1024 / D rows each: D / 4 lanes per row, and where
// that leaves lanes (few rows, many splits) the splits are dealt to several such
// parts, whose sums are added in order.  Each of the others adds to the
// weights of kJoinSlots slots what the group's rows gave them, row by row in
// order.  Bound by the latency of its few dependent loads, and with many rows by the
// logits: 4.3 us for 128 groups in 4 splits, 4 rows of up to 4096 logits; 9.3 us for 64
// groups in 8 splits, 28 rows of up to 3936 (24 MB; 8.5 us without the comparison of
// positions).
template <AttendSource SRC, typename T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a, int out_blocks) {
  const int tid = threadIdx.x, bg = blockIdx.y, RM = 16 * a.rt;
  int b = bg / a.Hkv, g = bg - b * a.Hkv, r0 = (int)blockIdx.x * a.join_rows;
  int64_t slot0 = (int64_t)bg * a.row_blocks * a.splits;   // of the group's first row block
  if constexpr (SRC == kOverWindow) {
    if (a.packed) {
      const int each = RM / a.join_rows, id = (int)blockIdx.x / each;
      RowBlock found;
      if (!find_row_block<false>(a, id, RM, found)) return;   // uniform
      b = found.b, g = found.g;
      r0 = found.rb * RM + ((int)blockIdx.x - id * each) * a.join_rows;
      slot0 = (int64_t)(found.part - found.rb) * a.splits;
    }
  }
  if ((int)blockIdx.x < out_blocks) {
    constexpr int LR = D / 4, NP = 256 / LR;      // lanes per row; rows x parts of the splits
    __shared__ __align__(16) f32x4 part_s[NP][LR];
    __shared__ float2 all_s[NP];
    const int q0 = SRC == kOverWindow ? a.cu_q[b] : 0;
    const int rows = SRC == kOverWindow ? (a.cu_q[b + 1] - q0) * a.G : a.rows;
    if (r0 >= rows) return;                       // uniform
    const int here = min(a.join_rows, rows - r0), parts = NP / a.join_rows;
    join_rows(a, slot0, r0, here, all_s);
    __syncthreads();
    const int e = tid / LR, mine = e / parts, part = e % parts, d = 4 * (tid % LR);
    const int r = r0 + min(mine, here - 1), rb = r / RM, rr = r - rb * RM;
    const float2 all = all_s[min(mine, here - 1)];
    const float2 *ml = a.part_ml + (slot0 + (int64_t)rb * a.splits) * RM + rr;
    const float *po = a.part_o + ((slot0 + (int64_t)rb * a.splits) * RM + rr) * D + d;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = part; s < a.splits; s += parts) {
      const float f = fast_exp2(ml[(int64_t)s * RM].x - all.x);
      const f32x4 x = *reinterpret_cast<const f32x4 *>(po + (int64_t)s * RM * D);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += x[k] * f;
    }
    part_s[e][tid % LR] = o;
    __syncthreads();
    if (part == 0 && mine < here) {
      for (int p = 1; p < parts; ++p) {
        const f32x4 x = part_s[e + p][tid % LR];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += x[k];
      }
      const int i = r / a.G, h = g * a.G + (r - i * a.G);
      const int64_t token = SRC == kOverWindow ? (int64_t)q0 + i : (int64_t)b * a.n_q + i;
      T *to = reinterpret_cast<T *>(a.out) + (token * ((int64_t)a.Hkv * a.G) + h) * D + d;
      typedef T Tx4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<Tx4 *>(to) = Tx4{(T)(o[0] * all.y), (T)(o[1] * all.y), (T)(o[2] * all.y),
                                         (T)(o[3] * all.y)};
    }
  } else if constexpr (SRC == kOverCache) {
    __shared__ float2 row_s[64];                  // (reference, 1 / sum)
    const int n = live_slots(a.c, bg);
    const int s0 = ((int)blockIdx.x - out_blocks) * kJoinSlots;
    if (s0 >= n) return;                          // uniform
    float got[kJoinSlots / 256] = {}, old[kJoinSlots / 256];
    int32_t pos[kJoinSlots / 256] = {};           // one token sees every slot
#pragma unroll
    for (int i = 0; i < kJoinSlots / 256; ++i) {
      const int64_t at = (int64_t)bg * a.c.capacity + min(s0 + tid + 256 * i, n - 1);
      old[i] = a.c.weight[at];
      if (a.masks) pos[i] = a.c.pos[at];
    }
    join_rows(a, slot0, 0, a.rows, row_s);
    __syncthreads();
    const float *z = a.logits + (int64_t)bg * a.rows * a.logit_stride;
    // A row whose sum is a NaN gives it to the slots that it sees and to no other: the logit of
    // those is -infinity, but 0 times a NaN is one.
    auto add = [&]<bool MASKS>() {
      int t = (int)((uint32_t)a.c.seen[bg] - (uint32_t)a.n_q), h = 0;   // the row's position, head
#pragma unroll 4
      for (int r = 0; r < a.rows; ++r) {
        const float2 all = row_s[r];
#pragma unroll
        for (int i = 0; i < kJoinSlots / 256; ++i) {
          const int s = min(s0 + tid + 256 * i, n - 1);
          const float p = fast_exp2(__builtin_fmaf(z[r * a.logit_stride + s], a.c1, -all.x)) * all.y;
          got[i] += !MASKS || pos[i] <= t ? p : 0.f;
        }
        if (MASKS && ++h == a.G) h = 0, ++t;
      }
    };
    a.masks ? add.template operator()<true>() : add.template operator()<false>();
#pragma unroll
    for (int i = 0; i < kJoinSlots / 256; ++i) {
      const int s = s0 + tid + 256 * i;
      if (s < n) a.c.weight[(int64_t)bg * a.c.capacity + s] = old[i] + got[i];
    }
  }
}

void launch_attend_join(AttendArgs a, AttendSource source, bool f32, int head_dim, int max_rows,
                        hipStream_t stream) {
  // rows per workgroup: as many as fill it, fewer where the splits are many
  a.join_rows = 1024 / head_dim;
  while (a.join_rows > 1 && a.splits > 4 * (1024 / head_dim / a.join_rows)) a.join_rows /= 2;
  const int out_blocks = a.splits == 1 ? 0
                         : a.packed    ? a.blocks * (16 * a.rt / a.join_rows)
                                       : (max_rows + a.join_rows - 1) / a.join_rows;
  const int weight_blocks = a.accumulate && !a.one ? (a.c.capacity + kJoinSlots - 1) / kJoinSlots : 0;
  if (out_blocks + weight_blocks == 0) return;
  const dim3 grid(out_blocks + weight_blocks, a.packed ? 1 : a.c.groups);
  auto go = [&]<AttendSource SRC, typename T, int D>() {
    hipLaunchKernelGGL((attend_join_kernel<SRC, T, D>), grid, dim3(256), 0, stream, a, out_blocks);
  };
  auto dim = [&]<AttendSource SRC, typename T>() {
    head_dim == 64 ? go.template operator()<SRC, T, 64>() : go.template operator()<SRC, T, 128>();
  };
  if (source == kOverCache)
    f32 ? dim.template operator()<kOverCache, float>() : dim.template operator()<kOverCache, __bf16>();
  else
    f32 ? dim.template operator()<kOverWindow, float>() : dim.template operator()<kOverWindow, __bf16>();
}

// One per row type (attend_fp4.hip, attend_bf16.hip, attend_f32.hip).
void launch_attend_fp4(const AttendArgs &a, bool f32, int head_dim, dim3 grid, hipStream_t stream);
void launch_attend_bf16(const AttendArgs &a, AttendSource source, int head_dim, dim3 grid,
                        hipStream_t stream);
void launch_attend_f32(const AttendArgs &a, AttendSource source, int head_dim, dim3 grid,
                       hipStream_t stream);

void launch_attend(const AttendArgs &a, AttendSource source, CacheType type, bool f32, int head_dim,
                   int max_rows, hipStream_t stream) {
  const dim3 grid = a.packed ? dim3(a.blocks, 1, a.splits) : dim3(a.row_blocks, a.c.groups, a.splits);
  if (type == kCacheFp4) launch_attend_fp4(a, f32, head_dim, grid, stream);
  else if (type == kCacheBf16) launch_attend_bf16(a, source, head_dim, grid, stream);
  else launch_attend_f32(a, source, head_dim, grid, stream);
  launch_attend_join(a, source, f32, head_dim, max_rows, stream);
}

// Row tiles per workgroup, by what widening or reading the rows again costs against the
// registers of more tiles (128 groups of 4096 keys, D = 128, 64 rows: one, two, four tiles).
// 4-bit rows: one (62, 66, 68 us; fp32 queries 72, 86).  fp32 rows: two at most (309, 180,
// 237 us).  bf16 rows: as many as there are rows for, up to four (155, 89, 77 us).
int attend_row_tiles(int rows, CacheType type) {
  const int tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  return type == kCacheFp4 ? 1 : type == kCacheF32 ? std::min(tiles, 2) : tiles;
}

// Whether one workgroup takes all keys of a group's rows, in one launch, instead of
// several workgroups and a join.  Where the groups alone fill half of the CUs, up to 2048
// keys; else as many as it reads about as fast as the second launch takes, 288 KB, with 4-bit
// rows, which are widened first, counted twice; and with weights 32 KB of logits at most.
// Per call without the host, one / split: 128 groups of 4-bit rows (D = 128), 512, 1024,
// 2048, 4096 keys: 6.4/9.7, 9.0/12.4, 15.9/15.5, 27.0/22.1 us, of bf16 rows 9.6/11.4,
// 16.4/19.6, 25.7/28.3, 51.8/48.4 us; 8 groups, 4-bit rows, 512, 1024, 2048 keys: 6.3/7.8,
// 8.7/8.1, 13.5/8.5 us, bf16 8.7/8.3, 14.0/8.6, 22.7/9.1 us.
bool attend_in_one(int64_t rows, int64_t keys, bool weights, int64_t groups, CacheType type, int head_dim) {
  const int64_t bytes = type == kCacheFp4 ? 2 * (head_dim + head_dim / 16)
                                          : head_dim * (type == kCacheF32 ? 8 : 4);
  return rows <= 16 && keys <= 2048 && (groups >= 128 || keys * bytes <= 288 << 10) &&
         (!weights || rows * ((keys + 31) / 32 * 32) <= 8192);
}

// Workgroups a row block's keys are split over: two per CU in all (as many as the
// registers let run at once), each with 128 keys (one step of every wave) at least.
// (256, 512, 1024 workgroups in all: 128 groups of 4096 4-bit rows 24.5, 22.2, 26.0 us, of
// 8192 bf16 rows 113.5, 116.5, 118.3 us; 8 groups of 32768 4-bit rows 16.9, 16.6, 20.8 us.)
// Where that leaves the last round of workgroups thin (more than half of them row blocks,
// but no multiple), more splits, of 1024 keys at least, if that takes a quarter off the rounds:
// 264 groups of up to 6144, 16384 4-bit slots 53.9 -> 44.1, 161 -> 117 us, bf16 161 -> 138,
// 465 -> 360 us; 320 groups of up to 4096 4-bit slots 40.3 -> 34.6 us.  (Not for less: 400 and
// 800 groups of up to 4096 41.3 -> 43.0, 84.6 -> 90.2 us.)
int attend_splits(int64_t blocks, int64_t keys) {
  blocks = std::max<int64_t>(1, blocks);
  const int64_t first = std::max<int64_t>(1, 512 / blocks), most = std::max<int64_t>(1, (keys + 127) / 128);
  int64_t best = std::min<int64_t>({first, most, (int64_t)kAttendMaxSplits});
  auto rounds = [&](int64_t s) { return (blocks * s + 511) / 512; };
  for (int64_t s = best + 1; s <= std::min<int64_t>(first + 6, kAttendMaxSplits) && s * 1024 <= keys; ++s)
    if (rounds(s) * best * 4 <= rounds(best) * s * 3) best = s;
  return (int)best;
}

}  // namespace ckv

using ckv_api::cache_view;
using ckv_api::check_cache;
using ckv_api::fail;
using ckv_api::launched;
using ckv_api::ok;
using ckv_api::round_up;

namespace {

struct AttendPlan {
  ckv::AttendArgs a;
  size_t ml_bytes, o_bytes, logit_bytes;
  size_t total() const { return ml_bytes + o_bytes + logit_bytes; }
};

int plan_attend(const ckv_cache *c, const ckv_attend_problem *p, AttendPlan &pl) {
  int st;
  if ((st = check_cache(c))) return st;
  if (!p) return fail(CKV_INVALID_ARGUMENT, "attend problem is NULL");
  if (p->reserved != 0) return fail(CKV_INVALID_ARGUMENT, "reserved must be 0");
  if (p->accumulate != 0 && p->accumulate != 1)
    return fail(CKV_INVALID_ARGUMENT, "accumulate must be 0 or 1 (got %d)", p->accumulate);
  if (p->n_q < 1) return fail(CKV_INVALID_ARGUMENT, "n_q must be >= 1 (got %d)", p->n_q);
  if (p->n_q_heads < 1 || p->n_q_heads % c->n_kv_heads)
    return fail(CKV_INVALID_ARGUMENT, "n_q_heads must be a multiple of n_kv_heads (got %d, %d)",
                p->n_q_heads, c->n_kv_heads);
  const float scale = p->scale > 0.f ? p->scale : 1.f / sqrtf((float)c->head_dim);
  if (!std::isfinite(p->scale) || !std::isfinite(scale * ckv::kLog2e))
    return fail(CKV_INVALID_ARGUMENT, "scale must be finite, times log2(e) too");
  if (p->dtype != CKV_F32 && p->dtype != CKV_BF16)
    return fail(CKV_UNSUPPORTED, "queries must be CKV_F32 or CKV_BF16 (got %d)", p->dtype);
  if (c->dtype != CKV_FP4 && p->dtype != c->dtype)
    return fail(CKV_UNSUPPORTED, "queries over full rows must have the rows' dtype");
  const int64_t rows = (int64_t)p->n_q * (p->n_q_heads / c->n_kv_heads);
  if (rows > 64)
    return fail(CKV_UNSUPPORTED, "n_q * n_q_heads / n_kv_heads must be <= 64 (got %lld)",
                (long long)rows);
  ckv::AttendArgs &a = pl.a;
  a = ckv::AttendArgs{};
  a.c = cache_view(c);
  a.Hkv = c->n_kv_heads;
  a.G = p->n_q_heads / c->n_kv_heads;
  a.n_q = p->n_q;
  a.rows = (int32_t)rows;
  a.rt = ckv::attend_row_tiles(a.rows, (ckv::CacheType)c->dtype);
  a.row_blocks = (a.rows + 16 * a.rt - 1) / (16 * a.rt);
  a.blocks = a.c.groups * a.row_blocks;
  a.logit_stride = round_up(c->capacity, 32);
  a.accumulate = p->accumulate;
  a.masks = p->n_q > 1;
  a.one = ckv::attend_in_one(rows, c->capacity, true,      // the same bits with and without
                             a.c.groups, (ckv::CacheType)c->dtype, c->head_dim);
  a.splits = a.one ? 1 : ckv::attend_splits(a.blocks, c->capacity);
  a.c1 = scale * ckv::kLog2e;
  const size_t parts = (size_t)a.blocks * a.splits * 16 * a.rt;
  pl.ml_bytes = a.splits > 1 || (p->accumulate && !a.one) ? round_up(parts * sizeof(float2), 256) : 0;
  pl.o_bytes = a.splits > 1 ? round_up(parts * c->head_dim * sizeof(float), 256) : 0;
  pl.logit_bytes =
      p->accumulate && !a.one
          ? round_up((size_t)a.c.groups * a.rows * a.logit_stride * sizeof(float), 256) : 0;
  return CKV_OK;
}

}  // namespace

extern "C" {

size_t compresskv_cache_attend_workspace_bytes(const ckv_cache *c, const ckv_attend_problem *p) {
  AttendPlan pl;
  if (plan_attend(c, p, pl)) return 0;
  ok();
  return std::max<size_t>(256, pl.total());
}

int compresskv_cache_attend(const ckv_cache *c, const ckv_attend_problem *p, const void *q,
                            void *out, void *ws, size_t ws_bytes, void *stream) {
  AttendPlan pl;
  int st;
  if ((st = plan_attend(c, p, pl))) return st;
  if (!q || !out) return fail(CKV_INVALID_ARGUMENT, "q and out are required");
  if (!ckv_api::aligned(q, 16) || !ckv_api::aligned(out, 16))
    return fail(CKV_UNSUPPORTED, "q and out must be 16-byte aligned");
  if (!ws) return fail(CKV_INVALID_ARGUMENT, "ws is NULL");
  if (!ckv_api::aligned(ws, 256)) return fail(CKV_UNSUPPORTED, "ws must be 256-byte aligned");
  if (ws_bytes < std::max<size_t>(256, pl.total()))
    return fail(CKV_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given",
                std::max<size_t>(256, pl.total()), ws_bytes);
  ckv::AttendArgs &a = pl.a;
  a.q = static_cast<const char *>(q);
  a.out = static_cast<char *>(out);
  char *w = static_cast<char *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(w);
  a.part_o = reinterpret_cast<float *>(w + pl.ml_bytes);
  a.logits = reinterpret_cast<float *>(w + pl.ml_bytes + pl.o_bytes);
  ckv::launch_attend(a, ckv::kOverCache, (ckv::CacheType)c->dtype, p->dtype == CKV_F32, c->head_dim,
                     a.rows, (hipStream_t)stream);
  return launched("cache attend");
}

}  // extern "C"
