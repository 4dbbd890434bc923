// Causal attention of new tokens over a paged cache (include/compresskv_paged.h): the entry
// point, the plan of its launches, and the join of split rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged_api.h"
#include "pages_attend.h"
#include "score_common.h"

namespace ckv {

constexpr int kJoinGrid = 2048;                  // workgroups of a join

// What the launches of a call have, for the kernels that serve two together (16 sequences, four of them
// with 512 new tokens, of up to 8192 8-bit ones: one join instead of two 242 -> 237 us).
struct PagesBoth {
  PagesArgs a[2];
};

// One of the two, in the kernel's arguments (which selected by a value of theirs would be copied).  They
// are the kernel's first argument, which lies at the start of them.
__device__ __forceinline__ const PagesArgs &pages_args(int which) {
  typedef const __attribute__((address_space(4))) PagesBoth *kernarg_ptr;
  return ((const PagesBoth *)(kernarg_ptr)__builtin_amdgcn_kernarg_segment_ptr())->a[which];
}

// Sums up the batch for find_page_unit.  One workgroup, a run of sequences a thread.
__device__ __forceinline__ void pages_index(const PagesArgs &a) {
  constexpr int NTH = 1024, NW = NTH / 64;
  __shared__ float work_s[NW];
  __shared__ int longest_s[NW];
  __shared__ int3 run_s[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.c.batch + NTH - 1) / NTH, b0 = min(tid * per, a.c.batch), b1 = min(b0 + per, a.c.batch);
  auto add = [](auto u, auto v) { return u + v; };
  float work = 0.f;
  int longest = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    const int nb = page_blocks(a, a.cu_q[b + 1] - a.cu_q[b]), len = paged_len(a.c, b, a.max_len);
    work += (float)nb * (float)len;
    longest = max(longest, nb ? len : 0);
  }
  work = lane_scan(work, add);
  longest = lane_scan(longest, [](int u, int v) { return max(u, v); });
  if (lane == 63) work_s[wave] = work, longest_s[wave] = longest;
  __syncthreads();
  work = 0.f, longest = 0;
  for (int w = 0; w < NW; ++w) work += work_s[w], longest = max(longest, longest_s[w]);
  const int keys = page_keys(a, work, longest, [&](int keys) {
    int n = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b)
      n += page_run(a, a.cu_q[b + 1] - a.cu_q[b], paged_len(a.c, b, a.max_len), keys).units;
    n = lane_scan(n, add);
    __syncthreads();                               // (the last sums have been read)
    if (lane == 63) longest_s[wave] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < NW; ++w) n += longest_s[w];
    return n;
  });
  PageRun mine{0, 0, 0};
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    const PageRun x = page_run(a, a.cu_q[b + 1] - a.cu_q[b], paged_len(a.c, b, a.max_len), keys);
    mine.units += x.units, mine.slots += x.slots, mine.joins += x.joins;
  }
  const int3 upto = make_int3(lane_scan(mine.units, add), lane_scan(mine.slots, add), lane_scan(mine.joins, add));
  if (lane == 63) run_s[wave] = upto;
  __syncthreads();
  int4 at = make_int4(upto.x - mine.units, upto.y - mine.slots, upto.z - mine.joins, keys);
  for (int w = 0; w < wave; ++w) at.x += run_s[w].x, at.y += run_s[w].y, at.z += run_s[w].z;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    a.index[b] = at;
    const PageRun x = page_run(a, a.cu_q[b + 1] - a.cu_q[b], paged_len(a.c, b, a.max_len), keys);
    at.x += x.units, at.y += x.slots, at.z += x.joins;
  }
  if (tid == NTH - 1) a.index[a.c.batch] = at;     // (its run is the last one, or empty)
}

__global__ __launch_bounds__(1024) void pages_index_kernel(const PagesArgs a) { pages_index(a); }
__global__ __launch_bounds__(1024) void pages_index_both_kernel(const PagesBoth) {
  pages_index(pages_args(blockIdx.x));
}

template <typename First, typename... Rest>
std::is_same<First, PagesBoth> both_come_first(void (*)(First, Rest...));
static_assert(decltype(both_come_first(pages_index_both_kernel))::value);

// Grid (blocks of several splits, a few workgroups for the rows of each), 256 threads: D / 4 lanes per
// row, and where that leaves lanes (few rows, many splits) the splits are dealt to several such
// parts, whose sums are added in order.
template <typename T, int D>
__device__ __forceinline__ void pages_join(const PagesArgs &a, int id) {
  constexpr int LR = D / 4, NP = 256 / LR;         // lanes per row; rows x parts of the splits
  __shared__ __align__(16) f32x4 part_s[NP][LR];
  PageUnit at;
  if (!find_page_unit<false, true>(a, id, at)) return;   // uniform
  const int splits = at.splits, r0 = at.rb << a.rm_log2;
  if (splits == 1) return;                         // uniform: written by its workgroup
  const int rows = min(at.lq * a.G - r0, 1 << a.rm_log2);        // of the block
  const int parts = NP / a.join_rows, e = (int)threadIdx.x / LR, sub = (int)threadIdx.x % LR;
  const int mine = e / parts, part = e - mine * parts;
  for (int first = (int)blockIdx.y * a.join_rows; first < rows; first += (int)gridDim.y * a.join_rows) {   // uniform
    const bool in = first + mine < rows;
    const int64_t slot = (int64_t)at.slot * a.part_rows + first + (in ? mine : 0);
    const float2 *ml = a.part_ml + slot;
    const float *po = a.part_o + slot * D + 4 * sub;
    float top = -INFINITY;
    for (int s = sub; s < splits; s += LR) top = fmaxf(top, ml[(int64_t)s * a.part_rows].x);
#pragma unroll
    for (int o = LR / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int s = sub; s < splits; s += LR) {
      const float2 x = ml[(int64_t)s * a.part_rows];
      sum += x.y * fast_exp2(x.x - ref);
    }
#pragma unroll
    for (int o = LR / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = part; s < splits; s += parts) {
      const float f = fast_exp2(ml[(int64_t)s * a.part_rows].x - ref);
      const f32x4 x = *reinterpret_cast<const f32x4 *>(po + (int64_t)s * a.part_rows * D);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += x[k] * f;
    }
    if (parts > 1) {                               // uniform
      __syncthreads();                             // (the last rows' sums have been read)
      part_s[e][sub] = o;
      __syncthreads();
      for (int p = 1; p < parts && part == 0; ++p) {
        const f32x4 x = part_s[e + p][sub];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += x[k];
      }
    }
    if (!in || part) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int r = r0 + first + mine, i = r / a.G, h = at.g * a.G + (r - i * a.G);
    typedef T Tx4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<Tx4 *>(reinterpret_cast<T *>(a.out) +
                             ((int64_t)(at.q0 + i) * ((int64_t)a.c.Hkv * a.G) + h) * D + 4 * sub) =
        Tx4{(T)(o[0] * inv), (T)(o[1] * inv), (T)(o[2] * inv), (T)(o[3] * inv)};
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void pages_join_kernel(const PagesArgs a) {
  pages_join<T, D>(a, blockIdx.x);
}

// Of two launches, where the first has `first_joins` of the blocks.
template <typename T, int D>
__global__ __launch_bounds__(256) void pages_join_both_kernel(const PagesBoth, int first_joins) {
  const int which = (int)blockIdx.x >= first_joins ? 1 : 0;     // uniform
  pages_join<T, D>(pages_args(which), (int)blockIdx.x - which * first_joins);
}

static_assert(decltype(both_come_first(pages_join_both_kernel<float, 64>))::value);

void launch_pages_join(PagesBoth &both, bool f32, int head_dim, hipStream_t stream) {
  const int joins = both.a[0].joins + both.a[1].joins;
  if (joins == 0) return;
  int most = 1;
  for (PagesArgs &a : both.a) {
    if (a.joins == 0) continue;
    // as many rows as fill a workgroup, one where there may be many splits of a block
    a.join_rows = 1;
    if (a.target <= 8 * a.blocks)
      while (2 * a.join_rows <= std::min(a.part_rows, 1024 / head_dim)) a.join_rows *= 2;
    most = std::max(most, (a.part_rows + a.join_rows - 1) / a.join_rows);
  }
  // (finding its block costs a workgroup more than some rows: 16384, 8192, 4096, 2048, 1024 workgroups 277,
  // 279, 275, 273, 276 us for 16 sequences, four of them with 512 new tokens, of up to 8192 8-bit ones)
  const dim3 grid(joins, std::clamp(kJoinGrid / joins, 1, most));
  const dim3 block(256);
  auto as = [&]<typename T, int D>() {
    const PagesArgs &first = both.a[0], &second = both.a[1];
    if (first.joins && second.joins)
      hipLaunchKernelGGL((pages_join_both_kernel<T, D>), grid, block, 0, stream, both, first.joins);
    else
      hipLaunchKernelGGL((pages_join_kernel<T, D>), grid, block, 0, stream, first.joins ? first : second);
  };
  auto go = [&]<typename T>() {
    head_dim == 64 ? as.template operator()<T, 64>() : as.template operator()<T, 128>();
  };
  f32 ? go.template operator()<float>() : go.template operator()<__bf16>();
}

}  // namespace ckv

using ckv_api::check_offsets;
using ckv_api::check_paged;
using ckv_api::check_paged_dtype;
using ckv_api::fail;
using ckv_api::launched;
using ckv_api::ok;
using ckv_api::paged_view;
using ckv_api::round_up;

namespace {

// Row blocks of a call: a launch has fewer than 2^32 threads, a workgroup 512 at most, and the splits and
// whole runs of workgroups (pages_prompt.hip) add fewer than 4096 of these.
constexpr int64_t kMaxBlocks = (1 << 23) - 4096;

// One launch of a call, over the sequences whose query rows per group lie in its range.
struct PagesLaunch {
  ckv::PagesArgs a{};
  bool prompt = false;          // the kernel for many rows
  bool masks = false;           // some sequence has more than one new token
  int rt = 1;
  size_t at = 0, ml_bytes = 0, o_bytes = 0, index_bytes = 0;   // of the workspace
};

struct PagesPlan {
  PagesLaunch launch[2];
  int launches = 0;
  size_t total = 0;
};

// bf16 queries: sequences with more rows per group than this (two row tiles) go to the kernel for many.
constexpr int32_t kFewRows = 32;

// Workgroups that the keys are split for, and keys of a split at least.
// Few rows: some workgroups per CU (768, 1024, 2048 of them: 64 sequences of 500 to 8192 8-bit tokens
// 130, 130, 129 us, four of up to 131072 bf16 ones 214, 198, 204 us, 64 of up to 8 new tokens
// and 4096 121, 123, 136 us), of a step of every wave at least; where that makes more than 160, of up
// to 512 keys (8 sequences of 500 to 2048 bf16 tokens 20.9 -> 17.6 us, 4 of 4096 8-bit ones
// 20.7 -> 16.8 us; one of 8192 16.1 -> 16.7 us).
// Many rows: as many as page_keys finds best.
constexpr int32_t kFewTarget = 1024, kFewLeast = 128, kFewGentle = 160;
constexpr int32_t kManyLeast = 256, kCus = 256;

int plan_pages(const ckv_paged_cache *c, const ckv_chunk *ch, const ckv_paged_attend_problem *p, PagesPlan &pl) {
  int st;
  if ((st = check_paged(c))) return st;
  if (!ch) return fail(CKV_INVALID_ARGUMENT, "chunk is NULL");
  if ((st = check_offsets(ch->cu_q, ch->cu_q_host, c->batch, "cu_q"))) return st;
  if (!p) return fail(CKV_INVALID_ARGUMENT, "attend problem is NULL");
  if (p->reserved[0] != 0 || p->reserved[1] != 0)
    return fail(CKV_INVALID_ARGUMENT, "reserved must be 0");
  if (p->n_q_heads < 1 || p->n_q_heads % c->n_kv_heads)
    return fail(CKV_INVALID_ARGUMENT, "n_q_heads must be a multiple of n_kv_heads (got %d, %d)",
                p->n_q_heads, c->n_kv_heads);
  if (p->n_q_heads > ckv::kMaxQHeads)
    return fail(CKV_UNSUPPORTED, "n_q_heads must be <= %d", ckv::kMaxQHeads);
  const int32_t most = c->max_pages * c->page_size;
  if (p->max_len < 0 || p->max_len > most)
    return fail(CKV_INVALID_ARGUMENT, "max_len must be in [0, max_pages * page_size] (got %d)", p->max_len);
  const float scale = p->scale > 0.f ? p->scale : 1.f / sqrtf((float)c->head_dim);
  if (!std::isfinite(p->scale) || !std::isfinite(scale * ckv::kLog2e))
    return fail(CKV_INVALID_ARGUMENT, "scale must be finite, times log2(e) too");
  if ((st = check_paged_dtype(c, p->dtype))) return st;
  const int size = p->dtype == CKV_BF16 ? 2 : 4;
  const int64_t strides[] = {p->q_stride_tok, p->q_stride_head};
  for (int64_t s : strides) {
    if (s < c->head_dim || s > (int64_t)1 << 40)
      return fail(CKV_INVALID_ARGUMENT, "strides of q must be in [head_dim, 2^40]");
    if (s * size % 16) return fail(CKV_UNSUPPORTED, "strides of q must be multiples of 16 bytes");
  }
  ckv::PagesArgs all{};
  all.c = paged_view(c);
  all.G = p->n_q_heads / c->n_kv_heads;
  all.q_tok = p->q_stride_tok * size, all.q_head = p->q_stride_head * size;
  all.cu_q = ch->cu_q;
  all.max_len = p->max_len ? p->max_len : most;
  all.c1 = scale * ckv::kLog2e;
  const bool two = p->dtype == CKV_BF16;           // kinds of sequences
  int64_t all_blocks = 0;
  for (int kind = 0; kind < (two ? 2 : 1); ++kind) {
    PagesLaunch &la = pl.launch[pl.launches];
    ckv::PagesArgs &a = la.a = all;
    la.prompt = kind == 1;
    a.above = la.prompt ? kFewRows : 0;
    a.upto = two && !la.prompt ? kFewRows : INT32_MAX;
    int64_t max_rows = 0, longest = 0;
    for (int b = 0; b < c->batch; ++b) {
      const int64_t n = ch->cu_q_host[b + 1] - ch->cu_q_host[b], rows = n * a.G;
      longest = std::max(longest, rows);
      if (rows <= a.above || rows > a.upto) continue;
      max_rows = std::max(max_rows, rows);
      la.masks |= n > 1;
    }
    if (longest > INT32_MAX)
      return fail(CKV_UNSUPPORTED, "a sequence has 2^31 or more query rows per group");
    if (max_rows == 0) continue;
    ++pl.launches;
    // Two row tiles where there are the rows for them.  fp32 queries over 8-bit rows take one: their three parts
    // do not leave the registers for two (64 sequences of up to 8 new tokens over up to 4096 97 us, with two
    // 202; four chunks of up to 750 tokens over up to 3000, 32 / 8 heads, D = 128: 305 and 458 us).
    if (c->dtype == p->dtype || p->dtype == CKV_BF16) la.rt = max_rows > 16 ? 2 : 1;
    const int rm = !la.prompt ? 16 * la.rt : max_rows > 128 ? 256 : 128;
    a.rm_log2 = __builtin_ctz(rm);
    a.part_rows = (int32_t)std::min<int64_t>(rm, max_rows);
    const bool many = max_rows > 32;               // bound by the products
    a.slots = !many ? 0 : rm == 256 ? kCus : la.prompt ? 2 * kCus : 3 * kCus;   // registers allow as many
    a.target = many ? 2 * a.slots : kFewTarget;
    a.least = many ? kManyLeast : kFewLeast;
    a.gentle = many ? 0 : kFewGentle;
    int64_t blocks = 0, may_split = 0;
    for (int b = 0; b < c->batch; ++b) {
      const int64_t rows = (int64_t)(ch->cu_q_host[b + 1] - ch->cu_q_host[b]) * a.G;
      if (rows <= a.above || rows > a.upto) continue;
      const int64_t n = (rows + rm - 1) / rm * c->n_kv_heads;
      blocks += n;
      if (n < a.target) may_split += n;
    }
    all_blocks += blocks;
    if (all_blocks > kMaxBlocks) return fail(CKV_UNSUPPORTED, "too many query rows for one launch");
    a.blocks = (int32_t)blocks;
    // A sequence is split where it has more keys than all blocks' keys / target, so that one with
    // `target` blocks never is, and blocks that are split are fewer than `target`.  A block's splits are
    // less than one more than its keys over those, so that all blocks have blocks + target at most, and
    // those that are split as many as they are + target.
    const int64_t most_splits = (a.max_len + a.least - 1) / a.least;
    if (most_splits == 1) may_split = 0;
    a.grid = (int32_t)(blocks + std::min<int64_t>(may_split * (most_splits - 1), may_split ? a.target : 0));
    a.joins = (int32_t)std::min<int64_t>(may_split, a.target);
    const size_t parts = (size_t)std::min<int64_t>(may_split * most_splits, a.joins + a.target) * a.part_rows;
    la.at = pl.total;
    la.ml_bytes = round_up(parts * sizeof(float2), 256);
    la.o_bytes = round_up(parts * c->head_dim * sizeof(float), 256);
    la.index_bytes = c->batch > 64 ? round_up(((size_t)c->batch + 1) * sizeof(int4), 256) : 0;
    pl.total += la.ml_bytes + la.o_bytes + la.index_bytes;
  }
  return CKV_OK;
}

}  // namespace

extern "C" {

size_t compresskv_paged_attend_workspace_bytes(const ckv_paged_cache *c, const ckv_chunk *ch,
                                               const ckv_paged_attend_problem *p) {
  PagesPlan pl;
  if (plan_pages(c, ch, p, pl)) return 0;
  ok();
  return std::max<size_t>(256, pl.total);
}

int compresskv_paged_attend(const ckv_paged_cache *c, const ckv_chunk *ch,
                            const ckv_paged_attend_problem *p, const void *q, void *out, void *ws,
                            size_t ws_bytes, void *stream) {
  PagesPlan pl;
  int st;
  if ((st = plan_pages(c, ch, p, pl))) return st;
  if (pl.launches == 0) return ok();   // no query anywhere
  if (!q || !out) return fail(CKV_INVALID_ARGUMENT, "q and out are required");
  if (!ckv_api::aligned(q, 16) || !ckv_api::aligned(out, 16))
    return fail(CKV_UNSUPPORTED, "q and out must be 16-byte aligned");
  if (!ws) return fail(CKV_INVALID_ARGUMENT, "ws is NULL");
  if (!ckv_api::aligned(ws, 256)) return fail(CKV_UNSUPPORTED, "ws must be 256-byte aligned");
  if (ws_bytes < std::max<size_t>(256, pl.total))
    return fail(CKV_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given",
                std::max<size_t>(256, pl.total), ws_bytes);
  const bool f32 = p->dtype == CKV_F32;
  const hipStream_t s = (hipStream_t)stream;
  ckv::PagesBoth both{};
  for (int i = 0; i < pl.launches; ++i) {
    const PagesLaunch &la = pl.launch[i];
    ckv::PagesArgs &a = both.a[i] = la.a;
    a.q = static_cast<const char *>(q);
    a.out = static_cast<char *>(out);
    char *at = static_cast<char *>(ws) + la.at;
    a.part_ml = reinterpret_cast<float2 *>(at);
    a.part_o = reinterpret_cast<float *>(at + la.ml_bytes);
    if (la.index_bytes) a.index = reinterpret_cast<int4 *>(at + la.ml_bytes + la.o_bytes);
  }
  if (both.a[0].index && pl.launches == 2)
    hipLaunchKernelGGL(ckv::pages_index_both_kernel, dim3(2), dim3(1024), 0, s, both);
  else if (both.a[0].index)
    hipLaunchKernelGGL(ckv::pages_index_kernel, dim3(1), dim3(1024), 0, s, both.a[0]);
  for (int i = 0; i < pl.launches; ++i) {
    const PagesLaunch &la = pl.launch[i];
    const ckv::PagesArgs &a = both.a[i];
    if (la.prompt) ckv::launch_pages_prompt(a, c->dtype == CKV_FP8, c->head_dim, s);
    else if (c->dtype == CKV_FP8) ckv::launch_pages_fp8(a, f32, c->head_dim, la.rt, la.masks, s);
    else if (c->dtype == CKV_BF16) ckv::launch_pages_bf16(a, c->head_dim, la.rt, la.masks, s);
    else ckv::launch_pages_f32(a, c->head_dim, la.rt, la.masks, s);
  }
  ckv::launch_pages_join(both, f32, c->head_dim, s);
  return launched("paged attend");
}

}  // extern "C"
