// Attention within a sliding window and the first tokens over packed sequences
// (include/compresskv_cache.h): the entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attend.h"
#include "cache_api.h"

using ckv_api::fail;
using ckv_api::launched;
using ckv_api::ok;
using ckv_api::round_up;

namespace {

constexpr int32_t kMaxTokens = 1 << 30;
// Row blocks of a call: 256 threads each, and a launch has 2^32 at most (the kernel for
// many rows rounds up by 255 blocks).
constexpr int64_t kMaxBlocks = (1 << 24) - 512;

struct WindowPlan {
  ckv::AttendArgs a;
  int64_t max_rows;             // query rows of one (sequence, group)
  bool prompt;                  // the kernel for many rows
  size_t ml_bytes, o_bytes;
  size_t total() const { return ml_bytes + o_bytes; }
};

// bf16 calls with more rows per group than this (a row tile) take the kernel for many
// rows.  One sequence of 8192 keys, 32 / 8 heads, with 16, 20, 32, 64 rows per group: 16.3, 19.0,
// 20.5, 40.5 us by the kernel for few, 16.3, 16.6, 17.1, 18.9 us by the one for many; eight:
// 49.0, 51.5, 52.7, 80.3 and 49.9, 51.5, 52.0, 56.2 us.
constexpr int64_t kFewRows = 16;

// Workgroups that a row block's keys are split over in the kernel for many
// rows: as many as two per CU in all leave room for, four tiles each at least.
// (64 queries over 8192 keys, 32 / 8 heads: 32.6 us; with twice as many workgroups, of two
// tiles at least, 46.2 us.)
int prompt_splits(int64_t blocks, int64_t keys) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / blocks, (keys + 255) / 256, 64}));
}

int check_cu(const int32_t *cu, int batch, const char *name) {
  if (cu[0] != 0) return fail(CKV_INVALID_ARGUMENT, "%s[0] must be 0", name);
  for (int b = 0; b < batch; ++b)
    if (cu[b + 1] < cu[b])
      return fail(CKV_INVALID_ARGUMENT, "%s must be non-decreasing (sequence %d)", name, b);
  return CKV_OK;
}

int plan_window(const ckv_window_problem *p, WindowPlan &pl) {
  if (!p) return fail(CKV_INVALID_ARGUMENT, "window problem is NULL");
  if (p->batch < 1 || p->n_kv_heads < 1)
    return fail(CKV_INVALID_ARGUMENT, "batch and n_kv_heads must be >= 1");
  if (p->n_q_heads < 1 || p->n_q_heads % p->n_kv_heads)
    return fail(CKV_INVALID_ARGUMENT, "n_q_heads must be a multiple of n_kv_heads (got %d, %d)",
                p->n_q_heads, p->n_kv_heads);
  if (p->window < 1) return fail(CKV_INVALID_ARGUMENT, "window must be >= 1 (got %d)", p->window);
  if (p->n_sinks < 0) return fail(CKV_INVALID_ARGUMENT, "n_sinks must be >= 0 (got %d)", p->n_sinks);
  const float scale = p->scale > 0.f ? p->scale : 1.f / sqrtf((float)p->head_dim);
  if (!std::isfinite(p->scale) || !std::isfinite(scale * ckv::kLog2e))
    return fail(CKV_INVALID_ARGUMENT, "scale must be finite, times log2(e) too");
  if (!p->cu_q || !p->cu_q_host || !p->cu_k || !p->cu_k_host)
    return fail(CKV_INVALID_ARGUMENT, "cu_q, cu_q_host, cu_k and cu_k_host are required");
  int st;
  if ((st = check_cu(p->cu_q_host, p->batch, "cu_q_host"))) return st;
  if ((st = check_cu(p->cu_k_host, p->batch, "cu_k_host"))) return st;
  if (p->dtype != CKV_F32 && p->dtype != CKV_BF16)
    return fail(CKV_UNSUPPORTED, "dtype must be CKV_F32 or CKV_BF16 (got %d)", p->dtype);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(CKV_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", p->head_dim);
  if (p->n_kv_heads > ckv::kMaxKvHeads || (int64_t)p->batch * p->n_kv_heads > 65535 ||
      p->n_q_heads > ckv::kMaxQHeads)
    return fail(CKV_UNSUPPORTED, "n_kv_heads must be <= %d, n_q_heads <= %d and batch * n_kv_heads "
                                 "<= 65535", ckv::kMaxKvHeads, ckv::kMaxQHeads);
  if (p->cu_q_host[p->batch] > kMaxTokens || p->cu_k_host[p->batch] > kMaxTokens)
    return fail(CKV_UNSUPPORTED, "at most 2^30 query tokens and keys");
  const int size = p->dtype == CKV_BF16 ? 2 : 4;
  const int64_t strides[] = {p->q_stride_tok, p->q_stride_head, p->k_stride_tok,
                             p->k_stride_head, p->v_stride_tok, p->v_stride_head};
  for (int64_t s : strides) {
    if (s < p->head_dim || s > (int64_t)1 << 40)
      return fail(CKV_INVALID_ARGUMENT, "strides must be in [head_dim, 2^40]");
    if (s * size % 16) return fail(CKV_UNSUPPORTED, "strides must be multiples of 16 bytes");
  }
  ckv::AttendArgs &a = pl.a;
  a = ckv::AttendArgs{};
  a.c.groups = p->batch * p->n_kv_heads;
  a.Hkv = p->n_kv_heads;
  a.G = p->n_q_heads / p->n_kv_heads;
  pl.max_rows = 0;
  int64_t keys = 0;              // that a row block may read, at most
  for (int b = 0; b < p->batch; ++b) {
    const int64_t lq = p->cu_q_host[b + 1] - p->cu_q_host[b];
    const int64_t lk = p->cu_k_host[b + 1] - p->cu_k_host[b];
    if (lq == 0) continue;
    pl.max_rows = std::max(pl.max_rows, lq * a.G);
    const int64_t span = std::min<int64_t>(lq, ckv::kPromptRows / a.G + 1);   // tokens of a block
    keys = std::max(keys, std::min<int64_t>(lk, (int64_t)p->window + p->n_sinks + span - 1));
  }
  if (pl.max_rows > INT32_MAX)
    return fail(CKV_UNSUPPORTED, "a sequence has 2^31 or more query rows per group");
  pl.prompt = p->dtype == CKV_BF16 && pl.max_rows > kFewRows &&
              std::max(p->k_stride_tok, p->v_stride_tok) * size <= ckv::kPromptMaxStride;
  a.rt = pl.prompt                ? ckv::kPromptRows / 16
         : p->dtype == CKV_BF16 ? 1
                                : ckv::attend_row_tiles((int)std::min<int64_t>(pl.max_rows, 64), ckv::kCacheF32);
  a.row_blocks = (int32_t)((pl.max_rows + 16 * a.rt - 1) / (16 * a.rt));
  a.masks = pl.max_rows > a.G;   // more than one token in some row block
  a.one = !pl.prompt && ckv::attend_in_one(pl.max_rows, keys, false, a.c.groups,
                                           p->dtype == CKV_F32 ? ckv::kCacheF32 : ckv::kCacheBf16,
                                           p->head_dim);
  // The row blocks that there are, where one per group is not all: sequences of other lengths
  // beside a long one cost no workgroups and no workspace then.
  const int64_t most = (int64_t)a.c.groups * a.row_blocks;
  int64_t blocks = most;
  if (pl.prompt || (a.masks && !a.one)) {
    blocks = 0;
    for (int b = 0; b < p->batch; ++b) {
      const int64_t rows = (int64_t)(p->cu_q_host[b + 1] - p->cu_q_host[b]) * a.G;
      blocks += (rows + 16 * a.rt - 1) / (16 * a.rt) * a.Hkv;
    }
  }
  if (blocks > kMaxBlocks) return fail(CKV_UNSUPPORTED, "too many query rows for one launch");
  a.blocks = (int32_t)blocks;
  a.packed = blocks < most;
  a.splits = pl.prompt ? prompt_splits(blocks, keys)
             : a.one   ? 1
                       : ckv::attend_splits(blocks, keys);
  a.window = std::min(p->window, kMaxTokens);   // positions plus or minus either stay in 32 bits
  a.sinks = std::min(p->n_sinks, kMaxTokens);
  a.q_tok = p->q_stride_tok * size, a.q_head = p->q_stride_head * size;
  a.k_tok = p->k_stride_tok * size, a.k_head = p->k_stride_head * size;
  a.v_tok = p->v_stride_tok * size, a.v_head = p->v_stride_head * size;
  a.cu_q = p->cu_q;
  a.cu_k = p->cu_k;
  a.c1 = scale * ckv::kLog2e;
  const size_t parts = (size_t)a.blocks * a.splits * 16 * a.rt;
  pl.ml_bytes = a.splits > 1 ? round_up(parts * sizeof(float2), 256) : 0;
  pl.o_bytes = a.splits > 1 ? round_up(parts * p->head_dim * sizeof(float), 256) : 0;
  return CKV_OK;
}

}  // namespace

extern "C" {

size_t compresskv_window_attention_workspace_bytes(const ckv_window_problem *p) {
  WindowPlan pl;
  if (plan_window(p, pl)) return 0;
  ok();
  return std::max<size_t>(256, pl.total());
}

int compresskv_window_attention(const ckv_window_problem *p, const void *q, const void *k,
                                const void *v, void *out, void *ws, size_t ws_bytes, void *stream) {
  WindowPlan pl;
  int st;
  if ((st = plan_window(p, pl))) return st;
  if (pl.max_rows == 0) return ok();   // no query anywhere
  const void *ptrs[] = {q, out, k, v};
  const char *names[] = {"q", "out", "k", "v"};
  const int needed = p->cu_k_host[p->batch] > 0 ? 4 : 2;   // without keys, k and v are not read
  for (int i = 0; i < needed; ++i) {
    if (!ptrs[i]) return fail(CKV_INVALID_ARGUMENT, "%s is NULL", names[i]);
    if (!ckv_api::aligned(ptrs[i], 16))
      return fail(CKV_UNSUPPORTED, "%s must be 16-byte aligned", names[i]);
  }
  if (pl.total() > 0) {
    if (!ws) return fail(CKV_INVALID_ARGUMENT, "ws is NULL");
    if (!ckv_api::aligned(ws, 256)) return fail(CKV_UNSUPPORTED, "ws must be 256-byte aligned");
    if (ws_bytes < pl.total())
      return fail(CKV_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given", pl.total(),
                  ws_bytes);
  }
  ckv::AttendArgs &a = pl.a;
  a.q = static_cast<const char *>(q);
  a.k = static_cast<const char *>(k);
  a.v = static_cast<const char *>(v);
  a.out = static_cast<char *>(out);
  a.part_ml = static_cast<float2 *>(ws);
  a.part_o = reinterpret_cast<float *>(static_cast<char *>(ws) + pl.ml_bytes);
  const bool f32 = p->dtype == CKV_F32;
  if (pl.prompt)
    ckv::launch_window_prompt(a, p->head_dim, (int)pl.max_rows, (hipStream_t)stream);
  else
    ckv::launch_attend(a, ckv::kOverWindow, f32 ? ckv::kCacheF32 : ckv::kCacheBf16, f32, p->head_dim,
                       (int)pl.max_rows, (hipStream_t)stream);
  return launched("window attention");
}

}  // extern "C"
