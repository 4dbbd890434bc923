// Host-side helpers of the entry points around the bounded cache.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/compresskv_cache.h"
#include "api_common.h"
#include "cache_device.h"

namespace ckv_api {

inline size_t round_up(size_t n, size_t a) { return (n + a - 1) / a * a; }

inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess)
    return fail(CKV_HIP_ERROR, "%s launch failed: %s", what, hipGetErrorString(e));
  return ok();
}

// Bytes of one K (or V) row, scales apart.
inline int row_bytes(const ckv_cache *c) {
  return c->dtype == CKV_FP4 ? c->head_dim / 2
                             : c->head_dim * (c->dtype == CKV_BF16 ? 2 : 4);
}

inline int check_cache(const ckv_cache *c) {
  if (!c) return fail(CKV_INVALID_ARGUMENT, "cache is NULL");
  if (c->batch < 1 || c->n_kv_heads < 1 || c->capacity < 1)
    return fail(CKV_INVALID_ARGUMENT, "batch, n_kv_heads and capacity must be >= 1");
  if (c->reserved != 0) return fail(CKV_INVALID_ARGUMENT, "reserved must be 0");
  if (c->dtype != CKV_F32 && c->dtype != CKV_BF16 && c->dtype != CKV_FP4)
    return fail(CKV_UNSUPPORTED, "dtype must be CKV_F32, CKV_BF16 or CKV_FP4 (got %d)", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(CKV_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", c->head_dim);
  if (c->n_kv_heads > ckv::kMaxKvHeads || (int64_t)c->batch * c->n_kv_heads > 65535)
    return fail(CKV_UNSUPPORTED, "n_kv_heads must be <= %d and batch * n_kv_heads <= 65535",
                ckv::kMaxKvHeads);
  if (c->capacity > (1 << 24))
    return fail(CKV_UNSUPPORTED, "capacity must be <= 2^24 (got %d)", c->capacity);
  if (c->dtype == CKV_FP4 && c->capacity % 32)
    return fail(CKV_UNSUPPORTED, "the capacity of a 4-bit cache must be a multiple of 32 (got %d)",
                c->capacity);
  struct Field { const void *p; const char *name; size_t align; };
  const Field need[] = {{c->k, "k", 16},     {c->v, "v", 16},      {c->pos, "pos", 16},
                        {c->weight, "weight", 16}, {c->len, "len", 4}, {c->seen, "seen", 4}};
  for (const Field &f : need) {
    if (!f.p) return fail(CKV_INVALID_ARGUMENT, "%s is NULL", f.name);
    if (!aligned(f.p, f.align))
      return fail(CKV_UNSUPPORTED, "%s must be %zu-byte aligned", f.name, f.align);
  }
  if (c->dtype == CKV_FP4) {
    if (!c->k_scale || !c->v_scale)
      return fail(CKV_INVALID_ARGUMENT, "a 4-bit cache needs k_scale and v_scale");
    if (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))
      return fail(CKV_UNSUPPORTED, "k_scale and v_scale must be 16-byte aligned");
  }
  return CKV_OK;
}

// Rows of `dtype` go in and out of the cache.
inline int check_rows_dtype(const ckv_cache *c, int dtype) {
  if (dtype != CKV_F32 && dtype != CKV_BF16)
    return fail(CKV_UNSUPPORTED, "rows must be CKV_F32 or CKV_BF16 (got %d)", dtype);
  if (c->dtype != CKV_FP4 && dtype != c->dtype)
    return fail(CKV_UNSUPPORTED, "a cache of full rows takes and gives rows of its own dtype");
  return CKV_OK;
}

inline ckv::CacheView cache_view(const ckv_cache *c) {
  ckv::CacheView v;
  v.k = static_cast<char *>(c->k);
  v.v = static_cast<char *>(c->v);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.pos = c->pos;
  v.weight = c->weight;
  v.len = c->len;
  v.seen = c->seen;
  v.groups = c->batch * c->n_kv_heads;
  v.Hkv = c->n_kv_heads;
  v.capacity = c->capacity;
  return v;
}

}  // namespace ckv_api
