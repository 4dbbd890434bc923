/*
 * compresskv_cache.h -- C ABI of what follows a compressed prefill in
 * libcompresskv.so: a bounded KV cache per layer that the kept rows are loaded
 * into, that decoding appends to and attends over, and that is held within its
 * budget by evicting the slots that received the least attention; and the
 * attention of layers whose cache is bounded by position instead (a sliding
 * window and the first few tokens).
 *
 * The conventions of compresskv.h hold here too: device pointers unless the
 * name ends in _host, caller-owned memory, work enqueued on `stream` (a stream
 * of the current device, on which the buffers live), validation on the host
 * before any HIP call, status codes CKV_*, compresskv_last_error() for the
 * reason of a failure, deterministic results.  No call allocates, copies to the
 * host or sets memory, so every call can be captured into a HIP graph.  Calls
 * that overlap in time need workspaces of their own, and calls that write one
 * cache must not overlap with any other call on it.
 */
#ifndef COMPRESSKV_CACHE_H
#define COMPRESSKV_CACHE_H

#include "compresskv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of a cache held in 4 bits: per block of 32 consecutive values a scale
 * 2^e, stored as the byte e + 127, and 32 codes of one sign bit, two exponent
 * bits and one mantissa bit, for 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale;
 * value 2i in the low half of byte i.  A stored block takes the smallest e with
 * max |x| <= 7 * 2^e, kept in [-100, 125], and the code nearest to x / 2^e
 * (ties: the even code; the largest code is 6).  A block that holds an infinity
 * or a NaN takes the byte 255 and reads as NaN. */
#define CKV_FP4 2

/* A cache of one layer.  `len` live slots per (sequence, KV group), the first
 * ones; a slot is a K row, a V row, the position of its token and the attention
 * weight that it has received.  The slots are in no particular order once an
 * eviction has moved rows.  Values of len outside [0, capacity] are taken as
 * the nearer end. */
typedef struct ckv_cache {
  int32_t batch;        /* sequences, >= 1 */
  int32_t n_kv_heads;   /* KV groups Hkv, 1 .. 128; batch * n_kv_heads <= 65535 */
  int32_t head_dim;     /* D: 64 or 128 */
  int32_t capacity;     /* slots per (sequence, group), 1 .. 2^24; CKV_FP4: a multiple of 32 */
  int32_t dtype;        /* of the rows: CKV_F32, CKV_BF16 or CKV_FP4 */
  int32_t reserved;     /* must be 0 */
  void *k, *v;          /* [batch][Hkv][capacity][D], CKV_FP4: codes [batch][Hkv][capacity][D/2];
                           16-byte aligned */
  uint8_t *k_scale, *v_scale; /* CKV_FP4: [batch][Hkv][capacity][D/32], 16-byte aligned; else NULL */
  int32_t *pos;         /* [batch][Hkv][capacity] positions, 16-byte aligned */
  float *weight;        /* [batch][Hkv][capacity] accumulated weights, 16-byte aligned */
  int32_t *len;         /* [batch][Hkv] live slots */
  int32_t *seen;        /* [batch][Hkv] tokens of the sequence so far (the next position) */
} ckv_cache;

/*
 * Fills the cache from kept rows, as compresskv_compress_layer (and _layers)
 * write them: slot j of (b, g) takes row j of k_rows / v_rows
 * [batch][Hkv][n_rows][D] (dtype CKV_F32 or CKV_BF16) with the position
 * idx[b][g][j], for the entries of idx that are >= 0 (these come first, then -1
 * past the kept count).  Their weights become 0, len their number, and
 * seen[b][g] the length cu_seqlens[b+1] - cu_seqlens[b] of the prompt.  The
 * other slots are left as they are.
 * group_rows_host: NULL, or int32 [Hkv] for the ragged outputs of
 *   compresskv_compress_layer_heads: group g has group_rows_host[g] >= 1 rows,
 *   row j of (b, g) at b * total + off[g] + j (n_rows is not read).
 * Rows are stored as they are (the dtype of the cache), or in 4 bits.
 * 1 <= rows <= capacity; a CKV_F32 / CKV_BF16 cache takes rows of its own dtype.
 */
int compresskv_cache_load(const ckv_cache *c, int32_t dtype, int32_t n_rows, const void *k_rows,
                          const void *v_rows, const int32_t *idx, const int32_t *group_rows_host,
                          const int32_t *cu_seqlens, void *stream);

/*
 * Appends the rows of n_new >= 1 tokens of every sequence: slot len + i of
 * (b, g) takes row i with the position seen + i and the weight 0; len and seen
 * grow by n_new.  Rows that would pass the capacity are dropped (len stays at
 * the capacity, seen grows).  k_new, v_new: element (b, i, g, d) at
 * b * strides[0] + i * strides[1] + g * strides[2] + d, D contiguous, strides in
 * elements (int64 [3], host), each a multiple of 16 bytes and >= 0; 16-byte
 * aligned; dtype as for compresskv_cache_load.
 */
int compresskv_cache_append(const ckv_cache *c, int32_t dtype, int32_t n_new, const void *k_new,
                            const int64_t *k_strides_host, const void *v_new,
                            const int64_t *v_strides_host, void *stream);

/*
 * The rows as values: k_out, v_out [batch][Hkv][capacity][D], slots past len as
 * zeros.  dtype: CKV_F32 or CKV_BF16 (either holds every value of a 4-bit row
 * exactly); a CKV_F32 / CKV_BF16 cache is read in its own dtype.
 */
int compresskv_cache_read(const ckv_cache *c, int32_t dtype, void *k_out, void *v_out,
                          void *stream);

/* The queries of one decoding step. */
typedef struct ckv_attend_problem {
  int32_t n_q_heads;    /* Hq, a multiple of n_kv_heads; head h reads group h / (Hq / Hkv) */
  int32_t n_q;          /* query tokens per sequence, >= 1; n_q * Hq / Hkv <= 64 */
  int32_t dtype;        /* of q and out: CKV_F32 or CKV_BF16; the cache's own unless it is CKV_FP4 */
  int32_t accumulate;   /* 1: add what each slot receives to its weight; 0: leave the weights */
  float scale;          /* softmax scale, below 2.3e38; <= 0 selects 1/sqrt(head_dim) */
  int32_t reserved;     /* must be 0 */
} ckv_attend_problem;

size_t compresskv_cache_attend_workspace_bytes(const ckv_cache *c, const ckv_attend_problem *a);

/*
 * Attention of a step's query tokens over the cache:
 *   out[b][i][h] = sum over slots s of p(i, h, s) * v_s,
 *   p(i, h, .) = softmax over s of scale * q[b][i][h] . k_s.
 * One query token attends to every live slot; of n_q > 1, the last n_q tokens
 * of the sequence, token i attends to the slots at positions <= seen - n_q + i
 * (their own rows have been appended before).  A row that sees no slot gives
 * zeros, and so does one whose every visible logit is -infinity.  With accumulate,
 * weight_s += sum over i and the heads h of the group of p(i, h, s), added in fp32.
 * q, out: [batch][n_q][Hq][D], 16-byte aligned.  Logits, sums and softmax are held
 * in fp32.  Before the product with V a probability is rounded to 16 bits (bf16
 * queries; the output's own rounding is 2^8 times as coarse) or to 24.  K and V of
 * slots past len, and of slots that a row does not see, do not reach that row,
 * whatever they hold.
 * ws: >= compresskv_cache_attend_workspace_bytes(), 256-byte aligned.
 */
int compresskv_cache_attend(const ckv_cache *c, const ckv_attend_problem *a, const void *q,
                            void *out, void *ws, size_t ws_bytes, void *stream);

size_t compresskv_cache_evict_workspace_bytes(const ckv_cache *c, int32_t budget);

/*
 * Holds every (sequence, group) within `budget` live slots: of a group with
 * more, the len - budget slots of the least accumulated weight go (ties: the
 * highest slots; NaN counts as less than any weight).  Slots of the first
 * n_sinks positions and of the last n_recent ones (>= seen - n_recent) go only
 * when no other is left, the highest slots first.  The kept slots from budget on
 * then move, in ascending order, into the freed slots below it, in ascending order:
 * rows, positions and weights; no other slot is written.  Groups within the budget
 * are left as they are.  1 <= budget <= capacity; n_sinks, n_recent >= 0.
 * ws: >= compresskv_cache_evict_workspace_bytes(), 256-byte aligned.
 */
int compresskv_cache_evict(const ckv_cache *c, int32_t budget, int32_t n_sinks, int32_t n_recent,
                           void *ws, size_t ws_bytes, void *stream);

/* Sizes of a windowed attention over packed sequences. */
typedef struct ckv_window_problem {
  int32_t batch;        /* packed sequences, >= 1 */
  int32_t n_q_heads;    /* Hq, a multiple of n_kv_heads; head h reads group h / (Hq / Hkv) */
  int32_t n_kv_heads;   /* Hkv, 1 .. 128; batch * n_kv_heads <= 65535 */
  int32_t head_dim;     /* D: 64 or 128 */
  int32_t dtype;        /* CKV_F32 or CKV_BF16, of q, k, v and out */
  int32_t window;       /* keys that a token sees, itself included, >= 1 */
  int32_t n_sinks;      /* first positions that every later token sees, >= 0 */
  float scale;          /* softmax scale, below 2.3e38; <= 0 selects 1/sqrt(head_dim) */
  const int32_t *cu_q, *cu_q_host; /* device and host [batch+1]: query tokens, cu[0] = 0 */
  const int32_t *cu_k, *cu_k_host; /* the same for the keys; non-decreasing both,
                                      at most 2^30 tokens.  The launch is laid out
                                      for the host's values: the device's are the same
                                      whenever the call, or a graph of it, runs */
  int64_t q_stride_tok, q_stride_head; /* elements, multiples of 16 bytes, >= D */
  int64_t k_stride_tok, k_stride_head;
  int64_t v_stride_tok, v_stride_head;
} ckv_window_problem;

size_t compresskv_window_attention_workspace_bytes(const ckv_window_problem *p);

/*
 * Causal attention within a sliding window and the first tokens.  The queries
 * of sequence b are its last Lq = cu_q[b+1] - cu_q[b] tokens: query i stands at
 * t = Lk - Lq + i (Lk = cu_k[b+1] - cu_k[b] keys) and sees the keys j <= t with
 * j > t - window or j < n_sinks.  So Lq = Lk is a prompt, 1 < Lq < Lk a chunk of
 * one, Lq = 1 a decoding step.  A query that sees nothing (t < 0) gives zeros, and
 * so does one whose every visible logit is -infinity.
 * q [Tq][Hq][D], k, v [Tk][Hkv][D] packed, with the problem's strides; out
 * [Tq][Hq][D] dense; all 16-byte aligned.  Rows of out past the last sequence
 * are not written.  Logits, sums and softmax are held in fp32.  Before the product
 * with V a bf16 call rounds a probability once more: to 16 bits where no sequence has
 * more than 16 query rows per group (tokens times Hq / Hkv) or tokens of K or V lie more
 * than 2^24 bytes apart, and otherwise to 8 bits, as the output (the error is then about
 * 1.3 times that of the output's own rounding).  K and V of a key that a query does
 * not see do not reach it, whatever they hold.  Without any query nothing is done, and q and out may be NULL; without any key k and v may be.
 * Refused besides: 2^31 query rows (tokens times Hq / Hkv) or more in one sequence, and
 * more than 2^24 - 512 blocks of query rows in all; a block is 128 rows (bf16, more than 16
 * rows in some sequence, and tokens of K and V at most 2^24 bytes apart) or else 16 or 32.
 * ws: >= compresskv_window_attention_workspace_bytes(), 256-byte aligned.
 */
int compresskv_window_attention(const ckv_window_problem *p, const void *q, const void *k,
                                const void *v, void *out, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* COMPRESSKV_CACHE_H */
