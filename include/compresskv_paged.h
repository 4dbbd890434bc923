/*
 * compresskv_paged.h -- C ABI of what comes before a prompt's compression in
 * libcompresskv.so: rotary positions, a paged KV cache that the rotated keys and
 * the values of new tokens are written into (as they are, or in 8 bits) and read
 * back from, packed as compresskv_compress_layer takes them, and the causal
 * attention of new tokens (a chunk of a prompt, or single tokens) over it.
 *
 * The conventions of compresskv.h and compresskv_cache.h hold here too: device
 * pointers unless the name ends in _host, caller-owned memory, work enqueued on
 * `stream` (a stream of the current device, on which the buffers live), validation
 * on the host before any HIP call, status codes CKV_*, compresskv_last_error()
 * for the reason of a failure, deterministic results.  No call allocates, copies
 * to the host or sets memory, so every call can be captured into a HIP graph.
 * Calls that overlap in time need workspaces of their own, and a call that writes
 * a cache must not overlap with any other call on its pages.
 */
#ifndef COMPRESSKV_PAGED_H
#define COMPRESSKV_PAGED_H

#include "compresskv_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows held in 8 bits: per block of 32 consecutive values a scale 2^e, stored as
 * the byte e + 127, and 32 codes of one sign bit, four exponent bits (bias 7) and
 * three mantissa bits (exponent 0: m / 8 * 2^-6; the largest code is 448, there are no
 * infinities, and the code with all lower bits set is a NaN).  A stored block takes
 * the smallest e in [-100, 119] with max |x| <= 448 * 2^e (119 if there is none) and the
 * code nearest to x / 2^e (ties: the even code; past 448: 448).  A block that holds an
 * infinity or a NaN takes the byte 255 and reads as NaN. */
#define CKV_FP8 3

/* which dimensions of a head turn together (n = rotary_dim) */
#define CKV_ROTARY_HALF 0  /* i and i + n / 2, i < n / 2 */
#define CKV_ROTARY_PAIRS 1 /* 2 i and 2 i + 1 */

/* how the frequencies are scaled for long contexts */
#define CKV_ROTARY_PLAIN 0  /* not at all */
#define CKV_ROTARY_LINEAR 1 /* every frequency divided by `factor` */
#define CKV_ROTARY_BLEND 2  /* by the turns t that a pair makes within original_len tokens: kept where
                               t >= high, divided by `factor` where t <= low, and in between
                               f * s + f / factor * (1 - s) with s = (t - low) / (high - low) */

/* A rotation of the heads: pair i of a token at position m turns by the angle m * f_i, and
 * is multiplied by `amplitude`.  Dimensions from rotary_dim on are left as they are. */
typedef struct ckv_rotary {
  int32_t head_dim;     /* D: 64 or 128 */
  int32_t rotary_dim;   /* dimensions that turn, the first ones: a multiple of 16, 16 .. D */
  int32_t layout;       /* CKV_ROTARY_HALF or CKV_ROTARY_PAIRS */
  float amplitude;      /* finite; 1 leaves lengths as they are */
  const uint64_t *turns; /* [rotary_dim / 2]: the part of a turn per position, f_i / (2 pi), as a
                            64-bit fraction (times 2^64); 8-byte aligned.  An angle is then exact
                            modulo one turn, to 2^-65 of a turn per position, at every position */
  int32_t reserved[2];  /* must be 0 */
} ckv_rotary;

/*
 * Fills turns_host [rotary_dim / 2] for f_i = base^(-2 i / rotary_dim), scaled by
 * `scaling`.  base >= 1; factor > 0 (LINEAR, BLEND); 0 <= low < high and
 * original_len >= 1 (BLEND).  Host code, in extended precision; copy the table to
 * the device once.
 */
int compresskv_rotary_turns(int32_t rotary_dim, double base, int32_t scaling, double factor,
                            double low, double high, int32_t original_len, uint64_t *turns_host);

/* Tokens' rows: element (t, h, d) at t * stride_tok + h * stride_head + d.  Strides in
 * elements, multiples of 16 bytes, >= 0 (inputs) or >= D (outputs); data 16-byte aligned. */
typedef struct ckv_rows {
  void *data;
  int64_t stride_tok, stride_head;
} ckv_rows;

/*
 * Rotates the rows of n_tokens >= 0 tokens: n_q_heads >= 0 heads of q to q_out and
 * n_k_heads >= 0 of k to k_out, at least one head in all (q, k: input rows, only
 * read).  pos: int32 [n_tokens], any values.  transposed: 0, or 1 for the transposed
 * rotation, which takes the gradient of an output to that of its input.  Values are computed in
 * fp32, from cosines and sines that are rounded to it once: off by 2^-22 (|x0 c| + |x1 s|) at most, besides
 * what the table's angles are.  A bf16 output is rounded once more.  dtype: CKV_F32 or CKV_BF16.  Outputs may be their
 * own inputs (same data and strides) and must not overlap otherwise.
 */
int compresskv_rotary(const ckv_rotary *r, int32_t dtype, int32_t transposed, int32_t n_tokens,
                      const int32_t *pos, int32_t n_q_heads, const ckv_rows *q, const ckv_rows *q_out,
                      int32_t n_k_heads, const ckv_rows *k, const ckv_rows *k_out, void *stream);

/* A paged cache of one layer.  Token j of sequence b lies in slot j % page_size of page
 * page_table[b][j / page_size]; len[b] tokens of it are there, those of the call's
 * own chunk included.  The table and the lengths are the layers' in common, and only
 * read.  Lengths outside [0, max_pages * page_size] are taken as the nearer end.  An
 * entry outside [0, n_pages) stands for no page: its tokens are not written, read as
 * zeros, and no query sees them.  Sequences may share pages that no call writes; the
 * slots that one call writes are different ones. */
typedef struct ckv_paged_cache {
  int32_t batch;        /* sequences, >= 1; batch * n_kv_heads <= 65535 */
  int32_t n_kv_heads;   /* KV groups Hkv, 1 .. 128 */
  int32_t head_dim;     /* D: 64 or 128 */
  int32_t page_size;    /* tokens per page: a power of two, 16 .. 65536 */
  int32_t n_pages;      /* pages of the pool, >= 1 */
  int32_t max_pages;    /* entries per sequence of the table, >= 1; max_pages * page_size <= 2^24 */
  int32_t dtype;        /* of the rows: CKV_F32, CKV_BF16 or CKV_FP8 */
  int32_t reserved;     /* must be 0 */
  void *k, *v;          /* [n_pages][Hkv][page_size][D], CKV_FP8: codes; 16-byte aligned */
  uint8_t *k_scale, *v_scale; /* CKV_FP8: [n_pages][Hkv][page_size][D / 32], 16-byte aligned; else NULL */
  const int32_t *page_table;  /* [batch][max_pages] */
  const int32_t *len;         /* [batch] */
} ckv_paged_cache;

/* The new tokens of a call, packed: sequence b's are the last cu_q[b+1] - cu_q[b] of its
 * len[b] tokens.  Device and host [batch + 1], cu_q[0] = 0, non-decreasing, at most 2^30
 * tokens.  The launch is laid out for the host's values: the device's are the same whenever
 * the call, or a graph of it, runs. */
typedef struct ckv_chunk {
  const int32_t *cu_q, *cu_q_host;
} ckv_chunk;

/*
 * Writes the rows of the chunk's tokens into the cache: token i of sequence b's n new
 * ones goes to position len[b] - n + i (positions below 0 are not written).
 * r: NULL, or the rotation of k_new (and of q, if n_q_heads > 0, to q_out), by that
 * position.  k_new, v_new, q: rows of dtype CKV_F32 or CKV_BF16 (the cache's own unless it is
 * CKV_FP8).  Without a rotation n_q_heads is 0.  q_out and rows stored in fp32 or bf16 are as
 * compresskv_rotary gives them; 8-bit rows are turned in fp64, so that a code is the nearest to the exact
 * value.  q_out may be q itself.
 */
int compresskv_paged_append(const ckv_paged_cache *c, const ckv_chunk *ch, const ckv_rotary *r,
                            int32_t dtype, const ckv_rows *k_new, const ckv_rows *v_new,
                            int32_t n_q_heads, const ckv_rows *q, const ckv_rows *q_out,
                            void *stream);

/*
 * The first cu_k[b+1] - cu_k[b] tokens of every sequence, packed: k_out, v_out
 * [cu_k[batch]][Hkv][D] dense, 16-byte aligned, as ckv_problem describes a prompt's.  Tokens
 * past len[b] are zeros.  dtype: CKV_F32 or CKV_BF16 (either holds every value that an 8-bit
 * row was stored with exactly); a CKV_F32 / CKV_BF16 cache is read in its own dtype.  cu_k,
 * cu_k_host: as ckv_chunk's.
 */
int compresskv_paged_read(const ckv_paged_cache *c, int32_t dtype, const int32_t *cu_k,
                          const int32_t *cu_k_host, void *k_out, void *v_out, void *stream);

/* The queries of a chunk. */
typedef struct ckv_paged_attend_problem {
  int32_t n_q_heads;    /* Hq, a multiple of n_kv_heads, <= 256; head h reads group h / (Hq / Hkv) */
  int32_t dtype;        /* of q and out: CKV_F32 or CKV_BF16; the cache's own unless it is CKV_FP8 */
  int32_t max_len;      /* no len[b] is larger (they are taken as this otherwise); 0: max_pages *
                           page_size.  It lays out the launch and the workspace, results but for
                           rounding do not depend on it */
  float scale;          /* softmax scale, below 2.3e38; <= 0 selects 1/sqrt(head_dim) */
  int64_t q_stride_tok, q_stride_head; /* elements, multiples of 16 bytes, >= D */
  int32_t reserved[2];  /* must be 0 */
} ckv_paged_attend_problem;

/* Bytes of workspace, by the chunk's tokens, the heads and max_len: what the splits of the keys need that
 * the lengths may make, 165 MiB at most (single tokens of 8 groups: 2 MiB; a chunk of 2048 tokens
 * of 8 groups of 4 heads of 128: 98 MiB).  Calls that follow each other on a stream can share one. */
size_t compresskv_paged_attend_workspace_bytes(const ckv_paged_cache *c, const ckv_chunk *ch,
                                               const ckv_paged_attend_problem *p);

/*
 * Causal attention of the chunk's tokens over their sequences' pages: token i of
 * sequence b's n new ones stands at t = len[b] - n + i and sees the keys j <= t (its
 * own has been appended before).  A row that sees nothing (t < 0, or no page) gives
 * zeros, and so does one whose every visible logit is -infinity.
 * q [cu_q[batch]][Hq][D] with the problem's strides, out dense; 16-byte aligned.  Rows of
 * out past the last sequence are not written.  Logits, sums and softmax are held in fp32.
 * Before the product with V a bf16 call rounds a probability once more: to 16 bits in
 * sequences of at most 32 query rows per group (tokens times Hq / Hkv), and to 8 bits, as the
 * output, in others.  The products with V are added up before they are divided by the sum, so
 * that values of V beyond 2^116 / (keys seen) may give infinities.  An infinite value of V
 * whose key has a weight of 2^-100 of the row's largest at least gives that infinity (NaN where both
 * signs meet); one of less weight may give a NaN instead.  K and V of keys that a row does not see
 * do not reach it, whatever they hold.
 * Refused besides: 2^31 query rows (tokens times Hq / Hkv) or more in one sequence, and
 * more than 2^23 - 4096 blocks of query rows in all.  A block is 256 rows of a bf16 sequence
 * (128 where none has more), and 32 of one of at most 32 rows and of fp32 (16 where none has more than 16,
 * and of fp32 over 8-bit rows).
 * ws: >= compresskv_paged_attend_workspace_bytes(), 256-byte aligned.
 */
int compresskv_paged_attend(const ckv_paged_cache *c, const ckv_chunk *ch,
                            const ckv_paged_attend_problem *p, const void *q, void *out, void *ws,
                            size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* COMPRESSKV_PAGED_H */
