// Attention of a few query rows per KV group over many keys, which may be split
// over several workgroups: the decoding step over a cache, and the windowed
// attention where it has few query rows or fp32 ones.
#pragma once

#include "cache_device.h"

namespace ckv {

constexpr int kAttendWaves = 4;       // waves of a workgroup, each on key steps of its own
constexpr int kAttendMaxSplits = 256;
constexpr float kLog2e = 1.44269504088896340736f;

// Rows of a group: row r is query token r / G, head g * G + r % G.
struct AttendArgs {
  CacheView c;                        // cache: rows, lengths, weights
  const char *q;                      // cache: [batch][n_q][Hq][D]; window: packed, strided
  char *out;                          // the same, dense
  const char *k, *v;                  // window: packed rows
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;   // window: byte strides
  const int32_t *cu_q, *cu_k;         // window
  float2 *part_ml;                    // [blocks][splits][16 RT] (reference, sum)
  float *part_o;                      // [blocks][splits][16 RT][D]
  float *logits;                      // accumulate (several splits): [groups][rows][logit_stride]
                                      // raw q . k
  int64_t logit_stride;
  int32_t Hkv, G, n_q;                // n_q: cache only
  int32_t rows;                       // cache: n_q * G
  int32_t rt;                         // row tiles per workgroup: 1, 2 or 4
  int32_t row_blocks, splits;         // row_blocks: of the group with the most rows
  int32_t blocks;                     // row blocks of all groups
  int32_t packed;                     // window: some group has fewer than row_blocks, and the
                                      // blocks are numbered without gaps (row_blocks.h)
  int32_t accumulate;                 // cache: add to the weights
  int32_t masks;                      // rows of a workgroup may see different keys
  int32_t join_rows;                  // rows per workgroup of the join (set by its launcher)
  int32_t one;                        // one workgroup per row block, no join (16 rows at most)
  int32_t window, sinks;              // window
  float c1;                           // softmax scale * log2(e)
};

// Which rows are attended over, and the precision of the products.
enum AttendSource : int { kOverCache = 0, kOverWindow = 1 };

// Enqueues the attention (and the join of its splits, with the accumulation of
// the weights if a.accumulate).  type: of the rows; f32: of q and out; max_rows: of
// the group with the most.  a.c.groups and a.Hkv are read for either source.
void launch_attend(const AttendArgs &a, AttendSource source, CacheType type, bool f32, int head_dim,
                   int max_rows, hipStream_t stream);

// bf16 prompts and chunks (window_prompt.hip): kPromptRows rows per workgroup, a.rt
// that many 16-row tiles.
constexpr int kPromptRows = 128;
constexpr int64_t kPromptMaxStride = 1 << 24;   // bytes between tokens: 64 rows stay within 32 bits
void launch_window_prompt(const AttendArgs &a, int head_dim, int max_rows, hipStream_t stream);

// Joins the splits' outputs, and adds to the weights if a.accumulate.
void launch_attend_join(AttendArgs a, AttendSource source, bool f32, int head_dim,
                        int max_rows, hipStream_t stream);

// Row tiles per workgroup for that many rows, and workgroups to split `keys` keys
// of each of `blocks` row blocks over.
int attend_row_tiles(int rows, CacheType type);
bool attend_in_one(int64_t rows, int64_t keys, bool weights, int64_t groups, CacheType type, int head_dim);
int attend_splits(int64_t blocks, int64_t keys);

}  // namespace ckv
