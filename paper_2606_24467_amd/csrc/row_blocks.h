// The numbering of the row blocks of packed sequences (the windowed attention's
// kernels and their join): those that there are, sequence by sequence and group by
// group, without gaps.
#pragma once

#include "attend.h"

namespace ckv {

struct RowBlock {
  int b, g, rb;                  // sequence, group, row block of the two
  int part;                      // its number: where its partial results lie
  int q0, lq, k0, lk;            // the sequence's queries and keys
};

// Row block `id` of rows_per_block rows; LATEST_FIRST: counted from a group's last rows.
// The wave calls this together and gets one answer.  The lanes look at 64 runs of sequences
// together, then at 64 runs within the one found, and so on to a single sequence (4096
// sequences of 64 tokens in window_prompt_kernel: 772 us looked for 64 after the other, 454
// by runs).  False: there is no such block.
template <bool LATEST_FIRST>
__device__ __forceinline__ bool find_row_block(const AttendArgs &a, int id, int rows_per_block, RowBlock &o) {
  const int lane = (int)threadIdx.x & 63;
  const int batch = a.c.groups / a.Hkv, number = id;
  auto blocks_of = [&](int tokens) {             // of a sequence, per group
    const int64_t n = ((int64_t)tokens * a.G + rows_per_block - 1) / rows_per_block;
    return (int)max((int64_t)0, min(n, (int64_t)a.row_blocks));
  };
  auto scan = [&](int x) {                       // inclusive, over the lanes
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int before = __shfl_up(x, s);
      x += lane >= s ? before : 0;
    }
    return x;
  };
  int b0 = 0;
  for (int per = batch; per > 64;) {             // sequences, then of a run
    per = (per + 63) / 64;
    int mine = 0, at = a.cu_q[min(b0 + lane * per, batch)];
#pragma unroll 8
    for (int i = 1; i <= per; ++i) {             // (past the last sequence there are no rows)
      const int next = a.cu_q[min(b0 + lane * per + i, batch)];
      mine += blocks_of(next - at);
      at = next;
    }
    const int upto = scan(mine * a.Hkv);
    const uint64_t beyond = __ballot(upto > id);
    const int src = beyond ? __builtin_ctzll(beyond) : 63;
    id -= __builtin_amdgcn_readlane(upto - mine * a.Hkv, src);
    b0 = min(b0 + src * per, batch);
  }
  const int q_at = a.cu_q[min(b0 + lane, batch)], q_to = a.cu_q[min(b0 + lane + 1, batch)];
  const int k_at = a.cu_k[min(b0 + lane, batch)], k_to = a.cu_k[min(b0 + lane + 1, batch)];
  const int mine = blocks_of(q_to - q_at), upto = scan(mine * a.Hkv);
  const uint64_t beyond = __ballot(upto > id);
  if (beyond == 0) return false;                 // uniform
  const int src = __builtin_ctzll(beyond), nb = __builtin_amdgcn_readlane(mine, src);
  id -= __builtin_amdgcn_readlane(upto, src) - nb * a.Hkv;
  o.b = b0 + src;
  o.g = id / nb;
  const int nth = id - o.g * nb;
  o.rb = LATEST_FIRST ? nb - 1 - nth : nth;
  o.part = number - nth + o.rb;
  o.q0 = __builtin_amdgcn_readlane(q_at, src);
  o.k0 = __builtin_amdgcn_readlane(k_at, src);
  o.lq = __builtin_amdgcn_readlane(q_to, src) - o.q0;
  o.lk = __builtin_amdgcn_readlane(k_to, src) - o.k0;
  return true;
}

}  // namespace ckv
