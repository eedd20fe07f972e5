// What the commit kernels of all cache types decide before they move a row.
#ifndef SMART_TREE_COMMIT_H_
#define SMART_TREE_COMMIT_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smart_tree.h"

namespace smart {

struct CommitInputs {
  int max_depth, block_size, max_blocks, num_blocks;
  const int32_t* cu_nodes;
  const int32_t* accept_len;
  const int32_t* accept_path;
  const int32_t* block_table;
  const int32_t* prefix_len;
};
struct CommitRow {
  int verdict, accepted, start;  // of the sequence
  int node, block;               // of path entry i (where the verdict is SMART_OK and i <= accepted)
};

// Path entry i of sequence b.  Every wavefront takes the same accept / refuse decision from the same inputs (a lane per path
// entry: two memory round trips per 64 entries).
__device__ inline CommitRow commit_row(const CommitInputs& in, int i, int b, int base, int n, int lane) {
  CommitRow r;
  r.accepted = in.accept_len[b];
  r.start = in.prefix_len[b];
  r.verdict = SMART_OK;
  r.node = r.block = 0;
  const int a = r.accepted, start = r.start;
  const int32_t* path = in.accept_path + (size_t)b * (in.max_depth + 1);
  if (base < 0 || a < 0 || a > in.max_depth) {
    r.verdict = SMART_ETREE;
  } else if (start < 0 || (int64_t)start + a + 1 > (int64_t)in.max_blocks * in.block_size) {
    r.verdict = SMART_ECAP;
  } else {
    for (int k0 = 0; k0 <= a; k0 += 64) {  // at most max_depth + 1 <= 129 entries
      const int k = min(k0 + lane, a);
      const int v = path[k];
      const int blk = in.block_table[(size_t)b * in.max_blocks + (start + k) / in.block_size];
      if (__any(v < 0 || v >= n || blk < 0 || blk >= in.num_blocks)) r.verdict = SMART_ETREE;
      if (i >= k0 && i < k0 + 64) {
        r.node = __builtin_amdgcn_readlane(v, i - k0);
        r.block = __builtin_amdgcn_readlane(blk, i - k0);
      }
    }
  }
  return r;
}

}  // namespace smart
#endif
