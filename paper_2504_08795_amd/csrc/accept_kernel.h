// Which of a tree's drafted words stand: the walk from the root of each sequence to the node below whose word the model drew.
//
// A node's parent is the highest node of its mask in front of it, and child[p] the first node below p whose word is what was drawn behind p, found for
// all nodes at once (a minimum in LDS, which no order changes).  The walk is then a chain of one read a node: of a register's lanes where the tree has
// 64 nodes at most, of LDS where it has more.  A wave a sequence; bound by latency: row_start -> masks, words and what was drawn ->
// outputs.  One tree of 26 nodes 1.7 us (a call 7.6), 512 of up to 200, 2.3 MB, 4.4 (10.1): the longest walk of LDS reads.
#pragma once
#include "step_common.h"

namespace daris {

__device__ __forceinline__ void accept_body(const AcceptArgs& a) {
  constexpr int kNone = 0x7fffffff;
  __shared__ int child[kTreeNodes], drawn[kTreeNodes], line[kTreeNodes];
  const int s = blockIdx.x, lane = threadIdx.x;
  CacheArgs c = {};
  c.row_start = a.row_start;
  c.n_rows = a.n_rows;
  c.n_seqs = a.n_seqs;
  const int row0 = first_row(c, s), rows = rows_of(c, s), nodes = rows < 64 * a.tree_words ? rows : 64 * a.tree_words;
  const int before = a.before ? a.before[s] : 0;
  for (int j = lane; j < nodes; j += 64) {
    child[j] = kNone;
    drawn[j] = a.answers[row0 + j];
  }
  __syncthreads();
  for (int j = lane; j < nodes; j += 64) {
    const uint64_t* mask = a.tree + (int64_t)(row0 + j) * a.tree_words;
    const int word = a.words[row0 + j];
    int parent = -1;
    for (int w = j >> 6; w >= 0 && parent < 0; --w) {
      const uint64_t above = w == j >> 6 ? mask[w] & ((1ull << (j & 63)) - 1) : mask[w];
      if (above) parent = 64 * w + 63 - __builtin_clzll(above);
    }
    if (parent >= 0 && word >= 0 && drawn[parent] == word) atomicMin(&child[parent], j);
  }
  __syncthreads();
  int count = 0, at = 0;
  if (nodes > 64) {
    for (int next = 0; next != kNone; ++count) {
      at = next;
      if (lane == 0) line[count] = at;
      next = uniform(child[at]);
    }
    __syncthreads();
    for (int j = lane; j < rows; j += 64) a.path[row0 + j] = j < count ? line[j] : -1;
  } else if (nodes > 0) {
    const int mine = lane < nodes ? child[lane] : kNone;
    uint64_t on = 0;
    for (int next = 0; next != kNone; ++count) {
      at = next;
      on |= 1ull << at;
      next = __builtin_amdgcn_readlane(mine, at);
    }
    // (children have higher numbers: the walk is the set of its nodes in order)
    if (on >> lane & 1) a.path[row0 + __popcll(on & ((1ull << lane) - 1))] = lane;
    for (int j = count + lane; j < rows; j += 64) a.path[row0 + j] = -1;
  }
  if (lane == 0) {
    a.count[s] = count;
    a.word[s] = count ? drawn[at] : -1;
    if (a.after) a.after[s] = (int)((uint32_t)before + (uint32_t)count);
  }
}

}  // namespace daris
