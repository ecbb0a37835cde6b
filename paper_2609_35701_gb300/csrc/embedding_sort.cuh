// Which cluster sorts the tokens of the embedding's gradient. Host code only, free of CUDA.
#pragma once

#include <cstdint>

namespace meq {

constexpr int kFewTokens = 256;  // up to which they are not sorted
// Tokens above which 16 blocks sort, not 8, us: 8192 16.7 with 8, 16.1 with 16, 16384 18.9 and 18.1, 32768 22.7 and 20.5,
// 65536 32.6 and 25.3, 131072 74 and 36 (launch and event 6 of them); 16 leave fewer SMs that can hold a cluster to zero rows.
constexpr int64_t kWideSort = 16384;

// The blocks of the cluster that sorts n tokens, 0 if none does. clusters_of(blocks) says how many such clusters the
// device holds at a time, < 1 for none, and is asked no more than needed: a part of a GPU may hold 8 blocks of a cluster
// but not 16, which more than 8 is not promised anywhere. *clusters < 1 where blocks are needed: there is no cluster.
template <typename F>
int sort_blocks(int64_t n, F clusters_of, int* clusters) {
  *clusters = 0;
  if (n <= kFewTokens) return 0;
  if (n > kWideSort) {
    *clusters = clusters_of(16);
    if (*clusters > 0) return 16;
  }
  *clusters = clusters_of(8);
  return 8;
}

}  // namespace meq
