// What the kernels of the attention over a cache in pages share.
#pragma once

#include "wf_tiles.hpp"

namespace wf {

// A sequence: its rows in the cache, its query rows, and what hides keys from them.
struct Sequence {
  int L, n, base;  // keys, query rows, first key that is not seen by all
  long first;      // token of query row 0
  __device__ __forceinline__ Sequence(const TreeArgs& a, int b) {
    L = min(max(a.len[b], 0), a.max_len);
    first = a.start ? a.start[b] : (long)b * a.max_rows;
    n = a.start ? (int)min(max((long)a.start[b + 1] - first, 0L), (long)a.max_rows) : a.max_rows;
    base = L - n;
  }
  __device__ __forceinline__ static bool there(const TreeArgs& a, long token) {
    return token >= 0 && token < a.tokens;
  }
};

// Which of the 32 keys from `key` on query row i of a sequence sees (bit b: key + b),
// the first nv of them at most; words: the row's mask (null: none).
__device__ __forceinline__ uint32_t seen_keys(const TreeArgs& a, const Sequence& s, int i,
                                              const uint32_t* words, int key, int nv) {
  const int j0 = key - s.base;  // the first key as a new row (below 0: seen by all)
  uint32_t seen = ~0u;
  if (a.mask) {
    auto word = [&](int k) { return k < 0 ? ~0u : k < a.words ? words[k] : 0u; };
    seen = (uint32_t)((((uint64_t)word((j0 >> 5) + 1) << 32) | word(j0 >> 5)) >> (j0 & 31));
  } else if (a.causal) {
    const int c = i - j0;
    seen = c < 0 ? 0u : c >= 31 ? ~0u : (2u << c) - 1u;
  }
  return nv < 32 ? seen & ((1u << nv) - 1u) : seen;
}

hipError_t launch_tree_few(const TreeArgs& a, int head_dim, int format, long items, hipStream_t s);

}  // namespace wf
