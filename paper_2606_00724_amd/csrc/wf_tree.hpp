// What the kernels of the attention over a cache in pages share.
#pragma once

#include "wf_tiles.hpp"

namespace wf {

// A sequence: its rows in the cache, its query rows, and what hides keys from them.
struct Sequence {
  int L, n, base;  // keys, query rows, first key that is not seen by all
  long first;      // token of query row 0
  // (no branch: the loads are queued together, scalar ones, since no kernel that runs
  // beside this writes lengths)
  __device__ __forceinline__ Sequence(const TreeArgs& a, int b) {
    const int len = word(a.len + b);
    const int r0 = word(a.start ? a.start + b : a.len + b);
    const int r1 = word(a.start ? a.start + b + 1 : a.len + b);
    L = min(max(len, 0), a.max_len);
    first = a.start ? r0 : (long)b * a.max_rows;
    n = a.start ? (int)min(max((long)r1 - r0, 0L), (long)a.max_rows) : a.max_rows;
    base = L - n;
  }
  __device__ __forceinline__ static int word(const int32_t* p) {
    return *(const __attribute__((address_space(4))) int32_t*)p;
  }
  __device__ __forceinline__ static bool there(const TreeArgs& a, long token) {
    return token >= 0 && token < a.tokens;
  }
};

// The workgroup's block of query rows, range of keys and (sequence, K/V head).  Blocks
// of query rows are innermost: those that read the same keys run at once on one XCD.
struct TreeItem {
  int mb, sp, seq, head;
  __device__ __forceinline__ TreeItem(const TreeArgs& a, int item) {
    const int range = a.by_mblocks(item), unit = a.by_splits(range);
    mb = item - range * a.mblocks;
    sp = range - unit * a.splits;
    seq = a.by_heads(unit);
    head = unit - seq * a.heads;
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

// Four channels from c on of row r of V as fp32 numbers.
template <typename T, int D, int FMT>
__device__ __forceinline__ f32x4 values4(const TreeArgs& a, long r, int c) {
  f32x4 v;
  if constexpr (FMT == WF_CACHE_PLAIN) {
    const T* p = static_cast<const T*>(a.V) + r * D + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = load_elem<T>(p, e);
  } else {
    const float s = block_scale(a.Vx[r * (D / 32) + c / 32]);
    u32x2 w = {0u, 0u};
    if constexpr (FMT == WF_CACHE_E4M3)
      w[0] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.V) + r * D + c);
    else
      w[0] = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(a.V) + r * (D / 2) +
                                                c / 2);
    float x[8];
    decode8<FMT>(w, s, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
  }
  return v;
}

// Values that are no numbers, which the kernels leave out of their products where not
// all rows see them (a weight of 0 times one would be NaN), put to the four channels
// c .. c + 3 of query row i: those of the keys from .. to - 1 that it sees.  A chain of
// loads for each key (0.27 us), which the callers keep to the tiles or blocks from the
// first one with a hidden key on: the new rows and a part of a tile before them.
template <typename T, int D, int FMT>
__device__ __forceinline__ void add_odd(const TreeArgs& a, const Sequence& s, int seq, int head,
                                        int i, int from, int to, int c, f32x4& o) {
  const uint32_t* words =
      a.mask ? a.mask + min(max(s.first + i, 0L), a.tokens - 1L) * a.words : nullptr;
  for (int k = from; k < to; ++k) {
    if (!(seen_keys(a, s, i, words, k, 32) & 1)) continue;
    const long page = min(max(a.table[(long)seq * a.tp + (k >> a.shift)], 0), a.pages - 1);
    const f32x4 v = values4<T, D, FMT>(
        a, ((page * a.heads + head) << a.shift) + (k & ((1 << a.shift) - 1)), c);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!(fabsf(v[e]) < INFINITY)) o[e] += v[e];
  }
}

// (rows: query rows of a workgroup, 16 or, in bf16, 32)
hipError_t launch_tree_few(const TreeArgs& a, int dtype, int head_dim, int format, int rows,
                           long items, hipStream_t s);
hipError_t load_tree_few_kernels();

}  // namespace wf
