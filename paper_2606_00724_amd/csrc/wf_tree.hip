// Attention of new rows over a cache in pages (wf_tree_attn).
//
// For a K/V head of a sequence the query rows of its new tokens and of the head's
// group are one block of M = n * group rows over the same keys.  A workgroup takes
// a block of those rows and a range of the keys; where there are several ranges it
// leaves an unnormalised output with the rows' reference (log2 units) and sum of
// weights, and a second kernel merges them.  The products, the softmax and the
// tiles are those of the attention over a prefix (wf_tiles.hpp); here a wave's
// sixteen rows of a tile lie in one page, whose number it takes from a part of the
// table in LDS, and the last tiles, which hold keys that some of the new rows do
// not see, are masked by a word of bits for each query row and 32 keys.
//
// What bounds it depends on M: 4 d operations for each query row and key against
// 4 d bytes of a bf16 key and value.  Up to M = 32 the cache's bytes do, in a kernel
// made for that (wf_tree_few.hip); from some 200 rows on the products (64 drafted rows
// of 4 heads, M = 256); between them whichever kernel plan_tree's cost prefers.
#include "wf_tree.hpp"
#include "wf_launch.hpp"

namespace wf {

constexpr int kPageKeys = 32768;                 // keys whose pages are in LDS at once
constexpr int kPageIds = kPageKeys / 16 + 1;     // (pages of 16 rows at least)

// The pages of a range's keys, kPageKeys of them at once.
struct PageIds {
  int32_t* ids;        // LDS
  const int32_t* row;  // the sequence's table
  int first;           // page of ids[0] in the table
  int last;            // the sequence's last page
  int shift, pages;
  // the pages of keys from `key` on
  __device__ __forceinline__ void stage(int key, int threads) {
    first = key >> shift;
    const int n = min((kPageKeys >> shift) + 1, last - first + 1);
    for (int i = threadIdx.x; i < n; i += threads)
      ids[i] = min(max(row[first + i], 0), pages - 1);  // a bad page cannot leave the pool
  }
  __device__ __forceinline__ int of(int key) const { return ids[min(key >> shift, last) - first]; }
};

// Tiles by direct loads: wave w loads rows 16 w .. + 15 of a tile, which are in one
// page, one 64-byte piece of each in an instruction (four lanes a row).
template <typename T, int D>
struct PageLoads {
  using Geom = TileGeom<T, D>;
  static constexpr int N = Geom::NP;  // instructions per wave and matrix
  const unsigned char* K;
  const unsigned char* V;
  uint32_t off[2];  // the lane's byte offsets in sixteen rows
  uint32_t lds;     // LDS offset of the wave's rows in tile slot 0
  int heads, head, shift;

  __device__ __forceinline__ void init(const TreeArgs& a, int head_, uint32_t lds0) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    K = static_cast<const unsigned char*>(a.K);
    V = static_cast<const unsigned char*>(a.V);
    off[0] = (lane >> 2) * Geom::RB + 16 * ((lane & 3) ^ ((lane >> 4) & 3));
    off[1] = (lane >> 2) * Geom::RB + 16 * (lane & 3);
    lds = lds0 + 1024 * wave;
    heads = a.heads;
    head = head_;
    shift = a.shift;
  }
  struct Tile {
    const unsigned char *k, *v;  // the wave's first rows
    uint32_t to;                 // LDS offset of the wave's rows in its slot
    int go;                      // whether it is loaded
  };
  // the tile whose first key is `key`
  __device__ __forceinline__ Tile at(const PageIds& pages, int key, uint32_t slot) const {
    const int k = key + 16 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long page = __builtin_amdgcn_readfirstlane(pages.of(k));
    const long r = ((page * heads + head) << shift) + (k & ((1 << shift) - 1));
    return Tile{K + r * Geom::RB, V + r * Geom::RB, lds + slot * 2 * Geom::MB, 1};
  }
  // instruction i of 2 N (K's, then V's)
  template <int I>
  __device__ __forceinline__ void one(const Tile& t) const {
    tile_load<(I % N) * 64, (I / N) * Geom::MB + (I % N) * kPiece>(I < N ? t.k : t.v, off[I / N],
                                                                   t.to);
  }
  // instructions I0 + i .. I0 + e - 1 (the bounds are constants after unrolling)
  template <int I0, int I = 0>
  __device__ __forceinline__ void some(int i, int e, const Tile& t) const {
    if constexpr (I0 + I < 2 * N) {
      if (I >= i && I < e) one<I0 + I>(t);
      if (I + 1 < e) some<I0, I + 1>(i, e, t);
    }
  }
};

// NaN and infinities in V's rows 0 .. nr - 1 of a tile are made 0; whether there are
// any in the granules that this thread looks at.
template <typename T, int D, int NW>
__device__ __forceinline__ bool odd_values(unsigned char* tile, int nr) {
  using Geom = TileGeom<T, D>;
  bool odd = false;
  for (int i = threadIdx.x; i < nr * 4 * Geom::NP; i += 64 * NW) {
    u32x4* g = reinterpret_cast<u32x4*>(tile + Geom::MB + i / (4 * nr) * kPiece + i % (4 * nr) * 16);
    u32x4 w = *g;
    bool here = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) {
        const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
        here |= lo | hi;
        w[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
      } else {
        const bool bad = (w[e] & 0x7f800000u) == 0x7f800000u;
        here |= bad;
        w[e] = bad ? 0u : w[e];
      }
    }
    if (here) *g = w;
    odd |= here;
  }
  return odd;
}

// A tile's codes as a thread stages them.  The rows of a wave's load lie in one page
// (or, two pieces a row, in one for each half of the wave): the lanes' offsets are
// constant.
template <typename T, int D, int FMT, int NW, int OF>
__device__ __forceinline__ void stage_pages(QuantStage<T, D, FMT, NW, OF>& st, const TreeArgs& a,
                                            const PageIds& pages, int head, int key) {
  using S = QuantStage<T, D, FMT, NW, OF>;
  if (S::idle()) return;
#pragma unroll
  for (int i = 0; i < S::N; ++i) {
    auto first = [&](int k) -> long {  // row of the pool of key k, the first of sixteen
      const long page = __builtin_amdgcn_readfirstlane(pages.of(k));
      return ((page * a.heads + head) << a.shift) + (k & ((1 << a.shift) - 1));
    };
    const int wave = __builtin_amdgcn_readfirstlane(S::wave());
    const int lane = threadIdx.x & 63, r16 = S::row(i) & 15;
    const uint32_t o = (r16 * S::PPR + S::piece()) * 16;
    const uint32_t e = r16 * (D / 32) + S::piece() * S::CPP / 32;
    const uint8_t* K = static_cast<const uint8_t*>(a.K);
    const uint8_t* V = static_cast<const uint8_t*>(a.V);
    if constexpr (S::PPR > 2) {  // 8 or 16 rows
      const long r = first(key + (i * NW + wave) * (64 / S::PPR) / 16 * 16);
      st.w[0][i] = *reinterpret_cast<const u32x4*>(K + r * (S::PPR * 16) + o);
      st.w[1][i] = *reinterpret_cast<const u32x4*>(V + r * (S::PPR * 16) + o);
      st.x[0][i] = (a.Kx + r * (D / 32))[e];
      st.x[1][i] = (a.Vx + r * (D / 32))[e];
    } else {
      const int k = key + (i * NW + wave) * 32;
      const long r0 = first(k), r1 = first(k + 16), r = lane < 32 ? r0 : r1;
      st.w[0][i] = *reinterpret_cast<const u32x4*>(K + r * (S::PPR * 16) + o);
      st.w[1][i] = *reinterpret_cast<const u32x4*>(V + r * (S::PPR * 16) + o);
      st.x[0][i] = a.Kx[r * (D / 32) + e];
      st.x[1][i] = a.Vx[r * (D / 32) + e];
    }
  }
}

// The query rows of a (sequence, head) over a range of its keys: the kernel of many
// rows.  In bf16 the tiles that every row sees run in the pipelined loop of PrefixWave
// (four tile slots in LDS filled three tiles ahead by direct loads, the softmax of a
// block beside the products of the next); the few behind them, and rows of other
// kinds, one tile at a time.  64 query rows a wave (QW = 2) read each tile from LDS
// for twice the products: where M > 128 that is what lets them run at the rate that
// the power limit leaves.  16 sequences of 64 rows, 32 heads over 8, 16K keys:
// 258 us in the first calls and 310 after, 0.89 PFLOP/s sustained, the matrix units
// busy in 53% of its cycles; with one range for each sequence and head, and so no
// merge, 340.  Codes (eight waves, two tile slots at once, decoded on their way to
// LDS): two blocks of 32 rows over 128K keys in 4 bits 168 us, 0.82 PFLOP/s.  The matrix
// units are busy in 39% of its cycles and the vector units in about half: all waves
// decode a tile, meet at its barrier and then multiply, so that the two of a SIMD do the
// same at once.  fp32: 8 sequences of 64 rows over 4K keys 332 us, 0.10 PFLOP/s, two
// thirds of the rate of large fp32 products; over codes 309 and 306.
template <typename T, int D, int FMT, int QW>
__global__ __launch_bounds__((64 * prefix_waves<T, FMT>())) void tree_attn_kernel(TreeArgs a) {
  constexpr int NW = prefix_waves<T, FMT>();
  using W = PrefixWave<T, D, QW>;
  using Geom = TileGeom<T, D>;
  constexpr int MB = Geom::MB, SLOTS = Geom::SLOTS, QS = W::QS;
  constexpr bool QUANT = FMT != WF_CACHE_PLAIN;
  extern __shared__ __align__(16) unsigned char smem[];  // tiles, pages, a flag, masks
  int32_t* ids = reinterpret_cast<int32_t*>(smem + SLOTS * 2 * MB);
  int32_t* flag = ids + kPageIds;
  uint32_t* masks = reinterpret_cast<uint32_t*>(flag + 1);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;

  const int item = xcd_swizzle(blockIdx.x, gridDim.x);
  if (item >= a.items) return;  // (the grid holds whole eights of them)
  const TreeItem it(a, item);
  const int mb = it.mb, sp = it.sp, head = it.head, seq = it.seq;
  const Sequence s(a, seq);
  const int M = s.n * a.g, m0 = mb * a.mrows;
  const int k0 = sp * a.rps, nk = min(a.rps, s.L - k0);  // the range's keys
  if (m0 >= M || (nk <= 0 && !a.whole)) return;
  const int KW = a.kw, kw = wave % KW, qw = wave / KW;
  const int i0 = a.by_g(m0);  // first token of the block
  auto token_of = [&](int m, int& x) {  // and the head in its group
    const int i = a.by_g(m);
    x = m - i * a.g;
    return s.first + i;
  };
  W w;
  w.init(a.scale);
  bool odd = false;  // values that are no numbers among the keys from odd_from on
  int odd_from = 0;

  if (nk > 0) {
    // a tile: the keys of one slot, or with eight waves of two
    constexpr int US = NW == 8 ? 2 : 1, NS = SLOTS / US, KT = US * kTileRows;
    const int nt = (nk + KT - 1) / KT;
    // tiles that every row sees whole
    const int nseen = min(max(s.base - k0, 0), nk) / KT;
    odd_from = k0 + nseen * KT;
    auto slot_of = [&](int t) { return t % NS * US; };
    PageIds pages;
    pages.ids = ids;
    pages.row = a.table + (long)seq * a.tp;
    pages.last = (s.L - 1) >> a.shift;
    pages.shift = a.shift;
    pages.pages = a.pages;
    // the pages of the next kPageKeys keys when tile t is the first of them (no wave
    // needs older ones: tile t - 1 has been queued by all)
    auto stage_ids = [&](int t) __attribute__((always_inline)) {
      if (t * KT % kPageKeys != 0) return;  // uniform
      if (t > 0) lds_barrier();
      pages.stage(k0 + t * KT, 64 * NW);
      if (t == 0) {
        if (threadIdx.x == 0) *flag = 0;
        if (a.mask && nseen < nt) {
          const int ntok = a.by_g(min(m0 + a.mrows, M) - 1) - i0 + 1;
          for (int i = threadIdx.x; i < ntok * a.words; i += 64 * NW) {
            const long tok = s.first + i0 + i / a.words;
            masks[i] = Sequence::there(a, tok) ? a.mask[tok * a.words + i % a.words] : 0u;
          }
        }
      }
      __syncthreads();
    };
    PageLoads<T, D> dma;
    // Codes of a slot that fewer waves than there are have pieces of: at 64 channels each
    // slot is loaded and decoded by waves of its own (64 query rows a head over 8K rows
    // of 32 sequences: 8 bits 94 -> 92 us, 4 bits 92 -> 84; at 128 channels, where two
    // waves of a SIMD share the same work either way, 4 bits over 128K 182 -> 188).
    constexpr int F = QUANT ? FMT : WF_CACHE_E4M3;
    constexpr int PW = QuantStage<T, D, F, NW>::PT / 64;
    constexpr bool APART = US > 1 && D == 64 && PW < NW;
    const int slot = APART ? wave / PW : 0;  // the first of the wave's
    QuantStage<T, D, F, APART ? PW : NW, NW> st[APART ? 1 : US];
    static_assert(!APART || US * PW <= NW, "a wave loads codes of one slot");
    if constexpr (!QUANT) dma.init(a, head, lds_offset(smem));
    // tile t queued: on its way to its slot, or to registers
    int queued = 0;
    auto queue = [&](int t) __attribute__((always_inline)) {
      stage_ids(t);
      queued = t + 1;
      if constexpr (QUANT) {
#pragma unroll
        for (int i = 0; i < (APART ? 1 : US); ++i)
          if (slot + i < US) stage_pages(st[i], a, pages, head, k0 + t * KT + (slot + i) * kTileRows);
      } else {
        dma.template some<0>(0, 2 * dma.N, dma.at(pages, k0 + t * KT, slot_of(t)));
      }
    };
    auto commit = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < (APART ? 1 : US); ++i)
        if (slot + i < US) st[i].commit(smem + (slot_of(t) + slot + i) * 2 * MB);
    };
    // tile t is in its slot once every wave has passed the barrier behind this
    auto landed = [&](int t) __attribute__((always_inline)) {
      wait_vmcnt_chunks<2 * PageLoads<T, D>::N>(queued - 1 - t);
    };
    queue(0);
    // whole tiles in the pipelined loop
    const int nf = W::BF && !QUANT ? nseen : 0;
    int row[QW];  // the lane's tokens, from i0 on
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      int x;
      const long tok = token_of(min(m0 + (qw * QW + b) * 32 + l32, M - 1), x);
      row[b] = (int)(tok - s.first);
      const u32x4* src = reinterpret_cast<const u32x4*>(
          static_cast<const T*>(a.Q) + min(max(tok, 0L), a.tokens - 1L) * a.qs +
          (long)(head * a.g + x) * D);
#pragma unroll
      for (int j = 0; j < QS; ++j) w.q[b][j] = src[2 * j + h];
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): and tile 0
    if constexpr (W::BF && QW * QS >= 16) {
#pragma unroll
      for (int b = 0; b < QW; ++b)
#pragma unroll
        for (int j = 0; j < QS; ++j) asm volatile("" : "+a"(w.q[b][j]));
    }

    // LDS offset of the wave's first block in tile t
    const uint32_t lds0 = lds_offset(smem) + kw * 2048;
    auto tile_at = [&](int t) { return lds0 + slot_of(t) * 2 * MB; };
    if constexpr (W::BF && !QUANT) {
      if (nf > 0) {
        // Before tile t: tile t + 1 visible, t - 1 left by all; t + 2 in flight
        // and t + 3 queued over the tile's blocks.
        if (nt > 1) queue(1);
        if (nt > 2) queue(2);
        landed(0);
        lds_barrier();
        u32x4 kf[QS];
        f32x16 s0[QW], s1[QW];
        float mx[QW];
        w.keys(tile_at(0), kf);
        w.scores(kf, s0);
#pragma unroll
        for (int b = 0; b < QW; ++b) {
          w.shift_one(b, s0[b], s0[b]);
          mx[b] = w.largest(s0[b]);
        }
        if (QW > 1 || KW == 1) w.keys(tile_at(0) + 2048, kf);
        auto begin = [&](int t) __attribute__((always_inline)) {
          if (t + 1 >= nt) return;
          landed(t + 1);
          lds_barrier();
        };
        // the loads of tile t + 3 go between the products of tile t
        auto next = [&](int t) __attribute__((always_inline)) {
          typename PageLoads<T, D>::Tile ahead{dma.K, dma.V, 0u, 0};
          if (t + 3 < nt) {  // uniform
            stage_ids(t + 3);
            queued = t + 4;
            ahead = dma.at(pages, k0 + (t + 3) * KT, slot_of(t + 3));
          }
          return ahead;
        };
        constexpr int N = PageLoads<T, D>::N;  // tile loads of K, of V
        if (QW > 1 || KW == 1) {
          for (int t = 0; t < nf; ++t) {
            begin(t);
            const auto ahead = next(t);
            const uint32_t now = tile_at(t) + MB, then = tile_at(t + 1 < nt ? t + 1 : t);
            w.template block<N>(now, then, kf, s0, s1, mx,
                                [&](int i, int e) __attribute__((always_inline)) {
                                  if (ahead.go) dma.template some<0>(i, e, ahead);
                                });
            w.template block<N>(now + 2048, then + 2048, kf, s1, s0, mx,
                                [&](int i, int e) __attribute__((always_inline)) {
                                  if (ahead.go) dma.template some<N>(i, e, ahead);
                                });
          }
        } else {
          auto one = [&](int t, f32x16(&sc)[QW], f32x16(&sn)[QW])
                         __attribute__((always_inline)) {
                           begin(t);
                           const auto ahead = next(t);
                           w.keys(tile_at(t + 1 < nt ? t + 1 : t), kf);
                           w.template block<2 * N>(
                               tile_at(t) + MB, tile_at(t), kf, sc, sn, mx,
                               [&](int i, int e) __attribute__((always_inline)) {
                                 if (ahead.go) dma.template some<0>(i, e, ahead);
                               });
                         };
          for (int t = 0; t < nf; t += 2) {
            one(t, s0, s1);
            if (t + 1 < nf) one(t + 1, s1, s0);
          }
        }
      }
    }
    // The other tiles: tile t visible, then computed, with up to NS - 1 tiles
    // behind it on their way.
    if (nf == 0 && !QUANT)
      for (int t = 1; t < min(nt, NS - 1); ++t) queue(t);
    for (int t = nf; t < nt; ++t) {
      if constexpr (QUANT) {
        commit(t);
        if (t + 1 < nt) queue(t + 1);
        lds_barrier();
      } else if (nf == 0 || t > nf) {  // (else visible since the last whole one)
        landed(t);
        lds_barrier();
        while (queued < min(nt, t + NS)) queue(queued);
      }
      const int nr = nk - t * KT;  // rows of the tile that are in the range
      if (nr < KT) {
        const int last = (nr - 1) / kTileRows;  // its last 64 rows
        if (nr % kTileRows)
          clear_rows<T, D, NW>(smem + (slot_of(t) + last) * 2 * MB, nr - last * kTileRows);
      }
      // Keys that some rows do not see: their scores are taken out, whatever they
      // are.  A weight of 0 times a value that is no number would still be NaN:
      // such values are cleared, and put to the rows that see them behind it all.
      const bool all = k0 + t * KT + min(nr, KT) <= s.base;  // uniform
      if (!all) {
        bool here = false;
#pragma unroll
        for (int i = 0; i < US; ++i)
          here |= odd_values<T, D, NW>(smem + (slot_of(t) + i) * 2 * MB,
                                       min(max(nr - i * kTileRows, 0), kTileRows));
        if (__builtin_amdgcn_ballot_w64(here) != 0 && lane == 0) *flag = 1;
        lds_barrier();
      }
      for (int r = 32 * kw; r < min(nr, KT); r += 32 * KW) {
        const int key = k0 + t * KT + r;
        const uint32_t at =
            lds_offset(smem) + (slot_of(t) + r / kTileRows) * 2 * MB + r % kTileRows * 64;
        uint32_t seen[QW];
#pragma unroll
        for (int b = 0; b < QW; ++b) seen[b] = ~0u;
        if (!all)
#pragma unroll
          for (int b = 0; b < QW; ++b)
            seen[b] = seen_keys(a, s, row[b], masks + (row[b] - i0) * a.words, key, nr - r);
        w.template step<true>(at, at + MB, all ? 32 : 0, seen);
      }
    }
    odd = __builtin_amdgcn_readfirstlane(*flag) != 0;
    lds_barrier();  // the tiles are idle
  }

  OutRows<D, QW, NW> out(smem);
  out.put(w, wave);
  constexpr int C4 = D / 4, RPP = 64 * NW / C4;  // rows per round
  const int c = threadIdx.x % C4;
  constexpr int NR = 4;
  const int mend = min(a.mrows, M - m0);
  for (int r0 = threadIdx.x / C4; r0 < mend; r0 += NR * RPP) {
    int v[NR];
    Merge4 g[NR];
    // row r of the workgroup is in row r % (32 QW) of the KW waves of its rows
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = min(r0 + i * RPP, mend - 1);
      v[i] = r / (32 * QW) * KW * 32 * QW + r % (32 * QW);
    }
    out.merged(v, KW, c, g);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = r0 + i * RPP;
      if (r >= mend) break;
      int x;
      const long tok = token_of(m0 + r, x);
      if (!Sequence::there(a, tok)) continue;
      if (odd)
        add_odd<T, D, FMT>(a, s, seq, head, (int)(tok - s.first), odd_from, k0 + nk, 4 * c, g[i].o);
      const int hq = head * a.g + x;
      const long row = tok * a.hq + hq;
      if (a.whole) {
        g[i].finish(static_cast<T*>(a.O) + tok * a.os + (long)hq * D + 4 * c,
                    a.lse ? a.lse + row : nullptr, c == 0);
      } else {
        const long at = row * a.splits + sp;
        *reinterpret_cast<f32x4*>(a.part + at * D + 4 * c) = g[i].o;
        if (c == 0) *reinterpret_cast<hw_f32x2*>(a.pstat + 2 * at) = hw_f32x2{g[i].M, g[i].z};
      }
    }
  }
}

// Merges the partials of each query row, as many as its sequence has ranges.  A
// thread takes four channels of every SG-th partial of a row, eight in flight; the
// SG threads of a row's channels meet in LDS.  Bound by its partials' bytes where they
// are many (16K rows of two ranges: 12.6 us) and else by its round trips: 4 us.
template <typename T, int D, int SG>
__global__ __launch_bounds__(kBlock) void tree_merge_kernel(TreeArgs a) {
  constexpr int C4 = D / 4, RPB = kBlock / (C4 * SG), F = 8;
  const int seq = a.by_merge(blockIdx.x), part = blockIdx.x - seq * a.merges;
  const int r = part * RPB + threadIdx.x / (C4 * SG);  // (query row, head) of the sequence
  const int c = threadIdx.x % C4, sg = threadIdx.x / C4 % SG;
  const int i = a.by_hq(r), hq = r - i * a.hq;
  const Sequence s(a, seq);
  const long tok = s.first + i;
  const bool mine = i < s.n && Sequence::there(a, tok);
  const long row = mine ? tok * a.hq + hq : 0;
  const int slots = (s.L + a.rps - 1) / a.rps;
  Merge4 g;
  for (int s0 = sg; s0 < (s0 == sg ? a.splits : slots); s0 += F * SG) {
    hw_f32x2 mz[F];
    f32x4 x[F];
#pragma unroll
    for (int k = 0; k < F; ++k) {  // (all queued; those past the last are dropped)
      const long at = row * a.splits + min(s0 + k * SG, a.splits - 1);
      mz[k] = *reinterpret_cast<const hw_f32x2*>(a.pstat + 2 * at);
      x[k] = *reinterpret_cast<const f32x4*>(a.part + at * D + 4 * c);
    }
#pragma unroll
    for (int k = 0; k < F; ++k) {
      const bool in = s0 + k * SG < slots;
      g.add(in ? mz[k][0] : -INFINITY, in ? mz[k][1] : 0.f, x[k]);
    }
  }
  if constexpr (SG > 1) {
    __shared__ float sh[kBlock][7];  // (odd stride: no bank met twice)
    float* put = sh[threadIdx.x];
    put[0] = g.M;
    put[1] = g.z;
#pragma unroll
    for (int e = 0; e < 4; ++e) put[2 + e] = g.o[e];
    __syncthreads();
    if (sg != 0) return;  // no barrier follows
#pragma unroll
    for (int k = 1; k < SG; ++k) {
      const float* x = sh[threadIdx.x + k * C4];
      g.add(x[0], x[1], f32x4{x[2], x[3], x[4], x[5]});
    }
  }
  if (mine)
    g.finish(static_cast<T*>(a.O) + tok * a.os + (long)hq * D + 4 * c, a.lse ? a.lse + row : nullptr,
             c == 0);
}

// ------------------------------------------------------------ host side

static int merge_threads(int splits) { return splits <= 8 ? 1 : splits <= 32 ? 4 : 8; }

// How a call's work is cut.  The cost of a choice in us, fitted to measured times (a
// kernel's ranges to 388 shapes of 1 to 48 sequences, 1K to 64K rows and every type and
// format: 1.5% slower than the best of some ten ranges, in the mean).  A workgroup takes
// a block of query rows and a range of keys: a fixed part (its first loads, its outputs)
// and its tiles, each at its products and softmax or at its bytes, which come at the
// chip's rate to all CUs and at 32 GB/s (many query rows) or 50 (few) to one; and D
// floats a query row and range are written and read where there are several ranges.
TreePlan plan_tree(const wf_tree_params& p, size_t have) {
  const bool bf = p.dtype == WF_BF16, quant = p.format != WF_CACHE_PLAIN;
  const int D = p.head_dim;
  const long M = (long)p.max_rows * p.group, U = (long)p.batch * p.heads;
  const long rows = (long)p.tokens * p.heads * p.group, cus = device_cu_count();
  const double row_bytes = quant ? D * (p.format == WF_CACHE_E4M3 ? 1.0 : 0.5) + D / 32
                                 : D * (bf ? 2.0 : 4.0);
  // ranges are as many as the workspace holds partials for, and one at least
  const long most = (long)std::min<size_t>(have / (rows * (D + 2) * sizeof(float)), 1L << 30);
  auto merge = [&](long s) { return s > 1 ? 4.0 + s * ((double)rows * D * 8 / 5e6) : 0.0; };
  TreePlan best{};
  double least = 0;
  auto take = [&](const TreePlan& l, long rps, double cost) {
    if (least != 0 && cost >= least) return;
    least = cost;
    best = l;
    best.rps = (int)rps;
  };
  // Few query rows: 32 a workgroup of four waves, two workgroups a CU; the blocks of
  // query rows read the same keys, mostly from the L2.  (Eight waves and one workgroup
  // a CU, with half as many ranges: within 3% either way over 27 shapes.)
  {
    TreePlan l{};
    l.few = !bf || M <= 16 ? 16 : 32;
    l.qw = 1;
    l.nw = l.kw = 4;
    l.mblocks = (int)((M + l.few - 1) / l.few);
    const long KT = 128, tiles = std::max(1L, (p.max_len + KT - 1) / KT);
    // a tile of a workgroup that has its CU alone, and of one that shares it
    const double slope = !bf ? 2.6 : l.few == 16 ? (quant ? 0.45 : 0.2) : quant ? 0.9 : 0.65;
    const double alone = (!bf ? 0.2 : l.few == 16 && !quant ? 0.6 : 0.4) + slope * D / 128.0;
    const double both = 1.6 * alone;
    const double most_at_once = !bf && !quant && D == 128 ? 1.0 : 2.0;
    // bytes a us: to the chip (more of a cache that stays on it), to one CU (more of what
    // another block of query rows has brought to the L2)
    const double rate = 2.0 * U * p.max_len * row_bytes < 2e8 ? 7.4e6 : 6e6;
    const double cu_rate = l.mblocks > 1 ? 75e3 : 50e3;
    for (long n = 1; n <= tiles; n += 1 + n / 16) {
      const long per = (tiles + n - 1) / n, s = (tiles + per - 1) / per;
      if (s > 1 && s > most) break;
      const double groups = (double)(U * l.mblocks * s), per_cu = std::ceil(groups / cus);
      const double at_once = std::min(per_cu, most_at_once);
      const double running = std::min(groups, at_once * cus);
      const double bytes = 2 * KT * row_bytes *
                           std::max({running / std::min(l.mblocks, 3) / rate, running / 14e6,
                                     at_once / cu_rate});
      const double tile = std::max(at_once > 1 ? both : alone, bytes);
      const double rounds = std::max(1.0, per_cu / most_at_once);
      // (lengths that differ leave some CUs idle at the end: a part of a workgroup's time)
      take(l, per * KT, rounds * per * tile + 4.0 + 6.0 * (rounds - 1) + 0.2 * per * tile +
                            (s > 1 ? merge(s) + 0.035 * s : 0.0));
    }
  }
  // Many: a block of query rows for the workgroup, as of the attention over a prefix.
  const bool many = M > (bf ? 32 : 16);
  const int nw = bf && quant ? 8 : 4;
  const long KT = nw == 8 ? 2 * kTileRows : kTileRows;
  const long tiles = std::max(1L, (p.max_len + KT - 1) / KT);
  auto consider = [&](int qw, int qwaves, double block, double fixed) {
    TreePlan l{};
    l.qw = qw;
    l.nw = nw;
    l.kw = nw / qwaves;
    l.mblocks = (int)((M + 32 * qw * qwaves - 1) / (32 * qw * qwaves));
    const double products = (double)(KT / 32) / l.kw * D / 128.0 * block + fixed;
    const long one = std::max(1L, cus / (U * l.mblocks));  // ranges that fill the chip once
    auto ranges = [&](long n) {
      const long per = (tiles + n - 1) / n, s = (tiles + per - 1) / per;
      if (s > 1 && s > most) return;
      const double groups = (double)(U * l.mblocks * s), at_once = std::min(groups, (double)cus);
      const double bytes = 2 * KT * row_bytes * std::max(at_once / l.mblocks / 6e6, 1 / 32e3);
      take(l, per * KT,
           std::ceil(groups / cus) * (per * std::max(products, bytes) + 9.0) + merge(s));
    };
    for (long n = 1; n < std::min(one, tiles); n += 1 + n / 16) ranges(n);
    ranges(std::min(one, tiles));
    ranges(std::min(2 * one, tiles));
  };
  for (int qwaves = 2; many && qwaves <= nw && (qwaves == 2 || 16 * qwaves < M); qwaves *= 2)
    if (!bf)
      consider(1, qwaves, 4.2, quant ? 0.4 : 0.1);
    else if (quant)
      consider(1, qwaves, 0.875, 0.7);
    else
      consider(1, qwaves, 0.45, 0.1);
  if (many && bf && !quant && M > 128) consider(2, nw, 0.82, 0.1);
  TreePlan l = best;
  l.splits = (int)std::max(1L, ((long)p.max_len + l.rps - 1) / l.rps);
  l.items = U * l.mblocks * l.splits;
  const int mb = kTileRows * D * (bf ? 2 : 4);  // bytes of a K (or V) tile
  const int slots = 8 * mb > 131072 ? 2 : 4;
  const int words = (p.max_rows + 31) / 32, mrows = l.nw / l.kw * 32 * l.qw;
  const size_t out = (size_t)l.nw * 32 * l.qw * (D + 6) * sizeof(float);
  l.lds_bytes = std::max((size_t)slots * 2 * mb + (kPageIds + 1) * sizeof(int32_t) +
                             (size_t)std::min(mrows + 1, p.max_rows) * words * sizeof(uint32_t),
                         out);
  if (l.splits > 1) {
    l.part_bytes = (size_t)rows * l.splits * D * sizeof(float);
    l.pstat_bytes = (size_t)rows * l.splits * 2 * sizeof(float);
    const long rpb = kBlock / (D / 4 * merge_threads(l.splits));
    l.merges = ((long)p.max_rows * p.heads * p.group + rpb - 1) / rpb;
  }
  return l;
}

hipError_t launch_tree(const wf_tree_params& p, const TreePlan& l, TreeArgs& a, hipStream_t s) {
  a.items = (int)l.items;
  a.splits = l.splits;
  a.rps = l.rps;
  a.mblocks = l.mblocks;
  a.mrows = l.nw / l.kw * 32 * l.qw;
  a.kw = l.kw;
  a.heads = p.heads;
  a.g = p.group;
  a.hq = p.heads * p.group;
  a.by_g = FastDiv::by(p.group);
  a.merges = (int)l.merges;
  a.by_merge = FastDiv::by(std::max(1, a.merges));
  a.by_hq = FastDiv::by(a.hq);
  a.by_mblocks = FastDiv::by(a.mblocks);
  a.by_splits = FastDiv::by(a.splits);
  a.by_heads = FastDiv::by(a.heads);
  a.pages = p.pages;
  a.shift = __builtin_ctz(p.page_rows);
  a.tp = p.table_pages;
  a.tokens = p.tokens;
  a.max_rows = p.max_rows;
  a.max_len = p.max_len;
  a.words = (p.max_rows + 31) / 32;
  a.causal = p.causal;
  a.whole = l.splits == 1;
  a.scale = p.scale != 0.f ? p.scale : (float)(1.0 / std::sqrt((double)p.head_dim));
  auto run = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    auto go = [&](auto kern) {
      if (l.lds_bytes > 65536) {
        const hipError_t e =
            hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                hipFuncAttributeMaxDynamicSharedMemorySize, (int)l.lds_bytes);
        if (e != hipSuccess) return e;
      }
      hipLaunchKernelGGL(kern, dim3((unsigned)((l.items + 7) & ~7L)), dim3(64 * l.nw), l.lds_bytes,
                         s, a);
      return hipGetLastError();
    };
    hipError_t e = hipErrorInvalidValue;
    if (l.few)
      e = launch_tree_few(a, p.dtype, D, p.format, l.few, l.items, s);
    else if (p.format == WF_CACHE_E4M3)
      e = go(tree_attn_kernel<T, D, WF_CACHE_E4M3, 1>);
    else if (p.format == WF_CACHE_E2M1)
      e = go(tree_attn_kernel<T, D, WF_CACHE_E2M1, 1>);
    else if (l.qw == 1)
      e = go(tree_attn_kernel<T, D, WF_CACHE_PLAIN, 1>);
    else if constexpr (sizeof(T) == 2)
      e = go(tree_attn_kernel<T, D, WF_CACHE_PLAIN, 2>);
    if (e != hipSuccess || l.merges == 0) return e;
    const dim3 grid((unsigned)(l.merges * p.batch));
    switch (merge_threads(l.splits)) {
      case 1: hipLaunchKernelGGL((tree_merge_kernel<T, D, 1>), grid, dim3(kBlock), 0, s, a); break;
      case 4: hipLaunchKernelGGL((tree_merge_kernel<T, D, 4>), grid, dim3(kBlock), 0, s, a); break;
      default: hipLaunchKernelGGL((tree_merge_kernel<T, D, 8>), grid, dim3(kBlock), 0, s, a);
    }
    return hipGetLastError();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (p.dtype == WF_BF16)
    return p.head_dim == 128 ? run(bf16_t{}, D128{}) : run(bf16_t{}, D64{});
  return p.head_dim == 128 ? run(float{}, D128{}) : run(float{}, D64{});
}

hipError_t load_tree_kernels() {
  hipFuncAttributes fa;
  const hipError_t e = hipFuncGetAttributes(
      &fa, reinterpret_cast<const void*>(tree_attn_kernel<bf16_t, 128, WF_CACHE_PLAIN, 1>));
  return e != hipSuccess ? e : load_tree_few_kernels();
}

}  // namespace wf
