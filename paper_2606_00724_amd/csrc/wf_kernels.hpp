// Kernel argument blocks and launch helpers shared by the WaveFilter
// kernels (device side) and the C-ABI (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wf {

constexpr int kBlock = 256;        // threads per workgroup, all kernels
constexpr int kMaxCoefTile = 64;   // coarse coefficients per skim tile
constexpr int kScanChunk = 128;    // tokens per chunk of the token skims
constexpr int kCoefPad = 4;        // fp32 pad per LDS coefficient row

// kHaarStream: kHaarSum with the keys read with the nt policy
enum CoefSource { kHaarSum = 0, kCascade = 1, kFromApprox = 2, kHaarStream = 3 };

struct DwtArgs {
  const void* K;       // [U][Ls][D]
  float* approx;       // [U][nJ][D]
  float* details;      // nullable, [U][L - nJ][D]
  long Ls;             // rows per unit in K (L: the transformed rows)
  int U, L, D, J, nJ;
  int cps;             // coefficients per stream
  int streams;         // streams per workgroup tile
  int ntiles;          // tiles per unit
  int boundary;        // 0 symmetric, 1 periodic
};

struct SkimTileArgs {
  const void* K;        // [U][L][D]      (Haar sum / cascade)
  const float* approx;  // [U][nJ][D]     (from approx)
  const void* Q;        // [U][B][D]
  float* logits;        // [U][B][nJ]
  float* stats;         // [U][ntiles][2][B]: row max, then row sum of exp
  const int32_t* parent;  // nullable: coefficient n is block 2 parent[n/2] + n%2
                          // of level J ([U][npar], ascending block ids at J + 1)
  int npar;
  long Ls;              // rows per unit in K (L: the filtered rows)
  int U, L, B, J, nJ;
  int cpt;              // coefficients per tile
  int ntiles;           // tiles per unit
  int boundary;
  float scale;
};

struct SkimSelectArgs {
  const float* logits;  // [U][B][nJ]
  const float* stats;   // [U][ntiles][2][B]
  float* W;             // [U][nJ] out
  int32_t* seg;         // [U][S] out (block ids), or [U][2S] tokens when pairs
  const int32_t* parent;  // nullable: candidate n is block 2 parent[n/2] + n%2
  int npar;
  int pairs;            // emit the two tokens of each kept 2-token block
  int U, B, nJ, ntiles, S;
};

struct ScanArgs {
  const void* Q;        // [U][B][D]
  const void* K;        // [U][L][D]
  const int32_t* seg;   // [U][S] (the regions; unused when the scan selects them)
  // the scan selects the regions itself (token-level path): W [U][nJ] of
  // the block weights kernel, the token skim's block rows [U][nJ][2][B]
  // (log-sum-exps of the selected blocks give the pool normalisers), and
  // seg_out [U][S] for the regions, written by the unit's first workgroup
  const float* W;
  const float* blocks;
  int32_t* seg_out;
  int nJ;
  int w_in_lds;         // W staged in LDS for the selection
  float* stats;         // [U][C][2][B]: reference (log2 units), sum of 2^(logit - reference)
  float* wpool;         // [U][P]  (weights mode)
  long Ls;              // rows per unit in K
  int U, L, B, J, S, P, C;
  int Cs;               // slices in `stats`
  int span;             // pool positions per workgroup (multiple of the chunk)
  int nbuf;             // LDS ring depth
  int seg_cap;          // region ids staged per workgroup
  int stream;           // statistics pass: pool rows read with the nt policy
  float scale;
  // units per selection: the selecting scan of unit u reads W and writes
  // seg_out of selection u / share (seg_out by the group's first unit only)
  int share = 1;
};

struct ScanSelectArgs {
  const float* wpool;   // [U][P]
  const int32_t* seg;   // [U][S]
  int32_t* tok;         // [U][keff]
  int U, J, S, P, keff;
};

struct GatherArgs {
  const void* K;        // [U][L][D]
  const void* V;
  const int32_t* tok;   // [U][keff]
  const void* Kg;       // [U][G][D]
  const void* Vg;
  void* Ks;             // [U][keff + R + G][D]
  void* Vs;
  long Lf;              // first always-kept row: rows Lf .. L-1 follow tok
  int U, L, D, keff, R, G, elem;
};

struct AttnArgs {
  const void* Q;        // [U][B][D]
  const void* K;        // rows: [U][L][D] indexed by tok, or [U][nrows][D]
  const void* V;
  const int32_t* tok;   // nullable: rows are contiguous when null
  // the attention selects the tokens itself (token-level path): the top
  // nsel of the scan weights wpool [U][P] over the pool of the regions seg
  // [U][S] (2^J tokens each); tok_out [U][nsel] (nullable) receives them
  const float* wpool;
  const int32_t* seg;
  int32_t* tok_out;
  int P, S, J;
  int w_in_lds;         // wpool staged in LDS for the selection
  const void* Kg;       // [U][G][D] tail (indexed mode only)
  const void* Vg;
  float* part;          // [U][NS][B][D] unnormalised partial outputs
  float* pstat;         // [U][NS][2][B] partial row max (log2 units), row sum
  void* O;              // [U][B][D]
  long Lf;              // indexed mode: rows Lf .. Lf + R - 1 of K/V follow tok
  int R;
  int U, L, B, nsel, G, nrows, NS;
  int rps;              // cache rows per split (multiple of the chunk)
  int nbuf;             // LDS ring depth
  float scale;
  // units per selection: the selecting attention of unit u reads wpool and
  // seg of selection u / share (tok_out by the group's first unit only)
  int share = 1;
  int tcap;             // token ids in LDS at once (multiple of the chunk)
};

constexpr int kFastMaxQBlocks = 4;  // query rows <= 64 on the token-level skim

struct TokenSkimArgs {
  const void* K;        // [U][L][D] bf16
  const void* Q;        // [U][B][D] bf16
  float* blocks;        // [U][nJ][2][B]: coarse logits, then log-sum-exps of
                        // the block's token logits; without the log-sum-exps
                        // [U][B][nJ] coarse logits
  float* wstats;        // [U][R][2][B] coarse-logit max and sum of exp per range
  long Ls;              // rows per unit in K (L: the filtered rows)
  int U, L, B, nJ, R;
  int span;             // tokens per range (multiple of the chunk)
  int nbuf;             // LDS ring depth
  float scale;          // logit scale
  float norm;           // 2^{-J/2}
  // nullable: the rows are the gathered sequence of the kept blocks
  // parent [U][npar] of 2^pshift tokens each (a refinement scale of the
  // recursion); L then counts gathered rows
  const int32_t* parent;
  int npar, pshift;
  int par_cap;          // parent ids staged in LDS per range
};

// Daubechies-2 at J = 6 for the token-level skim: the level-6 low-pass filter
// f_6 (190 taps, zero-padded) and the three symmetric-end filters E_0 | E_1
// | E_2 (64, 128 and 192 taps).
struct Db2TokenTaps {
  float band[3 << 6];
  float edge[6 << 6];
};

// out [groups][n] = the sum over h < H of in [groups H + h][n], h in order
struct HeadSumArgs {
  const float* in;
  float* out;
  long n;
  int H, groups;
};

struct BlockWeightsArgs {
  const float* blocks;  // [U][nJ][2][B] block rows of the token skim
  const float* wstats;  // [U][R][2][B]
  float* W;             // [U][nJ] out
  int U, B, nJ, R;
  int WPU;              // workgroups (block slices) per unit
};

struct CacheArgs {
  void* K;              // [U][rows][D]
  void* V;
  const int32_t* idx;   // nullable: store [batch][rows], load [U][rows]
  void* Kc;             // [U][cap][D] or [U][cap][D / 2] codes
  void* Kx;             // [U][cap][D / 32] exponent bytes
  void* Vc;
  void* Vx;
  int heads, rows, cap, first;
  int blocks;           // workgroups per unit
};

// Division of 0 <= n < 2^31 by a constant d >= 1: with 2^(l-1) < d <= 2^l, n times
// ceil(2^(31 + l) / d), shifted right by 31 + l, is the quotient (Granlund and
// Montgomery 1994).
struct FastDiv {
  uint32_t mul;
  int shift;            // l - 1; -1 for d = 1
  static FastDiv by(uint32_t d) {
    int l = 0;
    while ((1ull << l) < d) ++l;
    return FastDiv{(uint32_t)(((1ull << (31 + l)) + d - 1) / d), l - 1};
  }
  __device__ __forceinline__ int operator()(int n) const {
    return shift < 0 ? n : (int)(__umulhi((uint32_t)n, mul) >> shift);
  }
};

// Angles of rotated rows: positions of several axes times the pairs' frequencies.
struct TurnArgs {
  const int32_t* pos;   // [axes][rows in all]
  const float* freq;    // [half]
  long n;               // rows in all
  int half;             // pairs (0: nothing is rotated)
  int pairs;            // adjacent channels are a pair, not halves
  uint32_t axis[4];     // axis of pair i: bits 2 (i % 16) of word i / 16
  float factor;
};

struct RopeArgs {
  TurnArgs turn;
  const void* X;
  void* Y;
  long xs[3], ys[3];    // elements from batch to batch, head to head, row to row
  int heads, rows;
  int blocks;           // blocks of rows per batch
  int hgroups, iters;   // workgroups over the heads, eights of heads in each
};

struct AppendArgs {
  TurnArgs turn;
  const void* Q;        // nullable [tokens][hq][D]
  const void* K;        // [tokens][heads][D]
  const void* V;
  void* Qr;
  const int32_t* slot;  // [tokens]
  void* Kc;             // [pages][heads][page rows][D] or codes
  uint8_t* Kx;          // exponent bytes (quantised)
  void* Vc;
  uint8_t* Vx;
  long qs, ks, vs, os;  // elements from token to token
  long slots;           // rows of the pool per head
  int tokens, heads, hq;
  int shift;            // log2 of a page's rows
  int hgroups, iters;
};

struct MoveArgs {
  const int32_t* table;  // [batch][tp]
  const int32_t* first;  // [batch]
  const int32_t* src;    // [batch][moves]
  void* c[2];            // K, V: rows of rb bytes
  uint8_t* x[2];         // exponent bytes (quantised)
  int pages, heads, tp, moves, shift;
  int rb;
  int pshift, cols;      // log2 of a row's 16-byte pieces in a workgroup, workgroups a row takes
  FastDiv by_cols, by_heads;
};

// Work of the prefix kernel: units x ranges of their keys x blocks of their query
// rows.
struct PrefixPart {
  int items;            // workgroups
  int splits;           // key ranges per unit
  int rps;              // keys per range (multiple of the tile)
  int mblocks;          // blocks of query rows per unit
  int mrows;            // query rows per workgroup
  int M;                // query rows per unit
  int kw;               // waves that take the keys of a tile in turn
};
// Work of the kernel of the own keys: units x blocks of their query rows.
struct OwnPart {
  int mblocks, mrows;   // blocks per unit, query rows per workgroup
  int kw, qw;           // waves over the keys of a tile, waves over the query rows
};

struct PrefixArgs {
  const void* Q;        // [sequences][heads][R][D]
  const void* K;        // [prefixes][heads][cap][D], or codes
  const void* V;
  const uint8_t* Kx;    // exponent bytes (quantised prefix)
  const uint8_t* Vx;
  const int32_t* list;  // nullable [prefixes][heads][rows]
  const int32_t* plen;  // nullable [prefixes]
  const void* Kt;       // [sequences][heads][T][D]
  const void* Vt;
  const int32_t* tlen;  // nullable [sequences]
  void* O;              // [sequences][heads][R][D]
  float* lse;           // nullable [sequences][heads][R]
  float* part;          // [query rows][slots][D] unnormalised partial outputs
  float* pstat;         // [query rows][slots][2] reference (log2 units), sum
  PrefixPart p;
  OwnPart t;
  int heads, share, R;  // R: group * q_len
  FastDiv by_R;
  int cap, rows, T;
  int slots;            // partials per query row
  int whole;            // the prefix kernel writes O itself
  float scale;
};

struct TreeArgs {
  const void* Q;         // [tokens][hq][D]
  const void* K;         // [pages][heads][page rows][D], or codes
  const void* V;
  const uint8_t* Kx;     // exponent bytes (quantised)
  const uint8_t* Vx;
  const int32_t* table;  // [batch][tp]
  const int32_t* len;    // [batch]
  const int32_t* start;  // nullable [batch + 1]
  const uint32_t* mask;  // nullable [tokens][words]
  void* O;               // [tokens][hq][D]
  float* lse;            // nullable [tokens][hq]
  float* part;           // [tokens][hq][splits][D] unnormalised partial outputs
  float* pstat;          // [tokens][hq][splits][2] reference (log2 units), sum
  long qs, os;           // elements from token to token
  int items;             // workgroups: units x ranges x blocks of query rows
  int splits, rps;       // key ranges per unit at most, keys of a range (whole tiles)
  int mblocks, mrows;    // blocks per unit, query rows of a block
  int kw;                // waves that take the keys of a tile in turn
  int heads, g, hq;
  FastDiv by_g, by_hq, by_mblocks, by_splits, by_heads;
  int merges;            // workgroups of the merge per sequence
  FastDiv by_merge;
  int pages, shift, tp;  // log2 of a page's rows
  int tokens, max_rows, max_len, words;
  int causal;
  int whole;             // the kernel writes O itself
  float scale;
};

}  // namespace wf
