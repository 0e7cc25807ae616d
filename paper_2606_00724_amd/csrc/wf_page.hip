// A cache in pages: rows rotated by their positions (wf_rope), rotated and
// written into the pool on the way (wf_page_append), and brought together behind
// their context (wf_page_move).
//
// All three move bytes, and reach the rate of a plain device copy (5.0 TB/s read and
// written) or more where there are many (rotation: of eight heads and more); small calls
// are a launch, 2.7 to 3.8 us, of which two or three round trips to memory are most.
//
// A thread rotates sixteen channels of a row, eight pairs, in two vectors of eight:
// channels 8 i and half + 8 i on (halves), or 16 i on (adjacent pairs, and the
// channels behind the rotated ones).  So a pair is one thread's, a load is 16 bytes or
// more, and a block of 32 channels of the 8 and 4 bit formats is two or four threads'
// of one wave.  The angles of a token are the same for all its heads: a workgroup
// takes a few tokens, as many as give each thread one angle to turn into a cosine and
// a sine (some 60 operations in 64 bits, which would bound a thread that formed its
// own eight), shares these through LDS, and goes over the heads with them in
// registers.  The rows are asked for before the positions and frequencies, and loads
// return in order: angles are formed when the rows are there, and in a small call
// nothing runs beside that round trip.
#include "wf_cache.hpp"
#include "wf_kernels.hpp"
#include "wf_launch.hpp"

namespace wf {

// Tokens of a workgroup (one angle a thread) and heads that it takes at once.
template <int D>
constexpr int kTurnRows = 2 * kBlock / D;
constexpr int kTurnHeads = 8;
constexpr int kTurnBatch = 2;  // rows of a thread, both on their way at once

// Sine and cosine in 64 bits.  The angle is taken to [-pi/4, pi/4] by a multiple
// of pi/2 in two parts (Cody and Waite 1980; the product is not rounded before it
// is subtracted), where the Taylor polynomials to r^15 and r^16 are off by less
// than 2^-54: their fp32 rounding is that of the exact value but for one in some
// 10^8.  In 32 bits an angle of 10^5 would be off by 2^-8.
__device__ __forceinline__ void sine_cosine(double th, double& sn, double& cs) {
  const double k = __builtin_rint(th * 0.63661977236758134308);  // 2 / pi
  double r = fma(-k, 1.57079632679489661923, th);                // pi / 2, its first 53 bits
  r = fma(-k, 6.12323399573676588613e-17, r);                    // and the next
  const double r2 = r * r;
  double s = -1.0 / 1307674368000.0;  // -1 / 15!
  s = fma(s, r2, 1.0 / 6227020800.0);
  s = fma(s, r2, -1.0 / 39916800.0);
  s = fma(s, r2, 1.0 / 362880.0);
  s = fma(s, r2, -1.0 / 5040.0);
  s = fma(s, r2, 1.0 / 120.0);
  s = fma(s, r2, -1.0 / 6.0);
  s = fma(s * r2, r, r);
  double c = 1.0 / 20922789888000.0;  // 1 / 16!
  c = fma(c, r2, -1.0 / 87178291200.0);
  c = fma(c, r2, 1.0 / 479001600.0);
  c = fma(c, r2, -1.0 / 3628800.0);
  c = fma(c, r2, 1.0 / 40320.0);
  c = fma(c, r2, -1.0 / 720.0);
  c = fma(c, r2, 1.0 / 24.0);
  c = fma(c, r2, -0.5);
  c = fma(c, r2, 1.0);
  const int q = (int)(long)k & 3;  // quarter turns
  sn = q & 1 ? c : s;
  cs = q & 1 ? s : c;
  sn = q & 2 ? -sn : sn;
  cs = (q + 1) & 2 ? -cs : cs;
}

// A thread's place: sixteen channels of a row.
template <int D>
struct Place {
  static constexpr int C = D / 16;                  // threads a row
  int c, head, token;                               // part of the row, head of eight, token
  int oa, ob;                                       // the two vectors' channels
  bool turns;
  __device__ __forceinline__ explicit Place(const TurnArgs& t) {
    c = threadIdx.x % C;
    head = threadIdx.x / C % kTurnHeads;
    token = threadIdx.x / (C * kTurnHeads);
    turns = 8 * c < t.half;
    const bool apart = turns && !t.pairs;
    oa = apart ? 8 * c : 16 * c;
    ob = apart ? t.half + 8 * c : 16 * c + 8;
  }
};

// Cosines and sines of the workgroup's tokens, and a thread's eight of them.
template <int D>
struct Turns {
  static constexpr int TR = kTurnRows<D>;
  float c[TR][D / 2], s[TR][D / 2];

  // row(i): the row in all of the workgroup's token i (valid, whichever i).  Ends
  // with a barrier.
  template <typename Row>
  __device__ __forceinline__ void stage(const TurnArgs& t, const Row& row) {
    const int i = threadIdx.x / (D / 2), pair = threadIdx.x % (D / 2);
    if (pair < t.half) {
      const uint32_t w01 = pair & 16 ? t.axis[1] : t.axis[0];
      const uint32_t w23 = pair & 16 ? t.axis[3] : t.axis[2];
      const int axis = (pair & 32 ? w23 : w01) >> (2 * (pair & 15)) & 3;
      double sn, cs;
      sine_cosine((double)t.pos[axis * t.n + row(i)] * (double)t.freq[pair], sn, cs);
      c[i][pair] = (float)(cs * (double)t.factor);
      s[i][pair] = (float)(sn * (double)t.factor);
    }
    lds_barrier();
  }
};
struct Turn8 {
  float c[8], s[8];
  template <int D>
  __device__ __forceinline__ void read(const Turns<D>& t, int token, int first) {
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(&t.c[token][first + k]);
      const f32x4 y = *reinterpret_cast<const f32x4*>(&t.s[token][first + k]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[k + e] = x[e];
        s[k + e] = y[e];
      }
    }
  }
  // Each product and sum is rounded by itself, so that the rotated row that is
  // quantised does not depend on how a compiler contracts them.
  __device__ __forceinline__ static void pair(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
    const float u = x * c - y * s;
    y = y * c + x * s;
    x = u;
  }
  __device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], bool adjacent) const {
    if (adjacent) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        pair(a[2 * k], a[2 * k + 1], c[k], s[k]);
        pair(b[2 * k], b[2 * k + 1], c[4 + k], s[4 + k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) pair(a[k], b[k], c[k], s[k]);
    }
  }
};

// Eight channels as they are in memory.
template <typename T>
struct Raw8 {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<u32x4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(w[0][i]);
        v[2 * i + 1] = bf16_hi(w[0][i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i / 4][i % 4]);
    }
  }
};

// A workgroup has kTurnRows rows of a batch and eight or sixteen heads.  Queries of four
// sequences of 8K rows and 32 heads, slices of a fused projection, three axes: 96 us,
// 5.6 TB/s; of one block of 32 rows: 2.9 us.  With fewer than eight heads the places of the
// others are empty, and the angles bound: eight sequences of 32K rows of one, two and
// three heads 100, 105 and 114 us, where a copy takes 27, 54 and 80.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void rope_kernel(RopeArgs a) {
  __shared__ Turns<D> turns;
  const Place<D> at(a.turn);
  const int hg = blockIdx.x % a.hgroups, block = blockIdx.x / a.hgroups;
  const int b = block / a.blocks, r0 = block % a.blocks * kTurnRows<D>;
  const int r = r0 + at.token, h0 = hg * a.iters * kTurnHeads + at.head;
  const T* X = static_cast<const T*>(a.X) + b * a.xs[0] + min(r, a.rows - 1) * a.xs[2];
  T* Y = static_cast<T*>(a.Y) + b * a.ys[0] + min(r, a.rows - 1) * a.ys[2];
  Raw8<T> va[kTurnBatch], vb[kTurnBatch];
#pragma unroll
  for (int i = 0; i < kTurnBatch; ++i) {
    const long h = h0 + i * kTurnHeads;
    if (i >= a.iters || h >= a.heads || r >= a.rows) continue;
    va[i].load(X + h * a.xs[1] + at.oa);
    vb[i].load(X + h * a.xs[1] + at.ob);
  }
  turns.stage(a.turn, [&](int i) { return (long)b * a.rows + min(r0 + i, a.rows - 1); });
  Turn8 t;
  t.read(turns, at.token, at.turns ? 8 * at.c : 0);
#pragma unroll
  for (int i = 0; i < kTurnBatch; ++i) {
    const long h = h0 + i * kTurnHeads;
    if (i >= a.iters || h >= a.heads || r >= a.rows) continue;
    T* y = Y + h * a.ys[1];
    if (at.turns) {
      float x1[8], x2[8];
      va[i].values(x1);
      vb[i].values(x2);
      t.turn(x1, x2, a.turn.pairs);
      put8(y + at.oa, x1);
      put8(y + at.ob, x2);
    } else {
      va[i].store(y + at.oa);
      vb[i].store(y + at.ob);
    }
  }
}

// The rows of a token go one after the other: its queries, keys and values, eight
// at once, so that one set of angles serves queries and keys.  A row to be quantised
// is rotated in registers and rounded once, from fp32 to its code.  32K tokens of 32
// query and 8 K/V heads, 8 bits: 131 us, 5.6 TB/s; 64 tokens: 3.1 us.
template <typename T, int D, int FMT>
__global__ __launch_bounds__(kBlock) void append_kernel(AppendArgs a) {
  constexpr bool QUANT = FMT != WF_CACHE_PLAIN;
  constexpr int CB = FMT == WF_CACHE_E2M1 ? 4 : 8;  // bytes of eight codes
  constexpr int C = Place<D>::C;
  __shared__ Turns<D> turns;
  __shared__ uint32_t top[QUANT ? kBlock / C : 1][2 * C];  // largest magnitudes of eights
  const Place<D> at(a.turn);
  const int hg = blockIdx.x % a.hgroups, t0 = blockIdx.x / a.hgroups * kTurnRows<D>;
  const int n = t0 + at.token, h0 = hg * a.iters * kTurnHeads + at.head;
  const int all = a.hq + 2 * a.heads;
  const long token = min(n, a.tokens - 1);
  const long slot = a.slot[token];
  Raw8<T> va[kTurnBatch], vb[kTurnBatch];
#pragma unroll
  for (int i = 0; i < kTurnBatch; ++i) {
    const int h = h0 + i * kTurnHeads;
    if (i >= a.iters || h >= all || n >= a.tokens) continue;
    const T* x = h < a.hq ? static_cast<const T*>(a.Q) + token * a.qs + (long)h * D
                 : h < a.hq + a.heads
                     ? static_cast<const T*>(a.K) + token * a.ks + (long)(h - a.hq) * D
                     : static_cast<const T*>(a.V) + token * a.vs + (long)(h - a.hq - a.heads) * D;
    va[i].load(x + at.oa);
    vb[i].load(x + at.ob);
  }
  turns.stage(a.turn, [&](int i) { return (long)min(t0 + i, a.tokens - 1); });
  Turn8 t;
  t.read(turns, at.token, at.turns ? 8 * at.c : 0);
  const bool kept = slot >= 0 && slot < a.slots;
  const long page = slot >> a.shift, row = slot & ((1 << a.shift) - 1);
#pragma unroll
  for (int i = 0; i < kTurnBatch; ++i) {
    const int h = h0 + i * kTurnHeads;
    if (i >= a.iters || h >= all || n >= a.tokens) continue;
    const bool query = h < a.hq, value = h >= a.hq + a.heads;
    if (!query && !kept) continue;
    const int head = h - a.hq - (value ? a.heads : 0);  // of the pool
    const long to = ((page * a.heads + head) << a.shift) + row;
    float x1[8], x2[8];
    va[i].values(x1);
    vb[i].values(x2);
    const bool turned = at.turns && !value;
    if (turned) t.turn(x1, x2, a.turn.pairs);
    if (query || !QUANT) {
      T* y = query ? static_cast<T*>(a.Qr) + token * a.os + (long)h * D
                   : static_cast<T*>(value ? a.Vc : a.Kc) + to * D;
      if (turned) {
        put8(y + at.oa, x1);
        put8(y + at.ob, x2);
      } else {  // (their bits, NaN's too)
        va[i].store(y + at.oa);
        vb[i].store(y + at.ob);
      }
    } else {
      // a block's largest magnitude over its four eights, which may be other
      // threads' of the row: they are in one wave, whose LDS operations go in order
      uint32_t ma = 0, mb = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ma = max(ma, __float_as_uint(x1[e]) & 0x7fffffffu);
        mb = max(mb, __float_as_uint(x2[e]) & 0x7fffffffu);
      }
      uint32_t* m = top[threadIdx.x / C];
      m[at.oa / 8] = ma;
      m[at.ob / 8] = mb;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int o = k ? at.ob : at.oa;
        const u32x4 w = *reinterpret_cast<const u32x4*>(m + o / 32 * 4);
        const uint32_t x = block_exponent<FMT>(max(max(w[0], w[1]), max(w[2], w[3])));
        const float s = block_unscale(x);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x == 255u ? 0.f : (k ? x2 : x1)[e] * s;
        const u32x2 code = encode8<FMT>(y);
        uint8_t* c = static_cast<uint8_t*>(value ? a.Vc : a.Kc) + (to * (D / 8) + o / 8) * CB;
        if constexpr (CB == 8)
          *reinterpret_cast<u32x2*>(c) = code;
        else
          *reinterpret_cast<uint32_t*>(c) = code[0];
        if (o % 32 == 0) (value ? a.Vx : a.Kx)[to * (D / 32) + o / 32] = (uint8_t)x;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// A workgroup has a column of all rows that one head of a sequence moves, in K or
// in V: it reads every row before it writes the first.  Round trips bound a small
// call, one each for the sources, their pages and the rows: a thread's loads of one
// kind are queued together, those of the exponents' row beside the others, from
// places that are always there, and what moves nothing is left out at the end.  (How
// many there are is a constant, N: behind a branch the compiler waits for every load
// before it, and a thread's second piece and its exponents took four more trips.)  Six
// rows of 32 sequences of 8 heads: 2.7 us (3.4 behind branches); 64 of 128 in 8 bits, 34 MB
// read and written: 7.3 us (9.8).
constexpr int kMovePieces = 4;  // 16-byte pieces of a thread
// N pieces and, for codes, one load more: XB exponent bytes of a row
template <int N, int XB>
__global__ __launch_bounds__(kBlock) void move_kernel(MoveArgs a) {
  const int part = a.by_cols(blockIdx.x), col = blockIdx.x - part * a.cols;
  const int m = part & 1, unit = part >> 1, b = a.by_heads(unit), head = unit - b * a.heads;
  constexpr int ALL = N + (XB != 0), X = N;  // (the last one: a row's exponent bytes)
  const long first = a.first[b];
  const int32_t* src = a.src + (long)b * a.moves;
  const int32_t* table = a.table + (long)b * a.tp;
  const int in = (1 << a.shift) - 1;
  int row[ALL], s[ALL], pf[ALL], pt[ALL];
#pragma unroll
  for (int k = 0; k < ALL; ++k) {
    row[k] = k < N ? (int)(threadIdx.x + k * kBlock) >> a.pshift : (int)threadIdx.x;
    s[k] = src[min(row[k], a.moves - 1)];
  }
  // all queued before the first is waited for
  auto queued = [](int(&x)[ALL]) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < ALL; ++k) asm volatile("" : "+v"(x[k]));
  };
  queued(s);
  auto index = [&](long t) { return (int)min(max(t >> a.shift, 0L), a.tp - 1L); };
#pragma unroll
  for (int k = 0; k < ALL; ++k) {
    pf[k] = table[index(first + s[k])];
    pt[k] = table[index(first + row[k])];
  }
  queued(pf);
  // row t of the sequence, in page `page`, in its head's rows of the pool
  auto place = [&](long t, int page) {
    return (((long)min(max(page, 0), a.pages - 1) * a.heads + head) << a.shift) + (t & in);
  };
  auto there = [&](long t, int page) {
    return t >= 0 && t < (long)a.tp << a.shift && page >= 0 && page < a.pages;
  };
  auto moves = [&](int k) {
    return row[k] < a.moves && s[k] >= 0 && there(first + s[k], pf[k]) &&
           there(first + row[k], pt[k]);
  };
  const int piece = threadIdx.x & ((1 << a.pshift) - 1);
  char* c = static_cast<char*>(a.c[m]) + (((long)col << a.pshift) + piece) * 16;
  u32x4 v[N];
#pragma unroll
  for (int k = 0; k < N; ++k)
    v[k] = *reinterpret_cast<const u32x4*>(c + place(first + s[k], pf[k]) * a.rb);
  using Exps = std::conditional_t<XB == 4, uint32_t, uint16_t>;
  Exps x = 0;
  if constexpr (XB != 0)
    x = *reinterpret_cast<const Exps*>(a.x[m] + place(first + s[X], pf[X]) * XB);
  // (a barrier alone waits for no load: every row has come before another wave writes)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (moves(k)) *reinterpret_cast<u32x4*>(c + place(first + row[k], pt[k]) * a.rb) = v[k];
  if constexpr (XB != 0)
    if (col == 0 && moves(X))  // (the row's first column of workgroups writes them)
      *reinterpret_cast<Exps*>(a.x[m] + place(first + row[X], pt[X]) * XB) = x;
}

// ------------------------------------------------------------ host side

// Workgroups over `all` heads for `blocks` blocks of tokens: each takes two eights of
// heads where that leaves the chip several workgroups a CU.  (32K tokens of 48 heads
// in 8 bits 132 us, and 150 with four eights in flight, which leave a SIMD fewer
// waves, 141 with one, whose angles are as much work as the rows.)
static void split_heads(long blocks, int all, int& hgroups, int& iters) {
  const int eights = (all + kTurnHeads - 1) / kTurnHeads;
  iters = eights > 1 && blocks * ((eights + 1) / 2) >= 8L * device_cu_count() ? kTurnBatch : 1;
  hgroups = (eights + iters - 1) / iters;
}

static TurnArgs turn_args(int rot_dim, int layout, const uint8_t* axis, float factor,
                          const int32_t* pos, const float* freq, long n) {
  TurnArgs t{};
  t.pos = pos;
  t.freq = freq;
  t.n = n;
  t.half = rot_dim / 2;
  t.pairs = layout == WF_ROPE_PAIRS;
  t.factor = factor != 0.f ? factor : 1.f;
  for (int i = 0; i < t.half; ++i) t.axis[i / 16] |= (uint32_t)axis[i] << (2 * (i % 16));
  return t;
}

static int turn_rows(int head_dim) { return head_dim == 128 ? kTurnRows<128> : kTurnRows<64>; }

static long rope_split(const wf_rope_params& p, int& blocks, int& hgroups, int& iters) {
  const int tr = turn_rows(p.head_dim);
  blocks = (int)(((long)p.rows + tr - 1) / tr);
  split_heads((long)p.batch * blocks, p.heads, hgroups, iters);
  return (long)p.batch * blocks * hgroups;
}
long rope_groups(const wf_rope_params& p) {
  int b, h, i;
  return rope_split(p, b, h, i);
}

static long append_split(const wf_append_params& p, int& hgroups, int& iters) {
  const int tr = turn_rows(p.head_dim);
  const long blocks = ((long)p.tokens + tr - 1) / tr;
  split_heads(blocks, p.heads * (p.group + 2), hgroups, iters);
  return blocks * hgroups;
}
long append_groups(const wf_append_params& p) {
  int h, i;
  return append_split(p, h, i);
}

static int row_bytes(int head_dim, int dtype, int format) {
  return format == WF_CACHE_PLAIN ? head_dim * (dtype == WF_BF16 ? 2 : 4)
         : format == WF_CACHE_E4M3 ? head_dim
                                   : head_dim / 2;
}
static void move_split(const wf_move_params& p, int& pc, int& cols) {
  const int pieces = row_bytes(p.head_dim, p.dtype, p.format) / 16;  // a power of two
  pc = pieces;
  while (pc * p.moves > kMovePieces * kBlock) pc /= 2;
  cols = pieces / pc;
}
long move_groups(const wf_move_params& p) {
  int pc, cols;
  move_split(p, pc, cols);
  return 2L * cols * p.batch * p.heads;
}

template <typename F>
static hipError_t by_type(int dtype, int head_dim, const F& run) {
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (dtype == WF_BF16) return head_dim == 128 ? run(bf16_t{}, D128{}) : run(bf16_t{}, D64{});
  return head_dim == 128 ? run(float{}, D128{}) : run(float{}, D64{});
}

hipError_t launch_rope(const wf_rope_params& p, const void* X, const int32_t* pos,
                       const float* freq, void* Y, const long (&xs)[3], const long (&ys)[3],
                       hipStream_t s) {
  RopeArgs a{};
  a.turn = turn_args(p.rot_dim, p.layout, p.axis, p.factor, pos, freq, (long)p.batch * p.rows);
  a.X = X;
  a.Y = Y;
  for (int i = 0; i < 3; ++i) {
    a.xs[i] = xs[i];
    a.ys[i] = ys[i];
  }
  a.heads = p.heads;
  a.rows = p.rows;
  const unsigned grid = (unsigned)rope_split(p, a.blocks, a.hgroups, a.iters);
  return by_type(p.dtype, p.head_dim, [&](auto t, auto d) {
    hipLaunchKernelGGL((rope_kernel<decltype(t), decltype(d)::value>), dim3(grid), dim3(kBlock), 0,
                       s, a);
    return hipGetLastError();
  });
}

hipError_t launch_append(const wf_append_params& p, AppendArgs& a, const int32_t* pos,
                         const float* freq, hipStream_t s) {
  a.turn = turn_args(p.rot_dim, p.layout, p.axis, p.factor, pos, freq, p.tokens);
  a.tokens = p.tokens;
  a.heads = p.heads;
  a.hq = p.heads * p.group;
  a.slots = (long)p.pages * p.page_rows;
  a.shift = __builtin_ctz(p.page_rows);
  const unsigned grid = (unsigned)append_split(p, a.hgroups, a.iters);
  return by_type(p.dtype, p.head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    if (p.format == WF_CACHE_E4M3)
      hipLaunchKernelGGL((append_kernel<T, D, WF_CACHE_E4M3>), dim3(grid), dim3(kBlock), 0, s, a);
    else if (p.format == WF_CACHE_E2M1)
      hipLaunchKernelGGL((append_kernel<T, D, WF_CACHE_E2M1>), dim3(grid), dim3(kBlock), 0, s, a);
    else
      hipLaunchKernelGGL((append_kernel<T, D, WF_CACHE_PLAIN>), dim3(grid), dim3(kBlock), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_move(const wf_move_params& p, const int32_t* table, const int32_t* first,
                       const int32_t* source, void* Kc, void* Kx, void* Vc, void* Vx,
                       hipStream_t s) {
  MoveArgs a{};
  a.table = table;
  a.first = first;
  a.src = source;
  a.c[0] = Kc;
  a.c[1] = Vc;
  a.x[0] = static_cast<uint8_t*>(Kx);
  a.x[1] = static_cast<uint8_t*>(Vx);
  a.pages = p.pages;
  a.heads = p.heads;
  a.tp = p.table_pages;
  a.moves = p.moves;
  a.shift = __builtin_ctz(p.page_rows);
  a.rb = row_bytes(p.head_dim, p.dtype, p.format);
  int pc;
  move_split(p, pc, a.cols);
  a.pshift = __builtin_ctz(pc);
  a.by_cols = FastDiv::by(a.cols);
  a.by_heads = FastDiv::by(a.heads);
  const dim3 grid((unsigned)move_groups(p));
  auto by_pieces = [&](auto xb) {
    constexpr int XB = decltype(xb)::value;
    switch ((pc * p.moves + kBlock - 1) / kBlock) {  // of a thread
      case 1: hipLaunchKernelGGL((move_kernel<1, XB>), grid, dim3(kBlock), 0, s, a); break;
      case 2: hipLaunchKernelGGL((move_kernel<2, XB>), grid, dim3(kBlock), 0, s, a); break;
      case 3: hipLaunchKernelGGL((move_kernel<3, XB>), grid, dim3(kBlock), 0, s, a); break;
      default: hipLaunchKernelGGL((move_kernel<kMovePieces, XB>), grid, dim3(kBlock), 0, s, a);
    }
    return hipGetLastError();
  };
  if (p.format == WF_CACHE_PLAIN) return by_pieces(std::integral_constant<int, 0>{});
  if (p.head_dim == 128) return by_pieces(std::integral_constant<int, 4>{});
  return by_pieces(std::integral_constant<int, 2>{});
}

hipError_t load_page_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(&fa, reinterpret_cast<const void*>(move_kernel<1, 0>));
}

}  // namespace wf
