// Attention of few query rows over a cache in pages: a sequence's single token, or the
// few drafted ones whose rows and heads of a group are 16 or 32 query rows of a K/V
// head.  Bound by the cache's bytes: each key is read once, for 8 d operations or so a
// byte.
//
// Each wave has keys, in blocks of 32, and a part of LDS of its own: it loads their
// rows, or codes, straight to LDS as they are in memory, waits for them by the count
// of its loads and meets the workgroup's other waves only when its last block is
// done. Two workgroups a CU have 128 KB (64 KB of 8-bit codes) queued or being read.
// The scores are S^T = K Q^T and the outputs O^T = V^T P^T, so that a lane has all
// of its keys' scores of one query row, as the second product wants its weights.
// Which channels make up one step of the first product is free: a lane has
// consecutive ones of its row of K, 16-byte chunks.  V's rows are read transposed,
// by the LDS loads made for operands of 16, 8 and 4 bits (fp32: a channel of a lane,
// word by word).  Codes are decoded behind these reads, K's with their row's scale;
// V's scales, one for each key and 32 channels, are put to the weights instead,
// which are the other operand for those 32 channels, as powers of two: exact.
//
// For bf16 queries the weights are rounded to bf16 for the second product, as in the
// attention over a prefix: the type of its operands, and weights in two parts would
// double it.  Their sum is taken of the unrounded ones.  Outputs are off by 0.0023 of
// their norm, of which the outputs' own rounding is 0.0017.  fp32 queries keep fp32
// weights.
//
// Products of 16 x 16 where M <= 16 (half the softmax and decoding of 32 x 32: 16
// sequences of 32K rows in 8 bits 198 us, 204 with 32; single tokens over 16K 16.4,
// 18.1), and for all of fp32; else of 32 x 32.
//
// Single tokens, 32 query heads over 8 of 128 channels: 64 sequences of 8K bf16 rows
// (ragged) 271 to 283 us, 5.7 to 5.9 TB/s, where the loads alone reach 6.1; 32 of 32K
// rows in 8 bits 289 to 307, 5.4 to 5.7 TB/s, the rate of its loads alone; 32 of 8K
// fp32 rows 359 to 369 us, 5.8 to 6.0 TB/s.  fp32 queries over codes are bound by the fp32
// products, a group's four rows padded to sixteen (32 sequences of 8K rows: 17 GFLOP,
// 112 us), and the decoding before them: 182 us in 8 bits, 176 in 4.  24 drafted rows over
// 4K bf16 rows: 13.0 us, a chain of round trips (lengths, pages, four blocks a wave, each
// queued when the one before it has been read).
#include "wf_tree.hpp"
#include "wf_launch.hpp"

namespace wf {

constexpr int kFewWaves = 4;

typedef int v2i_few __attribute__((ext_vector_type(2)));

// A wave's part of LDS: a block's rows of K, of V, and the exponents of this block
// and of the next, which come before this one's values are through.  Each part is
// queued anew as soon as it has been read, K's while the softmax and V's product
// run, V's over the next block's scores.  (Two blocks of 4 KB or less instead of
// one: the same times, up to 4% longer at 64 channels.)  Rows of a block stand after
// each other, their 16-byte chunks in an order that lets the lanes that read at once
// meet all banks: eight rows at one chunk of K, and of V eight rows (8 bits),
// sixteen (4 bits), four at two chunks (bf16) or every fourth one at 64 bytes
// (fp32).
template <typename T, int D, int FMT>
struct FewGeom {
  static constexpr bool QUANT = FMT != WF_CACHE_PLAIN;
  static constexpr int RB = QUANT ? (FMT == WF_CACHE_E4M3 ? D : D / 2)
                                  : D * (int)sizeof(T);        // bytes of a row
  static constexpr int C = RB / 16;                            // chunks of a row
  static constexpr int KB = 32 * RB;                           // bytes of 32 rows
  static constexpr int NI = KB / 1024;                         // loads of 32 rows
  static constexpr int RPI = 64 / C;                           // rows of a load
  static constexpr int XB = D / 32;                            // exponent bytes of a row
  static constexpr int XL = QUANT ? 1 : 0;                     // loads of a block's exponents
  static constexpr int WAVE = 2 * KB + XL * 2 * 256;           // bytes of a wave
  // place of row r's chunk c
  __device__ __forceinline__ static constexpr int swz(int r) {
    return C >= 8 ? r & 7 : C == 4 ? (r >> 1) & 3 : (r >> 2) & 1;
  }
  __device__ __forceinline__ static constexpr int vswz(int r) {
    return QUANT ? swz(r) : sizeof(T) == 2 ? (r & 3) << 1 : (r >> 2 & 3) << 2;
  }
  __device__ __forceinline__ static int at(int r, int c) { return r * RB + 16 * (c ^ swz(r)); }
  __device__ __forceinline__ static int vat(int r, int c) { return r * RB + 16 * (c ^ vswz(r)); }
  // Loads Q, Q + 1, ... of 32 rows of K, or V, from b0 and b1 on (sixteen each); off:
  // the lane's place in the first one (row and chunk orders are xors of their bits).
  template <bool V, int Q = 0>
  __device__ __forceinline__ static void load(const unsigned char* b0, const unsigned char* b1,
                                              uint32_t off, uint32_t lds) {
    if constexpr (C == 2) {  // sixteen rows in each half of the wave
      row_load<0>(((threadIdx.x & 32) == 0 ? b0 : b1 - 16 * RB) + off, lds);
    } else if constexpr (Q < NI) {
      constexpr int in = Q * 1024 % (16 * RB), imm = in & 4095;
      constexpr uint32_t x = 16 * (V ? vswz(Q * RPI) : swz(Q * RPI));
      tile_load<imm, Q * 1024>((Q * 1024 >= 16 * RB ? b1 : b0) + (in - imm), off ^ x, lds);
      load<V, Q + 1>(b0, b1, off, lds);
    }
  }
};

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// 4 bytes per lane straight to LDS (lane l's at `lds` + 4 l); m0 as in tile_load.
__device__ __forceinline__ void word_load(const void* g, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %0, off"
      :
      : "v"(g), "s"(lds)
      : "memory", "m0");
}
template <typename V>
__device__ __forceinline__ V lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) V*)(size_t)at;
}

// The bits of those values of a word that are no numbers.
template <typename T, int FMT>
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
  uint32_t odd = 0;
  constexpr int B = FMT != WF_CACHE_PLAIN ? 8 : 8 * (int)sizeof(T);
  constexpr uint32_t top = FMT != WF_CACHE_PLAIN ? 0x7fu : sizeof(T) == 2 ? 0x7f80u : 0x7f800000u;
  constexpr uint32_t all = B == 32 ? ~0u : (1u << (B & 31)) - 1u;
#pragma unroll
  for (int k = 0; k < 32; k += B) odd |= (w >> k & top) == top ? all << k : 0u;
  return odd;
}

// Eight codes to the operand of a product, times `scale`: two words in 8 bits, one in 4.
template <int FMT>
__device__ __forceinline__ u32x4 operand(uint32_t c0, uint32_t c1, float scale) {
  u32x4 v;
  auto bits = [](auto x) { return __builtin_bit_cast(uint32_t, x); };
  if constexpr (FMT == WF_CACHE_E4M3) {
    v[0] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, false));
    v[1] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, true));
    v[2] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, false));
    v[3] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, true));
  } else {
    v[0] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, scale, 0));
    v[1] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, scale, 1));
    v[2] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, scale, 2));
    v[3] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c0, scale, 3));
  }
  return v;
}
__device__ __forceinline__ u32x2 read_tr16(uint32_t at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) v4i16p*)(size_t)at));
}
template <int FMT>
__device__ __forceinline__ u32x2 read_codes(uint32_t at) {
  auto p = (__attribute__((address_space(3))) v2i_few*)(size_t)at;
  if constexpr (FMT == WF_CACHE_E4M3)
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(p));
  else
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr4_b64_v2i32(p));
}
// V's exponents of four keys.
template <int XB>
__device__ __forceinline__ void exponents4(uint32_t at, uint32_t* x) {
  if constexpr (XB == 4) {
    const u32x4 w = lds_read<u32x4>(at);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = w[e];
  } else {
    const u32x2 w = lds_read<u32x2>(at);
#pragma unroll
    for (int e = 0; e < 2; ++e) x[e] = w[e];
  }
}
// w 2^b, b a signed byte of x
__device__ __forceinline__ float times_exponent(float w, uint32_t x, int b) {
  return __builtin_amdgcn_ldexpf(w, (int)(x << (24 - 8 * b)) >> 24);
}

// What a wave makes of a block of 32 keys for 32 query rows: products of 32 x 32.
// A lane has scores of query row l % 32, keys 8 (e / 4) + 4 h + e % 4.
template <int D, int FMT>
struct FewRows32 {
  using G = FewGeom<bf16_t, D, FMT>;
  using W = PrefixWave<bf16_t, D, 1>;
  static constexpr int QN = 32, RB = G::RB, XB = G::XB, DT = D / 32;
  W w;
  f32x16 sc, t;

  __device__ __forceinline__ void init(float scale) { w.init(scale); }
  __device__ __forceinline__ static int query() { return threadIdx.x & 31; }
  __device__ __forceinline__ static int half() { return (threadIdx.x & 63) >> 5; }
  // channels h D / 2 + 8 j of step j
  __device__ __forceinline__ void load(const bf16_t* row) {
#pragma unroll
    for (int j = 0; j < W::QS; ++j)
      w.q[0][j] = reinterpret_cast<const u32x4*>(row)[half() * (D / 16) + j];
  }
  __device__ __forceinline__ void scores(uint32_t kat, uint32_t xat) {
    const int h = half(), r = query();
    constexpr int HC = G::C / 2;  // chunks of a lane
    u32x4 kc[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c) kc[c] = lds_read<u32x4>(kat + G::at(r, h * HC + c));
    const uint32_t kx = !G::QUANT  ? 0u
                        : XB == 4 ? lds_read<uint32_t>(xat + 4 * r) >> (16 * h)
                                  : lds_read<uint8_t>(xat + 2 * r + h);
    __builtin_amdgcn_sched_barrier(0);  // (all reads queued before the first is waited for)
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
    for (int j = 0; j < W::QS; ++j) {
      const float scale = block_scale(j < 4 ? kx & 0xff : kx >> 8 & 0xff);
      u32x4 kf;
      if constexpr (!G::QUANT)
        kf = kc[j];
      else if constexpr (FMT == WF_CACHE_E4M3)
        kf = operand<FMT>(kc[j / 2][2 * (j & 1)], kc[j / 2][2 * (j & 1) + 1], scale);
      else
        kf = operand<FMT>(kc[j / 4][j & 3], 0, scale);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                   __builtin_bit_cast(bf16x8, w.q[0][j]), sc, 0, 0,
                                                   0);
    }
  }
  // The block's weights; masked: of the keys whose bits are set in seen.
  __device__ __forceinline__ void softmax(bool masked, uint32_t seen) {
    const int h = half();
    auto hide = [&](float by) __attribute__((always_inline)) {
      if (!masked) return;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        t[e] = seen >> (8 * (e >> 2) + 4 * h + (e & 3)) & 1 ? t[e] : by;
    };
    w.shift_one(0, sc, t);
    hide(-INFINITY);
    float mx[1] = {w.largest(t)};
    w.raise(
        mx, [&](int, float by) __attribute__((always_inline)) { w.drop(t, by); },
        [&](int, float& mn, float& al) __attribute__((always_inline)) {
          t = sc;
          hide(-w.c2 * INFINITY);
          w.anew(0, t, mn, al);
        });
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      t[e] = __builtin_amdgcn_exp2f(t[e]);
      z += t[e];
    }
    w.l[0] += z;
  }
  __device__ __forceinline__ void product(int d, const u32x4& vf, const u32x4& pf) {
    w.O[0][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf),
                                                        __builtin_bit_cast(bf16x8, pf), w.O[0][d],
                                                        0, 0, 0);
  }
  // The weighted values.  A lane's place in a transposed load is a part of a row of
  // eight in 8 bits, of sixteen in 4 bits, of four in bf16, each of 16 channels.
  __device__ __forceinline__ void values(uint32_t vat, uint32_t vx) {
    const int h = half(), i16 = threadIdx.x & 15, hi = (threadIdx.x >> 4) & 1;
    const int p = FMT == WF_CACHE_E4M3 ? i16 >> 1 : FMT == WF_CACHE_E2M1 ? i16 : i16 >> 2;
    const int row = 16 * (p >> 3) + 8 * (p >> 2 & 1) + 4 * h + (p & 3);
    uint32_t vb = vat + (FMT == WF_CACHE_E4M3   ? G::vat(row, hi) + 8 * (i16 & 1)
                         : FMT == WF_CACHE_E2M1 ? G::vat(row, 0) + 8 * hi
                                                : G::vat(row, 2 * hi + (i16 >> 1 & 1)) + 8 * (i16 & 1));
    asm volatile("" : "+v"(vb));
    if constexpr (!G::QUANT) {
      u32x2 v[2][DT][2];  // (all reads queued before the first is waited for, here too)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            v[kb][d][k] = read_tr16((vb ^ (64 * d)) + (2 * kb + k) * 8 * RB);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        u32x4 pf;
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[e] = pack_bf16x2(t[8 * kb + 2 * e], t[8 * kb + 2 * e + 1]);
#pragma unroll
        for (int d = 0; d < DT; ++d)
          product(d, u32x4{v[kb][d][0][0], v[kb][d][0][1], v[kb][d][1][0], v[kb][d][1][1]}, pf);
      }
    } else {
      u32x2 c[DT][FMT == WF_CACHE_E4M3 ? 2 : 1];
#pragma unroll
      for (int d = 0; d < DT; ++d)
        if constexpr (FMT == WF_CACHE_E4M3) {
          c[d][0] = read_codes<FMT>(vb ^ (32 * d));
          c[d][1] = read_codes<FMT>((vb ^ (32 * d)) + 16 * RB);
        } else {
          c[d][0] = read_codes<FMT>(vb ^ (16 * d));
        }
      uint32_t xs[4 * XB];
#pragma unroll
      for (int q = 0; q < 4; ++q) exponents4<XB>(vx + (8 * q + 4 * h) * XB, xs + XB * q);
      __builtin_amdgcn_sched_barrier(0);
      // (less 128, for which the weights are doubled)
#pragma unroll
      for (int e = 0; e < 4 * XB; ++e) xs[e] ^= 0x80808080u;
#pragma unroll
      for (int e = 0; e < 16; ++e) t[e] += t[e];
      // the weights of half the keys for channels 32 d ..: times 2^(x - 127)
      auto weights = [&](int kb, int d) __attribute__((always_inline)) {
        u32x4 pf;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = 8 * kb + 2 * e, b0 = k * XB + d, b1 = b0 + XB;
          pf[e] = pack_bf16x2(times_exponent(t[k], xs[b0 / 4], b0 & 3),
                              times_exponent(t[k + 1], xs[b1 / 4], b1 & 3));
        }
        return pf;
      };
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          product(d,
                  FMT == WF_CACHE_E4M3 ? operand<FMT>(c[d][kb][0], c[d][kb][1], 1.f)
                                       : operand<FMT>(c[d][0][kb], 0, 1.f),
                  weights(kb, d));
    }
  }
  // The row's outputs, reference and sum; o, st: of the wave's rows.
  __device__ __forceinline__ void put(float* o, float* st, int stride) {
    const int h = half(), r = query();
    const float l = w.l[0] + partner32(w.l[0]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(o + r * stride + 32 * d + 2 * i + 4 * h) =
            f32x4{w.O[0][d][i], w.O[0][d][i + 1], w.O[0][d][i + 2], w.O[0][d][i + 3]};
    if (h == 0) {
      st[2 * r] = w.reference(0);
      st[2 * r + 1] = l;
    }
  }
};

// For 16 query rows: products of 16 x 16, half the softmax and weights of 32 rows.
// A lane has scores of query row l % 16, keys 16 (e / 4) + 4 g + e % 4, g = l / 16.
// bf16 products take 32 channels, or the block's keys, at once (a lane's eight of
// them), fp32 ones four (a lane's one).
template <typename T, int D, int FMT>
struct FewRows16 {
  using G = FewGeom<T, D, FMT>;
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int QN = 16, RB = G::RB, XB = G::XB, CT = D / 16;
  static constexpr int QS = BF ? D / 32 : D / 16;  // 16-byte query operands of a lane
  u32x4 q[QS];
  f32x4 O[CT];  // channels 16 c + 4 g .. + 3
  float sc[8], t[8];
  float mref, l, nref, limit, f, c2, c2p;  // as in PrefixWave

  __device__ __forceinline__ void init(float scale) {
    c2 = scale * kLog2e;
    c2p = __uint_as_float(__float_as_uint(c2) & 0xff800000u);
    mref = limit = -INFINITY;
    nref = l = 0.f;
    f = c2;
#pragma unroll
    for (int c = 0; c < CT; ++c) O[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ static int query() { return threadIdx.x & 15; }
  __device__ __forceinline__ static int group() { return (threadIdx.x & 63) >> 4; }
  // channels g D / 4 on
  __device__ __forceinline__ void load(const T* row) {
#pragma unroll
    for (int j = 0; j < QS; ++j) q[j] = reinterpret_cast<const u32x4*>(row)[group() * QS + j];
  }
  __device__ __forceinline__ void scores(uint32_t kat, uint32_t xat) {
    const int g = group();
    // 16-byte chunks of a lane's part of a row; 4 bits of 64 channels: half a chunk
    constexpr int HC = G::C >= 4 ? G::C / 4 : 1;
    u32x4 kc[2][HC];
    uint32_t kx[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = 16 * k + query();
      if constexpr (G::QUANT) kx[k] = lds_read<uint8_t>(xat + XB * r + g * XB / 4);
      if constexpr (G::C >= 4) {
#pragma unroll
        for (int c = 0; c < HC; ++c) kc[k][c] = lds_read<u32x4>(kat + G::at(r, g * HC + c));
      } else {
        const u32x2 w = lds_read<u32x2>(kat + G::at(r, g >> 1) + 8 * (g & 1));
        kc[k][0] = u32x4{w[0], w[1], 0u, 0u};
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // (all reads queued before the first is waited for)
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if constexpr (BF) {
#pragma unroll
      for (int j = 0; j < QS; ++j)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float scale = block_scale(kx[k]);
          u32x4 kf;
          if constexpr (!G::QUANT)
            kf = kc[k][j];
          else if constexpr (FMT == WF_CACHE_E4M3)
            kf = operand<FMT>(kc[k][j / 2][2 * (j & 1)], kc[k][j / 2][2 * (j & 1) + 1], scale);
          else
            kf = operand<FMT>(kc[k][0][j], 0, scale);
          s[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf),
                                                         __builtin_bit_cast(bf16x8, q[j]), s[k], 0,
                                                         0, 0);
        }
    } else {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {  // eight channels
        float v[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if constexpr (FMT == WF_CACHE_E4M3) {
            decode8<FMT>(u32x2{kc[k][j / 2][2 * (j & 1)], kc[k][j / 2][2 * (j & 1) + 1]},
                         block_scale(kx[k]), v[k]);
          } else if constexpr (FMT == WF_CACHE_E2M1) {
            decode8<FMT>(u32x2{kc[k][0][j], 0u}, block_scale(kx[k]), v[k]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = __uint_as_float(kc[k][2 * j + e / 4][e & 3]);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            s[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                v[k][e], __uint_as_float(q[2 * j + e / 4][e & 3]), s[k], 0, 0, 0);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sc[e] = s[e >> 2][e & 3];
  }
  __device__ __forceinline__ float ratio() const {  // c2 / c2p
    return __uint_as_float((__float_as_uint(c2) & 0x7fffffu) | 0x3f800000u);
  }
  __device__ __forceinline__ float reference() const { return f == c2 ? mref : mref * ratio(); }
  // As PrefixWave's: the reference moves when a score passes it by 2^8, and the
  // scores, which are kept, are then made anew, a far reference with the power of two.
  __device__ __forceinline__ void softmax(bool masked, uint32_t seen) {
    const int g = group();
    auto hide = [&](float by) __attribute__((always_inline)) {
      if (!masked) return;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        t[e] = seen >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1 ? t[e] : by;
    };
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = fmaf(sc[e], f, nref);
    hide(-INFINITY);
    float mx = t[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, t[e]);
    if (__builtin_amdgcn_ballot_w64(mx > limit) != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = sc[e];
      hide(-c2 * INFINITY);
      float x = t[0] * c2p;  // (exact, and in the order of the products with c2)
#pragma unroll
      for (int e = 1; e < 8; ++e) x = fmaxf(x, t[e] * c2p);
      x = max_xor32(max_xor16(x));
      const float was = reference(), m = x * ratio();
      const bool up = m > was;
      const float by = !up ? f : fabsf(m) >= PrefixWave<bf16_t, D, 1>::kFar ? c2p : c2;
      const float mn = !up ? mref : by == c2 ? m : x;
      const float al = !up ? 1.f
                       : mref == -INFINITY ? 0.f
                                           : __builtin_amdgcn_exp2f(by == f ? mref - mn : was - m);
      f = by;
      mref = mn;
      nref = mn > -INFINITY ? -mn : 0.f;
      limit = mn > -INFINITY ? 8.f : -INFINITY;
      l *= al;
#pragma unroll
      for (int c = 0; c < CT; ++c) O[c] *= al;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = fmaf(t[e], f, nref);
    }
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] = __builtin_amdgcn_exp2f(t[e]);
      z += t[e];
    }
    l += z;
  }
  // A transposed load's rows: the lane's eight keys (in 4 bits twice).
  __device__ __forceinline__ void values(uint32_t vat, uint32_t vx) {
    const int g = group(), i16 = threadIdx.x & 15;
    if constexpr (!BF && !G::QUANT) {
      // (fp32: a channel of a lane, row by row)
      uint32_t vb = vat + G::vat(4 * g, i16 >> 2) + 4 * (i16 & 3);
      asm volatile("" : "+v"(vb));
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = lds_read<float>((vb ^ (64 * c)) + (16 * (e >> 2) + (e & 3)) * RB);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          O[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], t[e], O[c], 0, 0, 0);
      }
      return;
    }
    const int p = FMT == WF_CACHE_E4M3 ? i16 >> 1 : FMT == WF_CACHE_E2M1 ? i16 & 7 : i16 >> 2;
    const int row = 16 * (p >> 2) + 4 * g + (p & 3);
    uint32_t vb = vat + (FMT == WF_CACHE_E4M3   ? G::vat(row, 0) + 8 * (i16 & 1)
                         : FMT == WF_CACHE_E2M1 ? G::vat(row, 0)
                                                : G::vat(row, i16 >> 1 & 1) + 8 * (i16 & 1));
    asm volatile("" : "+v"(vb));
    // (all reads queued before the first is waited for)
    u32x2 w[CT][G::QUANT ? 1 : 2];
    uint32_t xs[2 * XB];
    if constexpr (G::QUANT) {
      exponents4<XB>(vx + 4 * g * XB, xs);
      exponents4<XB>(vx + (16 + 4 * g) * XB, xs + XB);
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if constexpr (G::QUANT) {
        w[c][0] = read_codes<FMT>(vb ^ ((FMT == WF_CACHE_E4M3 ? 16 : 8) * c));
      } else {
        w[c][0] = read_tr16(vb ^ (32 * c));
        w[c][1] = read_tr16((vb ^ (32 * c)) + 16 * RB);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (G::QUANT) {  // less 128; the weights are doubled for it
#pragma unroll
      for (int e = 0; e < 2 * XB; ++e) xs[e] ^= 0x80808080u;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] += t[e];
    }
    // the weight of the lane's key e for channels 32 d ..: times 2^(x - 127)
    auto weight = [&](int e, int d) __attribute__((always_inline)) {
      const int b = e * XB + d;
      return times_exponent(t[e], xs[b / 4], b & 3);
    };
    u32x4 pf;
    float pw[8];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (G::QUANT ? c % 2 == 0 : c == 0) {  // the weights for 32 channels, or for all
#pragma unroll
        for (int e = 0; e < 8; ++e) pw[e] = G::QUANT ? weight(e, c / 2) : t[e];
        if constexpr (BF)
          pf = u32x4{pack_bf16x2(pw[0], pw[1]), pack_bf16x2(pw[2], pw[3]),
                     pack_bf16x2(pw[4], pw[5]), pack_bf16x2(pw[6], pw[7])};
      }
      if constexpr (BF) {
        u32x4 vf;
        if constexpr (!G::QUANT)
          vf = u32x4{w[c][0][0], w[c][0][1], w[c][1][0], w[c][1][1]};
        else
          vf = operand<FMT>(w[c][0][0], w[c][0][1], 1.f);
        O[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf),
                                                       __builtin_bit_cast(bf16x8, pf), O[c], 0, 0,
                                                       0);
      } else if constexpr (G::QUANT) {
        float v[8];
        decode8<FMT>(w[c][0], 1.f, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          O[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], pw[e], O[c], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void put(float* o, float* st, int stride) {
    const float z = add_xor32(add_xor16(l));
#pragma unroll
    for (int c = 0; c < CT; ++c)
      *reinterpret_cast<f32x4*>(o + query() * stride + 16 * c + 4 * group()) = O[c];
    if (group() == 0) {
      st[2 * query()] = reference();
      st[2 * query() + 1] = z;
    }
  }
};

// The waves' outputs in LDS: row r of wave k at k QN + r, their references and sums
// behind them.
template <int D, int QN>
struct FewOut {
  static constexpr int STRIDE = D + 4;
  static constexpr size_t BYTES = (size_t)kFewWaves * QN * (STRIDE + 2) * sizeof(float);
};

// Two workgroups per CU, of which fp32 rows of 128 channels have the LDS for one.
// (Registers for three of 16 rows over codes: the same times.)
template <typename T, int D, int FMT>
constexpr int few_groups() {
  return FewGeom<T, D, FMT>::WAVE * kFewWaves > 80 * 1024 ? 1 : 2;
}

template <typename T, int D, int FMT, int QN>
__global__ __launch_bounds__(64 * kFewWaves, (few_groups<T, D, FMT>())) void tree_few_kernel(
    TreeArgs a) {
  using G = FewGeom<T, D, FMT>;
  constexpr int NI = G::NI, RB = G::RB, KB = G::KB, XB = G::XB;
  constexpr bool QUANT = G::QUANT;
  extern __shared__ __align__(16) unsigned char smem[];  // the waves' blocks, two flags
  // values that are no numbers: whether there are any in blocks of keys that not all
  // rows see; in the others, the top bit of the byte of each 32 channels that have one
  uint32_t* flag = reinterpret_cast<uint32_t*>(smem + kFewWaves * G::WAVE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int item = xcd_swizzle(blockIdx.x, gridDim.x);
  if (item >= a.items) return;  // (the grid holds whole eights of them)
  const TreeItem it(a, item);
  const int sp = it.sp, head = it.head, seq = it.seq;
  const int k0 = sp * a.rps, m0 = QN * it.mb;
  // the wave's blocks: wave, wave + 4, ... of the range
  auto key_of = [&](int i) { return k0 + 32 * (wave + kFewWaves * i); };
  // (scalar loads: uniform, and no kernel that runs beside this writes tables)
  const __attribute__((address_space(4))) int32_t* table =
      (const __attribute__((address_space(4))) int32_t*)(a.table + (long)seq * a.tp);
  // pages of a block's two sixteens of rows (past the last: whatever the table holds)
  struct Pages {
    int a, b;
  };
  auto pages_of = [&](int i) __attribute__((always_inline)) {
    const int k = key_of(i);
    return Pages{table[min(k >> a.shift, a.tp - 1)], table[min((k + 16) >> a.shift, a.tp - 1)]};
  };
  Pages pages = pages_of(0);
  const Sequence s(a, seq);
  asm volatile("" : "+s"(pages.a), "+s"(pages.b));  // (beside the sequence's length)
  const int M = s.n * a.g;
  const int nk = min(a.rps, s.L - k0);  // the range's keys
  if (m0 >= M || (nk <= 0 && !a.whole)) return;
  std::conditional_t<QN == 32, FewRows32<D, FMT>, FewRows16<T, D, FMT>> w;
  w.init(a.scale);
  if (threadIdx.x <= QUANT) flag[threadIdx.x] = 0;
  lds_barrier();

  const int nb = nk > 0 ? (nk + 31) / 32 : 0;
  const int mine = nb > wave ? (nb - wave + kFewWaves - 1) / kFewWaves : 0;
  if (mine > 0) {
    const int kend = k0 + nk;
    // their first rows in the pool
    auto rows_of = [&](int i, const Pages& p, long& r0, long& r1) __attribute__((always_inline)) {
      const int k = key_of(i), in = (1 << a.shift) - 1;
      r0 = (((long)min(max(p.a, 0), a.pages - 1) * a.heads + head) << a.shift) + (k & in);
      r1 = a.shift > 4 ? r0 + 16
                       : (((long)min(max(p.b, 0), a.pages - 1) * a.heads + head) << a.shift) +
                             ((k + 16) & in);
    };
    const uint32_t kat = lds_offset(smem) + wave * G::WAVE, vat = kat + KB, exps = vat + KB;
    // the lane's 16 bytes of a load: row of those that it holds, chunk
    const int lrow = lane / G::C;
    const uint32_t koff = lrow * RB + 16 * (lane % G::C ^ G::swz(lrow));
    const uint32_t voff = lrow * RB + 16 * (lane % G::C ^ G::vswz(lrow));
    // the lane's 4 bytes of the exponents: K's of the 32 rows, then V's (again in the
    // lanes behind them)
    constexpr int XD = 8 * XB;
    const int xl = lane % (2 * XD), xg = xl % XD / (XD / 2);
    const uint8_t* xbase = (xl / XD ? a.Vx : a.Kx) + 4 * (xl % (XD / 2));
    // block i's loads: rows from r0 and r1 on
    const unsigned char* K = static_cast<const unsigned char*>(a.K);
    const unsigned char* V = static_cast<const unsigned char*>(a.V);
    auto exp_load = [&](long r0, long r1, uint32_t lds) __attribute__((always_inline)) {
      word_load(xbase + (xg ? r1 : r0) * XB, lds);
    };
    auto queue_keys = [&](int i, long r0, long r1) __attribute__((always_inline)) {
      G::template load<false>(K + r0 * RB, K + r1 * RB, koff, kat);
      if constexpr (QUANT) exp_load(r0, r1, exps + (i & 1) * 256);
    };
    auto queue_vals = [&](long r0, long r1) __attribute__((always_inline)) {
      G::template load<true>(V + r0 * RB, V + r1 * RB, voff, vat);
    };

    long r0, r1;
    rows_of(0, pages, r0, r1);
    queue_keys(0, r0, r1);
    queue_vals(r0, r1);
    const int m = min(m0 + w.query(), M - 1), ti = a.by_g(m);  // the lane's query row
    const long tok = min(max(s.first + ti, 0L), a.tokens - 1L);
    w.load(static_cast<const T*>(a.Q) + tok * a.qs + (long)(head * a.g + m - ti * a.g) * D);
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): so that no later wait is for these
    pages = pages_of(1);  // of the block that is queued next
    const uint32_t* words = a.mask ? a.mask + tok * a.words : nullptr;

    for (int i = 0; i < mine; ++i) {
      const int key = key_of(i), nv = min(32, kend - key);
      const uint32_t xat = exps + (i & 1) * 256;
      const bool more = i + 1 < mine;
      if (more) rows_of(i + 1, pages, r0, r1);
      pages = pages_of(i + 2);
      wait_loads<NI>();  // (V's may still be on their way)
      w.scores(kat, xat);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the codes have been read
      if (more) queue_keys(i + 1, r0, r1);

      // softmax, with the keys that the row does not see taken out
      const bool masked = key + 32 > min(s.base, kend);
      uint32_t seen = ~0u;
      if (masked) seen = seen_keys(a, s, ti, words, key, nv);
      w.softmax(masked, seen);

      if (more)
        wait_loads<NI + G::XL>();
      else
        wait_loads<0>();
      const uint32_t vx = xat + 32 * XB;  // V's exponents
      if (nv < 32) {  // rows behind the last: they may hold codes that are no numbers
        for (int c = lane; c < (32 - nv) * G::C; c += 64)
          *(__attribute__((address_space(3))) u32x4*)(size_t)(vat + nv * RB + 16 * c) =
              u32x4{0u, 0u, 0u, 0u};
      }
      // Values that are no numbers: a block of channels with the exponent byte 255, and
      // in 8 bits codes of NaN, or NaN and infinities in bf16.  Where not all rows see
      // them they are cleared, and put to the rows that do behind the last block.  Where
      // all do, the product makes NaN of those codes and values; of a byte 255, which is
      // no power of two for the weights, the channels are noted, NaN in every row.
      bool odd = false;
      if constexpr (QUANT) {
        const int r = lane & 31;
        const uint32_t x =
            XB == 4 ? lds_read<uint32_t>(vx + 4 * r) : lds_read<uint16_t>(vx + 2 * r);
        const uint32_t bad = r < nv ? ((x & 0x7f7f7f7fu) + 0x01010101u) & x & 0x80808080u : 0u;
        if (masked)
          odd = bad != 0;
        else if (bad != 0)  // rare
          atomicOr(flag + 1, bad);
      }
      if (FMT != WF_CACHE_E2M1 && masked)
        for (int c = lane; c < nv * G::C; c += 64) {
          const u32x4 v = lds_read<u32x4>(vat + 16 * c);
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= odd_bits<T, FMT>(v[e]) != 0;
        }
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {  // rare
        if (lane == 0) *flag = 1;
        if constexpr (FMT != WF_CACHE_E2M1)
          for (int c = lane; c < 32 * G::C; c += 64) {
            u32x4 v = lds_read<u32x4>(vat + 16 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] &= ~odd_bits<T, FMT>(v[e]);
            *(__attribute__((address_space(3))) u32x4*)(size_t)(vat + 16 * c) = v;
          }
      }
      w.values(vat, vx);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the codes have been read
      if (more) queue_vals(r0, r1);
    }
  }

  lds_barrier();  // the blocks are idle
  const bool odd = __builtin_amdgcn_readfirstlane(*flag) != 0;
  const uint32_t none = QUANT ? __builtin_amdgcn_readfirstlane(flag[1]) : 0u;  // (channels)
  // the first block that not all rows see
  const int odd_from = k0 + max(min(s.base - k0, nk), 0) / 32 * 32;
  lds_barrier();
  using Out = FewOut<D, QN>;
  float* out = reinterpret_cast<float*>(smem);
  float* stats = out + kFewWaves * QN * Out::STRIDE;
  w.put(out + wave * QN * Out::STRIDE, stats + wave * QN * 2, Out::STRIDE);
  lds_barrier();
  constexpr int C4 = D / 4, RPP = 64 * kFewWaves / C4;  // rows per round
  const int c = threadIdx.x % C4;
  for (int r = threadIdx.x / C4; r < min(QN, M - m0); r += RPP) {
    Merge4 g;
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) {
      const hw_f32x2 mz = *reinterpret_cast<const hw_f32x2*>(stats + 2 * (k * QN + r));
      g.add(mz[0], mz[1], *reinterpret_cast<const f32x4*>(out + (k * QN + r) * Out::STRIDE + 4 * c));
    }
    const int i = a.by_g(m0 + r);
    const long tok = s.first + i;
    if (!Sequence::there(a, tok)) continue;
    if (odd) add_odd<T, D, FMT>(a, s, seq, head, i, odd_from, k0 + nk, 4 * c, g.o);
    if (QUANT && (none >> c / 8 * 8 & 0x80u)) g.o = f32x4{NAN, NAN, NAN, NAN};
    const int hq = head * a.g + m0 + r - i * a.g;
    const long row = tok * a.hq + hq;
    if (a.whole) {
      g.finish(static_cast<T*>(a.O) + tok * a.os + (long)hq * D + 4 * c,
                  a.lse ? a.lse + row : nullptr, c == 0);
    } else {
      const long at = row * a.splits + sp;
      *reinterpret_cast<f32x4*>(a.part + at * D + 4 * c) = g.o;
      if (c == 0) *reinterpret_cast<hw_f32x2*>(a.pstat + 2 * at) = hw_f32x2{g.M, g.z};
    }
  }
}

// ------------------------------------------------------------ host side

template <typename T, int D, int FMT, int QN>
static constexpr size_t few_lds() {
  const size_t blocks = (size_t)kFewWaves * FewGeom<T, D, FMT>::WAVE + 2 * sizeof(uint32_t);
  const size_t out = FewOut<D, QN>::BYTES;
  return blocks > out ? blocks : out;
}

hipError_t launch_tree_few(const TreeArgs& a, int dtype, int head_dim, int format, int rows,
                           long items, hipStream_t s) {
  auto go = [&](auto t, auto d, auto f, auto n) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, F = decltype(f)::value, QN = decltype(n)::value;
    constexpr size_t lds = few_lds<T, D, F, QN>();
    auto kern = tree_few_kernel<T, D, F, QN>;
    if (lds > 65536) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)((items + 7) & ~7L)), dim3(64 * kFewWaves), lds, s, a);
    return hipGetLastError();
  };
  auto by_rows = [&](auto d, auto f) {
    using N16 = std::integral_constant<int, 16>;
    if (dtype == WF_F32) return go(float{}, d, f, N16{});
    return rows == 16 ? go(bf16_t{}, d, f, N16{})
                      : go(bf16_t{}, d, f, std::integral_constant<int, 32>{});
  };
  auto by_format = [&](auto d) {
    if (format == WF_CACHE_E4M3) return by_rows(d, std::integral_constant<int, WF_CACHE_E4M3>{});
    if (format == WF_CACHE_E2M1) return by_rows(d, std::integral_constant<int, WF_CACHE_E2M1>{});
    return by_rows(d, std::integral_constant<int, WF_CACHE_PLAIN>{});
  };
  return head_dim == 128 ? by_format(std::integral_constant<int, 128>{})
                         : by_format(std::integral_constant<int, 64>{});
}

hipError_t load_tree_few_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(
      &fa, reinterpret_cast<const void*>(tree_few_kernel<bf16_t, 128, WF_CACHE_PLAIN, 16>));
}

}  // namespace wf
