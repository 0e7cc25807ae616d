// Tiles of 64 keys and values in LDS, and what a wave makes of them: scores,
// softmax and weighted values of its query rows, partial results and their merge.
// Shared by the attention kernels over a prefix and over a cache in pages.
#pragma once

#include "wf_cache.hpp"
#include "wf_kernels.hpp"

namespace wf {

// Waves of a workgroup.  bf16 rows that are read as codes take two per SIMD in a
// plain loop, one beside the other's waits, decodes and softmax (128 query rows
// over 32K keys in 8 bits: 40 us, and 49 with four waves that pipeline
// themselves, whose registers the codes on their way overfill); bf16 rows take one
// per SIMD with a loop that pipelines itself (2048 rows over 32K keys: 253 us, and on
// the same card 293 with eight waves in the plain loop, which read every key from LDS
// twice as often); fp32 rows one per SIMD in the plain loop,
// whose products, at an eighth of the rate, are the bound.
template <typename T, int FMT>
constexpr int prefix_waves() {
  return sizeof(T) == 2 && FMT != WF_CACHE_PLAIN ? 8 : 4;
}
constexpr int kTileRows = 64;     // keys of an LDS tile

typedef short v4i16p __attribute__((ext_vector_type(4)));

// A tile of K or V in LDS: the 64-byte pieces of its rows, piece-major, so that
// every operand of a lane is at a constant from its first one.  In a piece of K
// the 16-byte granule k is in slot k ^ ((r >> 2) & 3): the 16 rows that are read
// at one granule then meet all banks.  V, whose transposed reads take whole
// pieces of four rows, stays in order.
constexpr int kPiece = kTileRows * 64;  // bytes from piece to piece
template <typename T, int D>
struct TileGeom {
  static constexpr int RB = D * (int)sizeof(T);  // bytes of a row
  static constexpr int NP = RB / 64;             // pieces of a row
  static constexpr int MB = kTileRows * RB;      // bytes of a K (or V) tile
  // tiles in LDS: the pipelined loop has one in use, the next one visible, one
  // in flight and one being queued; four do not fit with fp32 rows of 128
  static constexpr int SLOTS = 8 * MB > 131072 ? 2 : 4;
};
// LDS offset of granule k of row r
__device__ __forceinline__ int key_offset(int r, int k) {
  return (k >> 2) * kPiece + r * 64 + 16 * ((k & 3) ^ ((r >> 2) & 3));
}
__device__ __forceinline__ int val_offset(int r, int k) {
  return (k >> 2) * kPiece + r * 64 + 16 * (k & 3);
}

// A wave's 32 QW query rows: operands, outputs and running softmax.
template <typename T, int D, int QW>
struct PrefixWave {
  using Geom = TileGeom<T, D>;
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int QS = BF ? D / 16 : D / 8; // 16-byte query operands per lane
  static constexpr int DT = D / 32;              // 32-channel output tiles

  u32x4 q[QW][QS];
  f32x16 O[QW][DT];
  float mref[QW], l[QW];
  float nref[QW];   // -mref, 0 while that is -inf
  float limit[QW];  // 8; -inf while the reference is -inf
  float f[QW];      // what scores are multiplied by: c2, or with a far reference c2p
  float c2, c2p;    // scale log2(e); its power of two
  // LDS byte offsets of the lane's first operands in a 32-row block of a tile
  uint32_t ko[2], vo;

  __device__ __forceinline__ void init(float scale) {
    c2 = scale * kLog2e;
    c2p = __uint_as_float(__float_as_uint(c2) & 0xff800000u);
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, i16 = lane & 15;
    ko[0] = key_offset(l32, h);
    ko[1] = key_offset(l32, 2 + h);
    // bf16: in each 16-lane group lane i points at row t0 + i / 4, channels c0 +
    // 4 (i % 4) .. + 3, and receives rows t0 .. t0 + 3 of channel c0 + i
    const int t0 = 4 * h + (i16 >> 2), c0 = (lane & 16) + 4 * (i16 & 3);
    vo = BF ? val_offset(t0, c0 >> 3) + 2 * (c0 & 7)
            : val_offset(4 * h, l32 >> 2) + 4 * (l32 & 3);
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      mref[b] = limit[b] = -INFINITY;
      nref[b] = l[b] = 0.f;
      f[b] = c2;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[b][d][i] = 0.f;
    }
  }

  // The lane's first operands in the block at LDS offset `at`.  (Opaque, so that
  // the others are read at constant offsets from them and not from sums kept in
  // registers.)
  struct KeyBase {
    uint32_t b[2];
  };
  __device__ __forceinline__ KeyBase key_base(uint32_t at) const {
    KeyBase k = {{at + ko[0], at + ko[1]}};
    asm volatile("" : "+v"(k.b[0]), "+v"(k.b[1]));
    return k;
  }
  __device__ __forceinline__ uint32_t val_base(uint32_t at) const {
    uint32_t v = at + vo;
    asm volatile("" : "+v"(v));
    return v;
  }
  // Operand j of K: 16 bytes of the lane's row, granule 2 j + h.
  __device__ __forceinline__ static u32x4 key(const KeyBase& k, int j) {
    return *(const __attribute__((address_space(3))) u32x4*)(size_t)(k.b[j & 1] +
                                                                     (j >> 1) * kPiece);
  }
  __device__ __forceinline__ void keys(uint32_t at, u32x4 (&kf)[QS]) const {
    const KeyBase k = key_base(at);
#pragma unroll
    for (int j = 0; j < QS; ++j) kf[j] = key(k, j);
  }
  // Half of the operand of V^T of 16 of the block's rows (bf16): rows 16 kb + 8 k
  // + 4 h .. + 3 of channel 32 d + l % 32.
  __device__ __forceinline__ static u32x2 val(uint32_t base, int kb, int d, int k) {
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) v4i16p*)(size_t)(
                       base + d * kPiece + (2 * kb + k) * 512)));
  }
  // s = scores of 32 keys; lane: keys 8 (i / 4) + 4 h + i % 4 of query l % 32
  __device__ __forceinline__ void scores(const u32x4 (&kf)[QS], f32x16 (&s)[QW]) const {
#pragma unroll
    for (int b = 0; b < QW; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int j = 0; j < QS; ++j) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        if constexpr (BF) {
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[j]),
                                                         __builtin_bit_cast(bf16x8, q[b][j]), s[b],
                                                         0, 0, 0);
        } else {
          const f32x4 kv = __builtin_bit_cast(f32x4, kf[j]), qv = __builtin_bit_cast(f32x4, q[b][j]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[e], qv[e], s[b], 0, 0, 0);
        }
      }
    }
  }

  // 32 keys at LDS offsets kat, vat, the first nv of which are valid; MASK: with nv
  // < 32 those whose bits are set in the word of the lane's query row (for each block
  // of rows)
  template <bool MASK = false>
  __device__ __forceinline__ void step(uint32_t kat, uint32_t vat, int nv,
                                       const uint32_t* words = nullptr) {
    const int h = (threadIdx.x & 63) >> 5;
    uint32_t seen[QW];  // the lane's keys: bits 8 (i / 4) + i % 4
#pragma unroll
    for (int b = 0; b < QW; ++b) seen[b] = MASK ? words[b] >> (4 * h) : 0u;
    u32x4 kf[QS];
    f32x16 s[QW];
    keys(kat, kf);
    // products before the other wave's softmax (256 rows over 128K keys in 4 bits
    // 140 us, and 145 at one priority, or at a fixed one for each wave)
    __builtin_amdgcn_s_setprio(1);
    scores(kf, s);
    __builtin_amdgcn_s_setprio(0);
    f32x16 t[QW];
    float mx[QW];
    auto shifted = [&](int b) __attribute__((always_inline)) {
      shift_one(b, s[b], t[b]);
      if (nv < 32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool hidden = MASK ? !(seen[b] >> (8 * (i >> 2) + (i & 3)) & 1)
                                   : 8 * (i >> 2) + 4 * h + (i & 3) >= nv;
          t[b][i] = hidden ? -INFINITY : t[b][i];
        }
      }
    };
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      shifted(b);
      mx[b] = largest(t[b]);
    }
    raise(
        mx,
        [&](int b, float by) __attribute__((always_inline)) {
          if constexpr (BF)
            drop(t[b], by);
          else
            shifted(b);  // (fp32: large scores keep their differences)
        },
        [&](int b, float& mn, float& al) __attribute__((always_inline)) {
          // (a count of its own: the comparisons are not kept for this)
          int n = nv;
          asm volatile("" : "+s"(n));
          if constexpr (BF)
            score_one(b, key_base(kat), t[b]);  // (s is not kept for this)
          else
            t[b] = s[b];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool hidden = MASK ? n < 32 && !(seen[b] >> (8 * (i >> 2) + (i & 3)) & 1)
                                     : 8 * (i >> 2) + 4 * h + (i & 3) >= n;
            t[b][i] = hidden ? -c2 * INFINITY : t[b][i];
          }
          anew(b, t[b], mn, al);
        });
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        t[b][i] = __builtin_amdgcn_exp2f(t[b][i]);
        z += t[b][i];
      }
      l[b] += z;
    }
    const uint32_t vb = val_base(vat);
    __builtin_amdgcn_s_setprio(1);
    if constexpr (BF) {
      // (each weight rounded to bf16, as the products' operands are)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        u32x4 pf[QW];
#pragma unroll
        for (int b = 0; b < QW; ++b)
          pf[b] = u32x4{pack_bf16x2(t[b][8 * kb], t[b][8 * kb + 1]),
                        pack_bf16x2(t[b][8 * kb + 2], t[b][8 * kb + 3]),
                        pack_bf16x2(t[b][8 * kb + 4], t[b][8 * kb + 5]),
                        pack_bf16x2(t[b][8 * kb + 6], t[b][8 * kb + 7])};
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const u32x2 lo = val(vb, kb, d, 0), hi = val(vb, kb, d, 1);
          const u32x4 vf = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
          for (int b = 0; b < QW; ++b)
            O[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf),
                                                              __builtin_bit_cast(bf16x8, pf[b]),
                                                              O[b][d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const float vf = *(const __attribute__((address_space(3))) float*)(size_t)(
              vb + 2 * d * kPiece + (8 * (i >> 2) + (i & 3)) * 64);
#pragma unroll
          for (int b = 0; b < QW; ++b)
            O[b][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, t[b][i], O[b][d], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
  }
  __device__ __forceinline__ void rescale(int b, float mn, float al) {
    mref[b] = mn;
    nref[b] = mn > -INFINITY ? -mn : 0.f;
    limit[b] = mn > -INFINITY ? 8.f : -INFINITY;
    l[b] *= al;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[b][d][i] *= al;
  }

  // Scores in log2 units less the reference: t = s f - mref, the product
  // unrounded (while every score so far is -inf, t is -inf and the weight 0).
  __device__ __forceinline__ void shift_one(int b, const f32x16& s, f32x16& t) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = fmaf(s[i], f[b], nref[b]);
  }
  __device__ __forceinline__ static void drop(f32x16& t, float by) {
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] -= by;
  }
  __device__ __forceinline__ static float largest(const f32x16& t) {
    float mx = fmaxf(t[0], t[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) mx = fmaxf(mx, fmaxf(t[i], t[i + 1]));
    return mx;
  }
  __device__ __forceinline__ float ratio() const {  // c2 / c2p
    return __uint_as_float((__float_as_uint(c2) & 0x7fffffu) | 0x3f800000u);
  }
  // The reference in log2 units.
  __device__ __forceinline__ float reference(int b) const {
    return f[b] == c2 ? mref[b] : mref[b] * ratio();
  }
  // The reference moves only when a score passes it by 2^8: weights then stay
  // below 2^8, their sums far from the fp32 range, and a rescale of the outputs
  // is rare.  again(b, by): the scores less the new reference, by above the old.
  // Scores less a reference that is far below them have lost their differences:
  // where a reference moves far, or to a far place, afresh(b, its place, the factor
  // of the sums) makes them anew.  (The factor in a register of its own and the code
  // that is not reached cost 1%: 2048 rows over 32K keys 240.5 -> 242.8 us.)
  template <typename Again, typename Afresh>
  __device__ __forceinline__ void raise(const float (&mx)[QW], const Again& again,
                                        const Afresh& afresh) {
    bool grow = false;
#pragma unroll
    for (int b = 0; b < QW; ++b) grow |= mx[b] > limit[b];
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      float mn[QW], by[QW], al[QW];
      bool far = false;
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        const float up = fmaxf(mx[b], partner32(mx[b]));
        const bool first = mref[b] == -INFINITY;
        mn[b] = first ? up : fmaxf(mref[b], mref[b] + up);
        by[b] = mn[b] > -INFINITY ? mn[b] + nref[b] : 0.f;  // (nref: 0 or -mref)
        al[b] = first ? 0.f : __builtin_amdgcn_exp2f(-by[b]);
        far |= fabsf(by[b]) > 1024.f || (mn[b] > -INFINITY && fabsf(mn[b]) >= kFar);
      }
      if (__builtin_amdgcn_ballot_w64(far) != 0) {
#pragma unroll
        for (int b = 0; b < QW; ++b) {
          afresh(b, mn[b], al[b]);
          by[b] = 0.f;
        }
      }
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        rescale(b, mn[b], al[b]);
        again(b, by[b]);
      }
    }
  }
  // A block's scores t made scores less the reference mn, which moves to their
  // maximum where that is above the old one; al: the factor of the sums so far.  The
  // unrounded product and the reference, a rounded one, differ by up to half a unit
  // in the last place: 32 below 2^30, and beyond it weights would leave the fp32
  // range.  There a row multiplies its scores by a power of two, which is exact, in
  // place of c2.  Two scores of that size that differ do so by 32 at least then: the
  // lower one's weight is nothing with either factor.
  static constexpr float kFar = 0x1p30f;
  __device__ __forceinline__ void anew(int b, f32x16& t, float& mn, float& al) {
    float x = t[0] * c2p;  // (c2p: in the order of the products with c2, and exact)
#pragma unroll
    for (int i = 1; i < 16; ++i) x = fmaxf(x, t[i] * c2p);
    x = fmaxf(x, partner32(x));
    const float was = reference(b), m = x * ratio();
    const bool up = m > was;
    const float g = !up ? f[b] : fabsf(m) >= kFar ? c2p : c2;
    mn = !up ? mref[b] : g == c2 ? m : x;
    // (equal factors: the difference of the references themselves)
    al = !up ? 1.f
         : mref[b] == -INFINITY ? 0.f
                                : __builtin_amdgcn_exp2f(g == f[b] ? mref[b] - mn : was - m);
    f[b] = g;
    const float n = mn > -INFINITY ? -mn : 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = fmaf(t[i], g, n);
  }
  // The scores of 32 keys of one block of query rows, an operand at a time (bf16).
  __device__ __forceinline__ void score_one(int b, const KeyBase& k, f32x16& s) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < QS; ++j) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, key(k, j)),
                                                  __builtin_bit_cast(bf16x8, q[b][j]), s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // A block of the pipelined loop (bf16): weights of one block (shifted scores s) and their
  // product with V (at LDS offset vat) beside the scores sn of the next block
  // (its keys kf in registers; refilled with those at knext).  A wave issues in
  // order, an instruction in about five cycles, and waits for the matrix pipe at
  // its next product: only what stands between two products runs beside them.
  // Every product (32 cycles) is followed by its share of the vector work, LDS
  // reads and tile loads (load(i), i < NL), and the barriers hold that order.
  template <int NL, typename Load>
  __device__ __forceinline__ void block(uint32_t vat, uint32_t knext, u32x4 (&kf)[QS],
                                        f32x16 (&s)[QW], f32x16 (&sn)[QW], float (&mx)[QW],
                                        const Load& load) {
    float z[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b) z[b] = 0.f;
    const uint32_t vb = val_base(vat);
    const KeyBase kn = key_base(knext);
    u32x4 p0[QW], p1[QW], v0[DT], v1[DT];
    // weight e of 16 keys (of the block's first or second half)
    auto weight = [&](int half, int e) __attribute__((always_inline)) {
      const int b = e >> 3, i = 8 * half + (e & 7);
      s[b][i] = __builtin_amdgcn_exp2f(s[b][i]);
      z[b] += s[b][i];
      if (e & 1) {
        // (each weight rounded to bf16, as the products' operands are)
        uint32_t w = pack_bf16x2(s[b][i - 1], s[b][i]);
        asm volatile("" : "+v"(w), "+v"(z[b]));  // here, and not where it is used
        (half ? p1 : p0)[b][(e & 7) >> 1] = w;
      }
    };
    auto value = [&](int r) __attribute__((always_inline)) {
      const int kb = r / (2 * DT), d = (r >> 1) % DT, k = r & 1;
      const u32x2 y = val(vb, kb, d, k);
      (kb ? v1 : v0)[d][2 * k] = y[0];
      (kb ? v1 : v0)[d][2 * k + 1] = y[1];
    };
    constexpr int NQ = QS * QW, NV = DT * QW;  // products with K, with half of V
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int j = n / QW, b = n % QW;
      f32x16 c;
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = j ? sn[b][i] : 0.f;
      sn[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[j]),
                                                      __builtin_bit_cast(bf16x8, q[b][j]), c, 0, 0,
                                                      0);
#pragma unroll
      for (int r = n * 4 * DT / NQ; r < (n + 1) * 4 * DT / NQ; ++r) value(r);
      if (n < QW) {  // (the first products run beside this)
        if (n == QW - 1) {
          __builtin_amdgcn_sched_barrier(0);
          raise(
              mx, [&](int g, float by) __attribute__((always_inline)) { drop(s[g], by); },
              [&](int g, float& mn, float& al) __attribute__((always_inline)) {
                // (the block's keys are still in LDS, before its values)
                score_one(g, key_base(vat - Geom::MB), s[g]);
                anew(g, s[g], mn, al);
              });
#pragma unroll
          for (int e = 0; e < QW * 8 * QW / NQ; ++e) weight(0, e);
        }
      } else {
#pragma unroll
        for (int e = n * 8 * QW / NQ; e < (n + 1) * 8 * QW / NQ; ++e) weight(0, e);
      }
      if constexpr (NL > 0) {
        if ((n + 1) * NL / NQ > n * NL / NQ) load(n * NL / NQ, (n + 1) * NL / NQ);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int d = n / QW, b = n % QW;
      O[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v0[d]),
                                                        __builtin_bit_cast(bf16x8, p0[b]), O[b][d],
                                                        0, 0, 0);
#pragma unroll
      for (int e = n * 8 * QW / NV; e < (n + 1) * 8 * QW / NV; ++e) weight(1, e);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int d = n / QW, b = n % QW;
      O[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v1[d]),
                                                        __builtin_bit_cast(bf16x8, p1[b]), O[b][d],
                                                        0, 0, 0);
#pragma unroll
      for (int j = n * QS / NV; j < (n + 1) * QS / NV; ++j) kf[j] = key(kn, j);
#pragma unroll
      for (int e = n * 8 * QW / NV; e < (n + 1) * 8 * QW / NV; ++e) {
        const int g = e >> 3, i = 2 * (e & 7);
        sn[g][i] = fmaf(sn[g][i], f[g], nref[g]);
        sn[g][i + 1] = fmaf(sn[g][i + 1], f[g], nref[g]);
        const float two = fmaxf(sn[g][i], sn[g][i + 1]);
        mx[g] = i ? fmaxf(mx[g], two) : two;
        asm volatile("" : "+v"(mx[g]));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      l[b] += z[b];
      asm volatile("" : "+v"(l[b]));
    }
  }
};

// 16 bytes per lane from base + off + OFF straight to LDS (lane l's at `lds` + AT
// + 16 l; the instruction adds OFF to both addresses).  Waited for as
// async_load16's.  m0 is named as overwritten, not saved and restored as there:
// nothing else in this file's kernels uses it (a test reads the built code for that).
template <int OFF, int AT>
__device__ __forceinline__ void tile_load(const void* base, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_add_u32 m0, %2, %4\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1 offset:%3"
      :
      : "v"(off), "s"(base), "s"(lds), "n"(OFF), "n"(AT - OFF)
      : "memory", "m0", "scc");
}
template <int OFF>
__device__ __forceinline__ void row_load(const void* g, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off offset:%2"
      :
      : "v"(g), "s"(lds - OFF), "n"(OFF)
      : "memory", "m0");
}

template <typename T>
__device__ __forceinline__ void put4(T* p, const f32x4& v);
template <>
__device__ __forceinline__ void put4<bf16_t>(bf16_t* p, const f32x4& v) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
template <>
__device__ __forceinline__ void put4<float>(float* p, const f32x4& v) {
  *reinterpret_cast<f32x4*>(p) = v;
}

// A tile of a cache as a thread stages it: pieces of 16 codes (E4M3) or 32
// (E2M1), 16 bytes, and their block's exponent byte.  Four lanes load 64 bytes in
// a row; they write their granules in an order of their own each (by x below), so
// that eight lanes meet all banks.
template <typename T, int D, int FMT, int NW, int OF = NW>
struct QuantStage {
  using Geom = TileGeom<T, D>;
  static constexpr int CPP = FMT == WF_CACHE_E2M1 ? 32 : 16;  // channels per piece
  static constexpr int PPR = D / CPP;                         // pieces per row
  static constexpr int PT = kTileRows * PPR;                  // pieces of a tile and matrix
  static constexpr int N = (PT + 64 * NW - 1) / (64 * NW);  // per thread
  u32x4 w[2][N];
  uint32_t x[2][N];

  // the wave of those that load a tile: NW of the workgroup's OF
  __device__ __forceinline__ static int wave() {
    return OF == NW ? threadIdx.x >> 6 : (threadIdx.x >> 6) % NW;
  }
  // a wave's 64 pieces: 8 rows of 8 (two halves of a row's pieces after each
  // other), 16 rows of 4 or 32 rows of 2
  __device__ __forceinline__ static int row(int i) {
    const int lane = threadIdx.x & 63, w64 = i * NW + wave();
    return PPR == 8 ? w64 * 8 + ((lane >> 2) & 7) : w64 * (64 / PPR) + lane / PPR;
  }
  __device__ __forceinline__ static int piece() {
    const int lane = threadIdx.x & 63;
    return PPR == 8 ? (lane & 3) + 4 * (lane >> 5) : lane % PPR;
  }

  // a thread has no piece of a tile that is smaller than the workgroup
  __device__ __forceinline__ static bool idle() { return PT < 64 * NW && (int)threadIdx.x >= PT; }
  // its piece i: row r of the cache
  __device__ __forceinline__ void load(int i, const void* K, const void* V, const uint8_t* Kx,
                                       const uint8_t* Vx, long r) {
    w[0][i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(K) +
                                              (r * PPR + piece()) * 16);
    w[1][i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(V) +
                                              (r * PPR + piece()) * 16);
    x[0][i] = Kx[r * (D / 32) + piece() * CPP / 32];
    x[1][i] = Vx[r * (D / 32) + piece() * CPP / 32];
  }
  __device__ __forceinline__ void commit(unsigned char* tile) const {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (PT < 64 * NW && (int)threadIdx.x >= PT) break;
        const int r = row(i), pc = piece();
        const float s = block_scale(x[m][i]);
        unsigned char* dst = tile + m * Geom::MB;
        auto at = [&](int k) { return dst + (m ? val_offset(r, k) : key_offset(r, k)); };
        // v_cvt_scalef32_pk_bf16: two codes times the power of two, rounded to
        // nearest even: equal to decode8 and pack_bf16x2 for every code and
        // exponent byte 1 .. 255 (byte 0 is 2^-127 here, and the store gives it to
        // no block: it stands in cleared rows, whose codes are 0)
        u32x4 c = w[m][i];
        constexpr bool TWO = FMT == WF_CACHE_E4M3 && sizeof(T) == 2;   // two granules a piece
        constexpr bool FOUR = !TWO && (sizeof(T) == 2 || FMT == WF_CACHE_E4M3);  // four, a word each
        const int o = TWO ? (pc >> 1) & 1 : FOUR ? pc & 3 : 0;
        if constexpr (TWO)
          c = o ? u32x4{c[2], c[3], c[0], c[1]} : c;
        if constexpr (FOUR) {
          c = o & 1 ? u32x4{c[1], c[0], c[3], c[2]} : c;
          c = o & 2 ? u32x4{c[2], c[3], c[0], c[1]} : c;
        }
        if constexpr (TWO) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            u32x4 g;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              g[2 * e] = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * k + e], s, false));
              g[2 * e + 1] = __builtin_bit_cast(
                  uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * k + e], s, true));
            }
            *reinterpret_cast<u32x4*>(at(2 * pc + (k ^ o))) = g;
          }
        } else if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            u32x4 g;
            g[0] = __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 0));
            g[1] = __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 1));
            g[2] = __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 2));
            g[3] = __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 3));
            *reinterpret_cast<u32x4*>(at(4 * pc + (k ^ o))) = g;
          }
        } else if constexpr (FOUR) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float v[8];
            decode8<FMT>(u32x2{c[2 * k], c[2 * k + 1]}, s, v);
            *reinterpret_cast<f32x4*>(at(4 * pc + ((2 * k) ^ o))) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(at(4 * pc + ((2 * k + 1) ^ o))) =
                f32x4{v[4], v[5], v[6], v[7]};
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float v[8];
            decode8<FMT>(u32x2{c[k], 0u}, s, v);
            *reinterpret_cast<f32x4*>(at(8 * pc + 2 * k)) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(at(8 * pc + 2 * k + 1)) = f32x4{v[4], v[5], v[6], v[7]};
          }
        }
      }
  }
};

// Rows nr .. 63 of the tile's V cleared: they repeat the range's last row or hold
// what was there before, and 0 times an infinite value is NaN.  Ends with a
// barrier.
template <typename T, int D, int NW>
__device__ __forceinline__ void clear_rows(unsigned char* tile, int nr) {
  using Geom = TileGeom<T, D>;
  unsigned char* V = tile + Geom::MB;
  const int n = (kTileRows - nr) * 4;  // granules of a piece's rows
  for (int i = threadIdx.x; i < n * Geom::NP; i += 64 * NW)
    *reinterpret_cast<u32x4*>(V + i / n * kPiece + nr * 64 + i % n * 16) = u32x4{0u, 0u, 0u, 0u};
  lds_barrier();
}

// Running merge of partials (reference, sum, four channels).
struct Merge4 {
  float M = -INFINITY, z = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  // (no branches: the loads of several partials stay in flight together)
  __device__ __forceinline__ void add(float m, float zs, const f32x4& x) {
    const bool none = m == -INFINITY && zs == 0.f;  // an empty range: it has no output
    const float mn = fmaxf(M, m);
    // (all scores -inf or NaN: zs says it)
    const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
    const float g = M > -INFINITY ? __builtin_amdgcn_exp2f(M - mn) : 1.f;
    M = mn;
    z = z * g + f * zs;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * g + f * (none ? 0.f : x[e]);
  }
  template <typename T>
  __device__ __forceinline__ void finish(T* O, float* lse, bool first) const {
    put4<T>(O, o * (z == 0.f ? 0.f : 1.f / z));
    if (lse && first) *lse = z == 0.f ? -INFINITY : (M + __log2f(z)) * kLn2;
  }
};

// The workgroup's outputs in LDS, so that they leave it in whole rows: wave w's
// row r at (w 32 QW + r), unnormalised, and its reference and sum behind them.
template <int D, int QW, int NW>
struct OutRows {
  static constexpr int STRIDE = D + 4;  // floats (eight rows at one channel meet all banks)
  static constexpr int ROWS = NW * 32 * QW;
  static constexpr size_t BYTES = (size_t)ROWS * (STRIDE + 2) * sizeof(float);
  float* o;
  float* st;
  __device__ __forceinline__ explicit OutRows(unsigned char* smem)
      : o(reinterpret_cast<float*>(smem)), st(o + ROWS * STRIDE) {}
  // (the tiles are idle: the caller has passed a barrier)
  template <typename T>
  __device__ __forceinline__ void put(PrefixWave<T, D, QW>& w, int wave) {
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      const float l = w.l[b] + partner32(w.l[b]);
      const int r = (wave * QW + b) * 32 + l32;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(o + r * STRIDE + 32 * d + 2 * i + 4 * h) =
              f32x4{w.O[b][d][i], w.O[b][d][i + 1], w.O[b][d][i + 2], w.O[b][d][i + 3]};
      if (h == 0) {
        st[2 * r] = w.reference(b);
        st[2 * r + 1] = l;
      }
    }
    lds_barrier();
  }
  // four channels of NR rows, each merged over the KW waves that have it (the
  // first in row v)
  template <int NR>
  __device__ __forceinline__ void merged(const int (&v)[NR], int KW, int c, Merge4 (&g)[NR]) const {
    for (int k = 0; k < KW; ++k) {
      hw_f32x2 mz[NR];
      f32x4 x[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int r = v[i] + k * 32 * QW;
        mz[i] = *reinterpret_cast<const hw_f32x2*>(st + 2 * r);
        x[i] = *reinterpret_cast<const f32x4*>(o + r * STRIDE + 4 * c);
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) g[i].add(mz[i][0], mz[i][1], x[i]);
    }
  }
};

}  // namespace wf
