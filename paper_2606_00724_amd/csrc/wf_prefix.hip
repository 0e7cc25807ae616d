// Attention of a batch whose sequences share a prefix (wf_prefix_attn).
//
// For a K/V head of a prefix, the query rows of all its sequences and of the
// head's group are one block of M = share * group * q_len rows that sees the
// same keys: the prefix is read once for all of them.  A workgroup of the
// first kernel takes a block of those rows and a range of the prefix's keys
// and leaves an unnormalised output with the rows' reference (log2 units) and
// sum of weights.  The second kernel takes a sequence's R = group * q_len rows
// over its own keys and merges the partials of the prefix into them; where
// there are no own keys it only merges, and where there is one range it is not
// needed.
//
// S^T = K Q^T on 32 x 32 products: a lane then holds 16 scores of one query
// row, so that the softmax needs no lane exchange except one of the maximum
// with the lane of the other 16, and its weights are in place as the B operand
// of O^T = V^T P^T (the order of the keys inside that product is free, and V^T
// is read from LDS in the order of the scores).
//
// Few query rows are bound by the cache's bytes, more than about 250 rows a
// K/V head by the products.  bf16, d = 128, 8 K/V heads, on one MI355X: 2048
// query rows a head over 32K keys take 243 to 253 us by the card, 1.1 PFLOP/s (a
// product of 8192 x 8192 matrices reaches 1.21, groups of four 1.34); 256 rows over
// 128K keys in 4 bits 138 to 143 us, 1.0 PFLOP/s; 32 rows over 32K bf16 keys 30 us,
// 4.5 TB/s with the merge.
#include "wf_cache.hpp"
#include "wf_kernels.hpp"
#include "wf_launch.hpp"

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
constexpr int kOwnWaves = 4;      // waves of a workgroup over a sequence's own keys
constexpr int kPrefixIds = 4096;  // row ids in LDS at once (whole tiles)
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

// The rows of a workgroup's key range: row i of the range is key k0 + i, at
// most its last one.
struct KeyRows {
  const int32_t* ids;   // LDS: rows of keys id0, id0 + 1, ... (list), or null
  int cap;              // rows of the unit
  int k0, last;         // first key, last key
  int id0;
  __device__ __forceinline__ long operator()(int i) const {
    const int k = min(k0 + i, last);
    // ids are clamped into the unit: a bad id cannot leave K / V
    return ids ? min(max(ids[k - id0], 0), cap - 1) : k;
  }
};

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

  // 32 keys at LDS offsets kat, vat, the first nv of which are valid
  __device__ __forceinline__ void step(uint32_t kat, uint32_t vat, int nv) {
    const int h = (threadIdx.x & 63) >> 5;
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
        for (int i = 0; i < 16; ++i)
          t[b][i] = 8 * (i >> 2) + 4 * h + (i & 3) >= nv ? -INFINITY : t[b][i];
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
          for (int i = 0; i < 16; ++i)
            t[b][i] = 8 * (i >> 2) + 4 * h + (i & 3) >= n ? -c2 * INFINITY : t[b][i];
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

// Tiles by direct loads.  Wave w loads rows 16 w .. + 15 of a tile, one 64-byte
// piece of each in an instruction (four lanes a row).
template <typename T, int D>
struct TileLoads {
  using Geom = TileGeom<T, D>;
  static constexpr int N = Geom::NP;  // instructions per wave and matrix
  const unsigned char* K;             // the unit's rows
  const unsigned char* V;
  uint32_t off[2];                    // the lane's byte offsets in a tile of consecutive rows
  uint32_t lds;                       // LDS offset of the wave's rows in tile slot 0
  int row;                            // the lane's row in a tile

  __device__ __forceinline__ void init(const void* Ku, const void* Vu, uint32_t lds0) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    K = static_cast<const unsigned char*>(Ku);
    V = static_cast<const unsigned char*>(Vu);
    row = 16 * wave + (lane >> 2);
    off[0] = row * Geom::RB + 16 * ((lane & 3) ^ ((lane >> 4) & 3));
    off[1] = row * Geom::RB + 16 * (lane & 3);
    lds = lds0 + 1024 * wave;
  }
  // instruction i of 2 N (K's, then V's) of a tile of consecutive rows
  struct Tile {
    const unsigned char *k, *v;  // its first rows
    uint32_t to;                 // LDS offset of the wave's rows in its slot
    int go;                      // whether it is loaded
  };
  __device__ __forceinline__ Tile at(long r0, uint32_t slot, bool go) const {
    return Tile{K + r0 * Geom::RB, V + r0 * Geom::RB, lds + slot * 2 * Geom::MB,
                __builtin_amdgcn_readfirstlane(go ? 1 : 0)};
  }
  template <int I>
  __device__ __forceinline__ void one(const Tile& t) const {
    tile_load<(I % N) * 64, (I / N) * Geom::MB + (I % N) * kPiece>(I < N ? t.k : t.v, off[I / N],
                                                                   t.to);
  }
  template <int I, int E>
  __device__ __forceinline__ void some(const Tile& t) const {
    if constexpr (I < E) {
      one<I>(t);
      some<I + 1, E>(t);
    }
  }
  // a whole tile whose row i is `at`(i)
  template <int I = 0>
  __device__ __forceinline__ void rows(const unsigned char* k, const unsigned char* v,
                                       uint32_t to) const {
    if constexpr (I < N) {
      row_load<I * 64>(k, to + I * kPiece);
      row_load<I * 64>(v, to + Geom::MB + I * kPiece);
      rows<I + 1>(k, v, to);
    }
  }
  __device__ __forceinline__ void tile(const KeyRows& at, int first, bool straight,
                                       uint32_t slot) const {
    if (straight) {  // uniform
      some<0, 2 * N>(this->at(at.k0 + first, slot, true));
    } else {
      const long r = at(first + row) - row;  // (the offsets hold the row in the tile)
      rows(K + r * Geom::RB + off[0], V + r * Geom::RB + off[1], lds + slot * 2 * Geom::MB);
    }
  }
};

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
template <typename T, int D, int FMT, int NW>
struct QuantStage {
  using Geom = TileGeom<T, D>;
  static constexpr int CPP = FMT == WF_CACHE_E2M1 ? 32 : 16;  // channels per piece
  static constexpr int PPR = D / CPP;                         // pieces per row
  static constexpr int PT = kTileRows * PPR;                  // pieces of a tile and matrix
  static constexpr int N = (PT + 64 * NW - 1) / (64 * NW);  // per thread
  u32x4 w[2][N];
  uint32_t x[2][N];

  // a wave's 64 pieces: 8 rows of 8 (two halves of a row's pieces after each
  // other), 16 rows of 4 or 32 rows of 2
  __device__ __forceinline__ static int row(int i) {
    const int lane = threadIdx.x & 63, w64 = i * NW + (threadIdx.x >> 6);
    return PPR == 8 ? w64 * 8 + ((lane >> 2) & 7) : w64 * (64 / PPR) + lane / PPR;
  }
  __device__ __forceinline__ static int piece() {
    const int lane = threadIdx.x & 63;
    return PPR == 8 ? (lane & 3) + 4 * (lane >> 5) : lane % PPR;
  }

  // the tile whose first row is `first` of the range; straight: whole and of
  // consecutive rows
  __device__ __forceinline__ void load(const PrefixArgs& a, const KeyRows& rows, long unit,
                                       int first, bool straight) {
    const uint8_t* K = static_cast<const uint8_t*>(a.K);
    const uint8_t* V = static_cast<const uint8_t*>(a.V);
    if (PT < 64 * NW && (int)threadIdx.x >= PT) return;
    if (straight) {  // uniform: the lanes' offsets are constant
      const long r0 = unit * a.cap + rows.k0 + first;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t o = (row(i) * PPR + piece()) * 16, e = row(i) * (D / 32) + piece() * CPP / 32;
        w[0][i] = *reinterpret_cast<const u32x4*>(K + r0 * (PPR * 16) + o);
        w[1][i] = *reinterpret_cast<const u32x4*>(V + r0 * (PPR * 16) + o);
        x[0][i] = (a.Kx + r0 * (D / 32))[e];
        x[1][i] = (a.Vx + r0 * (D / 32))[e];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long r = unit * a.cap + rows(first + row(i));
        w[0][i] = *reinterpret_cast<const u32x4*>(K + (r * PPR + piece()) * 16);
        w[1][i] = *reinterpret_cast<const u32x4*>(V + (r * PPR + piece()) * 16);
        x[0][i] = a.Kx[r * (D / 32) + piece() * CPP / 32];
        x[1][i] = a.Vx[r * (D / 32) + piece() * CPP / 32];
      }
    }
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

// Tile loads I0 + i .. I0 + e - 1 (the bounds are constants after unrolling).
template <typename T, int D, int I0, int I = 0>
__device__ __forceinline__ void load_some(const TileLoads<T, D>& dma, int i, int e,
                                          const typename TileLoads<T, D>::Tile& t) {
  if constexpr (I0 + I < 2 * TileLoads<T, D>::N) {
    if (I >= i && I < e) dma.template one<I0 + I>(t);
    if (I + 1 < e) load_some<T, D, I0, I + 1>(dma, i, e, t);
  }
}

// Partials first, first + step, ... of NR query rows into g, F of each in flight.
template <int D, int NR, int F>
__device__ __forceinline__ void merge_partials(const PrefixArgs& a, const long (&row)[NR], int c,
                                               int first, int step, Merge4 (&g)[NR]) {
  for (int s0 = first; s0 < a.slots; s0 += F * step) {
    hw_f32x2 mz[NR][F];
    f32x4 x[NR][F];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int k = 0; k < F; ++k) {  // (all queued; those past the last are dropped)
        const long s = row[i] * a.slots + min(s0 + k * step, a.slots - 1);
        mz[i][k] = *reinterpret_cast<const hw_f32x2*>(a.pstat + 2 * s);
        x[i][k] = *reinterpret_cast<const f32x4*>(a.part + s * D + 4 * c);
      }
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int k = 0; k < F; ++k) {
        const bool in = s0 + k * step < a.slots;
        g[i].add(in ? mz[i][k][0] : -INFINITY, in ? mz[i][k][1] : 0.f, x[i][k]);
      }
  }
}

// The prefix: query rows of all sequences of a (prefix, head) over a range of its
// keys.  Whole tiles of bf16 rows go through the pipelined loop, three tiles
// ahead in LDS; without its tile loads it is 14% faster, the products alone would
// take 70% of it (2048 rows over 32K keys).  Rows kept as codes are loaded to
// registers one tile ahead, decoded into LDS and multiplied from there: 128 keys
// take about 4.2 us for 256 query rows, 2.5 for 128 and 1.6 for 64, half of it
// products at 256 rows, and the decode and the LDS reads below.
template <typename T, int D, int FMT, int QW>
__global__ __launch_bounds__((64 * prefix_waves<T, FMT>())) void prefix_attn_kernel(
    PrefixArgs a) {
  constexpr int NW = prefix_waves<T, FMT>();
  using W = PrefixWave<T, D, QW>;
  using Geom = TileGeom<T, D>;
  constexpr int MB = Geom::MB, SLOTS = Geom::SLOTS, QS = W::QS;
  constexpr bool QUANT = FMT != WF_CACHE_PLAIN;
  extern __shared__ __align__(16) unsigned char smem[];  // [SLOTS][K, V] tiles, row ids
  int32_t* ids = reinterpret_cast<int32_t*>(smem + SLOTS * 2 * MB);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;

  // The workgroup's item, blocks of query rows innermost, so that those reading
  // the same keys run at once on one XCD.
  const int item = xcd_swizzle(blockIdx.x, gridDim.x);
  if (item >= a.p.items) return;  // (the grid holds whole eights of them)
  const int mb = item % a.p.mblocks, sp = item / a.p.mblocks % a.p.splits;
  const int unit = item / (a.p.mblocks * a.p.splits);  // (prefix, head)
  const int group = unit / a.heads, head = unit % a.heads;
  const int M = a.p.M, KW = a.p.kw;
  const int len = a.plen ? min(max(a.plen[group], 0), a.rows) : a.rows;
  const int k0 = sp * a.p.rps, nk = min(a.p.rps, len - k0);  // the range's keys (none: nk <= 0)
  const int kw = wave % KW, qw = wave / KW;
  const int mrows = a.p.mrows;  // NW / KW * 32 QW
  // query row m of the unit -> row of Q, O (at most 2^30 in all)
  auto row_of = [&](int m) {
    const int n = a.by_R(m);
    return ((group * a.share + n) * a.heads + head) * a.R + (m - n * a.R);
  };
  W w;
  w.init(a.scale);

  if (nk > 0) {
    // a tile: the keys of one slot, or with eight waves of two, for half the
    // barriers
    constexpr int US = NW == 8 ? 2 : 1, NS = SLOTS / US, KT = US * kTileRows;
    const int nt = (nk + KT - 1) / KT;
    KeyRows rows;
    rows.ids = a.list ? ids : nullptr;
    rows.cap = a.cap;
    rows.k0 = k0;
    rows.last = k0 + nk - 1;
    rows.id0 = k0;
    auto slot_of = [&](int t) { return t % NS * US; };
    // the next kPrefixIds ids of a list, from tile t on, when tile t starts them
    // (no wave reads older ones: tile t - 1 has been queued by all)
    auto stage_ids = [&](int t) __attribute__((always_inline)) {
      if (!rows.ids || t * KT % kPrefixIds != 0) return;  // uniform
      rows.id0 = k0 + t * KT;
      lds_barrier();
      for (int i = threadIdx.x; i < min(kPrefixIds, nk - t * KT); i += 64 * NW)
        ids[i] = a.list[(long)unit * a.rows + rows.id0 + i];
      __syncthreads();
    };
    TileLoads<T, D> dma;
    QuantStage<T, D, QUANT ? FMT : WF_CACHE_E4M3, NW> st[US];
    if constexpr (!QUANT)
      dma.init(static_cast<const T*>(a.K) + (long)unit * a.cap * D,
               static_cast<const T*>(a.V) + (long)unit * a.cap * D, lds_offset(smem));
    // tile t queued: on its way to its slot, or to registers
    int queued = 0;
    auto straight = [&](int t) { return !rows.ids && nk - t * KT >= KT; };
    auto queue = [&](int t) __attribute__((always_inline)) {
      stage_ids(t);
      queued = t + 1;
      if constexpr (QUANT) {
#pragma unroll
        for (int i = 0; i < US; ++i)
          st[i].load(a, rows, unit, t * KT + i * kTileRows, straight(t));
      } else {
        dma.tile(rows, t * KT, straight(t), slot_of(t));
      }
    };
    auto commit = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < US; ++i) st[i].commit(smem + (slot_of(t) + i) * 2 * MB);
    };
    // tile t is in its slot once every wave has passed the barrier behind this
    auto landed = [&](int t) __attribute__((always_inline)) {
      wait_vmcnt_chunks<2 * TileLoads<T, D>::N>(queued - 1 - t);
    };
    // The query operands: loaded beside the first tile, and waited for here, so
    // that the compiler's wait for them is no wait for a tile later on.  Those of
    // 64 rows of 128 channels are put into the accumulation half of the
    // registers, from where the products take them: in the other half they were
    // copied there and back in every block.
    queue(0);
    // whole tiles in the pipelined loop
    const int nf = W::BF && !QUANT ? nk / KT : 0;
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      const int m = mb * mrows + (qw * QW + b) * 32 + l32;
      const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const T*>(a.Q) +
                                                        (long)row_of(min(m, M - 1)) * D);
#pragma unroll
      for (int j = 0; j < QS; ++j) w.q[b][j] = src[2 * j + h];
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
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
        // Whether the loads of tile t + 3 go between the products of tile t; else
        // they are queued at once, if there are any.
        auto spread = [&](int t) __attribute__((always_inline)) {
          if (t + 3 >= nt) return false;
          if (!straight(t + 3)) {
            queue(t + 3);
            return false;
          }
          queued = t + 4;
          return true;
        };
        constexpr int N = TileLoads<T, D>::N;  // tile loads of K, of V
        if (QW > 1 || KW == 1) {  // (64 rows per wave: no waves share them)
          for (int t = 0; t < nf; ++t) {
            begin(t);
            const auto ahead = dma.at(k0 + (long)(t + 3) * KT, slot_of(t + 3), spread(t));
            const uint32_t now = tile_at(t) + MB, next = tile_at(t + 1 < nt ? t + 1 : t);
            w.template block<N>(now, next, kf, s0, s1, mx,
                                [&](int i, int e) __attribute__((always_inline)) {
                                  if (ahead.go) load_some<T, D, 0>(dma, i, e, ahead);
                                });
            w.template block<N>(now + 2048, next + 2048, kf, s1, s0, mx,
                                [&](int i, int e) __attribute__((always_inline)) {
                                  if (ahead.go) load_some<T, D, N>(dma, i, e, ahead);
                                });
          }
        } else {
          auto one = [&](int t, f32x16(&s)[QW], f32x16(&sn)[QW])
                         __attribute__((always_inline)) {
                           begin(t);
                           const auto ahead =
                               dma.at(k0 + (long)(t + 3) * KT, slot_of(t + 3), spread(t));
                           w.keys(tile_at(t + 1 < nt ? t + 1 : t), kf);
                           w.template block<2 * N>(
                               tile_at(t) + MB, tile_at(t), kf, s, sn, mx,
                               [&](int i, int e) __attribute__((always_inline)) {
                                 if (ahead.go) load_some<T, D, 0>(dma, i, e, ahead);
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
      if (nf == 0) {  // (else the tile has been visible since the last whole one)
        if constexpr (QUANT) {
          commit(t);
          if (t + 1 < nt) queue(t + 1);
        } else {
          landed(t);
        }
        lds_barrier();
        if (!QUANT && t + NS - 1 < nt) queue(t + NS - 1);
      }
      const int nr = nk - t * KT;  // rows of the tile that are in the range
      if (nr < KT) {
        const int last = (nr - 1) / kTileRows;  // its last 64 rows
        if (nr % kTileRows)
          clear_rows<T, D, NW>(smem + (slot_of(t) + last) * 2 * MB, nr - last * kTileRows);
      }
      for (int r = 32 * kw; r < min(nr, KT); r += 32 * KW) {
        const uint32_t at = lds_offset(smem) + (slot_of(t) + r / kTileRows) * 2 * MB +
                            r % kTileRows * 64;
        w.step(at, at + MB, min(32, nr - r));
      }
    }
    lds_barrier();  // the tiles are idle
  }

  OutRows<D, QW, NW> out(smem);
  out.put(w, wave);
  constexpr int C4 = D / 4, RPP = 64 * NW / C4;  // rows per round
  const int c = threadIdx.x % C4;
  constexpr int NR = 4;
  const int mend = min(mrows, M - mb * mrows);
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
      const int row = row_of(mb * mrows + r);
      if (a.whole) {
        g[i].finish(static_cast<T*>(a.O) + (long)row * D + 4 * c, a.lse ? a.lse + row : nullptr,
                    c == 0);
      } else {
        const long s = (long)row * a.slots + sp;
        if (nk > 0) *reinterpret_cast<f32x4*>(a.part + s * D + 4 * c) = g[i].o;
        if (c == 0) *reinterpret_cast<hw_f32x2*>(a.pstat + 2 * s) = hw_f32x2{g[i].M, g[i].z};
      }
    }
  }
}

// A sequence's rows over its own keys, merged with the partials of the prefix.
// The keys are few (a block, a generated tail): a workgroup takes all of them,
// and 32 rows per wave that does not share its rows' keys with others, or fewer
// where the partials of the rows are the work.
template <typename T, int D>
__global__ __launch_bounds__(64 * kOwnWaves, (TileGeom<T, D>::SLOTS / 2)) void prefix_own_kernel(
    PrefixArgs a) {  // (workgroups per CU: as its two tiles fit)
  using W = PrefixWave<T, D, 1>;
  using Geom = TileGeom<T, D>;
  constexpr int MB = Geom::MB, QS = W::QS, N = TileLoads<T, D>::N;
  extern __shared__ __align__(16) unsigned char smem[];  // [2][K, V] tiles
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int mb = blockIdx.x % a.t.mblocks, unit = blockIdx.x / a.t.mblocks;  // (sequence, head)
  const int KW = a.t.kw, kw = wave % KW, qw = wave / KW;
  const int mrows = a.t.mrows;
  const int m0 = mb * mrows;
  const int n = a.tlen ? min(max(a.tlen[unit / a.heads], 0), a.T) : a.T;
  const long row0 = (long)unit * a.R;
  W w;
  w.init(a.scale);
  if (n > 0) {
    const int nt = (n + kTileRows - 1) / kTileRows;
    TileLoads<T, D> dma;
    dma.init(static_cast<const T*>(a.Kt) + (long)unit * a.T * D,
             static_cast<const T*>(a.Vt) + (long)unit * a.T * D, lds_offset(smem));
    KeyRows rows;
    rows.ids = nullptr;
    rows.cap = a.T;
    rows.k0 = rows.id0 = 0;
    rows.last = n - 1;
    auto queue = [&](int t) __attribute__((always_inline)) {
      dma.tile(rows, t * kTileRows, n - t * kTileRows >= kTileRows, t & 1);
    };
    queue(0);
    const u32x4* src = reinterpret_cast<const u32x4*>(
        static_cast<const T*>(a.Q) + (row0 + min(m0 + qw * 32 + l32, a.R - 1)) * D);
#pragma unroll
    for (int j = 0; j < QS; ++j) w.q[0][j] = src[2 * j + h];
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the queries, and tile 0
    for (int t = 0; t < nt; ++t) {
      wait_vmcnt_chunks<2 * N>(0);
      lds_barrier();  // tile t visible, everyone is past tile t - 1
      if (t + 1 < nt) queue(t + 1);
      const int nr = n - t * kTileRows;
      unsigned char* tile = smem + (t & 1) * 2 * MB;
      if (nr < kTileRows) clear_rows<T, D, kOwnWaves>(tile, nr);
      if (qw < a.t.qw)
        for (int r = 32 * kw; r < min(nr, kTileRows); r += 32 * KW) {
          const uint32_t at = lds_offset(tile) + r * 64;
          w.step(at, at + MB, min(32, nr - r));
        }
    }
    lds_barrier();
  }
  OutRows<D, 1, kOwnWaves> out(smem);
  out.put(w, wave);
  constexpr int C4 = D / 4, RPP = 64 * kOwnWaves / C4;  // rows per round
  const int c = threadIdx.x % C4;
  const int mend = min(mrows, a.R - m0);
  if (2 * mend <= RPP && a.slots > 16) {
    // SG groups of threads take a row's partials in turn and meet in LDS (one row
    // a workgroup: 128 ranges 7.0 us and 18.2 without, 32 ranges 7.0 and 7.9; 16
    // ranges, which a thread has in flight at once, 6.8 and 6.2)
    int SG = 2;
    while (2 * SG * mend <= RPP) SG *= 2;
    const int r = (int)threadIdx.x / C4 / SG, sg = (int)threadIdx.x / C4 % SG;
    const int v[1] = {min(r, mend - 1)};
    const long row[1] = {row0 + m0 + v[0]};
    Merge4 g[1];
    if (sg == 0) out.merged(v, KW, c, g);
    merge_partials<D, 1, 16>(a, row, c, sg, SG, g);
    lds_barrier();  // the outputs have been read
    float* sh = reinterpret_cast<float*>(smem);
    constexpr int ST = 7;  // (odd: no bank met twice)
    float* mine = sh + threadIdx.x * ST;
    mine[0] = g[0].M;
    mine[1] = g[0].z;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[2 + e] = g[0].o[e];
    lds_barrier();
    if (sg != 0 || r >= mend) return;  // no barrier follows
    for (int k = 1; k < SG; ++k) {
      const float* x = mine + k * C4 * ST;
      g[0].add(x[0], x[1], f32x4{x[2], x[3], x[4], x[5]});
    }
    g[0].finish(static_cast<T*>(a.O) + row[0] * D + 4 * c, a.lse ? a.lse + row[0] : nullptr,
                c == 0);
    return;
  }
  auto rows_of = [&](auto nr, auto f) {
    constexpr int NR = decltype(nr)::value, F = decltype(f)::value;
    for (int r0 = threadIdx.x / C4; r0 < mend; r0 += NR * RPP) {
      int v[NR];
      long row[NR];
      Merge4 g[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int r = min(r0 + i * RPP, mend - 1);
        v[i] = r / 32 * KW * 32 + r % 32;
        row[i] = row0 + m0 + r;
      }
      out.merged(v, KW, c, g);
      if (a.slots > 0) merge_partials<D, NR, F>(a, row, c, 0, 1, g);
#pragma unroll
      for (int i = 0; i < NR; ++i)
        if (r0 + i * RPP < mend)
          g[i].finish(static_cast<T*>(a.O) + row[i] * D + 4 * c, a.lse ? a.lse + row[i] : nullptr,
                      c == 0);
    }
  };
  // Partials of a row in flight: about those it has, up to 32 of a thread's rows
  // together.  (Places past the last one are loaded too: 1024 rows of 32 heads over
  // 1K keys, one range, 39 us, and 50 with eight places a row; 128 rows over 4K,
  // eight ranges, 29.6, and 31.3 with 16.)
  auto rows_by = [&](auto nr) {
    constexpr int NR = decltype(nr)::value;
    if (a.slots <= 1)
      rows_of(nr, std::integral_constant<int, 1>{});
    else if (a.slots <= 2)
      rows_of(nr, std::integral_constant<int, 2>{});
    else if (a.slots <= 4)
      rows_of(nr, std::integral_constant<int, 4>{});
    else if (NR == 4 || a.slots <= 8)
      rows_of(nr, std::integral_constant<int, 8>{});
    else
      rows_of(nr, std::integral_constant<int, 16>{});
  };
  if (mend <= RPP)
    rows_by(std::integral_constant<int, 1>{});
  else if (mend <= 2 * RPP)
    rows_by(std::integral_constant<int, 2>{});
  else
    rows_by(std::integral_constant<int, 4>{});
}

// Merges the partials of each query row where there are no own keys.  A thread
// takes four channels of every SG-th partial of a row; the SG threads of a row's
// channels meet in LDS.  Bound by the latency of the loads with few rows, by the
// partials' bytes with many (8192 rows of four ranges: 7.0 us, 2.4 TB/s with the
// launch).
template <typename T, int D, int SG>
__global__ __launch_bounds__(kBlock) void prefix_merge_kernel(PrefixArgs a, long nrows) {
  constexpr int C4 = D / 4, RPB = kBlock / (C4 * SG);
  const int c = threadIdx.x % C4, sg = threadIdx.x / C4 % SG;
  const long row = (long)blockIdx.x * RPB + threadIdx.x / (C4 * SG);
  const long one[1] = {min(row, nrows - 1)};
  Merge4 gs[1];
  merge_partials<D, 1, 8>(a, one, c, sg, SG, gs);
  Merge4& g = gs[0];
  if constexpr (SG > 1) {
    __shared__ float sh[kBlock][7];  // (odd stride: no bank met twice)
    float* mine = sh[threadIdx.x];
    mine[0] = g.M;
    mine[1] = g.z;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[2 + e] = g.o[e];
    __syncthreads();
    if (sg != 0) return;  // no barrier follows
#pragma unroll
    for (int k = 1; k < SG; ++k) {
      const float* x = sh[threadIdx.x + k * C4];
      g.add(x[0], x[1], f32x4{x[2], x[3], x[4], x[5]});
    }
  }
  if (row < nrows)
    g.finish(static_cast<T*>(a.O) + row * D + 4 * c, a.lse ? a.lse + row : nullptr, c == 0);
}

// ------------------------------------------------------------ host side

PrefixPlan plan_prefix(const wf_prefix_params& p, size_t have) {
  PrefixPlan l{};
  const bool bf = p.dtype == WF_BF16;
  const int D = p.head_dim;
  const long R = (long)p.group * p.q_len, M = R * p.share, U = (long)p.prefixes * p.heads;
  const long rows = M * U, cus = device_cu_count();
  const int mb = kTileRows * D * (bf ? 2 : 4);  // bytes of a K (or V) tile
  const int slots = 8 * mb > 131072 ? 2 : 4;
  if (p.prefix_rows > 0) {
    // A workgroup's waves are over query rows (two at least, more as far as there
    // are any) and over the keys of a tile.  64 rows per wave halve the LDS reads of
    // 32, where the loop pipelines itself.  Fewer rows per workgroup give as many
    // workgroups with fewer ranges of the keys, and so fewer partials.  The cost of
    // a choice in us, fitted to measured times: whole rounds of workgroups, each
    // with a fixed part (its first loads, its outputs) and its tiles, and a write
    // and a read of D floats a row and range at 5 TB/s.  A tile costs its products
    // (`block` for each 32 keys of a wave at 128 channels, `fixed` once) or its
    // bytes, which come at 8 TB/s to all CUs (in part from the Infinity Cache) and
    // at 32 GB/s to one.  E.g. 128 rows over 16K keys of 32 heads take 69.5 us in
    // ranges for all CUs and 76 in fewer; 256 rows of two heads over 4K keys 17.6 in
    // blocks of 128 rows and 24 in one of 256, of 32 heads over 16K 89 in one of 256
    // and 98 in two.
    const bool quant = p.format != WF_CACHE_PLAIN;
    l.nw = bf && quant ? 8 : 4;
    const long KT = l.nw == 8 ? 2 * kTileRows : kTileRows;
    const long tiles = (p.prefix_rows + KT - 1) / KT;
    const double row_bytes = quant ? D * (p.format == WF_CACHE_E4M3 ? 1.0 : 0.5) + D / 32
                                   : D * (bf ? 2.0 : 4.0);
    const double partial = (double)rows * D * 8 / 5e6;
    // Ranges are as many as the workspace holds partials for, and one at least:
    // they need not grow with the rows (2304 rows of the prefix may take fewer than
    // 2048), and a caller keeps one workspace while its prompts and batches change.
    const long most = (long)std::min<size_t>(have / (rows * (D + 2) * sizeof(float)), 1L << 30);
    double least = 0;
    auto consider = [&](int qw, int qwaves, double block, double fixed) {
      const long mblocks = (M + 32 * qw * qwaves - 1) / (32 * qw * qwaves);
      const int kw = l.nw / qwaves;
      const double products = (double)(KT / 32) / kw * D / 128.0 * block + fixed;
      const long one = std::max(1L, cus / (U * mblocks));  // ranges that fill the chip once
      auto ranges = [&](long n) {
        const long per = (tiles + n - 1) / n, s = (tiles + per - 1) / per;
        if (s > 1 && s > most) return;
        const double groups = (double)(U * mblocks * s), at_once = std::min(groups, (double)cus);
        const double bytes = 2 * KT * row_bytes * std::max(at_once / mblocks / 8e6, 1 / 32e3);
        const double cost = std::ceil(groups / cus) * (per * std::max(products, bytes) + 5.0) +
                            (s > 1 || p.tail_cap > 0 ? s * partial : 0.0);
        if (least != 0 && cost >= least) return;
        least = cost;
        l.qw = qw;
        l.kw = kw;
        l.mblocks = (int)mblocks;
        l.rps = (int)(per * KT);
      };
      for (long n = 1; n < std::min(one, tiles); n += 1 + n / 16) ranges(n);
      ranges(std::min(one, tiles));
      ranges(std::min(2 * one, tiles));
    };
    for (int qwaves = 2; qwaves <= l.nw && (qwaves == 2 || 16 * qwaves < M); qwaves *= 2)
      if (!bf)
        consider(1, qwaves, 4.2, quant ? 0.4 : 0.1);
      else if (quant)
        consider(1, qwaves, 0.875, 0.7);
      else
        consider(1, qwaves, 0.45, 0.1);
    if (bf && !quant && M > 128) consider(2, l.nw, 0.82, 0.1);
    l.splits = (int)((p.prefix_rows + l.rps - 1) / l.rps);
    l.items = U * l.mblocks * l.splits;
    const size_t out = (size_t)l.nw * 32 * l.qw * (D + 6) * sizeof(float);
    l.lds_bytes = std::max((size_t)slots * 2 * mb, out);
    l.ids_bytes = (size_t)slots * 2 * mb + std::min(l.rps, kPrefixIds) * sizeof(int32_t);
  }
  if (p.tail_cap > 0) {
    // 32 rows per wave; a workgroup takes up to 128 of a sequence's rows, fewer
    // where that leaves CUs without one.  Below 32 rows the workgroups of a block
    // compute the same scores, and share the partials of its rows: worth it while
    // those are more bytes than the own keys, down to a row for each group of
    // threads that reads them, or where a thread has them in flight at once anyway
    // (two heads, four sequences of 32 rows over 16K keys: 7.4 us, and 32 with 32
    // rows each).
    const long units = U * p.share, blocks = (R + 31) / 32;
    l.tqw = (int)std::min(4L, blocks);
    if (l.tqw == 3) l.tqw = 4;
    while (l.tqw > 1 && units * ((blocks + l.tqw - 1) / l.tqw) < cus) l.tqw /= 2;
    l.tkw = l.tqw == 4 ? 1 : 2;
    l.trows = l.tqw == 1 ? (int)std::min(32L, R) : 32 * l.tqw;
    const int groups = 4 * kOwnWaves * kWave / D;
    while (l.tqw == 1 && l.trows > 1 && units * ((R + l.trows - 1) / l.trows) < cus &&
           (l.trows > groups || l.splits > 16) &&
           l.trows * l.splits * 4L > 2L * p.tail_cap * (bf ? 2 : 4))
      l.trows = (l.trows + 1) / 2;
    l.tmblocks = (int)((R + l.trows - 1) / l.trows);
    l.titems = units * l.tmblocks;
    l.tlds_bytes = std::max((size_t)4 * mb, (size_t)kOwnWaves * 32 * (D + 6) * sizeof(float));
  }
  l.slots = l.splits;
  if (l.splits > 1 || (l.splits == 1 && l.titems > 0)) {
    l.part_bytes = (size_t)rows * l.slots * D * sizeof(float);
    l.pstat_bytes = (size_t)rows * l.slots * 2 * sizeof(float);
  }
  return l;
}

template <typename Kernel>
static hipError_t launch_lds(Kernel kern, long grid, int waves, size_t lds, const PrefixArgs& a,
                             hipStream_t s) {
  if (lds > 65536) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * waves), lds, s, a);
  return hipGetLastError();
}

template <typename T, int D>
static hipError_t merge_launch(const PrefixArgs& a, long rows, hipStream_t s) {
  // threads per row and channels: as many as have every partial of a row in flight
  // (32 rows, 1, 4 and 8 threads: 8 ranges 2.8, 3.6, 3.8 us; 16 ranges 3.8, 3.4, 3.8;
  // 32 ranges 5.6, 3.6, 3.8; 128 ranges and 8 rows 17.5, 5.7, 4.7)
  auto go = [&](auto n) {
    constexpr int SG = decltype(n)::value;
    constexpr int RPB = kBlock / (D / 4 * SG);
    hipLaunchKernelGGL((prefix_merge_kernel<T, D, SG>), dim3((unsigned)((rows + RPB - 1) / RPB)),
                       dim3(kBlock), 0, s, a, rows);
  };
  if (a.slots <= 8)
    go(std::integral_constant<int, 1>{});
  else if (a.slots <= 32)
    go(std::integral_constant<int, 4>{});
  else
    go(std::integral_constant<int, 8>{});
  return hipGetLastError();
}

hipError_t launch_prefix(const wf_prefix_params& p, const PrefixPlan& l, PrefixArgs& a,
                         hipStream_t s) {
  a.heads = p.heads;
  a.share = p.share;
  a.R = p.group * p.q_len;
  a.by_R = FastDiv::by(a.R);
  a.cap = p.prefix_cap;
  a.rows = p.prefix_rows;
  a.T = p.tail_cap;
  a.slots = l.slots;
  a.whole = l.part_bytes == 0;
  a.scale = p.scale != 0.f ? p.scale : (float)(1.0 / std::sqrt((double)p.head_dim));
  const int M = a.R * p.share;
  if (l.items > 0)
    a.p = PrefixPart{(int)l.items, l.splits, l.rps, l.mblocks, l.nw / l.kw * 32 * l.qw, M, l.kw};
  a.t = OwnPart{l.tmblocks, l.trows, l.tkw, l.tqw};
  auto run = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    if (l.items > 0) {
      const long grid = (l.items + 7) & ~7L;
      const size_t lds = a.list ? std::max(l.lds_bytes, l.ids_bytes) : l.lds_bytes;
      auto go = [&](auto f) {
        constexpr int F = decltype(f)::value;
        if constexpr (sizeof(T) == 2 && F == WF_CACHE_PLAIN)
          if (l.qw == 2) return launch_lds(prefix_attn_kernel<T, D, F, 2>, grid, l.nw, lds, a, s);
        return launch_lds(prefix_attn_kernel<T, D, F, 1>, grid, l.nw, lds, a, s);
      };
      const hipError_t e =
          p.format == WF_CACHE_E4M3   ? go(std::integral_constant<int, WF_CACHE_E4M3>{})
          : p.format == WF_CACHE_E2M1 ? go(std::integral_constant<int, WF_CACHE_E2M1>{})
                                      : go(std::integral_constant<int, WF_CACHE_PLAIN>{});
      if (e != hipSuccess) return e;
    }
    if (l.titems > 0)
      return launch_lds(prefix_own_kernel<T, D>, l.titems, kOwnWaves, l.tlds_bytes, a, s);
    if (!a.whole)
      return merge_launch<T, D>(a, (long)p.prefixes * p.share * p.heads * a.R, s);
    return hipSuccess;
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (p.dtype == WF_BF16)
    return p.head_dim == 128 ? run(bf16_t{}, D128{}) : run(bf16_t{}, D64{});
  return p.head_dim == 128 ? run(float{}, D128{}) : run(float{}, D64{});
}

hipError_t load_prefix_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(
      &fa, reinterpret_cast<const void*>(prefix_attn_kernel<bf16_t, 128, WF_CACHE_PLAIN, 1>));
}

}  // namespace wf
