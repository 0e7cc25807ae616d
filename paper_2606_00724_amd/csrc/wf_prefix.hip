// Attention of a batch whose sequences share a prefix (wf_prefix_attn).
//
// For a K/V head of a prefix, the query rows of all its sequences and of the
// head's group are one block of M = share * group * q_len rows that sees the
// same keys: the prefix is read once for all of them.  A sequence's own rows
// are a second, shorter key range of its R = group * q_len rows.  A workgroup
// takes a block of query rows and a range of keys of either kind and leaves an
// unnormalised output with the rows' reference (log2 units) and sum of
// weights; a second kernel merges a row's partials (none is needed where it
// has one).
//
// S^T = K Q^T on 32 x 32 products: a lane then holds 16 scores of one query
// row, so that the softmax needs no lane exchange except one of the maximum
// with the lane of the other 16, and its weights are in place as the B operand
// of O^T = V^T P^T (the order of the keys inside that product is free, and V^T
// is read from LDS in the order of the scores).
#include "wf_cache.hpp"
#include "wf_kernels.hpp"
#include "wf_launch.hpp"

namespace wf {

constexpr int kPrefixBlock = 256;
constexpr int kPrefixWaves = kPrefixBlock / kWave;
constexpr int kPrefixIds = 4096;  // row ids in LDS at once (whole tiles)

typedef short v4i16p __attribute__((ext_vector_type(4)));

// keys per LDS tile
template <typename T>
constexpr int kTile = sizeof(T) == 2 ? 128 : 64;

// Granules (16 bytes) of a row are stored in slot k ^ tile_swz(r) so that no
// LDS read below meets a bank twice: 16 rows at one granule (K), four rows of
// 64 bytes (bf16 V, transposed reads), and rows r and r + 4 of 128 bytes (fp32
// V) lie on different banks.
template <typename T, int G>
__device__ __forceinline__ int tile_swz(int r) {
  if constexpr (sizeof(T) == 4) return ((r & 4) << 1) | ((r & 3) << 1) | ((r >> 3) & 1);
  if constexpr (G == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
  return ((r & 2) << 1) | ((r >> 2) & 3);  // 128-byte rows
}
template <typename T, int G>
__device__ __forceinline__ int tile_offset(int r, int k) {
  return r * (16 * G) + 16 * (k ^ tile_swz<T, G>(r));
}

// The rows of a workgroup's key range: row i of tile t is key k0 + t * tile +
// i, at most its last one.
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

template <typename T, int D, int FMT, int QW>
struct PrefixWave {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int ES = sizeof(T), EPV = 16 / ES;
  static constexpr int G = D / EPV;              // granules per row
  static constexpr int KT = kTile<T>;
  static constexpr int MB = KT * D * ES;         // bytes of a K (or V) tile
  static constexpr int QS = BF ? D / 16 : D / 8; // 16-byte query operands per lane
  static constexpr int DT = D / 32;              // 32-channel output tiles

  u32x4 q[QW][QS];
  f32x16 O[QW][DT];
  float mref[QW], l[QW];
  float nref[QW];  // -mref, 0 while that is -inf
  bool neg;  // a negative scale: the scores change sign (and c2 is positive)

  // LDS byte offsets of the lane's operands in a 32-row block (the swizzle goes
  // by the row mod 16, so one offset serves all blocks).  The granules of a row
  // differ in bits that the swizzle is XORed into, so that those of the other
  // operands are this one's XOR a constant.
  uint32_t ko, vo;
  __device__ __forceinline__ void offsets() {
    const int lane = threadIdx.x & 63, h = lane >> 5, i16 = lane & 15;
    ko = tile_offset<T, G>(lane & 31, h);
    // in each 16-lane group lane i points at row t0 + i / 4, channels c0 + 4 (i %
    // 4) .. + 3, and receives rows t0 .. t0 + 3 of channel c0 + i
    const int t0 = 4 * h + (i16 >> 2), c0 = (lane & 16) + 4 * (i16 & 3);
    vo = tile_offset<T, G>(t0, c0 >> 3) + 2 * (c0 & 7);
  }

  // The lane's operand j of K in the block at LDS offset `at`: 16 bytes of its
  // row, granule 2 j + h.
  __device__ __forceinline__ u32x4 key(uint32_t at, int j) const {
    return *(const __attribute__((address_space(3))) u32x4*)(size_t)((at + ko) ^ (32u * j));
  }
  __device__ __forceinline__ void keys(uint32_t at, u32x4 (&kf)[QS]) const {
#pragma unroll
    for (int j = 0; j < QS; ++j) kf[j] = key(at, j);
  }
  // Half of the lane's operand of V^T of 16 of the block's rows (bf16): rows 16
  // kb + 8 k + 4 h .. + 3 of channel 32 d + l % 32.  (Eight rows on, the swizzle
  // flips a granule's bit 1.)
  __device__ __forceinline__ u32x2 val(uint32_t at, int kb, int d, int k) const {
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) v4i16p*)(size_t)(
                       ((at + vo) ^ (64u * d + 32u * k)) + (2 * kb + k) * 128 * G)));
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
  __device__ __forceinline__ static void maxima(const f32x16 (&s)[QW], float (&mx)[QW]) {
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      float m = fmaxf(s[b][0], s[b][1]);
#pragma unroll
      for (int i = 2; i < 16; i += 2) m = fmaxf(m, fmaxf(s[b][i], s[b][i + 1]));
      mx[b] = m;
    }
  }
  // The reference moves only when a score passes it by 2^8: weights then stay
  // below 2^8, their sums far from the fp32 range, and a rescale of the outputs
  // is rare.
  __device__ __forceinline__ void raise(const float (&mx)[QW], float c2) {
    bool grow = false;
#pragma unroll
    for (int b = 0; b < QW; ++b) grow |= mx[b] * c2 > mref[b] + 8.f;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        const float mn = fmaxf(mref[b], fmaxf(mx[b], partner32(mx[b])) * c2);
        const float al = mref[b] > -INFINITY ? __builtin_amdgcn_exp2f(mref[b] - mn) : 0.f;
        mref[b] = mn;
        nref[b] = mn > -INFINITY ? -mn : 0.f;
        l[b] *= al;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[b][d][i] *= al;
      }
    }
  }
  // Weights of keys i0 .. i0 + 7 of the lane's, and their sum into l.  (The
  // unrounded product less the reference: scores of thousands keep their
  // differences.  While every score so far is -inf, their weights are 2^-inf =
  // 0.)
  __device__ __forceinline__ void weights(f32x16 (&s)[QW], int i0, float c2) {
#pragma unroll
    for (int b = 0; b < QW; ++b) {
#pragma unroll
      for (int i = i0; i < i0 + 8; ++i)
        s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c2, nref[b]));
      l[b] += ((s[b][i0] + s[b][i0 + 1]) + (s[b][i0 + 2] + s[b][i0 + 3])) +
              ((s[b][i0 + 4] + s[b][i0 + 5]) + (s[b][i0 + 6] + s[b][i0 + 7]));
    }
  }
  // O^T += V^T P^T over 16 keys (bf16: the weights rounded to half a step of
  // bf16, as the products' operands are)
  __device__ __forceinline__ void add16(const f32x16 (&s)[QW], int kb, const u32x4 (&vf)[DT]) {
    u32x4 pf[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b)
      pf[b] = u32x4{pack_bf16x2(s[b][8 * kb], s[b][8 * kb + 1]),
                    pack_bf16x2(s[b][8 * kb + 2], s[b][8 * kb + 3]),
                    pack_bf16x2(s[b][8 * kb + 4], s[b][8 * kb + 5]),
                    pack_bf16x2(s[b][8 * kb + 6], s[b][8 * kb + 7])};
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int b = 0; b < QW; ++b)
        O[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[d]),
                                                          __builtin_bit_cast(bf16x8, pf[b]),
                                                          O[b][d], 0, 0, 0);
  }
  // the same over the block's 32 keys in fp32
  __device__ __forceinline__ void add32(const f32x16 (&s)[QW], const unsigned char* Vb, int sb) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = sb + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int c = 32 * d + (lane & 31);
        const float vf =
            *reinterpret_cast<const float*>(Vb + tile_offset<T, G>(r, c >> 2) + 4 * (c & 3));
#pragma unroll
        for (int b = 0; b < QW; ++b)
          O[b][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[b][i], O[b][d], 0, 0, 0);
      }
    }
  }

  // 32 keys (rows sb .. sb + 31 of the tile, nr of the tile's rows valid)
  __device__ __forceinline__ void step(const unsigned char* Kb, const unsigned char* Vb, int sb,
                                       int nr, float c2) {
    const uint32_t kat = lds_offset(Kb) + sb * 16 * G, vat = lds_offset(Vb) + sb * 16 * G;
    const int h = (threadIdx.x & 63) >> 5;
    u32x4 kf[QS];
    f32x16 s[QW];
    float mx[QW];
    keys(kat, kf);
    scores(kf, s);
    if (neg) {
#pragma unroll
      for (int b = 0; b < QW; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = -s[b][i];
    }
    if (sb + 32 > nr) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool off = sb + 8 * (i >> 2) + 4 * h + (i & 3) >= nr;
#pragma unroll
        for (int b = 0; b < QW; ++b) s[b][i] = off ? -INFINITY : s[b][i];
      }
    }
    maxima(s, mx);
    raise(mx, c2);
    weights(s, 0, c2);
    weights(s, 8, c2);
    if constexpr (BF) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        u32x4 vf[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const u32x2 lo = val(vat, kb, d, 0), hi = val(vat, kb, d, 1);
          vf[d] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
        add16(s, kb, vf);
      }
    } else {
      add32(s, Vb, sb);
    }
  }

  // The pipelined loop (bf16) keeps the next block's scores in log2 units less
  // the reference, t = s c2 - mref, and their maximum mx.  Before the block's
  // weights are taken the reference is raised where t passes it (see raise).
  float limit[QW];  // 8; -inf while the reference is -inf
  __device__ __forceinline__ void raise_shifted(f32x16 (&t)[QW], const float (&mx)[QW]) {
    bool grow = false;
#pragma unroll
    for (int b = 0; b < QW; ++b) grow |= mx[b] > limit[b];
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        const float up = fmaxf(mx[b], partner32(mx[b]));
        const bool first = mref[b] == -INFINITY;
        const float mn = first ? up : fmaxf(mref[b], mref[b] + up);
        const float by = mn > -INFINITY ? mn + nref[b] : 0.f;  // (nref: 0 or -mref)
        const float al = first ? 0.f : __builtin_amdgcn_exp2f(-by);
        mref[b] = mn;
        nref[b] = mn > -INFINITY ? -mn : 0.f;
        limit[b] = mn > -INFINITY ? 8.f : -INFINITY;
        l[b] *= al;
#pragma unroll
        for (int i = 0; i < 16; ++i) t[b][i] -= by;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[b][d][i] *= al;
      }
    }
  }
  __device__ __forceinline__ void shift(f32x16 (&t)[QW], float (&mx)[QW], float c2) const {
#pragma unroll
    for (int b = 0; b < QW; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) t[b][i] = fmaf(t[b][i], c2, nref[b]);
      mx[b] = fmaxf(t[b][0], t[b][1]);
#pragma unroll
      for (int i = 2; i < 16; i += 2) mx[b] = fmaxf(mx[b], fmaxf(t[b][i], t[b][i + 1]));
    }
  }

  // A block of that loop: weights of one block (shifted scores s) and their
  // product with V (at LDS offset vat) beside the scores sn of the next block
  // (its keys kf in registers; refilled with those at knext).  A wave issues in
  // order and waits for the matrix pipe at its next product, so only what stands
  // between two products runs beside them: every product (32 cycles) is followed
  // by its share of the vector work, four to six instructions, and the barriers
  // hold that order.
  __device__ __forceinline__ void block(uint32_t vat, uint32_t knext, u32x4 (&kf)[QS],
                                        f32x16 (&s)[QW], f32x16 (&sn)[QW], float (&mx)[QW],
                                        float c2) {
    raise_shifted(s, mx);
    float z[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b) z[b] = 0.f;
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
      const u32x2 y = val(vat, kb, d, k);
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
#pragma unroll
      for (int e = n * 8 * QW / NQ; e < (n + 1) * 8 * QW / NQ; ++e) weight(0, e);
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
      for (int j = n * QS / NV; j < (n + 1) * QS / NV; ++j) kf[j] = key(knext, j);
#pragma unroll
      for (int e = n * 8 * QW / NV; e < (n + 1) * 8 * QW / NV; ++e) {
        const int g = e >> 3, i = 2 * (e & 7);
        sn[g][i] = fmaf(sn[g][i], c2, nref[g]);
        sn[g][i + 1] = fmaf(sn[g][i + 1], c2, nref[g]);
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

// 16 bytes per lane from base + off straight to LDS (lane l's at `lds` + 16 l).
// Waited for as async_load16's.
__device__ __forceinline__ void tile_load(const void* base, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(off), "s"(base), "s"(lds)
      : "memory", "m0");
}

template <typename T>
__device__ __forceinline__ void put4(T* p, float a, float b, float c, float d);
template <>
__device__ __forceinline__ void put4<bf16_t>(bf16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
}
template <>
__device__ __forceinline__ void put4<float>(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
}

// One row of a cache as a thread stages it: 16 codes (E4M3) or 32 (E2M1) in
// 16 bytes, and their block's exponent byte.
template <typename T, int D, int FMT>
struct QuantStage {
  static constexpr int CPP = FMT == WF_CACHE_E2M1 ? 32 : 16;  // channels per piece
  static constexpr int PPR = D / CPP;                         // pieces per row
  static constexpr int PT = kTile<T> * PPR;                   // pieces of a tile and matrix
  static constexpr int N = (PT + kPrefixBlock - 1) / kPrefixBlock;  // per thread
  static constexpr int G = D * (int)sizeof(T) / 16;
  u32x4 w[2][N];
  uint32_t x[2][N];

  __device__ __forceinline__ void load(const PrefixArgs& a, const KeyRows& rows, long unit,
                                       int t0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = i * kPrefixBlock + threadIdx.x, pc = p % PPR;
      if (PT % kPrefixBlock != 0 && p >= PT) break;
      const long row = unit * a.cap + rows(t0 + p / PPR);
      w[0][i] = reinterpret_cast<const u32x4*>(a.K)[row * PPR + pc];
      w[1][i] = reinterpret_cast<const u32x4*>(a.V)[row * PPR + pc];
      x[0][i] = a.Kx[row * (D / 32) + pc * CPP / 32];
      x[1][i] = a.Vx[row * (D / 32) + pc * CPP / 32];
    }
  }
  __device__ __forceinline__ void commit(unsigned char* Kb, unsigned char* Vb) const {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int p = i * kPrefixBlock + threadIdx.x, r = p / PPR, pc = p % PPR;
        if (PT % kPrefixBlock != 0 && p >= PT) break;
        const float s = block_scale(x[m][i]);
        unsigned char* dst = m ? Vb : Kb;
        if constexpr (sizeof(T) == 2) {
          // v_cvt_scalef32_pk_bf16: two codes times the power of two, rounded to
          // nearest even (equal to decode8 and pack_bf16x2 for every code and
          // exponent byte 1 .. 255; byte 0 means 0 and not 2^-127)
          const u32x4 c = x[m][i] ? w[m][i] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
          for (int k = 0; k < CPP / 8; ++k) {  // eight channels, one granule each
            u32x4 g;
            if constexpr (FMT == WF_CACHE_E4M3) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                g[2 * e] = __builtin_bit_cast(
                    uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * k + e], s, false));
                g[2 * e + 1] = __builtin_bit_cast(
                    uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * k + e], s, true));
              }
            } else {
              g[0] = __builtin_bit_cast(uint32_t,
                                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 0));
              g[1] = __builtin_bit_cast(uint32_t,
                                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 1));
              g[2] = __builtin_bit_cast(uint32_t,
                                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 2));
              g[3] = __builtin_bit_cast(uint32_t,
                                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[k], s, 3));
            }
            *reinterpret_cast<u32x4*>(dst + tile_offset<T, G>(r, pc * (CPP / 8) + k)) = g;
          }
        } else {
#pragma unroll
          for (int k = 0; k < CPP / 8; ++k) {  // eight channels, two granules each
            float v[8];
            const u32x2 c = FMT == WF_CACHE_E4M3 ? u32x2{w[m][i][2 * k % 4], w[m][i][(2 * k + 1) % 4]}
                                                 : u32x2{w[m][i][k], 0u};
            decode8<FMT>(c, s, v);
            const int g = 2 * (pc * (CPP / 8) + k);
            *reinterpret_cast<f32x4*>(dst + tile_offset<T, G>(r, g)) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(dst + tile_offset<T, G>(r, g + 1)) =
                f32x4{v[4], v[5], v[6], v[7]};
          }
        }
      }
  }
};

template <typename T, int D, int FMT, int QW>
__global__ __launch_bounds__(kPrefixBlock, 1) void prefix_attn_kernel(PrefixArgs a) {
  using W = PrefixWave<T, D, FMT, QW>;
  constexpr int KT = W::KT, G = W::G, MB = W::MB, DT = W::DT, QS = W::QS;
  extern __shared__ __align__(16) unsigned char smem[];  // [2][K, V] tiles, then row ids
  int32_t* ids = reinterpret_cast<int32_t*>(smem + 4 * MB);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;

  // The workgroup's item.  Prefix items first, their blocks of query rows
  // innermost, so that those reading the same keys run at once on one XCD.
  const int np8 = (a.p.items + 7) & ~7;  // (the grid holds whole eights of them)
  const bool own = (int)blockIdx.x >= np8;
  const int item = own ? (int)blockIdx.x - np8 : xcd_swizzle(blockIdx.x, np8);
  if (item >= (own ? a.t.items : a.p.items)) return;
  const int mblocks = own ? a.t.mblocks : a.p.mblocks;
  const int splits = own ? a.t.splits : a.p.splits;
  const int rps = own ? a.t.rps : a.p.rps;
  const int M = own ? a.t.M : a.p.M;
  const int KW = own ? a.t.kw : a.p.kw;
  const int mb = item % mblocks, sp = item / mblocks % splits;
  const int unit = item / (mblocks * splits);  // (prefix or sequence, head)
  const int group = unit / a.heads, head = unit % a.heads;
  const int slot = own ? a.p.splits + sp : sp;
  int len = own ? a.T : a.rows;
  if (own ? a.tlen != nullptr : a.plen != nullptr)
    len = min(max((own ? a.tlen : a.plen)[group], 0), len);
  const int k0 = sp * rps, nk = min(rps, len - k0);  // the range's keys (none: nk <= 0)

  const int kw = wave % KW, qw = wave / KW;
  const int m0 = (mb * (kPrefixWaves / KW) + qw) * 32 * QW;
  // query row m of the unit -> row of Q, O
  auto row_of = [&](int m) {
    const int n = own ? group : group * a.share + m / a.R;
    return ((long)n * a.heads + head) * a.R + (own ? m : m % a.R);
  };
  W w;
  w.offsets();
  const float c2 = fabsf(a.scale) * kLog2e;
  w.neg = a.scale < 0.f;
#pragma unroll
  for (int b = 0; b < QW; ++b) {
    const T* src = reinterpret_cast<const T*>(a.Q) + row_of(min(m0 + 32 * b + l32, M - 1)) * D;
#pragma unroll
    for (int j = 0; j < QS; ++j)
      w.q[b][j] = reinterpret_cast<const u32x4*>(src)[2 * j + h];
    w.mref[b] = -INFINITY;
    w.limit[b] = -INFINITY;
    w.nref[b] = w.l[b] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.O[b][d][i] = 0.f;
  }
  const bool active = m0 < M;

  if (nk > 0) {
    const int nt = (nk + KT - 1) / KT;
    KeyRows rows;
    rows.ids = !own && a.list ? ids : nullptr;
    rows.cap = own ? a.T : a.cap;
    rows.k0 = k0;
    rows.last = k0 + nk - 1;
    rows.id0 = k0;
    // the next kPrefixIds ids of a list, from tile t on, when tile t starts them
    // (no wave reads older ones: tile t - 1 has been queued by all)
    auto stage_ids = [&](int t) __attribute__((always_inline)) {
      if (!rows.ids || t * KT % kPrefixIds != 0) return;  // uniform
      rows.id0 = k0 + t * KT;
      lds_barrier();
      for (int i = threadIdx.x; i < min(kPrefixIds, nk - t * KT); i += kPrefixBlock)
        ids[i] = a.list[(long)unit * a.rows + rows.id0 + i];
      __syncthreads();
    };
    // The query operands, loaded above: here, so that the compiler's wait for them
    // is no wait for a tile later on.  Those of 64 rows of 128 channels are put
    // into the accumulation half of the registers, from where the products take
    // them: in the other half they were copied there and back in every block.
    auto queries = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
      if constexpr (W::BF && QW * QS >= 16) {
#pragma unroll
        for (int b = 0; b < QW; ++b)
#pragma unroll
          for (int j = 0; j < QS; ++j) asm volatile("" : "+a"(w.q[b][j]));
      }
    };
    // The tiles in turn, through two LDS slots.  arrive(t): tile t is in its slot
    // for every wave; leave(t): no wave reads tile t any more.
    auto run = [&](auto&& arrive, auto&& leave) __attribute__((always_inline)) {
      // whole tiles in the pipelined loop (bf16)
      const int nf = !W::BF || w.neg ? 0 : nk / KT;
      auto slot_of = [&](int t) { return smem + (t & 1) * 2 * MB; };
      arrive(0);
      if constexpr (W::BF) {
        if (nf > 0) {
          const int nb = KT / 32 / KW;  // blocks of a tile that are the wave's
          // LDS offset of the wave's i-th block in tile t
          const uint32_t lds0 = lds_offset(smem) + kw * 512 * G;
          const int stride = KW * 512 * G;
          auto at = [&](int t, int i) { return lds0 + (t & 1) * 2 * MB + i * stride; };
          u32x4 kf[QS];
          f32x16 s0[QW], s1[QW];
          float mx[QW];
          w.keys(at(0, 0), kf);
          w.scores(kf, s0);
          w.shift(s0, mx, c2);
          if (nb > 1) w.keys(at(0, 1), kf);
          const int n = nf * nb;
          int t = 0, i = 0;
          auto one = [&](f32x16(&s)[QW], f32x16(&sn)[QW]) __attribute__((always_inline)) {
            const bool last = i == nb - 1;
            if (last && t + 1 < nt) {
              arrive(t + 1);
              w.keys(at(t + 1, 0), kf);  // (a partial tile's: not used)
            }
            // the keys after next, where they are in the next block's tile
            const bool two = last ? nb > 1 && t + 1 < nt : i + 2 < nb;
            const uint32_t next = last ? at(t + two, two) : at(t, two ? i + 2 : i);
            // (also for query rows past the last: they repeat it)
            w.block(at(t, i) + MB, next, kf, s, sn, mx, c2);
            if (last) leave(t);
            t += last ? 1 : 0;
            i = last ? 0 : i + 1;
          };
          for (int j = 0; j < n; j += 2) {
            one(s0, s1);
            if (j + 1 < n) one(s1, s0);
          }
        }
      }
      for (int t = nf; t < nt; ++t) {
        if (t > nf) arrive(t);
        const int nr = min(KT, nk - t * KT);
        unsigned char* Vb = slot_of(t) + MB;
        if (nr < KT) {  // rows past the range repeat its last one: 0 there, as 0
                        // times an infinite value is NaN
          for (int i = nr * G + threadIdx.x; i < KT * G; i += kPrefixBlock)
            reinterpret_cast<u32x4*>(Vb)[i] = u32x4{0u, 0u, 0u, 0u};
          lds_barrier();
        }
        if (active)
          for (int sb = 32 * kw; sb < nr; sb += 32 * KW) w.step(slot_of(t), Vb, sb, nr, c2);
        leave(t);
      }
    };
    if (FMT == WF_CACHE_PLAIN || own) {
      // direct loads to LDS, up to two tiles ahead
      const T* Kg = reinterpret_cast<const T*>(own ? a.Kt : a.K) + (long)unit * rows.cap * D;
      const T* Vg = reinterpret_cast<const T*>(own ? a.Vt : a.V) + (long)unit * rows.cap * D;
      constexpr int IPW = KT * G / (64 * kPrefixWaves);  // loads per wave and matrix
      constexpr int RPI = 64 / G;
      constexpr int RB = D * W::ES;                      // bytes of a row
      const uint32_t lds0 = lds_offset(smem) + 1024u * IPW * wave;
      // byte offsets of the lane's loads in a tile of consecutive rows
      uint32_t off[IPW];
#pragma unroll
      for (int i = 0; i < IPW; ++i) {
        const int r = (wave * IPW + i) * RPI + lane / G;
        off[i] = r * RB + 16 * ((lane % G) ^ tile_swz<T, G>(r));
      }
      int issued = 0;  // tiles queued so far
      auto issue = [&](int t) __attribute__((always_inline)) {
        stage_ids(t);
        issued = t + 1;
        const uint32_t at = lds0 + (t & 1) * 2 * MB;
        if (!rows.ids && nk - t * KT >= KT) {  // uniform
          const T* kt = Kg + (long)(k0 + t * KT) * D;
          const T* vt = Vg + (long)(k0 + t * KT) * D;
#pragma unroll
          for (int i = 0; i < IPW; ++i) tile_load(kt, off[i], at + 1024u * i);
#pragma unroll
          for (int i = 0; i < IPW; ++i) tile_load(vt, off[i], at + MB + 1024u * i);
        } else {
#pragma unroll 1
          for (int i = 0; i < IPW; ++i) {
            const int r = (wave * IPW + i) * RPI + lane / G;
            const long o = rows(t * KT + r) * D + W::EPV * ((lane % G) ^ tile_swz<T, G>(r));
            async_load16<false>(Kg + o, __builtin_amdgcn_readfirstlane(at + 1024u * i));
            async_load16<false>(Vg + o, __builtin_amdgcn_readfirstlane(at + MB + 1024u * i));
          }
        }
      };
      issue(0);
      queries();
      if (nt > 1) issue(1);
      run(
          [&](int t) __attribute__((always_inline)) {
            // tile t + 1 may be in flight: it is queued when tile t - 1 is left,
            // after tile t arrives in the pipelined loop, before in the other
            wait_vmcnt_chunks<2 * IPW>(issued > t + 1 ? 1 : 0);
            lds_barrier();
          },
          [&](int t) __attribute__((always_inline)) {
            lds_barrier();
            if (t + 2 < nt) issue(t + 2);
          });
    } else {
      // codes are loaded to registers a tile ahead, and decoded into LDS
      if constexpr (FMT != WF_CACHE_PLAIN) {
        QuantStage<T, D, FMT> st;
        stage_ids(0);
        st.load(a, rows, unit, 0);
        queries();
        run(
            [&](int t) __attribute__((always_inline)) {
              unsigned char* Kb = smem + (t & 1) * 2 * MB;
              st.commit(Kb, Kb + MB);
              if (t + 1 < nt) {
                stage_ids(t + 1);
                st.load(a, rows, unit, (t + 1) * KT);
              }
              lds_barrier();
            },
            [&](int) __attribute__((always_inline)) { lds_barrier(); });
      }
    }
  }

  // merge the waves that took keys in turn: each adds up a share of the
  // channels (the tiles are idle: every wave passed the barrier after the loop)
#pragma unroll
  for (int b = 0; b < QW; ++b) w.l[b] += partner32(w.l[b]);
  constexpr int OW = QW * DT * 16 * 64;  // floats of a wave's output
  float* oo = reinterpret_cast<float*>(smem);
  float* sm = oo + kPrefixWaves * OW;    // [waves][QW][32] references, then sums
  float* sl = sm + kPrefixWaves * QW * 32;
  int dshare = DT, d0 = 0;               // the wave's output tiles
  if (KW > 1) {
    if (nk > 0 && active) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            oo[wave * OW + ((b * DT + d) * 16 + i) * 64 + lane] = w.O[b][d][i];
        if (h == 0) {
          sm[(wave * QW + b) * 32 + l32] = w.mref[b];
          sl[(wave * QW + b) * 32 + l32] = w.l[b];
        }
      }
    }
    lds_barrier();
    dshare = max(1, DT / KW);
    d0 = kw * dshare;
    if (nk > 0 && active) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        float M2 = -INFINITY, z = 0.f;
        for (int k = 0; k < KW; ++k) M2 = fmaxf(M2, sm[((wave - kw + k) * QW + b) * 32 + l32]);
        float acc[DT][16];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
        for (int k = 0; k < KW; ++k) {
          const int v = wave - kw + k;
          const float mk = sm[(v * QW + b) * 32 + l32];
          const float f = mk > -INFINITY ? __builtin_amdgcn_exp2f(mk - M2) : 0.f;
          z += f * sl[(v * QW + b) * 32 + l32];
#pragma unroll
          for (int d = 0; d < DT; ++d)
            if (d >= d0 && d < d0 + dshare)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                acc[d][i] += f * oo[v * OW + ((b * DT + d) * 16 + i) * 64 + lane];
        }
        w.mref[b] = M2;
        w.l[b] = z;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) w.O[b][d][i] = acc[d][i];
      }
    }
  }
  if (!active) return;
#pragma unroll
  for (int b = 0; b < QW; ++b) {
    const int m = m0 + 32 * b + l32;
    if (m >= M) continue;
    const long row = row_of(m);
    const float inv = w.l[b] == 0.f ? 0.f : 1.f / w.l[b];
    if (a.slots == 1) {
      T* dst = reinterpret_cast<T*>(a.O) + row * D;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        if (d >= d0 && d < d0 + dshare)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            put4<T>(dst + 32 * d + 2 * i + 4 * h, w.O[b][d][i] * inv, w.O[b][d][i + 1] * inv,
                    w.O[b][d][i + 2] * inv, w.O[b][d][i + 3] * inv);
      if (a.lse && kw == 0 && h == 0)
        a.lse[row] = w.l[b] == 0.f ? -INFINITY : (w.mref[b] + __log2f(w.l[b])) * kLn2;
    } else {
      float* dst = a.part + (row * a.slots + slot) * D;
      if (nk > 0) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
          if (d >= d0 && d < d0 + dshare)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              put4<float>(dst + 32 * d + 2 * i + 4 * h, w.O[b][d][i], w.O[b][d][i + 1],
                          w.O[b][d][i + 2], w.O[b][d][i + 3]);
      }
      if (kw == 0 && h == 0) {
        a.pstat[(row * a.slots + slot) * 2] = w.mref[b];
        a.pstat[(row * a.slots + slot) * 2 + 1] = w.l[b];
      }
    }
  }
}

// Merges the partials of each query row.  A thread takes eight channels of every
// SG-th partial of a row, four of them in flight; the SG threads of a row's
// channels meet in LDS.  (33 partials of 256 rows: 24 us with SG = 1.)
template <typename T, int SG>
__global__ __launch_bounds__(kBlock) void prefix_merge_kernel(PrefixArgs a, long rows, int D) {
  const int tpr = D / 8, rpb = kBlock / (tpr * SG);
  const int c = threadIdx.x % tpr, sg = threadIdx.x / tpr % SG, rl = threadIdx.x / (tpr * SG);
  const long row = (long)blockIdx.x * rpb + rl;
  float M = -INFINITY, z = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // one partial into the running ones; an empty range (-inf, 0) has no output
  auto add = [&](float m, float zs, const float* x) {
    if (m == -INFINITY && zs == 0.f) return;
    const float mn = fmaxf(M, m);
    // (all scores -inf or NaN: zs says it)
    const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
    const float g = M > -INFINITY ? __builtin_amdgcn_exp2f(M - mn) : 1.f;
    M = mn;
    z = z * g + f * zs;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * g + f * x[e];
  };
  if (row < rows) {
    const float* st = a.pstat + row * a.slots * 2;
    const float* src = a.part + row * a.slots * D + 8 * c;
    constexpr int F = 4;
    for (int s0 = sg; s0 < a.slots; s0 += F * SG) {
      float m[F], zs[F];
      f32x4 x[F][2];
#pragma unroll
      for (int k = 0; k < F; ++k) {
        const int s = min(s0 + k * SG, a.slots - 1);
        m[k] = s0 + k * SG < a.slots ? st[2 * s] : -INFINITY;
        zs[k] = s0 + k * SG < a.slots ? st[2 * s + 1] : 0.f;
        x[k][0] = reinterpret_cast<const f32x4*>(src + (long)s * D)[0];
        x[k][1] = reinterpret_cast<const f32x4*>(src + (long)s * D)[1];
      }
#pragma unroll
      for (int k = 0; k < F; ++k) {
        const float v[8] = {x[k][0][0], x[k][0][1], x[k][0][2], x[k][0][3],
                            x[k][1][0], x[k][1][1], x[k][1][2], x[k][1][3]};
        add(m[k], zs[k], v);
      }
    }
  }
  if constexpr (SG > 1) {
    __shared__ float sh[kBlock][11];  // (odd stride: no bank met twice)
    float* mine = sh[threadIdx.x];
    mine[0] = M;
    mine[1] = z;
#pragma unroll
    for (int e = 0; e < 8; ++e) mine[2 + e] = o[e];
    __syncthreads();
    if (sg != 0) return;  // no barrier follows
#pragma unroll
    for (int k = 1; k < SG; ++k) {
      const float* other = sh[threadIdx.x + k * tpr];
      add(other[0], other[1], other + 2);
    }
  }
  if (row >= rows) return;
  const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  T* dst = reinterpret_cast<T*>(a.O) + row * D + 8 * c;
  put4<T>(dst, o[0], o[1], o[2], o[3]);
  put4<T>(dst + 4, o[4], o[5], o[6], o[7]);
  if (a.lse && c == 0) a.lse[row] = z == 0.f ? -INFINITY : (M + __log2f(z)) * kLn2;
}

// ------------------------------------------------------------ host side

PrefixPlan plan_prefix(const wf_prefix_params& p) {
  PrefixPlan l{};
  const bool bf = p.dtype == WF_BF16;
  const int es = bf ? 2 : 4, KT = bf ? 128 : 64, nblk = KT / 32;
  const long R = (long)p.group * p.q_len, M = R * p.share, U = (long)p.prefixes * p.heads;
  const long rows = M * U;
  const long slots_at_once = device_cu_count();
  const long most = p.prefix_rows > 0 ? M : R;
  l.qw = bf && most > 32 ? 2 : 1;
  // waves over query rows (the others over keys), blocks of query rows
  auto shape = [&](long m, int* kw, int* mblocks) {
    const long blocks = (m + 32 * l.qw - 1) / (32 * l.qw);
    int qwaves = 1;
    while (qwaves < kPrefixWaves && qwaves < blocks) qwaves *= 2;
    while (kPrefixWaves / qwaves > nblk) qwaves *= 2;
    *kw = kPrefixWaves / qwaves;
    *mblocks = (int)((blocks + qwaves - 1) / qwaves);
  };
  // Key ranges per unit: whole rounds of workgroups, each with a fixed part of
  // about a tile, against the partials that every range adds.
  auto split = [&](long units, long keys, int mblocks, int* splits, int* rps) {
    const long tiles = (keys + KT - 1) / KT;
    const long top = std::min(tiles, 2 * slots_at_once / (units * mblocks) + 1);
    long best = 1;
    double best_cost = 0;
    for (long s = 1; s <= top; ++s) {
      const long per = (tiles + s - 1) / s;
      if ((tiles + per - 1) / per != s) continue;
      const long n = units * mblocks * s;
      const double cost = (double)((n + slots_at_once - 1) / slots_at_once) * ((double)per + 1.2) +
                          (double)s * rows * p.head_dim * 8 / 11e6;
      if (best_cost == 0 || cost < best_cost) {
        best_cost = cost;
        best = s;
      }
    }
    const long per = (tiles + best - 1) / best;
    *rps = (int)(per * KT);
    *splits = (int)((tiles + per - 1) / per);
  };
  if (p.prefix_rows > 0) {
    shape(M, &l.kw, &l.mblocks);
    split(U, p.prefix_rows, l.mblocks, &l.splits, &l.rps);
    l.items = U * l.mblocks * l.splits;
  }
  if (p.tail_cap > 0) {
    shape(R, &l.tkw, &l.tmblocks);
    split(U * p.share, p.tail_cap, l.tmblocks, &l.tsplits, &l.trps);
    l.titems = U * p.share * l.tmblocks * l.tsplits;
  }
  l.slots = l.splits + l.tsplits;
  l.ids = std::min(l.rps, kPrefixIds);
  if (l.slots > 1) {
    l.part_bytes = (size_t)rows * l.slots * p.head_dim * sizeof(float);
    l.pstat_bytes = (size_t)rows * l.slots * 2 * sizeof(float);
  }
  const size_t tiles = (size_t)4 * KT * es * p.head_dim;
  const size_t merge = (size_t)kPrefixWaves * l.qw * (p.head_dim * 32 + 64) * sizeof(float);
  l.lds_bytes = std::max(tiles + (size_t)l.ids * sizeof(int32_t), merge);
  return l;
}

template <typename T, int D, int FMT, int QW>
static hipError_t prefix_launch(const PrefixArgs& a, size_t lds, hipStream_t s) {
  auto kern = prefix_attn_kernel<T, D, FMT, QW>;
  if (lds > 65536) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)(((a.p.items + 7) & ~7) + a.t.items);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(kPrefixBlock), lds, s, a);
  return hipGetLastError();
}

// Threads per row and channels in the merge: enough for every partial of a row to
// be in flight.
template <typename T>
static hipError_t merge_launch(const PrefixArgs& a, long rows, int D, hipStream_t s) {
  const int sg = a.slots <= 4 ? 1 : a.slots <= 16 ? 4 : 16;
  auto go = [&](auto n) {
    constexpr int SG = decltype(n)::value;
    const int rpb = kBlock / (D / 8 * SG);
    hipLaunchKernelGGL((prefix_merge_kernel<T, SG>), dim3((unsigned)((rows + rpb - 1) / rpb)),
                       dim3(kBlock), 0, s, a, rows, D);
  };
  if (sg == 1)
    go(std::integral_constant<int, 1>{});
  else if (sg == 4)
    go(std::integral_constant<int, 4>{});
  else
    go(std::integral_constant<int, 16>{});
  return hipGetLastError();
}

hipError_t launch_prefix(const wf_prefix_params& p, PrefixArgs& a, hipStream_t s) {
  const PrefixPlan l = plan_prefix(p);
  a.heads = p.heads;
  a.share = p.share;
  a.R = p.group * p.q_len;
  a.cap = p.prefix_cap;
  a.rows = p.prefix_rows;
  a.T = p.tail_cap;
  a.slots = l.slots;
  a.ids = l.ids;
  a.scale = p.scale != 0.f ? p.scale : (float)(1.0 / std::sqrt((double)p.head_dim));
  a.p = PrefixPart{(int)l.items, l.splits, l.rps, l.mblocks, a.R * p.share, l.kw};
  a.t = PrefixPart{(int)l.titems, l.tsplits, l.trps, l.tmblocks, a.R, l.tkw};
  auto go = [&](auto t, auto d, auto f) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, F = decltype(f)::value;
    if constexpr (sizeof(T) == 2)
      if (l.qw == 2) return prefix_launch<T, D, F, 2>(a, l.lds_bytes, s);
    return prefix_launch<T, D, F, 1>(a, l.lds_bytes, s);
  };
  auto by_format = [&](auto t, auto d) {
    if (p.format == WF_CACHE_E4M3)
      return go(t, d, std::integral_constant<int, WF_CACHE_E4M3>{});
    if (p.format == WF_CACHE_E2M1)
      return go(t, d, std::integral_constant<int, WF_CACHE_E2M1>{});
    return go(t, d, std::integral_constant<int, WF_CACHE_PLAIN>{});
  };
  auto by_dim = [&](auto t) {
    return p.head_dim == 128 ? by_format(t, std::integral_constant<int, 128>{})
                             : by_format(t, std::integral_constant<int, 64>{});
  };
  hipError_t e = p.dtype == WF_BF16 ? by_dim(bf16_t{}) : by_dim(float{});
  if (e != hipSuccess || l.slots == 1) return e;
  const long rows = (long)p.prefixes * p.share * p.heads * a.R;
  return p.dtype == WF_BF16 ? merge_launch<bf16_t>(a, rows, p.head_dim, s)
                            : merge_launch<float>(a, rows, p.head_dim, s);
}

hipError_t load_prefix_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(
      &fa, reinterpret_cast<const void*>(prefix_attn_kernel<bf16_t, 128, WF_CACHE_PLAIN, 1>));
}

}  // namespace wf
