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

  // 32 keys (rows sb .. sb + 31 of the tile, nr of the tile's rows valid)
  __device__ __forceinline__ void step(const unsigned char* Kb, const unsigned char* Vb, int sb,
                                       int nr, float c2) {
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
    f32x16 s[QW];
#pragma unroll
    for (int b = 0; b < QW; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int j = 0; j < QS; ++j) {
      const u32x4 kf =
          *reinterpret_cast<const u32x4*>(Kb + tile_offset<T, G>(sb + l32, 2 * j + h));
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        if constexpr (BF) {
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                         __builtin_bit_cast(bf16x8, q[b][j]), s[b],
                                                         0, 0, 0);
        } else {
          const f32x4 kv = __builtin_bit_cast(f32x4, kf), qv = __builtin_bit_cast(f32x4, q[b][j]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[e], qv[e], s[b], 0, 0, 0);
        }
      }
    }
    // the lane holds keys sb + 8 (i / 4) + 4 h + i % 4 of query l % 32
    if (sb + 32 > nr) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool off = sb + 8 * (i >> 2) + 4 * h + (i & 3) >= nr;
#pragma unroll
        for (int b = 0; b < QW; ++b) s[b][i] = off ? -INFINITY : s[b][i];
      }
    }
    float mx[QW];
    bool grow = false;
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      float m = s[b][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) m = fmaxf(m, s[b][i]);
      mx[b] = m * c2;
      grow |= mx[b] > mref[b] + 8.f;
    }
    // The reference moves only when a score passes it by 2^8: weights then stay
    // below 2^8, their sums far from the fp32 range, and a rescale of the
    // outputs is rare.
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
      for (int b = 0; b < QW; ++b) {
        const float mn = fmaxf(mref[b], fmaxf(mx[b], partner32(mx[b])));
        const float al = mref[b] > -INFINITY ? __builtin_amdgcn_exp2f(mref[b] - mn) : 0.f;
        mref[b] = mn;
        l[b] *= al;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[b][d][i] *= al;
      }
    }
#pragma unroll
    for (int b = 0; b < QW; ++b) {
      // (while every score so far is -inf, their weights are 2^-inf = 0)
      const float ref = mref[b] > -INFINITY ? mref[b] : 0.f;
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        // (the unrounded product: scores of thousands keep their differences)
        s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c2, -ref));
        z += s[b][i];
      }
      l[b] += z;
    }
    if constexpr (BF) {
      const uint32_t vb = lds_offset(Vb);
      const int i16 = lane & 15;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        u32x4 pf[QW];
#pragma unroll
        for (int b = 0; b < QW; ++b)
          pf[b] = u32x4{pack_bf16x2(s[b][8 * kb], s[b][8 * kb + 1]),
                        pack_bf16x2(s[b][8 * kb + 2], s[b][8 * kb + 3]),
                        pack_bf16x2(s[b][8 * kb + 4], s[b][8 * kb + 5]),
                        pack_bf16x2(s[b][8 * kb + 6], s[b][8 * kb + 7])};
        const int t0 = sb + 16 * kb + 4 * h + (i16 >> 2);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          // in each 16-lane group lane i points at row t0 + i / 4, channels c0 +
          // 4 (i % 4) .. + 3, and receives rows t0 .. t0 + 3 of channel c0 + i
          const int c0 = 32 * d + (lane & 16) + 4 * (i16 & 3);
          const uint32_t o = 2 * (c0 & 7);
          const v4i16p lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4i16p*)(size_t)(
                  vb + tile_offset<T, G>(t0, c0 >> 3) + o));
          const v4i16p hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4i16p*)(size_t)(
                  vb + tile_offset<T, G>(t0 + 8, c0 >> 3) + o));
          const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
          const u32x4 vf = {l2[0], l2[1], h2[0], h2[1]};
#pragma unroll
          for (int b = 0; b < QW; ++b)
            O[b][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pf[b]), O[b][d], 0, 0,
                0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = sb + 8 * (i >> 2) + 4 * h + (i & 3);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const int c = 32 * d + l32;
          const float vf = *reinterpret_cast<const float*>(Vb + tile_offset<T, G>(r, c >> 2) +
                                                           4 * (c & 3));
#pragma unroll
          for (int b = 0; b < QW; ++b)
            O[b][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[b][i], O[b][d], 0, 0, 0);
        }
      }
    }
  }
};

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
#pragma unroll
        for (int k = 0; k < CPP / 8; ++k) {  // eight channels each
          float v[8];
          u32x2 c;
          if constexpr (FMT == WF_CACHE_E4M3)
            c = u32x2{w[m][i][2 * k], w[m][i][2 * k + 1]};
          else
            c = u32x2{w[m][i][k], 0u};
          decode8<FMT>(c, s, v);
          unsigned char* dst = m ? Vb : Kb;
          const int g = pc * (CPP / 8) + k;  // eight channels: one granule of bf16, two of fp32
          if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4*>(dst + tile_offset<T, G>(r, g)) =
                u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7])};
          } else {
            *reinterpret_cast<f32x4*>(dst + tile_offset<T, G>(r, 2 * g)) =
                f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(dst + tile_offset<T, G>(r, 2 * g + 1)) =
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
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
  const float c2 = fabsf(a.scale) * kLog2e;
  const uint32_t flip = a.scale < 0.f ? (W::BF ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
  for (int b = 0; b < QW; ++b) {
    const T* src = reinterpret_cast<const T*>(a.Q) + row_of(min(m0 + 32 * b + l32, M - 1)) * D;
#pragma unroll
    for (int j = 0; j < QS; ++j)
      w.q[b][j] = reinterpret_cast<const u32x4*>(src)[2 * j + h] ^ u32x4{flip, flip, flip, flip};
    w.mref[b] = -INFINITY;
    w.l[b] = 0.f;
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
    auto stage_ids = [&](int t) {
      if (!rows.ids || t * KT % kPrefixIds != 0) return;  // uniform
      rows.id0 = k0 + t * KT;
      lds_barrier();
      for (int i = threadIdx.x; i < min(kPrefixIds, nk - t * KT); i += kPrefixBlock)
        ids[i] = a.list[(long)unit * a.rows + rows.id0 + i];
      __syncthreads();
    };
    // the products of tile t, in `buf`
    auto compute = [&](int t, int buf) {
      unsigned char* Kb = smem + buf * 2 * MB;
      unsigned char* Vb = Kb + MB;
      const int nr = min(KT, nk - t * KT);
      if (nr < KT) {
        // rows past the range repeat its last one: 0 there, as 0 times an
        // infinite value is NaN
        for (int i = nr * G + threadIdx.x; i < KT * G; i += kPrefixBlock)
          reinterpret_cast<u32x4*>(Vb)[i] = u32x4{0u, 0u, 0u, 0u};
        lds_barrier();
      }
      if (active)
        for (int sb = 32 * kw; sb < nr; sb += 32 * KW) w.step(Kb, Vb, sb, nr, c2);
    };
    if (FMT == WF_CACHE_PLAIN || own) {
      // tiles stream through two LDS slots by direct loads
      const T* Kg = reinterpret_cast<const T*>(own ? a.Kt : a.K) + (long)unit * rows.cap * D;
      const T* Vg = reinterpret_cast<const T*>(own ? a.Vt : a.V) + (long)unit * rows.cap * D;
      constexpr int IPW = KT * G / (64 * kPrefixWaves);  // loads per wave and matrix
      constexpr int RPI = 64 / G;
      const uint32_t lds0 = lds_offset(smem);
      auto issue = [&](int t) {
        stage_ids(t);
        const uint32_t at = lds0 + (t & 1) * 2 * MB;
        long off[IPW];
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
          const int r = (wave * IPW + i) * RPI + lane / G;
          const int k = (lane % G) ^ tile_swz<T, G>(r);
          off[i] = rows(t * KT + r) * D + W::EPV * k;
        }
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
          const uint32_t to = at + 1024u * (wave * IPW + i);
          async_load16<false>(Kg + off[i], __builtin_amdgcn_readfirstlane(to));
          async_load16<false>(Vg + off[i], __builtin_amdgcn_readfirstlane(to + MB));
        }
      };
      // consume the q operands before loads are queued: the compiler's own wait
      // for them then sits here
#pragma unroll
      for (int b = 0; b < QW; ++b)
#pragma unroll
        for (int j = 0; j < QS; ++j) asm volatile("" ::"v"(w.q[b][j]));
      issue(0);
      for (int t = 0; t < nt; ++t) {
        if (t + 1 < nt) {
          issue(t + 1);
          wait_vmcnt_chunks<2 * IPW>(1);
        } else {
          wait_vmcnt_chunks<2 * IPW>(0);
        }
        lds_barrier();  // tile t visible
        compute(t, t & 1);
        lds_barrier();  // everyone is past tile t
      }
    } else {
      // codes are loaded to registers a tile ahead, and decoded into LDS
      if constexpr (FMT != WF_CACHE_PLAIN) {
        QuantStage<T, D, FMT> st;
        stage_ids(0);
        st.load(a, rows, unit, 0);
        for (int t = 0; t < nt; ++t) {
          unsigned char* Kb = smem + (t & 1) * 2 * MB;
          st.commit(Kb, Kb + MB);
          if (t + 1 < nt) {
            stage_ids(t + 1);
            st.load(a, rows, unit, (t + 1) * KT);
          }
          lds_barrier();  // tile t visible, everyone is past tile t - 1
          compute(t, t & 1);
        }
        lds_barrier();
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

// Merges the partials of each query row: a thread takes eight channels.
template <typename T>
__global__ __launch_bounds__(kBlock) void prefix_merge_kernel(PrefixArgs a, long rows, int D) {
  const int tpr = D / 8;
  const long row = (long)blockIdx.x * (kBlock / tpr) + threadIdx.x / tpr;
  if (row >= rows) return;
  const int c0 = (threadIdx.x % tpr) * 8;
  const float* st = a.pstat + row * a.slots * 2;
  float M = -INFINITY;
  for (int s = 0; s < a.slots; ++s) M = fmaxf(M, st[2 * s]);
  float z = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.slots; ++s) {
    const float m = st[2 * s], zs = st[2 * s + 1];
    if (m == -INFINITY && zs == 0.f) continue;  // an empty range has no output
    const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - M) : 1.f;  // (zs NaN)
    const f32x4* src = reinterpret_cast<const f32x4*>(a.part + (row * a.slots + s) * D + c0);
    const f32x4 x = src[0], y = src[1];
    z += f * zs;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] += f * x[e];
      o[4 + e] += f * y[e];
    }
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  T* dst = reinterpret_cast<T*>(a.O) + row * D + c0;
  put4<T>(dst, o[0], o[1], o[2], o[3]);
  put4<T>(dst + 4, o[4], o[5], o[6], o[7]);
  if (a.lse && c0 == 0) a.lse[row] = z == 0.f ? -INFINITY : (M + __log2f(z)) * kLn2;
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
  const int rpb = kBlock / (p.head_dim / 8);
  const dim3 grid((unsigned)((rows + rpb - 1) / rpb));
  if (p.dtype == WF_BF16)
    hipLaunchKernelGGL(prefix_merge_kernel<bf16_t>, grid, dim3(kBlock), 0, s, a, rows, p.head_dim);
  else
    hipLaunchKernelGGL(prefix_merge_kernel<float>, grid, dim3(kBlock), 0, s, a, rows, p.head_dim);
  return hipGetLastError();
}

hipError_t load_prefix_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(
      &fa, reinterpret_cast<const void*>(prefix_attn_kernel<bf16_t, 128, WF_CACHE_PLAIN, 1>));
}

}  // namespace wf
