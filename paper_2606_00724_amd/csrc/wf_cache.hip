// The quantised cache: rows quantised as they are written, and read back
// (formats in wf_cache.hpp).
//
// Both kernels move bytes: a thread takes eight channels (16 bytes of bf16,
// 32 of fp32), the four threads of a block find its largest magnitude on DPP
// lane swaps, and a workgroup takes kRowsPerGroup rows of one unit, K and V.
// Its rows' loads are all on their way before the first is used, and there are
// enough workgroups per CU to fill HBM's latency.  On one MI355X, bytes read and
// written: 128 units x 32K bf16 rows of 128 channels stored in 8 bits 573 us,
// 5.7 TB/s (a large copy reaches 5.1); 8 units x 128K rows read back from 4 bits
// 127 us, 5.4 TB/s; 128 units x 4096 listed rows from 8 bits 88 us, 4.6 TB/s.  A
// block of 32 rows takes 3.6 us: a launch and two round trips to memory.
#include "wf_cache.hpp"
#include "wf_kernels.hpp"
#include "wf_launch.hpp"

namespace wf {

// The bits of |v| where they are largest over the four lanes of a quad
// (quad_perm [1 0 3 2], then [2 3 0 1]).
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));
}

// Rows of a unit that a workgroup moves: two per thread group.
template <int D>
constexpr int kRowsPerGroup = 2 * kBlock / (D / 8);

template <typename T, int D, int FMT>
__global__ __launch_bounds__(kBlock) void cache_store_kernel(CacheArgs a) {
  constexpr int TPR = D / 8;                             // threads per row
  constexpr int CB = FMT == WF_CACHE_E4M3 ? 8 : 4;       // bytes of eight codes
  const int u = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const int c = threadIdx.x % TPR;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = part * kRowsPerGroup<D> + i * (kBlock / TPR) + threadIdx.x / TPR;
    if (r >= a.rows) continue;  // (the lanes of a block go together)
    const int at = a.idx ? a.idx[(long)(u / a.heads) * a.rows + r] : a.first + r;
    if (at < 0 || at >= a.cap) continue;
    const long src = ((long)u * a.rows + r) * D + 8 * c;
    const long row = (long)u * a.cap + at;
    float v[2][8];
    load8(reinterpret_cast<const T*>(a.K) + src, v[0]);
    load8(reinterpret_cast<const T*>(a.V) + src, v[1]);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t amax = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(v[m][e]) & 0x7fffffffu);
      const uint32_t x = block_exponent<FMT>(quad_max(amax));
      const float s = block_unscale(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[m][e] = x == 255u ? 0.f : v[m][e] * s;
      const u32x2 w = encode8<FMT>(v[m]);
      uint8_t* codes = static_cast<uint8_t*>(m ? a.Vc : a.Kc) + (row * TPR + c) * CB;
      if constexpr (CB == 8)
        *reinterpret_cast<u32x2*>(codes) = w;
      else
        *reinterpret_cast<uint32_t*>(codes) = w[0];
      if ((c & 3) == 0) static_cast<uint8_t*>(m ? a.Vx : a.Kx)[row * (D / 32) + c / 4] = (uint8_t)x;
    }
  }
}

template <typename T, int D, int FMT>
__global__ __launch_bounds__(kBlock) void cache_load_kernel(CacheArgs a) {
  constexpr int TPR = D / 8;
  constexpr int CB = FMT == WF_CACHE_E4M3 ? 8 : 4;
  const int u = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const int c = threadIdx.x % TPR;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = part * kRowsPerGroup<D> + i * (kBlock / TPR) + threadIdx.x / TPR;
    if (r >= a.rows) continue;
    const int at = a.idx ? a.idx[(long)u * a.rows + r] : a.first + r;
    const bool in = at >= 0 && at < a.cap;
    const long row = (long)u * a.cap + (in ? at : 0);
    const long dst = ((long)u * a.rows + r) * D + 8 * c;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const uint8_t* codes = static_cast<const uint8_t*>(m ? a.Vc : a.Kc) + (row * TPR + c) * CB;
      u32x2 w = {0u, 0u};
      if constexpr (CB == 8)
        w = *reinterpret_cast<const u32x2*>(codes);
      else
        w[0] = *reinterpret_cast<const uint32_t*>(codes);
      const uint32_t x = static_cast<const uint8_t*>(m ? a.Vx : a.Kx)[row * (D / 32) + c / 4];
      float v[8];
      decode8<FMT>(w, block_scale(x), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = in ? v[e] : 0.f;
      put8(reinterpret_cast<T*>(m ? a.V : a.K) + dst, v);
    }
  }
}

// ------------------------------------------------------------ host side

template <typename T, int D, int FMT>
static void cache_launch(bool store, const CacheArgs& a, unsigned grid, hipStream_t s) {
  if (store)
    hipLaunchKernelGGL((cache_store_kernel<T, D, FMT>), dim3(grid), dim3(kBlock), 0, s, a);
  else
    hipLaunchKernelGGL((cache_load_kernel<T, D, FMT>), dim3(grid), dim3(kBlock), 0, s, a);
}

long cache_groups(const wf_cache_params& p) {
  const long per = p.head_dim == 128 ? kRowsPerGroup<128> : kRowsPerGroup<64>;
  return (long)p.batch * p.heads * ((p.rows + per - 1) / per);
}

hipError_t launch_cache(const wf_cache_params& p, bool store, const void* K, const void* V,
                        const int32_t* idx, const void* Kc, const void* Kx, const void* Vc,
                        const void* Vx, hipStream_t s) {
  CacheArgs a;
  a.K = const_cast<void*>(K);
  a.V = const_cast<void*>(V);
  a.idx = idx;
  a.Kc = const_cast<void*>(Kc);
  a.Kx = const_cast<void*>(Kx);
  a.Vc = const_cast<void*>(Vc);
  a.Vx = const_cast<void*>(Vx);
  a.heads = p.heads;
  a.rows = p.rows;
  a.cap = p.capacity;
  a.first = p.first;
  const long groups = cache_groups(p);
  a.blocks = (int)(groups / ((long)p.batch * p.heads));
  auto go = [&](auto t, auto fmt) {
    using T = decltype(t);
    constexpr int F = decltype(fmt)::value;
    if (p.head_dim == 128)
      cache_launch<T, 128, F>(store, a, (unsigned)groups, s);
    else
      cache_launch<T, 64, F>(store, a, (unsigned)groups, s);
  };
  using E4 = std::integral_constant<int, WF_CACHE_E4M3>;
  using E2 = std::integral_constant<int, WF_CACHE_E2M1>;
  if (p.dtype == WF_BF16)
    p.format == WF_CACHE_E4M3 ? go(bf16_t{}, E4{}) : go(bf16_t{}, E2{});
  else
    p.format == WF_CACHE_E4M3 ? go(float{}, E4{}) : go(float{}, E2{});
  return hipGetLastError();
}

hipError_t load_cache_kernels() {
  hipFuncAttributes fa;
  return hipFuncGetAttributes(&fa, reinterpret_cast<const void*>(
                                       cache_store_kernel<bf16_t, 128, WF_CACHE_E4M3>));
}

}  // namespace wf
