// Writing rows into the paged cache and reading them back
// (include/mmi_cache.h). 16 lanes hold a row, 8 channels each, so that a
// group of 32 channels is 4 lanes and a row of K or V one 256-byte access; a
// wave takes 4 neighbouring tokens, which lie next to each other in a page,
// a thread up to PV of their rows (heads, K and V) with all loads in flight.
// Workgroups of neighbouring heads follow each other: together they read or
// write whole tokens. Bound by HBM: 262144 rows of 8 heads written as int8 in
// 301 us and read back in 314 us (5.3 TB/s each, rows of one head at a time
// and one a thread took 480 and 417 us).
#include "cache.hpp"
#include "codec.hpp"

namespace mmi {

constexpr int PV = 4;              // rows in flight per thread
constexpr int TOKENS = 16;         // of a workgroup

struct Place {                     // where a unit of 16 lanes works
  int64_t row;                     // token: row of k and v
  int first, lane;                 // rows first .. first + PV - 1 of the token's 2 Hkv: head, then K or V
  int64_t slot;                    // -1: no such token
};

__device__ __forceinline__ Place place(const RowsArgs& a) {
  const int parts = (2 * a.c.Hkv + PV - 1) / PV;
  const int group = blockIdx.x / parts;
  Place p;
  p.row = (int64_t)group * TOKENS + (threadIdx.x >> 4);
  p.first = (blockIdx.x - group * parts) * PV;
  p.lane = threadIdx.x & 15;
  p.slot = p.row < a.n ? a.slot[p.row] : -1;
  return p;
}

__device__ __forceinline__ bool inside(const CacheDev& c, int64_t slot) {
  return slot >= 0 && (slot >> c.shift) < c.n_pages;
}

template <int TYPE>
__device__ __forceinline__ uint8_t* row_codes(const CacheDev& c, int second, int64_t slot, int head) {
  const int64_t in = ((int64_t)head << c.shift) + (slot & ((1 << c.shift) - 1));
  return (second ? c.v : c.k) + (slot >> c.shift) * c.page_stride + in * Codec<TYPE>::ROW;
}

__device__ __forceinline__ uint8_t* row_scales(const CacheDev& c, int second, int64_t slot, int head) {
  const int64_t in = ((int64_t)head << c.shift) + (slot & ((1 << c.shift) - 1));
  return (uint8_t*)(second ? c.vs : c.ks) + (slot >> c.shift) * c.scale_stride + in * 4;
}

__device__ __forceinline__ uint16_t* row_of(const RowsArgs& a, const Place& p, int i) {
  const int head = (p.first + i) >> 1;
  return ((p.first + i) & 1 ? a.v + p.row * a.v_ss + head * a.v_sh : a.k + p.row * a.k_ss + head * a.k_sh) + 8 * p.lane;
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_cache_write(RowsArgs a) {
  const Place p = place(a);
  const bool put = inside(a.c, p.slot);
  const int n = min(PV, 2 * a.c.Hkv - p.first);
  bf16x8 rows[PV];
#pragma unroll
  for (int i = 0; i < PV; ++i) rows[i] = put && i < n ? load16(row_of(a, p, i)) : zero8();
#pragma unroll
  for (int i = 0; i < PV; ++i) {
    const int head = (p.first + i) >> 1, second = (p.first + i) & 1;
    const bf16x8 x = rows[i];
    if constexpr (TYPE == MMI_CACHE_BF16) {
      if (put && i < n) *reinterpret_cast<bf16x8*>(row_codes<TYPE>(a.c, second, p.slot, head) + 16 * p.lane) = x;
    } else {
      // every lane takes part in the exchanges
      const u32x4 bits = __builtin_bit_cast(u32x4, x);
      int amax = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        amax = max(amax, max((int)(bits[e] & 0x7fff), (int)(bits[e] >> 16 & 0x7fff)));
      amax = max(amax, __shfl_xor(amax, 1));
      amax = max(amax, __shfl_xor(amax, 2));
      const int b = scale_byte<TYPE>(amax);
      const float inv = b == 255 ? 0.0f : scale_inverse(b);
      const float most = __uint_as_float((uint32_t)most_bits<TYPE>() << 16);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        y[e] = b == 255 ? 0.0f : __builtin_amdgcn_fmed3f((float)x[e], -most, most) * inv;
      if (put && i < n) {
        uint8_t* at = row_codes<TYPE>(a.c, second, p.slot, head);
        if constexpr (TYPE == MMI_CACHE_FP4) {
          uint32_t w = 0;
          w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
          w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
          w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
          w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
          *reinterpret_cast<uint32_t*>(at + 4 * p.lane) = w;
        } else {
          const u32x2 w = {encode8<TYPE>(y[0], y[1], y[2], y[3]), encode8<TYPE>(y[4], y[5], y[6], y[7])};
          *reinterpret_cast<u32x2*>(at + 8 * p.lane) = w;
        }
        if ((p.lane & 3) == 0) row_scales(a.c, second, p.slot, head)[p.lane >> 2] = (uint8_t)b;
      }
    }
  }
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_cache_read(RowsArgs a) {
  const Place p = place(a);
  if (p.row >= a.n) return;
  const int n = min(PV, 2 * a.c.Hkv - p.first);
  const bool get = inside(a.c, p.slot);
  u32x4 raw[PV];
  uint32_t scale[PV];
#pragma unroll
  for (int i = 0; i < PV; ++i) {
    raw[i] = u32x4{};
    scale[i] = 0;
    if (get && i < n) {
      const int head = (p.first + i) >> 1, second = (p.first + i) & 1;
      const uint8_t* at = row_codes<TYPE>(a.c, second, p.slot, head);
      if constexpr (TYPE == MMI_CACHE_BF16) {
        raw[i] = *reinterpret_cast<const u32x4*>(at + 16 * p.lane);
      } else if constexpr (TYPE == MMI_CACHE_FP4) {
        raw[i][0] = *reinterpret_cast<const uint32_t*>(at + 4 * p.lane);
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(at + 8 * p.lane);
        raw[i][0] = w[0];
        raw[i][1] = w[1];
      }
      if constexpr (Codec<TYPE>::SCALED) scale[i] = row_scales(a.c, second, p.slot, head)[p.lane >> 2];
    }
  }
#pragma unroll
  for (int i = 0; i < PV; ++i) {
    if (i >= n) break;
    u32x4 x = raw[i];
    if constexpr (TYPE == MMI_CACHE_FP4) x = __builtin_bit_cast(u32x4, decode4(raw[i][0], scale_value(scale[i])));
    else if constexpr (TYPE != MMI_CACHE_BF16)
      x = __builtin_bit_cast(u32x4, decode8<TYPE>(raw[i][0], raw[i][1], scale_value(scale[i])));
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(row_of(a, p, i)));
  }
}

static dim3 rows_grid(const RowsArgs& a) {
  // n Hkv <= 2^26: at most 2^23 workgroups
  return dim3((unsigned)((a.n + TOKENS - 1) / TOKENS * ((2 * a.c.Hkv + PV - 1) / PV)));
}

hipError_t launch_cache_write(const RowsArgs& a, int type, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  switch (type) {
    case MMI_CACHE_BF16: hipLaunchKernelGGL(k_cache_write<MMI_CACHE_BF16>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_FP8: hipLaunchKernelGGL(k_cache_write<MMI_CACHE_FP8>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_INT8: hipLaunchKernelGGL(k_cache_write<MMI_CACHE_INT8>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_FP4: hipLaunchKernelGGL(k_cache_write<MMI_CACHE_FP4>, rows_grid(a), dim3(256), 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_cache_read(const RowsArgs& a, int type, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  switch (type) {
    case MMI_CACHE_BF16: hipLaunchKernelGGL(k_cache_read<MMI_CACHE_BF16>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_FP8: hipLaunchKernelGGL(k_cache_read<MMI_CACHE_FP8>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_INT8: hipLaunchKernelGGL(k_cache_read<MMI_CACHE_INT8>, rows_grid(a), dim3(256), 0, st, a); break;
    case MMI_CACHE_FP4: hipLaunchKernelGGL(k_cache_read<MMI_CACHE_FP4>, rows_grid(a), dim3(256), 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace mmi
