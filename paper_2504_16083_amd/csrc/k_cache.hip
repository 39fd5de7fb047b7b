// Writing rows into the paged cache and reading them back
// (include/mmi_cache.h). 16 lanes hold a row, 8 channels each, so that a
// group of 32 channels is 4 lanes and a row of K or V one 256-byte access; a
// wave takes 4 neighbouring rows of one head, which lie next to each other in
// a page. Bound by HBM.
#include "cache.hpp"
#include "codec.hpp"

namespace mmi {

struct Place {                     // where a unit of 16 lanes works
  int64_t row;                     // of k and v
  int head, lane, second;          // second: V, not K
  bool live;
};

__device__ __forceinline__ Place place(const RowsArgs& a) {
  const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
  const int64_t quads = (a.n + 3) / 4, u = unit >> 2;
  const int64_t hv = u / quads;
  Place p;
  p.row = (u - hv * quads) * 4 + (unit & 3);
  p.head = (int)(hv >> 1);
  p.second = (int)(hv & 1);
  p.lane = threadIdx.x & 15;
  p.live = p.row < a.n && p.head < a.c.Hkv;
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

template <int TYPE>
__global__ __launch_bounds__(256) void k_cache_write(RowsArgs a) {
  const Place p = place(a);
  int64_t slot = -1;
  bf16x8 x = zero8();
  if (p.live) {
    slot = a.slot[p.row];
    if (inside(a.c, slot))
      x = load16((p.second ? a.v + p.row * a.v_ss + p.head * a.v_sh : a.k + p.row * a.k_ss + p.head * a.k_sh) +
                 8 * p.lane);
  }
  // every lane takes part in the exchange below
  const bool put = p.live && inside(a.c, slot);
  if constexpr (TYPE == MMI_CACHE_BF16) {
    if (put) *reinterpret_cast<bf16x8*>(row_codes<TYPE>(a.c, p.second, slot, p.head) + 16 * p.lane) = x;
  } else {
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
    if (put) {
      uint8_t* at = row_codes<TYPE>(a.c, p.second, slot, p.head);
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
      if ((p.lane & 3) == 0) row_scales(a.c, p.second, slot, p.head)[p.lane >> 2] = (uint8_t)b;
    }
  }
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_cache_read(RowsArgs a) {
  const Place p = place(a);
  if (!p.live) return;
  const int64_t slot = a.slot[p.row];
  bf16x8 x = zero8();
  if (inside(a.c, slot)) {
    const uint8_t* at = row_codes<TYPE>(a.c, p.second, slot, p.head);
    if constexpr (TYPE == MMI_CACHE_BF16) {
      x = load16(at + 16 * p.lane);
    } else {
      const float s = scale_value(row_scales(a.c, p.second, slot, p.head)[p.lane >> 2]);
      if constexpr (TYPE == MMI_CACHE_FP4) {
        x = decode4(*reinterpret_cast<const uint32_t*>(at + 4 * p.lane), s);
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(at + 8 * p.lane);
        x = decode8<TYPE>(w[0], w[1], s);
      }
    }
  }
  uint16_t* to = p.second ? a.v + p.row * a.v_ss + p.head * a.v_sh : a.k + p.row * a.k_ss + p.head * a.k_sh;
  *reinterpret_cast<bf16x8*>(to + 8 * p.lane) = x;
}


static dim3 rows_grid(const RowsArgs& a) {
  const int64_t threads = (a.n + 3) / 4 * 4 * a.c.Hkv * 2 * 16;   // n Hkv <= 2^26: below 2^32
  return dim3((unsigned)((threads + 255) / 256));
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
