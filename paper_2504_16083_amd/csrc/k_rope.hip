// Rotary positions on Q and K (include/mmi_cache.h).
//
// A row of 128 channels is 16 chunks of 8; a thread turns two of them (8
// pairs), and 32 groups of 8 threads take the rows of a workgroup's tokens in
// the order in which they lie in memory (a token's Q heads, then its K heads).
// The sines and cosines of the tokens are found once, in LDS. Bound by HBM:
// 262144 tokens of 32 + 8 heads in 1010 us, 5.3 TB/s (1050 us where a thread
// kept one token and went from head to head: neighbouring lanes were then on
// tokens 8 KB apart; 20240 tokens 64 us for 72). The stores do not displace
// what is still to be read: 64 us for 67 at 20240 tokens, the same at 262144.
//
// Angles: turns a position as a 64-bit fraction, times the position, modulo
// 2^64: the fraction of a turn that is left, to 2^-32 at position 2^31 (in
// fp32 a position of 2^20 and more has lost the angle's fraction). Its upper
// 32 bits as a signed number are the angle in [-1/2, 1/2) turns; as fp32 that
// is off by up to 2^-26.
#include <algorithm>

#include "cache.hpp"
#include "device.hpp"

namespace mmi {

constexpr int RU = 4;              // rows in flight per thread
constexpr int RT = 8;              // most tokens of a workgroup

typedef __attribute__((__vector_size__(16))) unsigned int u32q;

template <bool HALF>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, int tokens) {
  __shared__ __align__(16) float2 cs[RT * D / 2];          // cosine, sine of every pair
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t x0 = (int64_t)blockIdx.x * tokens;
  const int n = (int)min((int64_t)tokens, a.S - x0);
  for (int i = tid; i < n * half; i += 256) {
    const int x = i / half, pair = i - x * half;
    const int axis = (pair >= a.sec1) + (pair >= a.sec2);
    const int64_t p = a.pos ? a.pos[(int64_t)axis * a.S + x0 + x] : x0 + x;
    const int32_t t = (int32_t)(((uint64_t)p * a.turn[pair]) >> 32);
    float s, c;
    sincospif((float)t * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
    cs[x * (D / 2) + pair] = make_float2(c * a.m, (a.inverse ? -s : s) * a.m);
  }
  __syncthreads();
  const int j = tid & 7, H = a.Hq + a.Hkv;
  const int turned = a.rot / 8;    // chunks that turn
  int ca, cb;                      // this thread's chunks, and whether they turn
  bool ta, tb;
  if (HALF) {
    const int m = a.rot / 16;
    ta = tb = j < m;
    ca = ta ? j : turned + 2 * (j - m);
    cb = ta ? j + m : ca + 1;
  } else {
    ca = j; cb = j + 8;
    ta = ca < turned; tb = cb < turned;
  }
  const int rows = n * H;
  for (int r0 = tid >> 3; r0 < rows; r0 += 32 * RU) {
    bf16x8 va[RU], vb[RU];
    uint16_t* dst[RU];
    int tok[RU];
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      const int r = min(r0 + 32 * u, rows - 1);
      tok[u] = r / H;
      const int h = r - tok[u] * H;
      const bool isq = h < a.Hq;
      const int64_t off = isq ? (x0 + tok[u]) * a.q_ss + (int64_t)h * a.q_sh
                              : (x0 + tok[u]) * a.k_ss + (int64_t)(h - a.Hq) * a.k_sh;
      const uint16_t* src = (isq ? a.q : a.k) + off;
      dst[u] = (isq ? a.qo : a.ko) + off;
      va[u] = load16(src + 8 * ca);
      vb[u] = load16(src + 8 * cb);
    }
#pragma unroll
    for (int u = 0; u < RU; ++u) {
      if (r0 + 32 * u >= rows) break;
      bf16x8 ra = va[u], rb = vb[u];
      const float2* t = cs + tok[u] * (D / 2);
      if (HALF) {
        if (ta) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 w = t[8 * j + e];
            const float p = (float)va[u][e], q = (float)vb[u][e];
            ra[e] = (__bf16)(p * w.x - q * w.y);
            rb[e] = (__bf16)(q * w.x + p * w.y);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (ta) {
            const float2 w = t[4 * ca + e];
            const float p = (float)va[u][2 * e], q = (float)va[u][2 * e + 1];
            ra[2 * e] = (__bf16)(p * w.x - q * w.y);
            ra[2 * e + 1] = (__bf16)(q * w.x + p * w.y);
          }
          if (tb) {
            const float2 w = t[4 * cb + e];
            const float p = (float)vb[u][2 * e], q = (float)vb[u][2 * e + 1];
            rb[2 * e] = (__bf16)(p * w.x - q * w.y);
            rb[2 * e + 1] = (__bf16)(q * w.x + p * w.y);
          }
        }
      }
      __builtin_nontemporal_store(__builtin_bit_cast(u32q, ra), reinterpret_cast<u32q*>(dst[u] + 8 * ca));
      __builtin_nontemporal_store(__builtin_bit_cast(u32q, rb), reinterpret_cast<u32q*>(dst[u] + 8 * cb));
    }
  }
}

hipError_t launch_rope(const RopeArgs& a, int layout, hipStream_t st) {
  // several tokens a workgroup once one each fills the chip
  const int tokens = (int)std::min<int64_t>(RT, std::max<int64_t>(1, a.S / 2048));
  const int64_t blocks = ((int64_t)a.S + tokens - 1) / tokens;
  if (layout == MMI_ROPE_HALF)
    hipLaunchKernelGGL(k_rope<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, tokens);
  else
    hipLaunchKernelGGL(k_rope<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, tokens);
  return hipGetLastError();
}

}  // namespace mmi
