// Rotary positions on Q and K (include/mmi_cache.h).
//
// A row of 128 channels is 16 chunks of 8; a thread turns two of them (8
// pairs) of one token, in several heads one after another, so that the
// angles, sines and cosines of a token are found once a group of heads.
//
// Angles: turns a position as a 64-bit fraction, times the position, modulo
// 2^64: the fraction of a turn that is left, exact at any position (in fp32 a
// position of 2^20 and more has lost the angle's fraction). Its upper 32 bits
// as a signed number are the angle in [-1/2, 1/2) turns.
#include "cache.hpp"
#include "device.hpp"

namespace mmi {

constexpr int ROPE_UNROLL = 4;     // heads in flight per thread

template <bool HALF>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, int groups) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(idx & 7);
  const int64_t unit = idx >> 3;
  if (unit >= (int64_t)a.S * groups) return;
  // neighbouring lanes take neighbouring tokens of one group of heads
  const int x = (int)(unit % a.S), grp = (int)(unit / a.S);
  const int H = a.Hq + a.Hkv, per = (H + groups - 1) / groups;
  const int h0 = grp * per, h1 = min(H, h0 + per);
  const int turned = a.rot / 8;    // chunks that turn
  int ca, cb;                      // this thread's chunks
  bool ta, tb;
  if (HALF) {
    const int n = a.rot / 16;
    ta = tb = j < n;
    ca = ta ? j : turned + 2 * (j - n);
    cb = ta ? j + n : ca + 1;
  } else {
    ca = j; cb = j + 8;
    ta = ca < turned; tb = cb < turned;
  }
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = HALF ? 8 * j + e : 4 * (e < 4 ? ca : cb) + (e & 3);
    cs[e] = 1.0f; sn[e] = 0.0f;
    if (HALF ? ta : (e < 4 ? ta : tb)) {
      const int axis = (i >= a.sec1) + (i >= a.sec2);
      const int64_t p = a.pos ? a.pos[(int64_t)axis * a.S + x] : x;
      const int32_t t = (int32_t)(((uint64_t)p * a.turn[i]) >> 32);
      float s, c;
      sincospif((float)t * 4.656612873077393e-10f, &s, &c);    // 2^-31: half turns
      cs[e] = c * a.m;
      sn[e] = (a.inverse ? -s : s) * a.m;
    }
  }
  for (int h = h0; h < h1; h += ROPE_UNROLL) {
    bf16x8 va[ROPE_UNROLL], vb[ROPE_UNROLL];
    uint16_t* dst[ROPE_UNROLL];
#pragma unroll
    for (int u = 0; u < ROPE_UNROLL; ++u) {
      const int hh = min(h + u, h1 - 1);
      const bool isq = hh < a.Hq;
      const int64_t off = isq ? (int64_t)x * a.q_ss + (int64_t)hh * a.q_sh
                              : (int64_t)x * a.k_ss + (int64_t)(hh - a.Hq) * a.k_sh;
      const uint16_t* src = (isq ? a.q : a.k) + off;
      dst[u] = (isq ? a.qo : a.ko) + off;
      va[u] = load16(src + 8 * ca);
      vb[u] = load16(src + 8 * cb);
    }
#pragma unroll
    for (int u = 0; u < ROPE_UNROLL; ++u) {
      if (h + u >= h1) break;
      bf16x8 ra = va[u], rb = vb[u];
      if (HALF) {
        if (ta) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = (float)va[u][e], q = (float)vb[u][e];
            ra[e] = (__bf16)(p * cs[e] - q * sn[e]);
            rb[e] = (__bf16)(q * cs[e] + p * sn[e]);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = (float)va[u][2 * e], q = (float)va[u][2 * e + 1];
          const float r = (float)vb[u][2 * e], s = (float)vb[u][2 * e + 1];
          if (ta) {
            ra[2 * e] = (__bf16)(p * cs[e] - q * sn[e]);
            ra[2 * e + 1] = (__bf16)(q * cs[e] + p * sn[e]);
          }
          if (tb) {
            rb[2 * e] = (__bf16)(r * cs[4 + e] - s * sn[4 + e]);
            rb[2 * e + 1] = (__bf16)(s * cs[4 + e] + r * sn[4 + e]);
          }
        }
      }
      *reinterpret_cast<bf16x8*>(dst[u] + 8 * ca) = ra;
      *reinterpret_cast<bf16x8*>(dst[u] + 8 * cb) = rb;
    }
  }
}

hipError_t launch_rope(const RopeArgs& a, int layout, hipStream_t st) {
  const int H = a.Hq + a.Hkv;
  // groups of heads: enough threads to fill the chip (2^18) where the tokens
  // alone are too few, at most one head a group
  int64_t want = (((int64_t)1 << 18) + 8 * (int64_t)a.S - 1) / (8 * (int64_t)a.S);
  const int per = want >= H ? 1 : (int)((H + want - 1) / want);
  const int groups = (H + per - 1) / per;
  const int64_t blocks = ((int64_t)a.S * groups * 8 + 255) / 256;
  if (layout == MMI_ROPE_HALF)
    hipLaunchKernelGGL(k_rope<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, groups);
  else
    hipLaunchKernelGGL(k_rope<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, groups);
  return hipGetLastError();
}

}  // namespace mmi
