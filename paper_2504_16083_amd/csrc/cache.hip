// Host checks of the operators around the prefill (include/mmi_cache.h):
// every argument that the host can see is validated here, before a context
// or a device is touched, and turned into the records that the launches take.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "cache.hpp"
#include "device.hpp"

namespace mmi {

namespace {

[[noreturn]] void fail(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  throw Error(code, buf);
}

void aligned(const void* p, int bytes, const char* name) {
  if (!p) fail(MMI_ERR_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % bytes) fail(MMI_ERR_INVALID_ARG, "%s must be %d-byte aligned", name, bytes);
}

// 0, 0 = packed; a row offset of any token and head stays far from 2^63
void strides(int64_t& ss, int64_t& sh, int H, const char* name) {
  if (ss == 0 && sh == 0) { ss = (int64_t)H * D; sh = D; }
  if (ss <= 0 || sh <= 0 || ss % 8 || sh % 8)
    fail(MMI_ERR_INVALID_ARG, "%s strides must be positive multiples of 8 elements", name);
  if (ss > ((int64_t)1 << 40) || sh > ((int64_t)1 << 40)) fail(MMI_ERR_UNSUPPORTED, "%s strides exceed 2^40", name);
}

constexpr double TWO_PI = 6.283185307179586476925286766559;
constexpr double PER_TURN = 0x1.45f306dc9c883p-3, PER_TURN_REST = -0x1.6b01ec5417056p-57;   // 1 / (2 pi) as the sum of two
constexpr double MOST_FREQ = 0x1p40;
constexpr int ROW_BYTES[4] = {256, 128, 128, 64};

}  // namespace

// Radians a position of every pair, and the factor of cos and sin.
double rope_freq(const mmi_rope_cfg* cfg, double* freq) {
  if (!cfg) fail(MMI_ERR_INVALID_ARG, "rope config is NULL");
  const mmi_rope_cfg& c = *cfg;
  if (c.rot_dim < 16 || c.rot_dim > D || c.rot_dim % 16)
    fail(MMI_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16 in [16, 128]", c.rot_dim);
  if (c.scaling < MMI_ROPE_SCALE_NONE || c.scaling > MMI_ROPE_SCALE_PARTS)
    fail(MMI_ERR_BAD_CONFIG, "unknown rope scaling %d", c.scaling);
  if (!c.inv_freq && !(c.theta > 0 && std::isfinite(c.theta))) fail(MMI_ERR_BAD_CONFIG, "theta must be positive");
  if (c.scaling != MMI_ROPE_SCALE_NONE && !(c.factor >= 1 && std::isfinite(c.factor)))
    fail(MMI_ERR_BAD_CONFIG, "factor must be at least 1");
  if (c.scaling == MMI_ROPE_SCALE_PARTS && !c.inv_freq &&
      !(c.orig_len > 0 && std::isfinite(c.orig_len) && c.beta_slow >= 0 && c.beta_fast > c.beta_slow &&
        std::isfinite(c.beta_fast)))
    fail(MMI_ERR_BAD_CONFIG, "orig_len must be positive and beta_fast > beta_slow >= 0");
  if (!(c.attn_factor >= 0 && std::isfinite((float)c.attn_factor)))
    fail(MMI_ERR_BAD_CONFIG, "attn_factor must not be negative");
  double theta = c.theta;
  if (c.scaling == MMI_ROPE_SCALE_NTK) theta *= std::pow(c.factor, (double)c.rot_dim / (c.rot_dim - 2));
  for (int i = 0; i < c.rot_dim / 2; ++i) {
    double f;
    if (c.inv_freq) {
      f = c.inv_freq[i];
    } else {
      f = std::pow(theta, -2.0 * i / c.rot_dim);
      if (c.scaling == MMI_ROPE_SCALE_LINEAR) f /= c.factor;
      if (c.scaling == MMI_ROPE_SCALE_PARTS) {
        const double g = std::fmin(std::fmax((c.orig_len * f / TWO_PI - c.beta_slow) / (c.beta_fast - c.beta_slow),
                                             0.0), 1.0);
        f *= g + (1.0 - g) / c.factor;
      }
    }
    if (!(f >= 0 && f <= MOST_FREQ)) fail(MMI_ERR_BAD_CONFIG, "frequency %d is not in [0, 2^40]", i);
    freq[i] = f;
  }
  return c.attn_factor > 0 ? c.attn_factor : c.scaling == MMI_ROPE_SCALE_PARTS ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
}

// Of the problem only what the rotation uses: the limits that the attention
// kernel sets to K's strides are not its own.
RopeArgs rope_args(const mmi_problem* prob, const mmi_rope_cfg* cfg, const int32_t* pos, const void* q, const void* k,
                   void* q_out, void* k_out) {
  if (!prob) fail(MMI_ERR_INVALID_ARG, "problem is NULL");
  mmi_problem p = *prob;
  if (p.S < 1) fail(MMI_ERR_INVALID_ARG, "S must be >= 1");
  if (p.S > MMI_MAX_SEQ) fail(MMI_ERR_UNSUPPORTED, "S = %lld exceeds %d", (long long)p.S, MMI_MAX_SEQ);
  if (p.Hq < 1 || p.Hkv < 1) fail(MMI_ERR_INVALID_ARG, "head counts must be >= 1");
  if (p.Hq % p.Hkv) fail(MMI_ERR_UNSUPPORTED, "Hq %% Hkv != 0");
  if (p.D != D) fail(MMI_ERR_UNSUPPORTED, "head dim %d (only 128)", p.D);
  if (p.block != MMI_BLOCK) fail(MMI_ERR_UNSUPPORTED, "block %d (only 64)", p.block);
  strides(p.q_stride_s, p.q_stride_h, p.Hq, "q");
  strides(p.k_stride_s, p.k_stride_h, p.Hkv, "k");
  double freq[D / 2];
  const double m = rope_freq(cfg, freq);
  const mmi_rope_cfg& c = *cfg;
  if (c.layout != MMI_ROPE_HALF && c.layout != MMI_ROPE_INTERLEAVED)
    fail(MMI_ERR_BAD_CONFIG, "unknown rope layout %d", c.layout);
  if (c.inverse != 0 && c.inverse != 1) fail(MMI_ERR_BAD_CONFIG, "inverse must be 0 or 1");
  if (c.reserved) fail(MMI_ERR_INVALID_ARG, "reserved must be 0");
  const int half = c.rot_dim / 2;
  int64_t sum = 0;
  for (int s : c.sections) {
    if (s < 0) fail(MMI_ERR_BAD_CONFIG, "a section is negative");
    sum += s;
  }
  if (sum != 0 && sum != half) fail(MMI_ERR_BAD_CONFIG, "sections add up to %lld of %d pairs", (long long)sum, half);
  if (!q && !k) fail(MMI_ERR_INVALID_ARG, "q and k are NULL");
  if (!q != !q_out || !k != !k_out) fail(MMI_ERR_INVALID_ARG, "an input without its output, or the other way round");
  if (q) { aligned(q, 16, "q"); aligned(q_out, 16, "q_out"); }
  if (k) { aligned(k, 16, "k"); aligned(k_out, 16, "k_out"); }
  if (pos) aligned(pos, 4, "pos");

  RopeArgs a{};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k;
  a.qo = (uint16_t*)q_out; a.ko = (uint16_t*)k_out;
  a.q_ss = p.q_stride_s; a.q_sh = p.q_stride_h; a.k_ss = p.k_stride_s; a.k_sh = p.k_stride_h;
  a.pos = pos;
  a.S = (int32_t)p.S;
  a.Hq = q ? p.Hq : 0;
  a.Hkv = k ? p.Hkv : 0;
  a.rot = c.rot_dim;
  a.inverse = c.inverse;
  a.sec1 = sum ? c.sections[0] : half;
  a.sec2 = sum ? c.sections[0] + c.sections[1] : half;
  a.m = (float)m;
  for (int i = 0; i < half; ++i) {
    // turns to 2^-63: a product of doubles alone would be off by up to 2^-53
    // of itself, which a far position multiplies. f <= 2^40, so the second
    // part stays below 2^50 in units of 2^-64.
    const double t = freq[i] * PER_TURN, rest = std::fma(freq[i], PER_TURN, -t) + freq[i] * PER_TURN_REST;
    const double part = t - std::floor(t);                   // exact, at most 1 - 2^-53
    a.turn[i] = (uint64_t)(part * 0x1p64) + (uint64_t)std::llrint(rest * 0x1p64);
  }
  return a;
}

CacheDev cache_dev(const mmi_cache* c) {
  if (!c) fail(MMI_ERR_INVALID_ARG, "cache is NULL");
  if (c->type < MMI_CACHE_BF16 || c->type > MMI_CACHE_FP4) fail(MMI_ERR_BAD_CONFIG, "unknown cache type %d", c->type);
  if (c->D != D) fail(MMI_ERR_UNSUPPORTED, "head dim %d (only 128)", c->D);
  int shift = 4;
  while (shift < 8 && (1 << shift) != c->page) ++shift;
  if ((1 << shift) != c->page) fail(MMI_ERR_UNSUPPORTED, "page of %d tokens (16, 32, 64, 128 or 256)", c->page);
  if (c->Hkv < 1) fail(MMI_ERR_INVALID_ARG, "head counts must be >= 1");
  if (c->Hkv > 1024) fail(MMI_ERR_UNSUPPORTED, "more than 1024 KV heads");
  if (c->n_pages < 1) fail(MMI_ERR_INVALID_ARG, "the cache has no pages");
  if (c->n_pages > 0x7fffffff) fail(MMI_ERR_UNSUPPORTED, "page numbers must fit 32 bits");
  CacheDev d{};
  d.shift = shift;
  d.Hkv = c->Hkv;
  d.n_pages = c->n_pages;
  const int64_t rows = (int64_t)c->Hkv * c->page, packed = rows * ROW_BYTES[c->type];
  d.page_stride = c->page_stride ? c->page_stride : packed;
  d.scale_stride = c->scale_stride ? c->scale_stride : rows * 4;
  if (d.page_stride < packed || d.page_stride % 16)
    fail(MMI_ERR_INVALID_ARG, "page_stride must be a multiple of 16 and hold a page");
  aligned(c->k, 16, "cache k");
  aligned(c->v, 16, "cache v");
  d.k = (uint8_t*)c->k;
  d.v = (uint8_t*)c->v;
  if (c->type != MMI_CACHE_BF16) {
    if (d.scale_stride < rows * 4 || d.scale_stride % 4)
      fail(MMI_ERR_INVALID_ARG, "scale_stride must be a multiple of 4 and hold a page");
    aligned(c->k_scale, 4, "cache k_scale");
    aligned(c->v_scale, 4, "cache v_scale");
    d.ks = (uint32_t*)c->k_scale;
    d.vs = (uint32_t*)c->v_scale;
  }
  if (d.page_stride > ((int64_t)1 << 40) || d.scale_stride > ((int64_t)1 << 40))
    fail(MMI_ERR_UNSUPPORTED, "page strides exceed 2^40 bytes");
  return d;
}

RowsArgs rows_args(const mmi_cache* c, const void* k, int64_t k_ss, int64_t k_sh, const void* v, int64_t v_ss,
                   int64_t v_sh, const int64_t* slot, int64_t n) {
  RowsArgs a{};
  a.c = cache_dev(c);
  if (n < 0) fail(MMI_ERR_INVALID_ARG, "negative number of rows");
  if (n > ((int64_t)1 << 26) / c->Hkv) fail(MMI_ERR_UNSUPPORTED, "more than 2^26 rows of all heads");
  strides(k_ss, k_sh, c->Hkv, "k");
  strides(v_ss, v_sh, c->Hkv, "v");
  if (n > 0) {                     // an empty call may have no arrays
    aligned(k, 16, "k");
    aligned(v, 16, "v");
    aligned(slot, 8, "slot");
  }
  a.k = (uint16_t*)k; a.v = (uint16_t*)v;
  a.k_ss = k_ss; a.k_sh = k_sh; a.v_ss = v_ss; a.v_sh = v_sh;
  a.slot = slot;
  a.n = n;
  return a;
}

mmi_tree tree_checked(const mmi_cache* c, const mmi_tree* tree) {
  if (!tree) fail(MMI_ERR_INVALID_ARG, "tree is NULL");
  mmi_tree t = *tree;
  if (t.n_seq < 0 || t.n_rows < 0) fail(MMI_ERR_INVALID_ARG, "negative number of sequences or rows");
  if (t.n_seq > 4096 || t.n_rows > (1 << 20)) fail(MMI_ERR_UNSUPPORTED, "more than 4096 sequences or 2^20 rows");
  if (t.Hq < 1) fail(MMI_ERR_INVALID_ARG, "head counts must be >= 1");
  if (t.Hq > 1024 || t.Hq % c->Hkv) fail(MMI_ERR_UNSUPPORTED, "Hq %% Hkv != 0 or more than 1024 query heads");
  if (t.max_rows < 1) fail(MMI_ERR_INVALID_ARG, "max_rows must be >= 1");
  if (t.max_rows > 256) fail(MMI_ERR_UNSUPPORTED, "more than 256 drafted tokens of a sequence");
  if (t.max_len < 0) fail(MMI_ERR_INVALID_ARG, "max_len is negative");
  if (t.max_len > LONGEST) fail(MMI_ERR_UNSUPPORTED, "max_len exceeds 2^30");
  if (t.max_pages < 0 || (int64_t)t.max_pages * c->page < t.max_len)
    fail(MMI_ERR_INVALID_ARG, "max_pages pages of %d tokens do not hold max_len", c->page);
  if (t.mask && t.mask_words < (t.max_rows + 63) / 64)
    fail(MMI_ERR_INVALID_ARG, "%d words of mask for %d drafted tokens", t.mask_words, t.max_rows);
  if (!(t.scale >= 0 && std::isfinite(t.scale * LOG2E))) fail(MMI_ERR_INVALID_ARG, "scale must be positive, or 0");
  if (t.reserved) fail(MMI_ERR_INVALID_ARG, "reserved must be 0");
  strides(t.q_stride_s, t.q_stride_h, t.Hq, "q");
  strides(t.k_stride_s, t.k_stride_h, c->Hkv, "k");
  strides(t.v_stride_s, t.v_stride_h, c->Hkv, "v");
  strides(t.o_stride_s, t.o_stride_h, t.Hq, "o");
  return t;
}

TreeArgs tree_args(const mmi_cache* c, const mmi_tree& t, const void* q, const void* k, const void* v, void* o,
                   float* lse) {
  TreeArgs a{};
  a.c = cache_dev(c);
  if (t.n_seq > 0 && t.n_rows > 0) {
    aligned(q, 16, "q"); aligned(k, 16, "k"); aligned(v, 16, "v"); aligned(o, 16, "o");
    aligned(t.row_start, 4, "row_start");
    aligned(t.length, 4, "length");
    if (t.max_len > 0) aligned(t.pages, 4, "pages");
    if (t.mask) aligned(t.mask, 8, "mask");
    if (lse) aligned(lse, 4, "lse");
  }
  a.q = {q, t.q_stride_s, t.q_stride_h};
  a.k = {k, t.k_stride_s, t.k_stride_h};
  a.v = {v, t.v_stride_s, t.v_stride_h};
  a.o = (uint16_t*)o;
  a.o_ss = t.o_stride_s; a.o_sh = t.o_stride_h;
  a.lse = lse;
  a.row_start = t.row_start; a.length = t.length; a.pages = t.pages;
  a.mask = (const uint32_t*)t.mask;
  a.n_seq = t.n_seq; a.n_rows = t.n_rows; a.g = t.Hq / c->Hkv;
  a.max_rows = t.max_rows; a.max_len = (int32_t)t.max_len; a.max_pages = t.max_pages; a.mask_words = t.mask_words;
  a.sc = (t.scale > 0 ? t.scale : 0.08838834764831845f) * LOG2E;   // finite, above zero
  return a;
}

}  // namespace mmi
