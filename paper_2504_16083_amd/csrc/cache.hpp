// Descriptors and launches of the operators around the prefill
// (include/mmi_cache.h): rotary positions, the paged cache, and the attention
// of drafted tokens over it. Host checks: cache.hip.
#pragma once

#include "../../include/mmi_cache.h"
#include "internal.hpp"

namespace mmi {

constexpr int GROUP = 32;          // channels of a quantised row that share a scale

// ---------------------------------------------------------------- k_rope.hip
struct RopeArgs {
  const uint16_t *q, *k;           // nullptr: left out
  uint16_t *qo, *ko;
  int64_t q_ss, q_sh, k_ss, k_sh;
  const int32_t* pos;              // [axes][S] or nullptr
  int32_t S, Hq, Hkv;
  int32_t rot, inverse;
  int32_t sec1, sec2;              // first pair of axis 1 and of axis 2 (rot / 2: none)
  float m;                         // factor of cos and sin
  uint64_t turn[D / 2];            // turns a position of every pair, modulo one, as 64-bit fractions
};
hipError_t launch_rope(const RopeArgs& a, int layout, hipStream_t st);

// --------------------------------------------------------------- k_cache.hip
struct CacheDev {
  uint8_t *k, *v;
  uint32_t *ks, *vs;               // four scale bytes a row
  int64_t page_stride, scale_stride;
  int64_t n_pages;
  int32_t shift, Hkv;              // page = 1 << shift
};
struct RowsArgs {
  CacheDev c;
  uint16_t *k, *v;
  int64_t k_ss, k_sh, v_ss, v_sh;
  const int64_t* slot;
  int64_t n;
};
hipError_t launch_cache_write(const RowsArgs& a, int type, hipStream_t st);
hipError_t launch_cache_read(const RowsArgs& a, int type, hipStream_t st);

// ---------------------------------------------------------------- k_tree.hip
struct TreeArgs {
  CacheDev c;
  Tensor q, k, v;
  uint16_t* o;
  int64_t o_ss, o_sh;
  float* lse;                      // [Hq][n_rows] or nullptr
  const int32_t *row_start, *length, *pages;
  const uint32_t* mask;            // rows of 2 * mask_words words, or nullptr
  int32_t n_seq, n_rows, g, max_rows, max_len, max_pages, mask_words;
  float sc;                        // scale of the scores times log2(e)
  int32_t target;                  // workgroups that a batch is cut into, if it is long enough
  int32_t items;                   // launched workgroups = partials the workspace holds
  int32_t cus;                     // compute units
  float* part_o;                   // [items][rows of a tile][128], sums over P as it entered the product
  float* part_ml;                  // [items][rows of a tile][4]: maximum (log2 units), sum of that P, fp32-P sum
  int32_t* rec;                    // [n_seq][2]: a sequence's first item and the chunks of its keys
};
struct TreeShape {                 // how a batch is cut, from its bounds alone
  int32_t rows;                    // query rows of a workgroup's tile
  int32_t target, items;
  size_t part_o, part_ml, rec, bytes;   // offsets into the workspace, and its size
};
TreeShape tree_shape(const mmi_tree& t, int Hkv, int type, int cus);
hipError_t launch_tree(const TreeArgs& a, int type, int rows, hipStream_t st);

// ---------------------------------------------------------------- cache.hip
// Host checks (they throw Error) and the records for the launches.
double rope_freq(const mmi_rope_cfg* cfg, double* freq);
RopeArgs rope_args(const mmi_problem& p, const mmi_rope_cfg* cfg, const int32_t* pos, const void* q, const void* k,
                   void* q_out, void* k_out);
CacheDev cache_dev(const mmi_cache* c);
RowsArgs rows_args(const mmi_cache* c, const void* k, int64_t k_ss, int64_t k_sh, const void* v, int64_t v_ss,
                   int64_t v_sh, const int64_t* slot, int64_t n);
mmi_tree tree_checked(const mmi_cache* c, const mmi_tree* t);   // strides filled in
TreeArgs tree_args(const mmi_cache* c, const mmi_tree& t, const void* q, const void* k, const void* v, void* o,
                   float* lse);

}  // namespace mmi
