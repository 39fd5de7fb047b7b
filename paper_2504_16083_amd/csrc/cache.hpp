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
  int32_t items;                   // launched workgroups
  int32_t parts;                   // partials that the workspace holds
  int32_t cus;                     // compute units
  float* part_o;                   // [parts][rows of a tile][128], sums over P as it entered the product
  float* part_ml;                  // [parts][rows of a tile][4]: maximum (log2 units), sum of that P, fp32-P sum
  int32_t* rec;                    // [n_seq][2]: place of a sequence's first partial, and the chunks of its keys
};
struct TreeShape {                 // how a batch is cut, from its bounds alone
  int32_t rows;                    // query rows of a workgroup's tile
  int32_t target, items, parts;
  size_t part_o, part_ml, rec, bytes;   // offsets into the workspace, and its size
};
TreeShape tree_shape(const mmi_tree& t, int Hkv, int type, int cus);
hipError_t launch_tree(const TreeArgs& a, int type, int rows, hipStream_t st);

// How the device cuts a batch. The chunk length follows from the work of the
// whole batch (cached tokens x tiles x heads, cut into `target` parts), so long
// sequences get many chunks and short ones few, whatever the bounds were. The
// last chunks are shorter than the others, so that there are more items than
// parts; as `target` of them run at once, the chunks are then made longer
// until all start together (a second round of a few items takes as long as
// the first: a ragged batch of 32 decoded tokens took 74 us for 65).
constexpr int CHUNK = 128;         // chunks are multiples of a step of the four waves
constexpr int64_t LONGEST = 1 << 30;   // cached tokens a sequence, and so a chunk: a multiple of CHUNK

// No chunk is longer than a sequence may be: work / parts alone can be the
// tokens of all sequences, more than 31 bits hold.
__host__ __device__ inline int chunk_of(int64_t work, int64_t parts) {
  const int64_t len = work < (1 << 30) ? ((int)work + (int)parts - 1) / (int)parts : (work + parts - 1) / parts;
  return ((int)(len < 1 ? 1 : len < LONGEST ? len : LONGEST) + CHUNK - 1) / CHUNK * CHUNK;
}

// Chunks of a sequence of L tokens; the sum stays below 2^31.
__host__ __device__ inline int chunks_of(int L, int chunk) { return L > chunk ? (L + chunk - 1) / chunk : 1; }

// Chunk of a batch with this work (cached tokens x tiles) and these tiles;
// count(chunk): its tiles x chunks.
template <typename F>
__host__ __device__ inline int choose_chunk(int64_t work, int64_t tiles, int Hkv, int target, F&& count) {
  work *= Hkv;
  const int chunk = chunk_of(work, target);
  const int64_t items = count(chunk) * Hkv, units = tiles * Hkv;
  if (items <= target || units >= target) return chunk;
  // at most units + work / chunk items: the second length always fits
  const int64_t fewer = target * (int64_t)target / items;
  const int longer = chunk_of(work, fewer > 1 ? fewer : 1);
  const int safe = chunk_of(work, target - units);
  return longer < safe && count(longer) * Hkv <= target ? longer : safe;
}

// ---------------------------------------------------------------- cache.hip
// Host checks (they throw Error) and the records for the launches.
double rope_freq(const mmi_rope_cfg* cfg, double* freq);
RopeArgs rope_args(const mmi_problem* prob, const mmi_rope_cfg* cfg, const int32_t* pos, const void* q, const void* k,
                   void* q_out, void* k_out);
CacheDev cache_dev(const mmi_cache* c);
RowsArgs rows_args(const mmi_cache* c, const void* k, int64_t k_ss, int64_t k_sh, const void* v, int64_t v_ss,
                   int64_t v_sh, const int64_t* slot, int64_t n);
mmi_tree tree_checked(const mmi_cache* c, const mmi_tree* t);   // strides filled in
TreeArgs tree_args(const mmi_cache* c, const mmi_tree& t, const void* q, const void* k, const void* v, void* o,
                   float* lse);

}  // namespace mmi
