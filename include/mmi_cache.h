/*
 * mmi_cache.h - the operators around the prefill of mmi.h: rotary positions
 * on Q and K before it, a paged cache that keeps K and V in 16, 8 or 4 bits
 * for the tokens that follow, and the attention of those tokens (one decoded
 * token a sequence, or a tree of drafted ones) over the cache.
 *
 * The conventions of mmi.h hold: status codes and mmi_last_error, device
 * pointers owned by the caller, work enqueued on the caller's stream, head
 * dimension 128, bfloat16 tensors [tokens][heads][128] with element strides
 * (0, 0 = packed; multiples of 8 elements), rows 16-byte aligned. Arguments
 * on the host are validated before the first launch. Every call takes a
 * context and runs on its device, whichever is current (that one is current
 * again afterwards). No call here allocates, synchronises or keeps state, so
 * each may be captured into a graph; host structures (configurations, the
 * strides and pointers of a cache or a batch) are read during the call only,
 * arrays named "device" when the work runs. Calls on several streams may
 * overlap as long as none writes what another one uses.
 */
#ifndef MMI_CACHE_H
#define MMI_CACHE_H

#include "mmi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------- rotary positions
 * Pair i of the first rot_dim channels of every row turns by the angle
 * a = position * f_i and is multiplied by attn_factor m:
 *   (x, y) -> (m (x cos a - y sin a), m (y cos a + x sin a)),
 * f_i = theta^(-2 i / rot_dim) radians a position, changed by `scaling`; the
 * other channels stay as they are. The angle of a position and of f_i as a
 * double (what mmi_rope_freq returns, or inv_freq) is held to 2^-25 of a turn
 * at any 32-bit position (64-bit fixed point); mmi_rope_freq's double is off
 * from the formula by up to (ln theta + 8) 2^-53 of itself, which a position p
 * multiplies. The products are taken in fp32 and rounded to bfloat16 once. */
#define MMI_ROPE_HALF 0          /* pair i = channels i and i + rot_dim / 2 */
#define MMI_ROPE_INTERLEAVED 1   /* pair i = channels 2 i and 2 i + 1 */

#define MMI_ROPE_SCALE_NONE 0
#define MMI_ROPE_SCALE_LINEAR 1  /* f / factor (position interpolation) */
#define MMI_ROPE_SCALE_NTK 2     /* theta * factor^(rot_dim / (rot_dim - 2)) in place of theta */
#define MMI_ROPE_SCALE_PARTS 3   /* by the turns t = orig_len f / (2 pi) of the original context (YaRN,
                                    arXiv 2309.00071): g = (t - beta_slow) / (beta_fast - beta_slow)
                                    clamped to [0, 1]; f (g + (1 - g) / factor) */

typedef struct mmi_rope_cfg {
  int32_t rot_dim;               /* rotated channels: a multiple of 16 in [16, 128] */
  int32_t layout;                /* MMI_ROPE_HALF or MMI_ROPE_INTERLEAVED */
  int32_t scaling;               /* MMI_ROPE_SCALE_* */
  int32_t inverse;               /* 1: angles negated, the factor m as before: the gradient of the
                                    rotation (and for m = 1 its inverse) */
  int32_t sections[3];           /* pairs, in order, that take their position from axis 0, 1 and 2 (the
                                    t, h, w of a video token), sum rot_dim / 2; 0, 0, 0: one axis */
  int32_t reserved;              /* 0 */
  double theta;                  /* > 0 */
  double factor;                 /* LINEAR, NTK, PARTS: >= 1 */
  double orig_len;               /* PARTS: > 0 */
  double beta_fast, beta_slow;   /* PARTS: beta_fast > beta_slow >= 0 */
  double attn_factor;            /* m > 0; 0: 0.1 ln(factor) + 1 for PARTS, else 1 */
  const double* inv_freq;        /* HOST array [rot_dim / 2] of f_i in [0, 2^40], in place of theta
                                    and scaling (factor still sets m of PARTS), or NULL */
} mmi_rope_cfg;

/* The frequencies f_i of a configuration (up to 2^40, else
 * MMI_ERR_BAD_CONFIG): HOST array [rot_dim / 2]. Computing
 * them takes longer than a short call's other host work; a program that calls
 * mmi_rope for single tokens keeps them in inv_freq. */
int mmi_rope_freq(const mmi_rope_cfg* cfg, double* inv_freq);

/* Rotates Q [S, Hq, 128] and K [S, Hkv, 128] of `prob` (its strides; v, o and
 * modality are not read) into q_out and k_out, laid out as q and k. q_out = q
 * or k_out = k rotates in place; otherwise an output overlaps no input. q or
 * k (with its output) may be NULL. pos: device int32 [S], or [3][S] with
 * sections; NULL: token x has position x (on every axis). */
int mmi_rope(mmi_ctx* ctx, const mmi_problem* prob, const mmi_rope_cfg* cfg, const int32_t* pos, const void* q,
             const void* k, void* q_out, void* k_out, void* stream);

/* ------------------------------------------------------------------ the cache
 * Pages of `page` tokens; k and v each hold [n_pages][Hkv][page] rows of 128
 * channels. A quantised row is four groups of 32 channels, each with a scale
 * 2^e of its own: e is the smallest integer >= -126 with max |x| <= M 2^e,
 * a channel's code the nearest value of the type to x 2^-e (ties to even),
 * its scale byte e + 127 (magnitudes that would round to 2^128 are cut to the
 * code below it). A group that holds an infinity or a NaN has scale
 * byte 255 and stands for NaN in all its channels. What a row stands for,
 * code times 2^e, is exact in bfloat16 (in a group that is zero or reaches
 * 2^-100): reading back adds no rounding. */
#define MMI_CACHE_BF16 0         /* 256 bytes a row, values as they are, no scales */
#define MMI_CACHE_FP8 1          /* 128 bytes: E4M3 codes, M = 448 */
#define MMI_CACHE_INT8 2         /* 128 bytes: two's complement codes, M = 127 */
#define MMI_CACHE_FP4 3          /* 64 bytes: E2M1 codes, M = 6; channel 2 i in the low half of byte i */

typedef struct mmi_cache {
  int32_t type;                  /* MMI_CACHE_* */
  int32_t page;                  /* tokens a page: 16, 32, 64, 128 or 256 */
  int32_t Hkv;
  int32_t D;                     /* must be 128 */
  int64_t n_pages;               /* >= 1 */
  void *k, *v;                   /* device, 16-byte aligned */
  void *k_scale, *v_scale;       /* device, 4-byte aligned: [n_pages][Hkv][page][4] scale bytes (BF16: unused) */
  int64_t page_stride;           /* bytes from page to page of k and v, a multiple of 16 (0: packed) */
  int64_t scale_stride;          /* the same of the scales, a multiple of 4 (0: packed) */
} mmi_cache;

/* Row i of k and v [n, Hkv, 128] goes to slot[i] = page number * page + place
 * in the page (device int64 [n]); rows whose slot lies outside the cache (-1,
 * the padding of a batch) go nowhere. Two rows of one call must not name the
 * same slot: what that slot then holds is undefined (the others are not
 * affected). Nothing but the named slots changes. n * Hkv <= 2^26. */
int mmi_cache_write(mmi_ctx* ctx, const mmi_cache* cache, const void* k, int64_t k_stride_s, int64_t k_stride_h,
                    const void* v, int64_t v_stride_s, int64_t v_stride_h, const int64_t* slot, int64_t n,
                    void* stream);

/* Rows i of k and v become what slot[i] stands for; zeros where the slot lies
 * outside the cache. Slots may repeat. n * Hkv <= 2^26. */
int mmi_cache_read(mmi_ctx* ctx, const mmi_cache* cache, const int64_t* slot, int64_t n, void* k, int64_t k_stride_s,
                   int64_t k_stride_h, void* v, int64_t v_stride_s, int64_t v_stride_h, void* stream);

/* ------------------------------------------------- drafted tokens over a cache
 * A batch of sequences, each with cached tokens (in the cache, in order of
 * the page table's pages) and drafted tokens: the rows of q, k, v and o.
 * Every drafted token sees all cached tokens of its sequence and the drafted
 * ones that its mask row names; one drafted token a sequence with mask NULL
 * is plain decoding. The drafted tokens' own K and V are read from k and v as
 * they are: those that are accepted go into the cache afterwards
 * (mmi_cache_write, the others' slots -1). */
typedef struct mmi_tree {
  int32_t n_seq;                 /* sequences, 0 .. 4096 */
  int32_t n_rows;                /* rows of q, k, v, o and mask, 0 .. 2^20 */
  int32_t Hq;                    /* query heads, a multiple of the cache's Hkv, at most 1024 */
  int32_t max_rows;              /* most drafted tokens of a sequence, 1 .. 256 */
  int64_t max_len;               /* most cached tokens of a sequence, 0 .. 2^30 */
  int32_t max_pages;             /* pages a row of the page table, max_pages * page >= max_len */
  int32_t mask_words;            /* 64-bit words a row of mask, at least max_rows / 64 rounded up */
  const int32_t* row_start;      /* device [n_seq + 1]: the rows of sequence b are row_start[b] up to
                                    row_start[b + 1], ascending; rows from row_start[n_seq] on (padding)
                                    are neither read nor written */
  const int32_t* length;         /* device [n_seq]: cached tokens */
  const int32_t* pages;          /* device [n_seq][max_pages]: page numbers; entries behind a sequence's
                                    last token are not read (NULL if max_len is 0) */
  const uint64_t* mask;          /* device [n_rows][mask_words]: bit j of a row: it sees drafted token j of
                                    its sequence (its own bit too). NULL: token i sees 0 .. i */
  int64_t q_stride_s, q_stride_h;  /* element strides; 0, 0 = packed */
  int64_t k_stride_s, k_stride_h;
  int64_t v_stride_s, v_stride_h;
  int64_t o_stride_s, o_stride_h;
  float scale;                   /* of the scores, > 0 (and below 2^127); 0: 1 / sqrt(128) */
  int32_t reserved;              /* 0 */
} mmi_tree;

/* Bytes of device workspace that a batch of these bounds needs; it depends on
 * the integers of `tree` and the cache's type and Hkv only. MMI_ERR_UNSUPPORTED for
 * bounds that ask for more than 2^22 workgroups. */
int mmi_tree_workspace(mmi_ctx* ctx, const mmi_cache* cache, const mmi_tree* tree, size_t* bytes);

/* o [n_rows, Hq, 128] = softmax(scale q k^T) v over the keys that a row sees,
 * scores and softmax in fp32; the weights enter the product with V in 15 bits
 * up to 32 rows a KV head (max_rows * Hq / Hkv), with more rounded to bfloat16
 * (8 bits); o rounded once; lse: device float [Hq][n_rows] natural-log sums, or NULL. A
 * row that sees no key gets o = 0 and lse = -inf. A drafted token that a row
 * does not see has no part in it, whatever its K and V hold (infinities and
 * NaN too). In what a row sees an infinity or a NaN of V acts by the formula,
 * but that weights under 2^-126 of the row's largest may be 0 (times an
 * infinity: NaN). Query head h reads KV head h / (Hq / Hkv). o must not overlap an
 * input. workspace: 16-byte aligned device memory of at least
 * mmi_tree_workspace bytes; its contents do not matter before and after, but
 * calls (and replays of captured ones) that may run at the same time need one
 * each. The device arrays are not trusted with addresses: lengths are cut to
 * [0, max_len], a sequence's rows to [0, n_rows) and its first max_rows (the
 * rest is left as it was), and the tokens of a page whose number lies outside
 * the cache are seen by no row. */
int mmi_tree_attention(mmi_ctx* ctx, const mmi_cache* cache, const mmi_tree* tree, const void* q, const void* k,
                       const void* v, void* o, float* lse, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MMI_CACHE_H */
