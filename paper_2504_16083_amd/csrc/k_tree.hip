// Attention of drafted tokens over the paged cache (include/mmi_cache.h).
//
// The query rows of a KV head are (drafted token, query head of its group):
// row r of sequence b is token r / g, head r % g. A workgroup takes a tile of
// them and a chunk of the sequence's cached tokens; the last chunk takes the
// drafted tokens too. Every type is turned into bfloat16 on the way to the
// matrix cores; a row keeps an online softmax over blocks of 32 keys:
//   S^T (keys x rows) = K Q^T, P = 2^(S - m) with a running maximum m,
//   O^T (128 x rows) += V^T P^T, sums of P in fp32.
// S^T has one row a lane, so P is already the operand of the second product
// (the keys of its contraction in the order that the lanes hold them).
// Up to 32 rows a head the cache's bytes bound the work (k_tree_few), with
// more the products (k_tree_wide). A sequence of several chunks leaves
// partials that k_tree_join merges in a fixed order.
#include <algorithm>
#include <type_traits>

#include "cache.hpp"
#include "codec.hpp"

namespace mmi {

#define INLINE __attribute__((always_inline))   // of lambdas: called twice they would become functions of memory

constexpr int KB = 32;                 // keys of a block
constexpr int TK = 136, TV = 160;      // bf16 a staged K / V row: operand reads without bank conflicts
constexpr int OP = 132;                // floats a row of the join buffer
constexpr float SLACK = 8.0f;          // the maximum moves when a block's passes it by this (log2 units)

typedef __attribute__((address_space(3))) bf16x4 lds4;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

struct Seq {
  int row0, T, L;                      // first row, drafted tokens, cached tokens
};

__device__ __forceinline__ Seq sequence(const TreeArgs& a, int b) {
  Seq s;
  s.row0 = clampi(a.row_start[b], 0, a.n_rows);
  s.T = clampi(a.row_start[b + 1], s.row0, min(a.n_rows, s.row0 + a.max_rows)) - s.row0;
  s.L = clampi(a.length[b], 0, a.max_len);
  return s;
}

// Between one lane's LDS accesses and another's of the same wave: the wave's
// are done in order, the compiler must keep that order.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Sum over the workgroup's NT threads, and the sum before this thread.
template <int NT>
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* before, int64_t* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == 63) sh[wave] = s;
  __syncthreads();
  int64_t base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) base += sh[w];
    all += sh[w];
  }
  *before = base + s - x;
  return all;
}

struct Item {
  int b, first, chunks, chunk, tile, head;   // sequence, its first item, its chunks; this one's chunk, tile, head
  int part;                                  // place of its partial, if the sequence is cut
  int c0, c1;                                // cached tokens
  Seq seq;
};

template <int ROWS>
__device__ __forceinline__ int tiles_of(const TreeArgs& a, const Seq& s) { return (s.T * a.g + ROWS - 1) / ROWS; }

// first, part: items of the sequences before it, and those of them that are cut.
__device__ __forceinline__ void set_item(const TreeArgs& a, Item& r, int it, int b, int first, int part, int tiles,
                                         int chunk, const Seq& s) {
  const int at = it - first;
  r.b = b;
  r.first = first;
  r.part = part + at;
  r.seq = s;
  r.chunks = chunks_of(s.L, chunk);
  r.chunk = at / (tiles * a.c.Hkv);
  const int rest = at - r.chunk * tiles * a.c.Hkv;
  r.head = rest / tiles;
  r.tile = rest - r.head * tiles;
  r.c0 = min(s.L, r.chunk * chunk);
  r.c1 = (int)min((int64_t)s.L, (int64_t)r.c0 + chunk);
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// Item `it` of the batch. Up to 64 sequences every wave finds it by itself, a
// sequence a lane; more are scanned by the workgroup, NT at a time.
template <int ROWS, int NT>
__device__ __forceinline__ bool find_item(const TreeArgs& a, int it, Item& r, int64_t* sh64, int* sh) {
  const int tid = threadIdx.x;
  if (a.n_seq == 1) {
    const Seq s = sequence(a, 0);
    const int tiles = tiles_of<ROWS>(a, s);
    auto count = [&](int chunk) -> int64_t { return (int64_t)tiles * chunks_of(s.L, chunk); };
    const int chunk = choose_chunk((int64_t)tiles * s.L, tiles, a.c.Hkv, a.target, count);
    if (it >= count(chunk) * a.c.Hkv) return false;
    set_item(a, r, it, 0, 0, 0, tiles, chunk, s);
  } else if (a.n_seq <= 64) {
    const int lane = tid & 63;
    Seq s = {0, 0, 0};
    if (lane < a.n_seq) s = sequence(a, lane);
    const int tiles = tiles_of<ROWS>(a, s);
    int64_t work = (int64_t)tiles * s.L;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) work += __shfl_xor(work, d);
    // fewer than 2^31 items: each has a workgroup
    auto count = [&](int chunk) -> int64_t { return wave_sum(tiles * chunks_of(s.L, chunk)); };
    const int chunk = choose_chunk(work, wave_sum(tiles), a.c.Hkv, a.target, count);
    const int n = tiles * a.c.Hkv * chunks_of(s.L, chunk), cut = s.L > chunk ? n : 0;
    int end = n, parts = cut;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(end, d), z = __shfl_up(parts, d);
      if (lane >= d) {
        end += y;
        parts += z;
      }
    }
    const uint64_t mine = __ballot(it >= end - n && it < end);
    if (!mine) return false;
    const int b = __builtin_ctzll(mine);
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, b); };
    const Seq sb = {of(s.row0), of(s.T), of(s.L)};
    set_item(a, r, it, b, of(end - n), of(parts - cut), of(tiles), chunk, sb);
  } else {
    int64_t work = 0, tiles = 0, before;
    for (int b = tid; b < a.n_seq; b += NT) {
      const Seq s = sequence(a, b);
      work += (int64_t)tiles_of<ROWS>(a, s) * s.L;
      tiles += tiles_of<ROWS>(a, s);
    }
    work = block_scan<NT>(work, &before, sh64);
    tiles = block_scan<NT>(tiles, &before, sh64);
    auto count = [&](int chunk) -> int64_t {
      int64_t n = 0, bef;
      for (int b = tid; b < a.n_seq; b += NT) {
        const Seq s = sequence(a, b);
        n += (int64_t)tiles_of<ROWS>(a, s) * chunks_of(s.L, chunk);
      }
      return block_scan<NT>(n, &bef, sh64);
    };
    const int chunk = choose_chunk(work, tiles, a.c.Hkv, a.target, count);
    if (tid == 0) sh[0] = -1;
    uint64_t base = 0;                     // items in the lower half, those of cut sequences in the upper one
    for (int b0 = 0; b0 < a.n_seq && (uint32_t)base <= (uint32_t)it; b0 += NT) {
      const int b = b0 + tid;
      Seq s = {0, 0, 0};
      if (b < a.n_seq) s = sequence(a, b);
      const uint32_t n = tiles_of<ROWS>(a, s) * a.c.Hkv * chunks_of(s.L, chunk);
      const int64_t all = block_scan<NT>((int64_t)(s.L > chunk ? (uint64_t)n << 32 | n : n), &before, sh64);
      const uint64_t at = base + (uint64_t)before;
      if ((uint32_t)it >= (uint32_t)at && (uint32_t)it < (uint32_t)at + n) {
        sh[0] = b;
        sh[1] = (int)(uint32_t)at;
        sh[2] = (int)(at >> 32);
      }
      base += (uint64_t)all;
    }
    __syncthreads();
    const int b = __builtin_amdgcn_readfirstlane(sh[0]);
    if (b < 0) return false;
    const Seq s = sequence(a, b);
    set_item(a, r, it, b, __builtin_amdgcn_readfirstlane(sh[1]), __builtin_amdgcn_readfirstlane(sh[2]),
             tiles_of<ROWS>(a, s), chunk, s);
  }
  // the same in every lane: into scalar registers, or every branch on them is a divergent one
  for (int* x : {&r.b, &r.first, &r.part, &r.chunks, &r.chunk, &r.tile, &r.head, &r.c0, &r.c1, &r.seq.row0, &r.seq.T, &r.seq.L})
    *x = __builtin_amdgcn_readfirstlane(*x);
  if (it == r.first && tid == 0) {         // for the join
    a.rec[2 * r.b] = r.part;
    a.rec[2 * r.b + 1] = r.chunks;
  }
  return r.chunks == 1 || (uint32_t)r.part < (uint32_t)a.parts;   // always: see tree_shape
}

// One 16-byte piece as bfloat16 into a staged row.
template <int TYPE>
__device__ __forceinline__ void put_piece(uint16_t* to, u32x4 w, uint32_t scales, int piece) {
  if constexpr (TYPE == MMI_CACHE_BF16) {
    *reinterpret_cast<u32x4*>(to + piece * 8) = w;
  } else {
    const float s = scale_value(scales >> (TYPE == MMI_CACHE_FP4 ? 8 * piece : 8 * (piece >> 1)) & 255);
    if constexpr (TYPE == MMI_CACHE_FP4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<bf16x8*>(to + piece * 32 + 8 * e) = decode4(w[e], s);
    } else {
      *reinterpret_cast<bf16x8*>(to + piece * 16) = decode8<TYPE>(w[0], w[1], s);
      *reinterpret_cast<bf16x8*>(to + piece * 16 + 8) = decode8<TYPE>(w[2], w[3], s);
    }
  }
}

// Bits of the eight bfloat16 in w that are an infinity or a NaN, as a word of
// eight flags; `keep` gets w with those set to zero.
__device__ __forceinline__ bool not_finite(u32x4 w, u32x4& keep) {
  bool any = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
    any |= lo | hi;
    keep[e] = (lo ? 0u : w[e] & 0xffffu) | (hi ? 0u : w[e] & 0xffff0000u);
  }
  return any;
}

struct Rows {                          // a wave's 32 rows
  f32x16 o[4];
  bf16x8 q[8];
  float m, l, lo;                      // maximum (log2 units) of a row; sums of this lane's P (fp32, bf16)
  float base, most;                    // m, or 0 while it is -inf; what a unit's sum may be before m has to move
};

__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ bf16x8 v_operand(const uint16_t* v, int vlane, int half, int dt) {
  const uint16_t* p = v + vlane + 16 * half * TV + 32 * dt;
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p + 8 * TV));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16e2;

// Drafted keys d0 .. d0 + 31 that a row of token `tok` sees.
__device__ __forceinline__ uint32_t seen_drafts(const TreeArgs& a, const Seq& sq, int tok, int d0) {
  const uint32_t seen = sq.T - d0 >= KB ? 0xffffffffu : (1u << (sq.T - d0)) - 1;
  if (a.mask) return seen & a.mask[(int64_t)(sq.row0 + min(tok, sq.T - 1)) * (2 * a.mask_words) + (d0 >> 5)];
  const int n = tok + 1 - d0;                // keys d0 .. tok
  return seen & (n >= KB ? 0xffffffffu : n > 0 ? (1u << n) - 1 : 0u);
}

// Infinities and NaN in the V of drafted keys reach only the rows that see
// them (a product over the block would spread them as 0 x inf): the block was
// staged without them, and here what they add is found from products of 0/1
// flags, of the rows that see a key and of the channels where it holds +inf
// (what 0), -inf (1) or a NaN (2). v: V of the block's first key, n: its keys.
__device__ __forceinline__ void flag_not_finite(uint16_t* flags, const uint16_t* v, int64_t ss, int n, int what,
                                                int lane) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(v + (int64_t)min(4 * i + lane / 16, n - 1) * ss + lane % 16 * 8);
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t f = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t u = raw[e] >> (16 * s) & 0xffff;
        const bool hit = what == 2 ? (u & 0x7fff) > 0x7f80 : u == (what ? 0xff80u : 0x7f80u);
        f |= hit ? 0x3f80u << (16 * s) : 0u;
      }
      w[e] = f;
    }
    *reinterpret_cast<u32x4*>(flags + (4 * i + lane / 16) * TV + lane % 16 * 8) = w;
  }
}

__device__ __forceinline__ void add_not_finite(f32x16 (&o)[4], uint16_t* flags, const uint16_t* v, int64_t ss, int n,
                                               uint32_t seen, int h, int vlane, int lane) {
  bf16x8 sees[2];
#pragma unroll
  for (int x = 0; x < 16; ++x)
    sees[x >> 3][x & 7] = (__bf16)((seen >> (8 * (x >> 2) + 4 * h + (x & 3)) & 1) ? 1.0f : 0.0f);
  for (int what = 0; what < 3; ++what) {
    flag_not_finite(flags, v, ss, n, what, lane);
    wave_fence();
    const float add = what == 2 ? __uint_as_float(0x7fc00000u) : what ? -INFINITY : INFINITY;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      f32x16 c = {};
#pragma unroll
      for (int half = 0; half < 2; ++half) c = mfma32(v_operand(flags, vlane, half, dt), sees[half], c);
#pragma unroll
      for (int x = 0; x < 16; ++x) o[dt][x] += c[x] > 0.0f ? add : 0.0f;
    }
    wave_fence();
  }
}

// ------------------------------------------------------------------ few rows
// Up to 32 rows: RN tiles of 16. The four waves of a workgroup split the keys:
// each takes every fourth block of 32 and shares nothing until the end, so the
// loop has no barrier. The MFMAs are 16x16x32 (a decoded token with its 4 to
// 16 query heads fills a third of a 32-wide tile at most): lane (r = l % 16,
// q = l / 16) holds row r of an operand and 8 of its 32 contracted entries.
// K comes from the cache straight into that layout (64 contiguous bytes of a
// row a load; which channels an MFMA contracts does not matter, Q follows);
// only V goes through LDS, to be read transposed. Two or three workgroups a
// compute unit (tree_shape) keep about 100 KB of loads in flight. One token
// over 524288, 32 heads on 8: bfloat16 364 us (5.9 TB/s of cache), E4M3 201
// (5.5), int8 229 (4.9), E2M1 121 (4.7); two tiles, 4 drafts of 7 heads a KV
// head over 262144: 121 to 125 us (4.3), 59 (4.7), 80 (3.5), 52 (2.7). The
// smaller types wait for the vector ALU that decodes them and, with two tiles,
// makes the weights of 32 rows for each of their bytes.
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// First channel of lane group q's eight in MFMA x of QK.
template <int TYPE>
__device__ __forceinline__ int channel(int x, int q) {
  return TYPE == MMI_CACHE_BF16 ? 32 * x + 8 * q : TYPE == MMI_CACHE_FP4 ? 32 * q + 8 * x : 64 * (x >> 1) + 16 * q + 8 * (x & 1);
}

template <int TYPE>
struct Raw32 {                                        // a block of 32 keys as it lies in the cache
  static constexpr int KN = Codec<TYPE>::ROW / 64;    // K pieces of a lane and tile of 16 keys
  static constexpr int CPR = Codec<TYPE>::ROW / 16, RP = 64 / CPR, N = KB / RP;   // V: piece i = key i * RP + lane / CPR
  u32x4 k[2][KN], v[N];
  uint32_t ks[2], vs[N];
  uint32_t seen;                                      // keys that exist
};

// Numbers of the two pages (16 keys each) of the block from token t on, read a
// block before its loads: they wait for nothing then. `zero` in a vector
// register keeps these vector loads, whose counter the LDS reads do not share.
__device__ __forceinline__ void block_pages(int (&p)[2], const TreeArgs& a, const int32_t* pages, int t, int len,
                                            int zero) {
#pragma unroll
  for (int half = 0; half < 2; ++half) p[half] = pages[(min(t + 16 * half, len - 1) >> a.c.shift) + zero];
}

template <int TYPE>
__device__ __forceinline__ void load_block(Raw32<TYPE>& r, const TreeArgs& a, const int (&pages)[2], int head, int t0,
                                           int len, int lane) {
  typedef Raw32<TYPE> R;
  r.seen = len - t0 >= KB ? 0xffffffffu : (1u << (len - t0)) - 1;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int t = t0 + 16 * half, p = __builtin_amdgcn_readfirstlane(pages[half]);
    const bool ok = (uint32_t)p < (uint64_t)a.c.n_pages;
    if (!ok) r.seen &= half ? 0x0000ffffu : 0xffff0000u;
    const int64_t page = ok ? p : 0;
    const int64_t in = ((int64_t)head << a.c.shift) + (t & ((1 << a.c.shift) - 1));
    const uint8_t* kp = a.c.k + page * a.c.page_stride + in * Codec<TYPE>::ROW;
    const uint8_t* vp = a.c.v + page * a.c.page_stride + in * Codec<TYPE>::ROW;
#pragma unroll
    for (int j = 0; j < R::KN; ++j)
      r.k[half][j] = *reinterpret_cast<const u32x4*>(kp + (lane & 15) * Codec<TYPE>::ROW + 64 * j + 16 * (lane >> 4));
#pragma unroll
    for (int i = half * R::N / 2; i < (half + 1) * R::N / 2; ++i)
      r.v[i] = *reinterpret_cast<const u32x4*>(vp + ((i - half * R::N / 2) * R::RP * R::CPR + lane) * 16);
    if constexpr (Codec<TYPE>::SCALED) {
      const uint32_t* ks = (const uint32_t*)((const uint8_t*)a.c.ks + page * a.c.scale_stride) + in;
      const uint32_t* vs = (const uint32_t*)((const uint8_t*)a.c.vs + page * a.c.scale_stride) + in;
      r.ks[half] = ks[lane & 15];
#pragma unroll
      for (int i = half * R::N / 2; i < (half + 1) * R::N / 2; ++i)
        r.vs[i] = vs[(i - half * R::N / 2) * R::RP + lane / R::CPR];
    }
  }
}

// V of the block, transposed on the way out: [key][TV].
template <int TYPE>
__device__ __forceinline__ void stage_v(uint16_t* v, const Raw32<TYPE>& r, int lane) {
  typedef Raw32<TYPE> R;
#pragma unroll
  for (int i = 0; i < R::N; ++i) {
    const int key = i * R::RP + lane / R::CPR;
    // a key that does not exist weighs nothing, whatever its place in the page holds
    const bool ok = r.seen >> key & 1;
    const u32x4 none = {};
    put_piece<TYPE>(v + key * TV, ok ? r.v[i] : none, ok ? r.vs[i] : 0u, lane % R::CPR);
  }
}

// The K operands of one tile of 16 keys.
template <int TYPE>
__device__ __forceinline__ void k_operands(bf16x8 (&op)[4], const Raw32<TYPE>& r, int half, int q) {
  if constexpr (TYPE == MMI_CACHE_BF16) {
#pragma unroll
    for (int x = 0; x < 4; ++x) op[x] = __builtin_bit_cast(bf16x8, r.k[half][x]);
  } else if constexpr (TYPE == MMI_CACHE_FP4) {
    const float s = scale_value(r.ks[half] >> (8 * q) & 255);
#pragma unroll
    for (int x = 0; x < 4; ++x) op[x] = decode4(r.k[half][0][x], s);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float s = scale_value(r.ks[half] >> (8 * (2 * j + (q >> 1))) & 255);
      op[2 * j] = decode8<TYPE>(r.k[half][j][0], r.k[half][j][1], s);
      op[2 * j + 1] = decode8<TYPE>(r.k[half][j][2], r.k[half][j][3], s);
    }
  }
}

template <int RN>
struct FewRows {                       // a wave's RN tiles of 16 rows
  f32x4 o[RN][8];
  bf16x8 q[RN][4];
  float m[RN], l[RN];                  // maximum (log2 units) of a row; sum of this lane's P
};

__device__ __forceinline__ float group_max(float x) {   // over the four lane groups
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

__device__ __forceinline__ bf16x8 v_operand16(const uint16_t* v, int vlane, int dt) {
  const uint16_t* p = v + vlane + 16 * dt;
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p + 16 * TV));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Scores of the block (s[n][half]: keys 16 half + 4 q + i) and the staged V
// against the wave's rows; bit k of seen[n]: this lane's row sees key k.
// P enters the product in two bfloat16 pieces that hold 15 bits of it: its
// first 8 bits, cut, and what is left plus 2^-17 of it (in all weights alike;
// without it the rest might be 0, and meet an infinity in V). Rounded to one
// piece, O was off by up to 2^-8 of the spread of V. The matrix cores have
// the time, the vector ALU has it but for the small types: one token over
// 524288, 32 heads on 8, bfloat16 365 us for 364 with one piece, E4M3 200 for
// 200, int8 229 for 224, E2M1 121 for 115; 4 drafts of 7 heads a KV head over
// 262144 125 for 124, 59 for 58, 80 for 75 and 52 for 47.
template <int RN>
__device__ __forceinline__ void attend_few(FewRows<RN>& r, f32x4 (&s)[RN][2], const uint16_t* v,
                                           const uint32_t (&seen)[RN], float sc, int q, int vlane) {
  bf16x8 p[RN], rest[RN];
#pragma unroll
  for (int n = 0; n < RN; ++n) {
    if (__any(seen[n] != 0xffffffffu)) {
      const uint32_t mine = seen[n] >> (4 * q);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (!(mine >> (16 * (x >> 2) + (x & 3)) & 1)) s[n][x >> 2][x & 3] = -INFINITY;
    }
    float mx = s[n][0][0];
#pragma unroll
    for (int x = 1; x < 8; ++x) mx = fmaxf(mx, s[n][x >> 2][x & 3]);
    mx = group_max(mx) * sc;                 // sc > 0
    if (__any(mx > r.m[n] + SLACK)) {
      const float m = fmaxf(r.m[n], mx), alpha = r.m[n] == m ? 1.0f : fast_exp2(r.m[n] - m);
      r.m[n] = m;
      r.l[n] *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int x = 0; x < 4; ++x) r.o[n][dt][x] *= alpha;
    }
    const float base = r.m[n] == -INFINITY ? 0.0f : r.m[n];   // nothing seen yet: every P is 2^-inf = 0
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float e = fast_exp2(fmaf(s[n][x >> 2][x & 3], sc, -base));
      r.l[n] += e;
      const uint32_t top = __float_as_uint(e) & 0xffff0000u;
      p[n][x] = __builtin_bit_cast(__bf16, (uint16_t)(top >> 16));
      rest[n][x] = (__bf16)fmaf(e, 1.0f + 0x1p-17f, -__uint_as_float(top));
    }
  }
#pragma unroll
  for (int dt = 0; dt < 8; ++dt) {
    const bf16x8 av = v_operand16(v, vlane, dt);
#pragma unroll
    for (int n = 0; n < RN; ++n) r.o[n][dt] = mfma16(av, rest[n], mfma16(av, p[n], r.o[n][dt]));
  }
}

// Infinities and NaN in the V of drafted keys, as in add_not_finite.
template <int RN>
__device__ __forceinline__ void add_not_finite_few(FewRows<RN>& r, uint16_t* flags, const uint16_t* v, int64_t ss,
                                                   int n, const uint32_t (&seen)[RN], int q, int vlane, int lane) {
  bf16x8 sees[RN];
#pragma unroll
  for (int t = 0; t < RN; ++t)
#pragma unroll
    for (int x = 0; x < 8; ++x) sees[t][x] = (__bf16)((seen[t] >> (16 * (x >> 2) + 4 * q + (x & 3)) & 1) ? 1.0f : 0.0f);
  for (int what = 0; what < 3; ++what) {
    flag_not_finite(flags, v, ss, n, what, lane);
    wave_fence();
    const float add = what == 2 ? __uint_as_float(0x7fc00000u) : what ? -INFINITY : INFINITY;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const bf16x8 av = v_operand16(flags, vlane, dt);
#pragma unroll
      for (int t = 0; t < RN; ++t) {
        f32x4 c = {};
        c = mfma16(av, sees[t], c);
#pragma unroll
        for (int x = 0; x < 4; ++x) r.o[t][dt][x] += c[x] > 0.0f ? add : 0.0f;
      }
    }
    wave_fence();
  }
}

template <int TYPE, int RN>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RN == 1 ? 3 : 2))) void k_tree_few(TreeArgs a) {
  constexpr int ROWS = 16 * RN;
  // V blocks of the four waves; at the end their O, a tile of 16 rows at a time
  __shared__ __align__(16) uint16_t vs[4 * KB * TV];
  static_assert(sizeof(vs) >= 4 * 16 * OP * sizeof(float), "the join buffer lies in the V blocks");
  __shared__ __align__(8) float ml[4][ROWS][2];
  __shared__ int64_t sh64[4];
  __shared__ int sh[8];
  Item it;
  if (!find_item<ROWS, 256>(a, blockIdx.x, it, sh64, sh)) return;
  const Seq sq = it.seq;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int c = lane & 15, q = lane >> 4;
  uint16_t* const v = vs + wave * KB * TV;
  // transpose-read source of this lane in a staged V block: in each 16-lane
  // group, output lane i, element e is element i % 4 of the 8 bytes addressed
  // by lane 4 e + i / 4
  const int vlane = (4 * q + (c >> 2)) * TV + 4 * (c & 3);

  FewRows<RN> r;
  int tok[RN];
#pragma unroll
  for (int n = 0; n < RN; ++n) {
    const int row = it.tile * ROWS + 16 * n + c;
    tok[n] = row / a.g;
    const bool live = tok[n] < sq.T;
    const uint16_t* qp = (const uint16_t*)a.q.p + (int64_t)(sq.row0 + (live ? tok[n] : 0)) * a.q.ss +
                         (int64_t)(it.head * a.g + (live ? row - tok[n] * a.g : 0)) * a.q.sh;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const bf16x8 y = load16(qp + channel<TYPE>(x, q));
      r.q[n][x] = live ? y : zero8();
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) r.o[n][dt] = f32x4{};
    r.m[n] = -INFINITY;
    r.l[n] = 0.0f;
  }

  const int32_t* pages = a.pages + (int64_t)it.b * a.max_pages;
  Raw32<TYPE> raw;
  int pid[2], zero = 0;
  asm("" : "+v"(zero));
  int t0 = it.c0 + KB * wave;
  if (t0 < it.c1) {
    block_pages(pid, a, pages, t0, it.c1, zero);
    load_block<TYPE>(raw, a, pid, it.head, t0, it.c1, lane);
    block_pages(pid, a, pages, t0 + 4 * KB, it.c1, zero);
  }
  for (; t0 < it.c1; t0 += 4 * KB) {
    uint32_t seen[RN];
#pragma unroll
    for (int n = 0; n < RN; ++n) seen[n] = raw.seen;
    stage_v<TYPE>(v, raw, lane);
    f32x4 s[RN][2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      bf16x8 op[4];
      k_operands<TYPE>(op, raw, half, q);
#pragma unroll
      for (int n = 0; n < RN; ++n) {
        s[n][half] = f32x4{};
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][half] = mfma16(op[x], r.q[n][x], s[n][half]);
      }
    }
    if (t0 + 4 * KB < it.c1) {
      load_block<TYPE>(raw, a, pid, it.head, t0 + 4 * KB, it.c1, lane);
      block_pages(pid, a, pages, t0 + 8 * KB, it.c1, zero);
    }
    wave_fence();
    attend_few<RN>(r, s, v, seen, a.sc, q, vlane);
    wave_fence();
  }
  if (it.chunk == it.chunks - 1) {
    const uint16_t* kb = (const uint16_t*)a.k.p + (int64_t)sq.row0 * a.k.ss + (int64_t)it.head * a.k.sh;
    const uint16_t* vb = (const uint16_t*)a.v.p + (int64_t)sq.row0 * a.v.ss + (int64_t)it.head * a.v.sh;
    for (int d0 = KB * wave; d0 < sq.T; d0 += 4 * KB) {
      uint64_t odd = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = 4 * i + lane / 16;
        const u32x4 raw_v = *reinterpret_cast<const u32x4*>(vb + (int64_t)min(d0 + key, sq.T - 1) * a.v.ss + lane % 16 * 8);
        u32x4 keep;
        const u32x4 none = {};
        odd |= __ballot(not_finite(raw_v, keep));
        *reinterpret_cast<u32x4*>(v + key * TV + lane % 16 * 8) = d0 + key < sq.T ? keep : none;
      }
      f32x4 s[RN][2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint16_t* kp = kb + (int64_t)min(d0 + 16 * half + c, sq.T - 1) * a.k.ss;
#pragma unroll
        for (int n = 0; n < RN; ++n) s[n][half] = f32x4{};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const bf16x8 op = load16(kp + channel<TYPE>(x, q));
#pragma unroll
          for (int n = 0; n < RN; ++n) s[n][half] = mfma16(op, r.q[n][x], s[n][half]);
        }
      }
      uint32_t seen[RN];
#pragma unroll
      for (int n = 0; n < RN; ++n) seen[n] = seen_drafts(a, sq, tok[n], d0);
      wave_fence();
      attend_few<RN>(r, s, v, seen, a.sc, q, vlane);
      wave_fence();
      if (odd) add_not_finite_few<RN>(r, v, vb + (int64_t)d0 * a.v.ss, a.v.ss, sq.T - d0, seen, q, vlane, lane);
    }
  }

  // the waves' parts of each row, weighed by their maxima
#pragma unroll
  for (int n = 0; n < RN; ++n) {
    r.l[n] += __shfl_xor(r.l[n], 16);
    r.l[n] += __shfl_xor(r.l[n], 32);
    if (q == 0) *reinterpret_cast<float2*>(ml[wave][16 * n + c]) = make_float2(r.m[n], r.l[n]);
  }
#pragma unroll
  for (int n = 0; n < RN; ++n) {
    __syncthreads();                       // the staged blocks, or the tile before, are done with
    float* buf = reinterpret_cast<float*>(vs) + wave * 16 * OP;
    {
      float m = ml[0][16 * n + c][0];
#pragma unroll
      for (int w = 1; w < 4; ++w) m = fmaxf(m, ml[w][16 * n + c][0]);
      const float f = r.m[n] == -INFINITY ? 0.0f : fast_exp2(r.m[n] - m);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
        *reinterpret_cast<float4*>(buf + c * OP + 16 * dt + 4 * q) =
            make_float4(r.o[n][dt][0] * f, r.o[n][dt][1] * f, r.o[n][dt][2] * f, r.o[n][dt][3] * f);
    }
    __syncthreads();
    const int jr = tid >> 4, part = tid & 15;              // row of the tile, 8 channels
    const int row = it.tile * ROWS + 16 * n + jr, jtok = row / a.g;
    if (jtok >= sq.T) continue;
    const float (*mr)[ROWS][2] = ml;
    float m = mr[0][16 * n + jr][0];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, mr[w][16 * n + jr][0]);
    float l = 0.0f, o[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) o[x] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float wm = mr[w][16 * n + jr][0], f = wm == -INFINITY ? 0.0f : fast_exp2(wm - m);
      l += mr[w][16 * n + jr][1] * f;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(vs) + (w * 16 + jr) * OP +
                                                          part * 8 + 4 * x);
        o[4 * x] += y.x; o[4 * x + 1] += y.y; o[4 * x + 2] += y.z; o[4 * x + 3] += y.w;
      }
    }
    if (it.chunks == 1) {
      const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;       // no key seen: 0; NaN stays
      const int head = it.head * a.g + row - jtok * a.g;
      bf16x8 y;
#pragma unroll
      for (int x = 0; x < 8; ++x) y[x] = (__bf16)(o[x] * inv);
      *reinterpret_cast<bf16x8*>(a.o + (int64_t)(sq.row0 + jtok) * a.o_ss + (int64_t)head * a.o_sh + part * 8) = y;
      if (a.lse && part == 0)
        a.lse[(int64_t)head * a.n_rows + sq.row0 + jtok] = l == 0.0f ? -INFINITY : (m + fast_log2(l)) * LN2;
    } else {
      const int64_t at = (int64_t)it.part * ROWS + 16 * n + jr;
      float* to = a.part_o + at * D + part * 8;
      *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
      if (part == 0) *reinterpret_cast<float4*>(a.part_ml + at * 4) = make_float4(m, l, l, 0.0f);
    }
  }
}

// ------------------------------------------------------------------ many rows
// With more than 32 rows a head the products, not the cache's bytes, bound the
// work (up to 64 about both): keys are staged once for all rows of a workgroup's tile. Its eight
// waves (two a SIMD) are WR groups of 32 rows times 8 / WR groups of keys;
// the keys go through four LDS stages of 64, one barrier a stage.
//
// A unit is 32 keys against a wave's 32 rows. Slot u issues QK of unit u + 1
// and PV of unit u - 1 (8 MFMAs each, in turn) with the softmax of unit u
// spread between them, since the vector ALU overlaps only MFMAs of the same
// wave; operands are read from LDS three MFMAs ahead.
// 64 drafts over 131072 tokens, 28 heads on 4, bfloat16: 151 us, 797 TFLOP/s.
// The matrix cores are busy 37% of the cycles, the vector ALU 35%, LDS (an
// operand serves one MFMA) about half; what is left is the barrier and steps
// that wait for each other. Measured against it, in turn: two tiles a wave and
// one wave a SIMD (512 registers, half the LDS reads) 209 us for 168, the
// compiler moves what it keeps in the accumulator half back and forth; a
// SIMD's waves strictly in turn, one attending while the other stages, 183 for
// 170; staging spread between a slot's MFMAs 176 for 169; operands seven ahead
// no change.
constexpr int SK = 64;                 // keys of a stage
constexpr int NST = 4;
constexpr int NTW = 512;               // threads

struct __align__(16) Stage64 {
  uint16_t k[SK * TK];
  uint16_t v[SK * TV];
};

template <int TYPE>
struct Raw64 {                         // a thread's pieces of a stage: piece i is number tid + i * NTW
  static constexpr int CPR = Codec<TYPE>::ROW / 16;        // pieces a row
  static constexpr int N = SK * CPR / NTW > 0 ? SK * CPR / NTW : 1;
  static constexpr int LIVE = SK * CPR < NTW ? SK * CPR / 64 : NTW / 64;   // waves that hold one of K and V
  // E2M1: the first waves take K (in k), the others V (in k too). Leaving all
  // to the first ones took 330 us for 314 (64 drafts over 262144
  // tokens, 32 heads on 8).
  static constexpr bool SPLIT = LIVE < NTW / 64;
  u32x4 k[N], v[N];
  uint32_t ks[N], vs[N];
  typedef int Ids[N];                                      // page numbers
};

// A pointer that is the same in every lane, kept in scalar registers: a load
// from it then takes a lane's offset in one register, not an address in two.
template <typename T>
__device__ __forceinline__ const __attribute__((address_space(1))) T* scalar(const void* p) {
  asm("" : "+s"(p));
  return (const __attribute__((address_space(1))) T*)p;
}

// Where a wave's pieces come from. Its 64 pieces i are 4, 8 or 16 whole rows,
// which lie in one page and follow each other: one page number and scalar base
// a load, and a lane's offset that never changes.
struct KeySource {
  const int32_t* pages;
  int head, c1, wave, lane;
  uint32_t zero;                       // in a vector register: keeps the page table's loads vector loads
};

template <int TYPE>
__device__ __forceinline__ int first_key(int wave, int i) {
  return (wave % Raw64<TYPE>::LIVE * 64 + i * NTW) / Raw64<TYPE>::CPR;
}

// The numbers stay in a vector register until they are used, a stage later: a
// scalar load would share its counter with the LDS reads of the slots between.
template <int TYPE>
__device__ __forceinline__ void page_ids(typename Raw64<TYPE>::Ids& p, const TreeArgs& a, const KeySource& s, int t0) {
#pragma unroll
  for (int i = 0; i < Raw64<TYPE>::N; ++i)
    p[i] = scalar<int32_t>(s.pages + (min(t0 + first_key<TYPE>(s.wave, i), s.c1 - 1) >> a.c.shift))[s.zero];
}

// Pages outside the cache are read as page 0, which is there; their keys are
// masked, and their V staged as zero.
template <int TYPE>
__device__ __forceinline__ void load_stage(Raw64<TYPE>& r, const typename Raw64<TYPE>::Ids& p, const TreeArgs& a,
                                           const KeySource& s, int t0) {
  typedef Raw64<TYPE> R;
  const bool second = s.wave >= R::LIVE;                   // of SPLIT
  static_assert(!R::SPLIT || R::LIVE == NTW / 128, "half the waves take K, half V");
#pragma unroll
  for (int i = 0; i < R::N; ++i) {
    const int t = t0 + first_key<TYPE>(s.wave, i);
    const int id = __builtin_amdgcn_readfirstlane(p[i]);
    const int64_t page = (uint32_t)id < (uint64_t)a.c.n_pages ? id : 0;
    const int in = (s.head << a.c.shift) + (t & ((1 << a.c.shift) - 1));
    const int64_t at = page * a.c.page_stride + (int64_t)in * Codec<TYPE>::ROW;
    r.k[i] = scalar<u32x4>((second ? a.c.v : a.c.k) + at)[(uint32_t)s.lane];
    if constexpr (!R::SPLIT) r.v[i] = scalar<u32x4>(a.c.v + at)[(uint32_t)s.lane];
    if constexpr (Codec<TYPE>::SCALED) {
      const int64_t sat = page * a.c.scale_stride + (int64_t)in * 4;
      const uint32_t row = (uint32_t)s.lane / R::CPR;
      r.ks[i] = scalar<uint32_t>((const uint8_t*)(second ? a.c.vs : a.c.ks) + sat)[row];
      if constexpr (!R::SPLIT) r.vs[i] = scalar<uint32_t>((const uint8_t*)a.c.vs + sat)[row];
    }
  }
}

// `there`: the stage's keys that exist; the others weigh nothing, whatever
// their places hold.
template <int TYPE>
__device__ __forceinline__ void write_stage(Stage64& st, const Raw64<TYPE>& r, int wave, int lane, uint64_t there) {
  typedef Raw64<TYPE> R;
#pragma unroll
  for (int i = 0; i < R::N; ++i) {
    const int key = first_key<TYPE>(wave, i) + lane / R::CPR, piece = lane % R::CPR;
    const bool ok = there == ~0ull || (there >> key & 1);
    const u32x4 none = {};
    if constexpr (R::SPLIT) {
      if (wave < R::LIVE) put_piece<TYPE>(&st.k[key * TK], r.k[i], r.ks[i], piece);
      else put_piece<TYPE>(&st.v[key * TV], ok ? r.k[i] : none, ok ? r.ks[i] : 0u, piece);
    } else {
      put_piece<TYPE>(&st.k[key * TK], r.k[i], r.ks[i], piece);
      put_piece<TYPE>(&st.v[key * TV], ok ? r.v[i] : none, ok ? r.vs[i] : 0u, piece);
    }
  }
}

// MFMA operand i of a slot: first the K rows of the next unit, then the
// transposed V of the last.
__device__ __forceinline__ bf16x8 slot_operand(int i, const uint16_t* kp, const uint16_t* vp) {
  const int x = i & 7;
  if (i < 8) return *reinterpret_cast<const bf16x8*>(kp + x * 8);
  const uint16_t* p = vp + 16 * (x >> 2) * TV + 32 * (x & 3);
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p + 8 * TV));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ void mask_unit(f32x16& s, uint32_t seen, int h) {
  const uint32_t mine = seen >> (4 * h);     // element 4 i + j is key 8 i + 4 h + j
#pragma unroll
  for (int x = 0; x < 16; ++x)
    if (!(mine >> (8 * (x >> 2) + (x & 3)) & 1)) s[x] = -INFINITY;
}

// A use that keeps the computation of x where it is written: nothing reads
// much of a slot's results before the next slot, and the compiler would move
// it there, in one lump behind the MFMAs that it is to run beside.
template <typename T>
__device__ __forceinline__ void pin(T& x) { asm volatile("" : "+v"(x)); }

// The softmax of a unit in pieces that fit between MFMAs: one exponential
// each, and after eight their packing and the sum of the packed. It takes the
// running maximum as it is and looks at no score: the sums tell, at the slot's
// end, where some row's scores have passed its maximum by so much (P of up to
// 2^12 do no harm) that it has to move, and soft_again makes P anew. (Finding
// a unit's maxima first put 20 dependent instructions before the exponentials
// of every slot: six ragged trees 402 us for 383, 16 drafts over 1M tokens in
// four bits 451 for 425.)
// P is rounded to bfloat16 for the product and O divided by the sum of the
// rounded, so that only the roundings' scatter is left: each weight is off by
// up to 2^-8, the mean of many by less. P in two pieces as with few rows makes
// a slot's 16 MFMAs 24: 64 drafts over 131072, 28 heads on 4, bfloat16 243 us
// for 173, 16 over 1048576 in E2M1 485 for 378, 256 of 64 sequences over 400 in
// E4M3 345 for 295.
constexpr int PIECES = 18;
constexpr float MOST = 4096.0f;
struct SoftState {
  float e[8], rs, ro;
};

template <bool WL>
__device__ __forceinline__ void soft_piece(int piece, const f32x16& s, float sc, const Rows& r, bf16x8 (&p)[2],
                                           SoftState& z) {
  const int half = piece / 9, x = piece % 9;
  if (piece == 0) z.rs = z.ro = 0.0f;
  if (x < 8) {
    float e = fast_exp2(fmaf(s[8 * half + x], sc, -r.base));
    pin(e);
    z.e[x] = e;
    if (WL) z.rs += e;
  } else {
    const bf16e2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 8; ++i) p[half][i] = (__bf16)z.e[i];   // rounded for the product; O is divided by the sum of these
#pragma unroll
    for (int i = 0; i < 4; ++i)
      z.ro = __builtin_amdgcn_fdot2_f32_bf16(bf16e2{p[half][2 * i], p[half][2 * i + 1]}, one, z.ro, false);
    pin(z.ro);
    pin(p[half]);
  }
}

// The unit's maxima move m, with O, l and lo; P and its sums once more.
template <bool WL>
__device__ __forceinline__ void soft_again(const f32x16& s, float sc, Rows& r, bf16x8 (&p)[2], SoftState& z) {
  float mx = s[0];
#pragma unroll
  for (int x = 1; x < 16; ++x) mx = fmaxf(mx, s[x]);
  mx = half_max(mx) * sc;                                  // sc > 0
  const float m = fmaxf(r.m, mx), alpha = r.m == m ? 1.0f : fast_exp2(r.m - m);
  r.m = m;
  r.base = m == -INFINITY ? 0.0f : m;                      // nothing seen yet: every P is 2^-inf = 0
  r.most = m == -INFINITY ? -1.0f : MOST;
  r.l *= alpha;
  r.lo *= alpha;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) r.o[dt][x] *= alpha;
#pragma unroll
  for (int pc = 0; pc < PIECES; ++pc) soft_piece<WL>(pc, s, sc, r, p, z);
}

constexpr int AHEAD = 3;

// PRE: the first operands are there, read in the slot before; this one reads
// the next one's (from kn, vn).
template <bool WL, bool PRE>
__device__ __forceinline__ void slot(Rows& r, bf16x8 (&op)[AHEAD + 1], f32x16& s_sm, f32x16& s_qk,
                                     const bf16x8 (&p_pv)[2], bf16x8 (&p_sm)[2], float sc, const uint16_t* kp,
                                     const uint16_t* vp, const uint16_t* kn, const uint16_t* vn) {
  SoftState z;
  const f32x16 zero = {};
  __builtin_amdgcn_s_setprio(1);       // before the SIMD's other wave while that stages
  if (!PRE) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) op[i] = slot_operand(i, kp, vp);
  }
  int pc = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = i + AHEAD;
    if (j < 16) op[j % (AHEAD + 1)] = slot_operand(j, kp, vp);
    else if (PRE) op[j % (AHEAD + 1)] = slot_operand(j - 16, kn, vn);
    const bf16x8 av = op[i % (AHEAD + 1)];
    const int x = i & 7;
    if (i < 8) {
      s_qk = mfma32(av, r.q[x], x == 0 ? zero : s_qk);
      pin(s_qk);
    } else r.o[x & 3] = mfma32(av, p_pv[x >> 2], r.o[x & 3]);
    const int end = (i + 1) * PIECES / 16;
#pragma unroll
    for (; pc < end; ++pc) soft_piece<WL>(pc, s_sm, sc, r, p_sm, z);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  // O holds PV up to unit u - 1, by the maximum of unit u - 1
  if (__any(z.ro > r.most)) soft_again<WL>(s_sm, sc, r, p_sm, z);
  if (WL) r.l += z.rs;
  r.lo += z.ro;
}

// A staged block of 32 keys, nothing overlapped.
__device__ __forceinline__ void unit_alone(Rows& r, uint32_t seen, float sc, int h, const uint16_t* kp,
                                           const uint16_t* vp) {
  f32x16 s = {};
#pragma unroll
  for (int x = 0; x < 8; ++x) s = mfma32(slot_operand(x, kp, vp), r.q[x], s);
  mask_unit(s, seen, h);
  SoftState z;
  bf16x8 p[2];
  soft_again<true>(s, sc, r, p, z);
  r.l += z.rs;
  r.lo += z.ro;
#pragma unroll
  for (int x = 0; x < 8; ++x) r.o[x & 3] = mfma32(slot_operand(8 + x, kp, vp), p[x >> 2], r.o[x & 3]);
}

template <int TYPE, int WR, bool WL>
__global__ __launch_bounds__(NTW) __attribute__((amdgpu_waves_per_eu(2))) void k_tree_wide(TreeArgs a) {
  constexpr int ROWS = 32 * WR, WK = 8 / WR;               // rows of a workgroup, groups of keys
  static_assert(WK == 1 || WK == 2, "a stage holds two units");
  __shared__ Stage64 st[NST];
  __shared__ int64_t sh64[8];
  __shared__ int sh[8];
  Item it;
  if (!find_item<ROWS, NTW>(a, blockIdx.x, it, sh64, sh)) return;
  const Seq sq = it.seq;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // waves w and w + 4 share a SIMD: the key groups take the rows in different
  // orders, so that up to 64 rows keep all four SIMDs busy (8 drafts of 7 heads
  // a KV head over 262144 tokens in E4M3: 78 us for 91, with both in order)
  const int wk = wave / WR, wr = wave % WR ^ (wk * (WR / 2));
  const int c = lane & 31, h = lane >> 5;
  // this lane's K row and transpose-read source inside a staged block of 32 keys
  const int grp = lane >> 4, li = lane & 15;
  const int klane = c * TK + h * 64;
  const int vlane = (4 * (grp >> 1) + (li >> 2)) * TV + 16 * (grp & 1) + 4 * (li & 3);
  const int row = it.tile * ROWS + 32 * wr + c, tok = row / a.g;
  const bool live = tok < sq.T;
  const bool active = it.tile * ROWS + 32 * wr < sq.T * a.g;   // some row of the wave's is

  Rows r;
  {
    const uint16_t* q = (const uint16_t*)a.q.p + (int64_t)(sq.row0 + (live ? tok : 0)) * a.q.ss +
                        (int64_t)(it.head * a.g + (live ? row - tok * a.g : 0)) * a.q.sh + h * 64;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const bf16x8 y = load16(q + 8 * x);
      r.q[x] = live ? y : zero8();
    }
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) r.o[dt][x] = 0.0f;
  r.m = -INFINITY;
  r.l = r.lo = r.base = 0.0f;
  r.most = -1.0f;

  // Stages: what lies behind c1 is staged as nothing. Two key groups take an
  // even number; with one a last single stage is worth its branch (16 sequences
  // of 128 drafts over 300 tokens 49 us for 52; 64 over 131072 158.4 for 157.5).
  const int steps = (it.c1 - it.c0 + WK * SK - 1) / (WK * SK) * WK;
  uint32_t zero = 0;
  asm("" : "+v"(zero));
  const KeySource src = {a.pages + (int64_t)it.b * a.max_pages, it.head, it.c1, wave, lane, zero};
  // Two stages are on their way in registers, in turn: a load has two steps to arrive.
  Raw64<TYPE> even, odd;
  typename Raw64<TYPE>::Ids pid, next;
  auto load = [&](Raw64<TYPE>& raw, int t) INLINE { load_stage<TYPE>(raw, pid, a, src, it.c0 + t * SK); };
  auto ids = [&](typename Raw64<TYPE>::Ids& to, int t) INLINE { page_ids<TYPE>(to, a, src, it.c0 + min(t, steps - 1) * SK); };
  auto advance = [&]() INLINE {
#pragma unroll
    for (int i = 0; i < Raw64<TYPE>::N; ++i) pid[i] = next[i];
  };
  bool any_bad = false;
  if (steps > 0) {
    ids(pid, 0);
    ids(next, 1);
    load(even, 0);
    advance();
    ids(next, 2);
    load(odd, 1);
    advance();
    // pages outside the cache are rare enough to ask once for the whole chunk
    int bad = 0;
    for (int p = (it.c0 >> a.c.shift) + tid; p <= (it.c1 - 1) >> a.c.shift; p += NTW)
      bad |= (uint32_t)src.pages[p] >= (uint64_t)a.c.n_pages;
    any_bad = __syncthreads_or(bad);
  }
  // The drafted tokens come first: these loads are on their way meanwhile (64
  // drafts over 8192 tokens 36.8 us for 37.9 with the drafted tokens last).
  const uint16_t* vb = (const uint16_t*)a.v.p + (int64_t)sq.row0 * a.v.ss + (int64_t)it.head * a.v.sh;
  int not_all_finite = 0;
  if (it.chunk == it.chunks - 1) {
    const uint16_t* kb = (const uint16_t*)a.k.p + (int64_t)sq.row0 * a.k.ss + (int64_t)it.head * a.k.sh;
    // without a mask no row sees a token behind the tile's last
    const int n = a.mask ? sq.T : min(sq.T, (it.tile * ROWS + ROWS - 1) / a.g + 1);
    u32x4 kv[2], vv[2];
    uint32_t seen[2 / WK], next_seen[2 / WK];
    auto fetch = [&](int d0) INLINE {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int d = min(d0 + tid / 16 + 32 * i, sq.T - 1);
        kv[i] = *reinterpret_cast<const u32x4*>(kb + (int64_t)d * a.k.ss + tid % 16 * 8);
        vv[i] = *reinterpret_cast<const u32x4*>(vb + (int64_t)d * a.v.ss + tid % 16 * 8);
      }
#pragma unroll
      for (int x = 0; x < 2 / WK; ++x) {
        const int k0 = d0 + 32 * (wk + WK * x);
        next_seen[x] = k0 < sq.T ? seen_drafts(a, sq, tok, k0) : 0u;
      }
    };
    // the next stage on its way while this one is attended, in two places in
    // turn: one barrier a stage (64 sequences of 256 drafts and 400 cached
    // tokens, no mask, 523 us for 563 with everything after one another)
    fetch(0);
    for (int d0 = 0; d0 < n; d0 += SK) {
      Stage64& to = st[d0 / SK & 1];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int key = tid / 16 + 32 * i;
        u32x4 keep;
        const u32x4 none = {};
        not_all_finite |= not_finite(vv[i], keep);
        *reinterpret_cast<u32x4*>(&to.k[key * TK + tid % 16 * 8]) = kv[i];
        *reinterpret_cast<u32x4*>(&to.v[key * TV + tid % 16 * 8]) = d0 + key < sq.T ? keep : none;
      }
#pragma unroll
      for (int x = 0; x < 2 / WK; ++x) seen[x] = next_seen[x];
      __syncthreads();
      if (d0 + SK < n) fetch(d0 + SK);
#pragma unroll
      for (int x = 0; x < 2 / WK; ++x) {
        const int sub = wk + WK * x;
        if (active && __any(seen[x] != 0))
          unit_alone(r, seen[x], a.sc, h, to.k + klane + 32 * sub * TK, to.v + vlane + 32 * sub * TV);
      }
    }
    not_all_finite = __syncthreads_or(not_all_finite);
  }
  if (steps > 0) {
    auto there = [&](int t) INLINE -> uint64_t {                  // keys of stage t that exist
      const int t0 = it.c0 + t * SK, n = it.c1 - t0;
      uint64_t m = n >= SK ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
      if (any_bad)
        for (int part = 0; part < 4; ++part) {
          const int p = src.pages[min(t0 + 16 * part, it.c1 - 1) >> a.c.shift];
          if ((uint32_t)p >= (uint64_t)a.c.n_pages) m &= ~(0xffffull << (16 * part));
        }
      return m;
    };
    write_stage<TYPE>(st[0], even, wave, lane, there(0));
    ids(next, 3);
    load(even, min(2, steps - 1));
    advance();
    write_stage<TYPE>(st[1], odd, wave, lane, there(1));
    // the numbers of the next stage before the loads of this one, here as below
    ids(next, 4);
    __builtin_amdgcn_sched_barrier(0);
    load(odd, min(3, steps - 1));
    advance();
    // The slot before unit 0 has no V yet: its P is zero, and what it takes for
    // V, the stage before stage 0, has to be finite (step 1 overwrites it).
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 none = {};
      *reinterpret_cast<u32x4*>(&st[NST - 1].v[(tid / 16 + 32 * i) * TV + tid % 16 * 8]) = none;
    }
    __syncthreads();
    // unit u: stage u / 2, block u % 2 (one key group), or stage u, block wk (two)
    const int units = WK == 1 ? 2 * steps : steps;
    auto k_at = [&](int u) INLINE -> const uint16_t* {
      return st[(WK == 1 ? u >> 1 : u) & (NST - 1)].k + klane + 32 * TK * (WK == 1 ? u & 1 : wk);
    };
    auto v_at = [&](int u) INLINE -> const uint16_t* {
      return st[(WK == 1 ? u >> 1 : u) & (NST - 1)].v + vlane + 32 * TV * (WK == 1 ? u & 1 : wk);
    };
    f32x16 s0 = {}, s1 = {};
    bf16x8 p0[2], p1[2], op[AHEAD + 1];
#pragma unroll
    for (int x = 0; x < 2; ++x) p0[x] = p1[x] = zero8();
#pragma unroll
    for (int x = 0; x < 8; ++x) s0 = mfma32(slot_operand(x, k_at(0), nullptr), r.q[x], s0);
    constexpr bool PRE = WK == 1;
    if (PRE) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) op[i] = slot_operand(i, k_at(1), nullptr);
    }
    // Stage t + 2 into LDS, t + 4 on its way. Nothing here is left out at the
    // end (the last stage is loaded again, from the caches): where loads are
    // issued on some paths only, the compiler waits for all of them. The next
    // page numbers are asked for before the loads, and wait for none of them.
    auto stage_on = [&](Raw64<TYPE>& raw, int t) INLINE {
      write_stage<TYPE>(st[(t + 2) & (NST - 1)], raw, wave, lane, there(t + 2));
      ids(next, t + 5);
      __builtin_amdgcn_sched_barrier(0);
      load(raw, min(t + 4, steps - 1));
      advance();
    };
    auto mask = [&](f32x16& s, int u) INLINE {
      const uint64_t m = there(WK == 1 ? u >> 1 : u);
      if (m != ~0ull) mask_unit(s, (uint32_t)(m >> (32 * (WK == 1 ? u & 1 : wk))), h);
    };
    // One key group, units 2 t and 2 t + 1 in step t: behind the barrier before
    // it stage t + 1 is whole, and the one that takes stage t + 2 (t - 2's) has
    // been read for the last time in step t - 1.
    // Two key groups, unit u = stage u: behind the barrier of slot u stage
    // u + 1 is whole, and everybody is through with slot u - 1, the last to
    // read stage u - 2.
    auto first_slot = [&](int u) INLINE {                         // u even: scores in s0
      if (!active) return;
      mask(s0, u);
      slot<WL, PRE>(r, op, s0, s1, p1, p0, a.sc, k_at(u + 1), v_at(u - 1), k_at(u + 2), v_at(u));
    };
    auto second_slot = [&](int u) INLINE {
      if (!active) return;
      mask(s1, u);
      slot<WL, PRE>(r, op, s1, s0, p0, p1, a.sc, k_at(u + 1), v_at(u - 1), k_at(u + 2), v_at(u));
    };
    if (WK == 2) {
      for (int u = 0; u < units; u += 2) {
        __syncthreads();
        first_slot(u);
        stage_on(even, u);
        __syncthreads();
        second_slot(u + 1);
        stage_on(odd, u + 1);
      }
    } else {
      auto step = [&](Raw64<TYPE>& raw, int t) INLINE {
        first_slot(2 * t);
        stage_on(raw, t);
        second_slot(2 * t + 1);
        __syncthreads();
      };
      for (int t = 0; t < steps; t += 2) {
        step(even, t);
        if (t + 1 == steps) break;
        step(odd, t + 1);
      }
    }
    if (active) {
      const uint16_t* vp = v_at(units - 1);
#pragma unroll
      for (int x = 0; x < 8; ++x) r.o[x & 3] = mfma32(slot_operand(8 + x, nullptr, vp), p1[x >> 2], r.o[x & 3]);
    }
    __syncthreads();
  }
  if (not_all_finite) {                                    // at the end: nothing scales what these put into O
    uint16_t* own = st[0].k + wave * (KB * TV);            // flags in a place of the wave's own
    static_assert(8 * KB * TV * 2 <= sizeof(st), "the flags lie in the stages");
    for (int k0 = 32 * wk; active && k0 < sq.T; k0 += 32 * WK)
      add_not_finite(r.o, own, vb + (int64_t)k0 * a.v.ss, a.v.ss, sq.T - k0, seen_drafts(a, sq, tok, k0), h, vlane, lane);
    __syncthreads();
  }

  r.l = half_sum(r.l);
  r.lo = half_sum(r.lo);
  if constexpr (WK == 2) {                                 // the second key group's part joins the first's
    float* buf = reinterpret_cast<float*>(st) + wr * (32 * OP + 128);
    static_assert(sizeof(st) >= WR * (32 * OP + 128) * sizeof(float), "the join buffer lies in the stages");
    float* ml = buf + 32 * OP;
    if (wk == 1) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(buf + c * OP + 32 * dt + 8 * i + 4 * h) =
              make_float4(r.o[dt][4 * i], r.o[dt][4 * i + 1], r.o[dt][4 * i + 2], r.o[dt][4 * i + 3]);
      if (h == 0) {
        ml[c * 4] = r.m;
        ml[c * 4 + 1] = r.lo;
        ml[c * 4 + 2] = r.l;
      }
    }
    __syncthreads();
    if (wk == 1) return;
    const float m1 = ml[c * 4], m = fmaxf(r.m, m1);
    const float f0 = r.m == -INFINITY ? 0.0f : fast_exp2(r.m - m);
    const float f1 = m1 == -INFINITY ? 0.0f : fast_exp2(m1 - m);
    r.m = m;
    r.lo = r.lo * f0 + ml[c * 4 + 1] * f1;
    r.l = r.l * f0 + ml[c * 4 + 2] * f1;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 y = *reinterpret_cast<const float4*>(buf + c * OP + 32 * dt + 8 * i + 4 * h);
        r.o[dt][4 * i] = r.o[dt][4 * i] * f0 + y.x * f1;
        r.o[dt][4 * i + 1] = r.o[dt][4 * i + 1] * f0 + y.y * f1;
        r.o[dt][4 * i + 2] = r.o[dt][4 * i + 2] * f0 + y.z * f1;
        r.o[dt][4 * i + 3] = r.o[dt][4 * i + 3] * f0 + y.w * f1;
      }
  }
  if (!live) return;
  if (it.chunks == 1) {
    const float inv = r.lo > 0.0f ? 1.0f / r.lo : r.lo == 0.0f ? 0.0f : r.lo;
    const int head = it.head * a.g + row - tok * a.g;
    uint16_t* to = a.o + (int64_t)(sq.row0 + tok) * a.o_ss + (int64_t)head * a.o_sh;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(r.o[dt][4 * i + e] * inv);
        *reinterpret_cast<bf16x4*>(to + 32 * dt + 8 * i + 4 * h) = y;
      }
    if (WL && h == 0)
      a.lse[(int64_t)head * a.n_rows + sq.row0 + tok] = r.l == 0.0f ? -INFINITY : (r.m + fast_log2(r.l)) * LN2;
  } else {
    const int64_t at = (int64_t)it.part * ROWS + 32 * wr + c;
    float* to = a.part_o + at * D;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(to + 32 * dt + 8 * i + 4 * h) =
            make_float4(r.o[dt][4 * i], r.o[dt][4 * i + 1], r.o[dt][4 * i + 2], r.o[dt][4 * i + 3]);
    if (h == 0) *reinterpret_cast<float4*>(a.part_ml + at * 4) = make_float4(r.m, r.lo, r.l, 0.0f);
  }
}

// Joins the partials of the sequences that were cut into chunks. A workgroup
// joins one of their rows after another (row, KV head, sequence): its waves
// take every fourth partial, two channels a lane, JU of them in flight (the
// statistics of those a lane each), and meet in LDS. Bound by latency, or with
// many rows by reading the partials. The host does not know which sequences
// were cut: with a workgroup for every row that may exist, 16 sequences of 128
// drafts and 300 cached tokens took 87 us for 52 in all, 64 of 256 and 400
// (28 heads on 4) 525 us for 290.
constexpr int JU = 8;                 // a lane each of max8 and sum8
constexpr int JOINS = 8;              // workgroups a compute unit

struct JoinShared {
  float2 o[4][64];
  float m[4], lo[4], l[4];
};

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// Over eight neighbouring lanes: the other one of two, the other two of four,
// and, those being alike, the mirrored of eight.
__device__ __forceinline__ float max8(float x) {
  x = fmaxf(x, dpp<0xb1>(x));
  x = fmaxf(x, dpp<0x4e>(x));
  return fmaxf(x, dpp<0x141>(x));
}

__device__ __forceinline__ float sum8(float x) {
  x += dpp<0xb1>(x);
  x += dpp<0x4e>(x);
  return x + dpp<0x141>(x);
}

__device__ __forceinline__ void join_row(const TreeArgs& a, int64_t at0, int64_t step, int chunks, int64_t token,
                                         int qh, JoinShared& sh) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float m = -INFINITY, l = 0.0f, lo = 0.0f;
  float2 o = make_float2(0.0f, 0.0f);
  for (int p0 = wave; p0 < chunks; p0 += 4 * JU) {
    const int mine = p0 + 4 * (lane % JU);
    const float4 e = *reinterpret_cast<const float4*>(a.part_ml + (at0 + min(mine, chunks - 1) * step) * 4);
    float2 y[JU];
#pragma unroll
    for (int u = 0; u < JU; ++u)
      y[u] = *reinterpret_cast<const float2*>(a.part_o + (at0 + min(p0 + 4 * u, chunks - 1) * step) * D + 2 * lane);
    // used here: the compiler would load each where it is added, one after another
#pragma unroll
    for (int u = 0; u < JU; ++u) {
      pin(y[u].x);
      pin(y[u].y);
    }
    const bool there = mine < chunks;
    const float mn = fmaxf(m, max8(there ? e.x : -INFINITY));
    const float f = m == -INFINITY ? 0.0f : fast_exp2(m - mn);
    const float w = there && e.x != -INFINITY ? fast_exp2(e.x - mn) : 0.0f;
    m = mn;
    lo = lo * f + sum8(there ? e.y * w : 0.0f);
    l = l * f + sum8(there ? e.z * w : 0.0f);
    o.x *= f; o.y *= f;
#pragma unroll
    for (int u = 0; u < JU; ++u) {
      if (p0 + 4 * u >= chunks) break;
      const float wu = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), u));
      o.x += y[u].x * wu; o.y += y[u].y * wu;
    }
  }
  sh.o[wave][lane] = o;
  if (lane == 0) {
    sh.m[wave] = m;
    sh.lo[wave] = lo;
    sh.l[wave] = l;
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int x = 1; x < 4; ++x) m = fmaxf(m, sh.m[x]);
  l = lo = 0.0f;
  o = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float f = sh.m[x] == -INFINITY ? 0.0f : fast_exp2(sh.m[x] - m);
    const float2 y = sh.o[x][lane];
    lo += sh.lo[x] * f;
    l += sh.l[x] * f;
    o.x += y.x * f; o.y += y.y * f;
  }
  const float inv = lo > 0.0f ? 1.0f / lo : lo == 0.0f ? 0.0f : lo;
  const bf16e2 y = {(__bf16)(o.x * inv), (__bf16)(o.y * inv)};
  *reinterpret_cast<bf16e2*>(a.o + token * a.o_ss + (int64_t)qh * a.o_sh + 2 * lane) = y;
  if (a.lse && lane == 0) a.lse[(int64_t)qh * a.n_rows + token] = l == 0.0f ? -INFINITY : (m + fast_log2(l)) * LN2;
}

// A sequence without rows, or (row_start not ascending) behind the items that
// were launched, has no record: whatever the workspace held is no index.
__device__ __forceinline__ bool was_cut(const TreeArgs& a, const Seq& s, int first, int chunks, int tiles) {
  return s.T > 0 && chunks > 1 && first >= 0 && first + (int64_t)chunks * a.c.Hkv * tiles <= a.parts;
}

template <int ROWS>
__device__ __forceinline__ void join_row_of(const TreeArgs& a, const Seq& s, int first, int chunks, int tiles, int at,
                                            JoinShared& sh) {
  const int rows = s.T * a.g, head = at / rows, row = at - head * rows, tok = row / a.g;
  join_row(a, ((int64_t)first + (int64_t)head * tiles + row / ROWS) * ROWS + row % ROWS, (int64_t)a.c.Hkv * tiles * ROWS,
           chunks, s.row0 + tok, head * a.g + row - tok * a.g, sh);
}

// EACH: a workgroup for every row that may exist. Few as they are, a workgroup
// then has nothing to search for (64 drafts over 8192 tokens 35.9 us for 37.2).
template <int ROWS, bool EACH>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(JOINS))) void k_tree_join(TreeArgs a) {
  __shared__ JoinShared sh;
  if constexpr (EACH) {
    const int most = a.max_rows * a.g * a.c.Hkv, b = blockIdx.x / most, at = blockIdx.x - b * most;
    const Seq s = sequence(a, b);
    const int first = a.rec[2 * b], chunks = a.rec[2 * b + 1], tiles = tiles_of<ROWS>(a, s);
    if (was_cut(a, s, first, chunks, tiles) && at < s.T * a.g * a.c.Hkv)
      join_row_of<ROWS>(a, s, first, chunks, tiles, at, sh);
    return;
  }
  int next = blockIdx.x, base = 0;                         // this workgroup's next row; rows of the sequences before
  for (int b0 = 0; b0 < a.n_seq; b0 += 64) {               // a sequence a lane, in every wave
    const int lane = threadIdx.x & 63, b = b0 + lane;
    Seq s = {0, 0, 0};
    int first = 0, chunks = 0;
    if (b < a.n_seq) {
      s = sequence(a, b);
      first = a.rec[2 * b];
      chunks = a.rec[2 * b + 1];
    }
    const int tiles = tiles_of<ROWS>(a, s);
    const int n = was_cut(a, s, first, chunks, tiles) ? s.T * a.g * a.c.Hkv : 0;   // host: below 2^23 of all sequences
    int end = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(end, d);
      if (lane >= d) end += y;
    }
    const int all = __builtin_amdgcn_readlane(end, 63);
    for (; next < base + all; next += gridDim.x) {
      const int at = next - base, l = __builtin_ctzll(__ballot(at >= end - n && at < end));
      auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
      const Seq sl = {of(s.row0), of(s.T), of(s.L)};
      join_row_of<ROWS>(a, sl, of(first), of(chunks), of(tiles), at - of(end - n), sh);
      __syncthreads();
    }
    base += all;
  }
}

TreeShape tree_shape(const mmi_tree& t, int Hkv, int type, int cus) {
  TreeShape s{};
  const int g = t.Hq / Hkv;
  // what bounds the work changes at 32 rows a head (16 rows: half the softmax
  // and products of 32); a wide workgroup holds a compute unit, three or two
  // of the few-row ones share it. 16-bit rows are read by two (16 sequences of
  // 20000 tokens, 32 heads on 8, 123 us for 126 with three), smaller ones by
  // three (32 of 8192: E2M1 63 us for 65 with two, int8 129 for 131, E4M3 110
  // for 108), 32 rows of any type by two (their registers; E4M3, 4 drafts of 7
  // heads a KV head over 262144, 59 us for 65).
  const int rows = t.max_rows * g;
  s.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 128 ? 128 : 256;
  s.target = cus * (s.rows > 32 ? 1 : s.rows == 32 || type == MMI_CACHE_BF16 ? 2 : 3);
  // tiles of all sequences, and `target` chunks more (each sequence's last chunk may be short)
  const int64_t most = (t.max_rows * (int64_t)g + s.rows - 1) / s.rows;
  const int64_t tiles = std::min<int64_t>(most * t.n_seq, ((int64_t)t.n_rows * g + (int64_t)t.n_seq * (s.rows - 1)) / s.rows);
  const int64_t items = tiles * Hkv + s.target;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  const int64_t limit = (int64_t)1 << 22;
  if (items > limit || (int64_t)t.max_rows * t.Hq * t.n_seq > 2 * limit) throw Error(MMI_ERR_UNSUPPORTED, "the batch is cut into more than 2^22 workgroups");
  s.items = (int32_t)items;
  // Only cut sequences leave partials. Each is longer than a chunk, so its
  // chunks are fewer than twice its length in chunks, and a chunk is at least
  // the batch's work / target: fewer than 2 target of them in all.
  s.parts = t.max_len <= CHUNK ? 0 : (int32_t)std::min<int64_t>(items, 2 * s.target);
  s.part_o = 0;
  s.part_ml = up((size_t)s.parts * s.rows * D * 4);
  s.rec = s.part_ml + up((size_t)s.parts * s.rows * 16);
  s.bytes = s.rec + up((size_t)std::max(t.n_seq, 1) * 8);
  return s;
}

template <int TYPE>
static void launch_type(const TreeArgs& a, int rows, hipStream_t st) {
  const dim3 grid((unsigned)a.items);
  if (rows == 16) hipLaunchKernelGGL((k_tree_few<TYPE, 1>), grid, dim3(256), 0, st, a);
  else if (rows == 32) hipLaunchKernelGGL((k_tree_few<TYPE, 2>), grid, dim3(256), 0, st, a);
  else if (rows == 128 && a.lse) hipLaunchKernelGGL((k_tree_wide<TYPE, 4, true>), grid, dim3(NTW), 0, st, a);
  else if (rows == 128) hipLaunchKernelGGL((k_tree_wide<TYPE, 4, false>), grid, dim3(NTW), 0, st, a);
  else if (a.lse) hipLaunchKernelGGL((k_tree_wide<TYPE, 8, true>), grid, dim3(NTW), 0, st, a);
  else hipLaunchKernelGGL((k_tree_wide<TYPE, 8, false>), grid, dim3(NTW), 0, st, a);
}

template <int ROWS>
static void launch_join(const TreeArgs& a, hipStream_t st) {
  // rows of the largest batch within the bounds (below 2^23), and as many workgroups as run at once
  const int64_t rows = (int64_t)a.max_rows * a.n_seq * a.g * a.c.Hkv, most = JOINS * (int64_t)a.cus;
  if (rows <= most) hipLaunchKernelGGL((k_tree_join<ROWS, true>), dim3((unsigned)rows), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_tree_join<ROWS, false>), dim3((unsigned)most), dim3(256), 0, st, a);
}

hipError_t launch_tree(const TreeArgs& a, int type, int rows, hipStream_t st) {
  if (a.n_seq <= 0 || a.n_rows <= 0) return hipSuccess;
  switch (type) {
    case MMI_CACHE_BF16: launch_type<MMI_CACHE_BF16>(a, rows, st); break;
    case MMI_CACHE_FP8: launch_type<MMI_CACHE_FP8>(a, rows, st); break;
    case MMI_CACHE_INT8: launch_type<MMI_CACHE_INT8>(a, rows, st); break;
    case MMI_CACHE_FP4: launch_type<MMI_CACHE_FP4>(a, rows, st); break;
    default: return hipErrorInvalidValue;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.max_len <= CHUNK) return e;   // one chunk a sequence at most
  switch (rows) {
    case 16: launch_join<16>(a, st); break;
    case 32: launch_join<32>(a, st); break;
    case 128: launch_join<128>(a, st); break;
    default: launch_join<256>(a, st);
  }
  return hipGetLastError();
}

}  // namespace mmi
