// Declarations shared by the host layer and the kernels of the paged cache
// (include/stlite_paged.h).
#pragma once

#include "stlite_internal.h"

namespace stlite {

// The cache and the batch of new tokens, as the kernels see them.
struct PagedDev {
  uint16_t* k;  // [units][n_pages][page][d]; of a 4-bit pool: [units][n_pages][page * 68 bytes]
  uint16_t* v;
  const int32_t* page_table;  // [n_seqs][max_pages]
  int32_t* seq_lens;          // [n_seqs], new tokens included
  const int32_t* cu_new;      // [n_seqs + 1]
  int32_t n_layers, n_q_heads, n_kv_heads, n_units, group;
  int32_t n_seqs, n_pages, max_pages, max_len;
  int32_t page_shift;  // log2(page_size), >= 4
  int64_t total_new;
};

struct PagedCompactArgs {
  PagedDev c;
  const int32_t* cu_budget;
  int64_t total_tokens, total_budget;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* kept;
  int32_t kept_per_layer;
};

struct PagedReadArgs {
  PagedDev c;
  uint16_t* k_out;  // [layers][total_new][kv_heads][d], nullable
  uint16_t* v_out;
};

struct PagedPagesArgs {
  PagedDev c;
  int32_t* free_pages;  // [n_pages]
  int32_t* n_free;      // [1]
  int32_t* held;        // [n_seqs]
  int32_t* page_table;  // the cache's
  int32_t* slots;       // growing: [total_new], nullable
  const int32_t* lens;  // releasing: [n_seqs], nullable
};

struct RowsIn {
  const uint16_t* data;  // nullable (no queries)
  int64_t token_stride, layer_stride;
};

struct PagedAppendArgs {
  PagedDev c;
  RowsIn q, k, v;
  uint16_t* q_out;
  const uint16_t* q_norm;  // [layers][d], nullable
  const uint16_t* k_norm;
  float eps;
  const int32_t* positions;  // [axes][total_new], nullable: no rotation
  int32_t interleaved;
  int32_t axis1, axis2;  // pairs >= axis1 go by the second position, >= axis2 by the third
  double turns[64];      // theta^(-i/64) / (2 pi): turns of pair i per position
  double low[64];        // what they lack of it (a 4-bit pool's)
};

// Attention runs as a flat range of places, cut into equal shares.  The queries of a (unit,
// sequence) are cut into items of `tokens` new tokens (all heads of the kv head: tokens *
// group rows; the kernels of few rows: one token, or over a 4-bit pool a sequence's few, at
// most `rows` of their rows, one token's heads in `parts` where they are more); item i of a
// sequence with n new tokens behind c cached ones counts c + min((i + 1) tokens, n) keys,
// what its last token sees, and takes item_cost places before them.  Items lie one after
// another, units outermost; work-group w takes the keys in [w share, (w + 1) share) of that
// range, but an item of up to `keep` keys is not cut: it is all of the share's that its
// middle lies in.  A share that holds a whole item writes its output; the parts of an item
// that several shares cut leave (max, sum, O) in the workspace and are joined by a second
// launch, which does not go where no item can be cut.  The lengths are read on the device
// only, so the grid does not depend on them.
constexpr int32_t kExtRows = 256;  // rows of an item of several tokens
struct PagedAttnArgs {
  PagedDev c;
  const uint16_t* q;  // [layers][total_new][q_heads][d]
  uint16_t* out;
  float scale2;       // scale * log2(e)
  int32_t parts;      // head groups of a kv head (few rows: `rows` heads each; else 1)
  int32_t tokens;     // new tokens per item
  int32_t rows;       // rows of an item's partial (few rows 16, 32 or, over 4 bits, 64; else kExtRows)
  int32_t shares;     // work-groups
  int32_t min_share;  // places
  int32_t item_cost;  // places that beginning an item takes
  int32_t keep;       // items of up to so many keys are not cut (a 16-bit pool: 0)
  bool joins;         // items may be cut
  int32_t join_items;  // joining by item: their number; 0: by boundary
  int32_t join_rows;  // rows of an item per joining work-group
  int32_t join_groups;  // rows that a joining work-group takes at once, 8 or 32
  int32_t join_split;  // joining work-groups per item or boundary
  float* pm;          // workspace [shares][2][rows]: max (log2 units)
  float* pl;          // workspace [shares][2][rows]: sum
  float* po;          // workspace [shares][2][rows][d]: O, unnormalised
};

// four: a 4-bit pool; half: fp16, else bf16
hipError_t launch_paged_compact(const PagedCompactArgs& a, bool four, bool half, hipStream_t stream);
hipError_t launch_paged_read(const PagedReadArgs& a, bool four, bool half, hipStream_t stream);
hipError_t launch_paged_append(const PagedAppendArgs& a, bool four, bool half, hipStream_t stream);
hipError_t launch_paged_decode(const PagedAttnArgs& a, bool half, hipStream_t stream);
hipError_t launch_paged4_few(const PagedAttnArgs& a, bool half, hipStream_t stream);
hipError_t launch_paged_extend(const PagedAttnArgs& a, bool four, bool half, hipStream_t stream);
hipError_t launch_paged_grow(const PagedPagesArgs& a, hipStream_t stream);
hipError_t launch_paged_release(const PagedPagesArgs& a, hipStream_t stream);
hipError_t launch_paged_join(const PagedAttnArgs& a, bool half, hipStream_t stream);

// ---------------------------------------------------------------------------
// Device helpers
// ---------------------------------------------------------------------------

template <typename T>
__device__ inline uint32_t elem_pack(float lo, float hi) {  // each rounded to nearest
  typedef T pair_t __attribute__((ext_vector_type(2)));
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, pair_t));
}

// 16-bit element types: bf16 or IEEE half.
template <typename T>
struct Elem;
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
template <>
struct Elem<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x16_t mfma32(x8 a, x8 b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  __device__ static f32x4_t mfma16(x8 a, x8 b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  // Pairs of a dword whose exponent is all ones (bits 15 and 31).
  __device__ static uint32_t not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
  // Weights are formed at most 2^-20 large (2^8 of those at the reference, with kLazy),
  // so that the sums of 2^20 keys' values of any size stay finite before the division.
  static constexpr float kBias = -28.0f;

  static __device__ f32x4_t mfma16(u32x2_t a, u32x2_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, a), __builtin_bit_cast(s16x4_t, b), c, 0, 0, 0);
  }
  // x as a sum of terms of this type: 3 x 8 bits are all of it.  A term is taken off.
  static constexpr int kTerms = 3;
  static constexpr float kTermsBias = -20.0f;  // (as kBias)
  static __device__ uint32_t take(float& x0, float& x1, bool) {
    const uint32_t b0 = __builtin_bit_cast(uint32_t, x0) & 0xffff0000u, b1 = __builtin_bit_cast(uint32_t, x1) & 0xffff0000u;
    x0 -= __builtin_bit_cast(float, b0);
    x1 -= __builtin_bit_cast(float, b1);
    return b0 >> 16 | b1;
  }
};
template <>
struct Elem<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x16_t mfma32(x8 a, x8 b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  __device__ static f32x4_t mfma16(x8 a, x8 b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  __device__ static uint32_t not_finite(uint32_t w) { return ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u; }
  // Half weights lose bits below 2^-14: they are formed 2^7 times as large, at
  // most 2^15 with kLazy.
  static constexpr float kBias = 7.0f;

  static __device__ f32x4_t mfma16(u32x2_t a, u32x2_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4_t, a), __builtin_bit_cast(f16x4_t, b), c, 0, 0, 0);
  }
  // Two terms of 11 bits, of weights of at most 2^15, the second rounded to nearest (cut
  // off, the sums of the weights in the numerator would all lie below the denominator's):
  // they are off by at most 2^-22 of the weight itself, or 2^-40 of the greatest.
  static constexpr int kTerms = 2;
  static constexpr float kTermsBias = 15.0f;
  static __device__ uint32_t take(float& x0, float& x1, bool last) {
    if (last) return elem_pack<_Float16>(x0, x1);
    const auto h = __builtin_amdgcn_cvt_pkrtz(x0, x1);
    x0 -= float(h[0]);
    x1 -= float(h[1]);
    return __builtin_bit_cast(uint32_t, h);
  }
};

template <typename T>
__device__ inline float elem_lo(uint32_t w) {
  return float(__builtin_bit_cast(T, uint16_t(w)));
}
template <typename T>
__device__ inline float elem_hi(uint32_t w) {
  return float(__builtin_bit_cast(T, uint16_t(w >> 16)));
}

// A logit in base 2, rounded: what a maximum is taken of and what it is taken from have
// to be the same number.  (Contracted, s scale - maximum is the unrounded product's
// distance, which for logits of 2^31 is up to 2^7.)
__device__ inline float base2(float s, float scale2) {
#pragma clang fp contract(off)
  return s * scale2;
}

__device__ inline int32_t paged_len(const PagedDev& c, int32_t s) { return min(max(c.seq_lens[s], 0), c.max_len); }

// What growing writes behind the pages of an empty sequence that it parks.
constexpr int32_t kPagesEnd = -2;

// Whether a compaction of `keeps` rows leaves sequence s of length `len` as it is: it is
// parked, and not an empty one whose row of the table has pages for them.  A length of -1 that
// no call has written is told from an empty parked sequence's by that row: without pages its
// first entry is none, with some growing has marked where they end.
__device__ inline bool stays_parked(const PagedDev& c, int32_t s, int32_t len, int32_t keeps) {
  if (len >= 0) return false;
  if (len < -1) return true;
  const int32_t* row = c.page_table + int64_t(s) * c.max_pages;
  bool parked = uint32_t(row[0]) >= uint32_t(c.n_pages);
  const int32_t last = min((keeps - 1) >> c.page_shift, c.max_pages - 1);
  for (int32_t e = 1; e <= last; ++e) parked |= row[e] == kPagesEnd;
  return parked;
}

// First row of page `page` of a unit, in rows of the pool.
__device__ inline int64_t page_row(const PagedDev& c, int32_t unit, int32_t page) {
  return ((int64_t(unit) * c.n_pages + page) << c.page_shift);
}

}  // namespace stlite
