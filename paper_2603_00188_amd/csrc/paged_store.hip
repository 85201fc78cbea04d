// Rows into a paged cache: the compression's kept rows (a gather, as the dense
// compaction) and the new tokens of a serving step (norm and rotation on the way).
#include "paged4.h"
#include "tile_lds.h"

namespace stlite {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Kept rows into pages
// ---------------------------------------------------------------------------

constexpr int kRowsPerGroup = 64;

// The sequence of entry j of a prefix-sum array (cu[0] = 0 <= j < cu[n]).
__device__ inline int32_t seq_of(const int32_t* cu, int32_t n, int64_t j) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (cu[mid] <= j) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A compaction's lengths, by one work-group.  (The others may read a length before or after:
// it is negative and stays, is not and remains so, or is -1 and its row of the table says.)
__device__ inline void set_lengths(const PagedCompactArgs& a) {
  for (int32_t s = threadIdx.x; s < a.c.n_seqs; s += 256) {
    const int32_t keeps = a.cu_budget[s + 1] - a.cu_budget[s];
    if (!stays_parked(a.c, s, a.c.seq_lens[s], keeps)) a.c.seq_lens[s] = keeps;
  }
}

// Sixteen lanes move one 256-byte row of K and one of V; a work-group 64 rows of
// a unit.  HBM-bound: all of a thread's loads are issued before its stores, and
// both bypass the caches (each byte is touched once).  3.47 GB (a trajectory of 150528
// tokens, a fifth kept, 112 units) take 601 us, 5.8 TB/s; 78 MB (one screen) 16 us, 4.9.
__global__ __launch_bounds__(256) void paged_compact_kernel(PagedCompactArgs a) {
  constexpr int kPer = kRowsPerGroup / 16;
  const int unit = blockIdx.y;
  const int64_t j0 = int64_t(blockIdx.x) * kRowsPerGroup;
  const int sub = threadIdx.x >> 4, part = threadIdx.x & 15;
  const int64_t ubase = int64_t(unit) * a.total_tokens;
  if (blockIdx.x == 0 && unit == 0) set_lengths(a);
  const int64_t kbase = int64_t(a.kept_per_layer ? unit / a.c.n_kv_heads : unit) * a.total_budget;
  int32_t tok[kPer];
  int64_t dst[kPer];  // row of the pool, or -1
#pragma unroll
  for (int r = 0; r < kPer; ++r) {
    const int64_t j = j0 + r * 16 + sub;
    tok[r] = -1;
    dst[r] = -1;
    if (j < a.total_budget) {
      tok[r] = a.kept[kbase + j];
      const int32_t s = seq_of(a.cu_budget, a.c.n_seqs, j);
      const int32_t at = int32_t(j - a.cu_budget[s]), keeps = a.cu_budget[s + 1] - a.cu_budget[s], len = a.c.seq_lens[s];
      const int32_t entry = at >> a.c.page_shift;
      const int32_t page = entry < a.c.max_pages ? a.c.page_table[int64_t(s) * a.c.max_pages + entry] : -1;
      if (page >= 0 && page < a.c.n_pages && !stays_parked(a.c, s, len, keeps))
        dst[r] = page_row(a.c, unit, page) + (at & ((1 << a.c.page_shift) - 1));
    }
  }
  if (a.total_budget == 0) return;
  u32x4_t kv[kPer], vv[kPer];
#pragma unroll
  for (int r = 0; r < kPer; ++r) {
    const bool ok = tok[r] >= 0 && tok[r] < a.total_tokens;
    const int64_t src = (ubase + (ok ? tok[r] : 0)) * kHeadDim + part * 8;
    kv[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.k + src));
    vv[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.v + src));
  }
#pragma unroll
  for (int r = 0; r < kPer; ++r) {
    if (!(tok[r] >= 0 && tok[r] < a.total_tokens)) {
      kv[r] = u32x4_t{0u, 0u, 0u, 0u};
      vv[r] = u32x4_t{0u, 0u, 0u, 0u};
    }
    if (dst[r] < 0) continue;
    __builtin_nontemporal_store(kv[r], reinterpret_cast<u32x4_t*>(a.c.k + dst[r] * kHeadDim + part * 8));
    __builtin_nontemporal_store(vv[r], reinterpret_cast<u32x4_t*>(a.c.v + dst[r] * kHeadDim + part * 8));
  }
}

// v of lane ^ M as bits.
template <int M>
__device__ __forceinline__ uint32_t lane_xor_bits(uint32_t v) {
  return __float_as_uint(lane_xor<M>(__uint_as_float(v)));
}

// Kept rows into the pages of a 4-bit pool: the same walk, sixteen lanes to a row.  Four
// lanes hold a block: its greatest magnitude by two exchanges, then 4 bytes of codes each;
// the row's four scale bytes meet in one lane.
// HBM-bound: 30105 rows of 112 units (1.73 GB in, 0.46 out) take 390 us, 5.6 TB/s; 678 rows
// 15.  (With codes stored past the caches 369, but what reads them next then takes more
// than that longer.)
template <typename T>
__global__ __launch_bounds__(256) void paged4_compact_kernel(PagedCompactArgs a) {
  constexpr int kPer = kRowsPerGroup / 16;
  const int unit = blockIdx.y;
  const int64_t j0 = int64_t(blockIdx.x) * kRowsPerGroup;
  const int sub = threadIdx.x >> 4, part = threadIdx.x & 15;
  const int64_t ubase = int64_t(unit) * a.total_tokens;
  if (blockIdx.x == 0 && unit == 0) set_lengths(a);
  if (a.total_budget == 0) return;
  const int64_t kbase = int64_t(a.kept_per_layer ? unit / a.c.n_kv_heads : unit) * a.total_budget;
  const int32_t in_page = (1 << a.c.page_shift) - 1;
  u32x4_t rows[2][kPer];
  int64_t page_at[kPer];  // first byte of the page, or -1
  int32_t row_at[kPer];
#pragma unroll
  for (int r = 0; r < kPer; ++r) {
    const int64_t j = j0 + r * 16 + sub;
    int32_t tok = -1;
    page_at[r] = -1;
    row_at[r] = 0;
    if (j < a.total_budget) {
      tok = a.kept[kbase + j];
      const int32_t s = seq_of(a.cu_budget, a.c.n_seqs, j);
      const int32_t at = int32_t(j - a.cu_budget[s]), keeps = a.cu_budget[s + 1] - a.cu_budget[s], len = a.c.seq_lens[s];
      const int32_t entry = at >> a.c.page_shift;
      const int32_t page = entry < a.c.max_pages ? a.c.page_table[int64_t(s) * a.c.max_pages + entry] : -1;
      row_at[r] = at & in_page;
      if (page >= 0 && page < a.c.n_pages && !stays_parked(a.c, s, len, keeps)) page_at[r] = page4(a.c, unit, page);
    }
    const bool ok = tok >= 0 && tok < a.total_tokens;
    const int64_t src = (ubase + (ok ? tok : 0)) * kHeadDim + part * 8;
    rows[0][r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.k + src));
    rows[1][r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.v + src));
    if (!ok) rows[0][r] = rows[1][r] = u32x4_t{0u, 0u, 0u, 0u};
  }
#pragma unroll
  for (int r = 0; r < kPer; ++r) {
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint32_t w[4] = {rows[kv][r][0], rows[kv][r][1], rows[kv][r][2], rows[kv][r][3]};
      uint32_t top = top_of(w);
      top = max(top, lane_xor_bits<1>(top));
      top = max(top, lane_xor_bits<2>(top));
      const uint32_t byte = scale_byte<T>(Four<T>::wide(top));
      const uint32_t code = codes_of<T>(w, byte);
      uint32_t scales = byte << (8 * (part >> 2));
      scales |= lane_xor_bits<4>(scales);
      scales |= lane_xor_bits<8>(scales);
      if (page_at[r] < 0) continue;
      uint8_t* p = reinterpret_cast<uint8_t*>(kv ? a.c.v : a.c.k) + page_at[r];
      *reinterpret_cast<uint32_t*>(p + row_at[r] * kCodes4 + part * 4) = code;
      if (part == 0) *reinterpret_cast<uint32_t*>(p + (in_page + 1) * kCodes4 + row_at[r] * 4) = scales;
    }
  }
}

// ---------------------------------------------------------------------------
// Rows out of pages
// ---------------------------------------------------------------------------

constexpr int kReadRows = 16;

// The new tokens' rows, sixteen lanes to a row, a work-group 16 rows in the output's order
// (a token's heads one after another), so that what it writes is contiguous.
// HBM-bound, a row's 68 (or 256) bytes in and 256 out: 30105 tokens of 112 units in 4 bits
// (2.2 GB, four fifths of it written) take 410 us behind the compaction, 5.3 TB/s, with the
// codes past the caches, 475 through them; 678 tokens 8.6 through them and 9.9 past, so
// PAST where the rows are more than the caches hold.
// (In a unit's order, whose writes are 256 bytes apart, 584; with 32, 64, 128 rows to a
// work-group 14, 14 and 37 more; with stores that go through the caches 30 more.)
template <typename T, bool FOUR, bool PAST>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedReadArgs a) {
  const PagedDev& c = a.c;
  const int layer = blockIdx.y;
  const int64_t n = c.total_new * c.n_kv_heads;
  const int64_t i = (int64_t(blockIdx.z) * gridDim.x + blockIdx.x) * kReadRows + (threadIdx.x >> 4), tok = i / c.n_kv_heads;
  if (i >= n) return;
  const int part = threadIdx.x & 15, unit = layer * c.n_kv_heads + int(i - tok * c.n_kv_heads);
  const int32_t in_page = (1 << c.page_shift) - 1;
  int32_t page = -1, row = 0;
  const int32_t s = seq_of(c.cu_new, c.n_seqs, tok);
  const int64_t at = int64_t(paged_len(c, s)) - c.cu_new[s + 1] + tok;
  if (at >= 0) {
    page = c.page_table[int64_t(s) * c.max_pages + (at >> c.page_shift)];
    row = int32_t(at) & in_page;
  }
  u32x4_t rows[2] = {u32x4_t{0u, 0u, 0u, 0u}, u32x4_t{0u, 0u, 0u, 0u}};
  if (page >= 0 && page < c.n_pages) {
    if constexpr (FOUR) {
      uint32_t codes[2], scales[2];
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint8_t* p = reinterpret_cast<const uint8_t*>(kv ? c.v : c.k) + page4(c, unit, page);
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(p + row * kCodes4 + part * 4);
        codes[kv] = PAST ? __builtin_nontemporal_load(from) : *from;
        scales[kv] = p[(in_page + 1) * kCodes4 + row * 4 + (part >> 2)];
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        uint32_t w[4];
        values_of<T>(codes[kv], scale_of(scales[kv]), w);
        rows[kv] = u32x4_t{w[0], w[1], w[2], w[3]};
      }
    } else {
      const int64_t from = (page_row(c, unit, page) + row) * kHeadDim + part * 8;
      rows[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(c.k + from));
      rows[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(c.v + from));
    }
  }
  const int64_t to = (layer * n + i) * kHeadDim + part * 8;
  if (a.k_out) __builtin_nontemporal_store(rows[0], reinterpret_cast<u32x4_t*>(a.k_out + to));
  if (a.v_out) __builtin_nontemporal_store(rows[1], reinterpret_cast<u32x4_t*>(a.v_out + to));
}

// ---------------------------------------------------------------------------
// New tokens
// ---------------------------------------------------------------------------

constexpr int64_t kMaxBlocks = int64_t(1) << 23;  // along x

// Sums of squares that fp32 holds to its full precision.  A row outside (bf16 values above
// 2^60 or all below 2^-50) is scaled by a power of two, and eps by its square, before its
// norm; a small one only where eps does not hide it, so that the scaled eps stays finite.
// (3136 normed tokens of 28 layers take 298 us; without it 295.5, in 64 bits 310.)
constexpr float kLeastSum = 0x1p-100f, kMostSum = 0x1p120f, kLeastEps = 0x1p-80f;

// y in fp32 rounded to odd (toward zero, the last bit set where something was cut off): it
// lies on the same side of every number with fewer bits as y, or is that number as y is.
__device__ inline float odd32(double y) {
  const float f = float(y);
  uint32_t b = __float_as_uint(f);
  if (double(f) != y) b = (b - (fabs(double(f)) > fabs(y) ? 1u : 0u)) | 1u;
  return __uint_as_float(b);
}

template <int M>
__device__ __forceinline__ double lane_xor64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = lane_xor_bits<M>(uint32_t(u)), hi = lane_xor_bits<M>(uint32_t(u >> 32));
  return __builtin_bit_cast(double, hi << 32 | lo);
}

// A key's or a value's row into a 4-bit pool, lane c of its eight with the dimensions
// 8 c .. and 64 + 8 c ..: blocks c / 4 and 2 + c / 4, four lanes to each.
template <typename T>
__device__ __forceinline__ void store4(const PagedAppendArgs& a, bool key, int layer, int h, int64_t slot, u32x4_t lo,
                                       u32x4_t hi, const double2* cs) {
  const PagedDev& c = a.c;
  const int cidx = threadIdx.x & 7;
  uint32_t code[2], byte[2];
  if (key && (a.k_norm || a.positions)) {
    double x[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = elem_lo<T>(lo[j]);
      x[2 * j + 1] = elem_hi<T>(lo[j]);
      x[8 + 2 * j] = elem_lo<T>(hi[j]);
      x[9 + 2 * j] = elem_hi<T>(hi[j]);
    }
    if (a.k_norm) {
      double ss = 0.0;
#pragma unroll
      for (int j = 0; j < 16; ++j) ss = fma(x[j], x[j], ss);
      ss += lane_xor64<1>(ss);
      ss += lane_xor64<2>(ss);
      ss += lane_xor64<4>(ss);
      const double rs = 1.0 / sqrt(ss * (1.0 / kHeadDim) + double(a.eps));
      const uint16_t* wl = a.k_norm + layer * kHeadDim + 8 * cidx;
      const u32x4_t w0 = *reinterpret_cast<const u32x4_t*>(wl), w1 = *reinterpret_cast<const u32x4_t*>(wl + 64);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] *= rs * elem_lo<T>(w0[j]);
        x[2 * j + 1] *= rs * elem_hi<T>(w0[j]);
        x[8 + 2 * j] *= rs * elem_lo<T>(w1[j]);
        x[9 + 2 * j] *= rs * elem_hi<T>(w1[j]);
      }
    }
    if (a.positions) {
      if (a.interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const double2 t = cs[4 * cidx + (j & 3) + 32 * (j >> 2)];
          const double y0 = x[2 * j] * t.x - x[2 * j + 1] * t.y;
          x[2 * j + 1] = x[2 * j + 1] * t.x + x[2 * j] * t.y;
          x[2 * j] = y0;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const double2 t = cs[8 * cidx + j];
          const double y0 = x[j] * t.x - x[8 + j] * t.y;
          x[8 + j] = x[8 + j] * t.x + x[j] * t.y;
          x[j] = y0;
        }
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float y[8];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = odd32(x[8 * b + j]);
        top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
      }
      top = max(top, lane_xor_bits<1>(top));
      top = max(top, lane_xor_bits<2>(top));
      byte[b] = scale_byte<T>(top);
      code[b] = codes_of(y, byte[b]);
    }
  } else {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const u32x4_t e = b ? hi : lo;
      const uint32_t w[4] = {e[0], e[1], e[2], e[3]};
      uint32_t top = top_of(w);
      top = max(top, lane_xor_bits<1>(top));
      top = max(top, lane_xor_bits<2>(top));
      byte[b] = scale_byte<T>(Four<T>::wide(top));
      code[b] = codes_of<T>(w, byte[b]);
    }
  }
  uint32_t scales = (byte[0] | byte[1] << 16) << (8 * (cidx >> 2));
  scales |= lane_xor_bits<4>(scales);
  if (slot < 0) return;
  const int32_t row = int32_t(slot) & ((1 << c.page_shift) - 1);
  uint8_t* p = reinterpret_cast<uint8_t*>(key ? c.k : c.v) + page4(c, layer * c.n_kv_heads + h, int32_t(slot >> c.page_shift));
  *reinterpret_cast<uint32_t*>(p + row * kCodes4 + 4 * cidx) = code[0];
  *reinterpret_cast<uint32_t*>(p + row * kCodes4 + 32 + 4 * cidx) = code[1];
  if (cidx == 0) *reinterpret_cast<uint32_t*>(p + (kCodes4 << c.page_shift) + row * 4) = scales;
}

// One (token, layer) by `WAVES` waves.  Eight lanes hold a head: lane c the
// dimensions 8c .. 8c+7 and 64+8c .. 64+8c+7, so both members of every pair of
// either pairing lie in one lane.  The 64 (cos, sin) of the token are formed
// once, one pair per lane, and kept in registers over the token's heads.
// Angles: position * turns in 64 bits, reduced to a fraction of a turn there;
// the sine of the reduced angle in fp32.
// HBM-bound once there are a few thousand rows: 3136 tokens of 28 layers (1.62 GB read
// and written) take 298 us, 5.4 TB/s; 64 tokens of 28 layers (44 MB) 12.3 us, 3.6 TB/s,
// where the chain of dependent loads (sequence, length, page, row) is half of it.
//
// FOUR: keys and values are stored in 4 bits.  Which code a key gets turns on the side of
// a border that it lies on, so it is formed in 64 bits, which this card multiplies and adds
// at the rate of single 32-bit operations, and the token's sines too, of turns to 105 bits
// (their product with a position of 2^31 is off by 10^-16 of a turn then, not 10^-8); on the
// way to codes it passes through fp32 rounded to odd, which keeps the side.
template <typename T, int WAVES, bool FOUR>
__global__ __launch_bounds__(256, FOUR ? 4 : 1) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int kTok = 4 / WAVES;  // tokens per work-group
  __shared__ float2 sm_cs[kTok][64];
  __shared__ double2 sm_cs64[FOUR ? kTok : 1][64];
  const PagedDev& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tl = wave / WAVES, part = wave % WAVES;
  const int layer = blockIdx.y;
  const int64_t tok = (int64_t(blockIdx.z) * gridDim.x + blockIdx.x) * kTok + tl;
  const bool live = tok < c.total_new;
  const int cidx = lane & 7, sub = lane >> 3;
  const int nq = a.q.data ? c.n_q_heads : 0, nk = c.n_kv_heads;
  const int rows = nq + 2 * nk;
  const uint16_t* q = a.q.data + layer * a.q.layer_stride + tok * a.q.token_stride;
  const uint16_t* k = a.k.data + layer * a.k.layer_stride + tok * a.k.token_stride;
  const uint16_t* v = a.v.data + layer * a.v.layer_stride + tok * a.v.token_stride;
  const int64_t unit_rows = int64_t(c.n_pages) << c.page_shift;
  // Row r of the token: queries, keys, values.  The first one's load runs under the
  // angles and the search, each further one's under the row before it.
  auto source = [&](int r) {
    return r < nq ? q + r * kHeadDim : r < nq + nk ? k + (r - nq) * kHeadDim : v + (r - nq - nk) * kHeadDim;
  };
  u32x4_t lo_next{}, hi_next{};
  auto load = [&](int r) {
    const uint16_t* src = source(r) + 8 * cidx;
    lo_next = *reinterpret_cast<const u32x4_t*>(src);
    hi_next = *reinterpret_cast<const u32x4_t*>(src + 64);
  };
  if (live && part * 8 + sub < rows) load(part * 8 + sub);
  if (a.positions && live && part == 0) {
    const int axis = (lane >= a.axis1) + (lane >= a.axis2);
    const double at = double(a.positions[axis * c.total_new + tok]), turn = at * a.turns[lane];
    if constexpr (FOUR) {
      double sn, cs;
      sincospi(2.0 * fma(at, a.low[lane], fma(at, a.turns[lane], -rint(turn))), &sn, &cs);
      sm_cs64[tl][lane] = make_double2(cs, sn);
      sm_cs[tl][lane] = make_float2(float(cs), float(sn));
    } else {
      const float r = float(turn - rint(turn));
      sm_cs[tl][lane] = make_float2(cospif(2.0f * r), sinpif(2.0f * r));
    }
  }
  __syncthreads();
  if (!live) return;

  float cs[16], sn[16];  // of the low chunk's and the high chunk's pairs
  if (a.positions) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // half split: pair 8c + j; interleaved: pairs 4c + j/2 and 32 + 4c + j/2
      const float2 lo = sm_cs[tl][a.interleaved ? 4 * cidx + (j >> 1) : 8 * cidx + j];
      const float2 hi = sm_cs[tl][a.interleaved ? 32 + 4 * cidx + (j >> 1) : 8 * cidx + j];
      cs[j] = lo.x;
      sn[j] = lo.y;
      cs[8 + j] = hi.x;
      sn[8 + j] = hi.y;
    }
  }
  // Where the token's keys and values go.
  int64_t slot = -1;  // row of the pool within a unit
  {
    int32_t s = 0;
    for (int32_t n = c.n_seqs; n > 1;) {  // a wave's 64 probes at once: one round for 64 sequences
      const int32_t step = (n + 63) / 64, at = lane * step;
      s += step * (63 - __builtin_clzll(__ballot(at < n && c.cu_new[min(s + at, c.n_seqs)] <= tok) | 1));
      n = min(step, c.n_seqs - s);
    }
    const int64_t at = int64_t(paged_len(c, s)) - c.cu_new[s + 1] + tok;
    if (at >= 0) {
      const int32_t page = c.page_table[int64_t(s) * c.max_pages + (at >> c.page_shift)];
      if (page >= 0 && page < c.n_pages) slot = (int64_t(page) << c.page_shift) + (at & ((1 << c.page_shift) - 1));
    }
  }
  for (int r = part * 8 + sub; r < rows; r += 8 * WAVES) {
    const u32x4_t lo = lo_next, hi = hi_next;
    if (r + 8 * WAVES < rows) load(r + 8 * WAVES);
    if constexpr (FOUR) {
      if (r >= nq) {  // (the lanes of a head take the same side)
        const int h = (r - nq) % nk;
        const bool key = r - nq < nk;
        store4<T>(a, key, layer, h, slot, lo, hi, sm_cs64[tl]);
        continue;
      }
    }
    uint16_t* dst;
    const uint16_t* w = nullptr;
    bool turn = a.positions != nullptr;
    if (r < nq) {
      dst = a.q_out + ((layer * c.total_new + tok) * c.n_q_heads + r) * kHeadDim;
      w = a.q_norm;
    } else {
      const int h = (r - nq) % nk;
      const bool key = r - nq < nk;
      const int64_t row = int64_t(layer * nk + h) * unit_rows + slot;
      dst = slot < 0 ? nullptr : (key ? c.k : c.v) + row * kHeadDim;
      w = key ? a.k_norm : nullptr;
      turn = turn && key;
    }
    u32x4_t ylo = lo, yhi = hi;
    if (w || turn) {
      float x[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = elem_lo<T>(lo[j]);
        x[2 * j + 1] = elem_hi<T>(lo[j]);
        x[8 + 2 * j] = elem_lo<T>(hi[j]);
        x[9 + 2 * j] = elem_hi<T>(hi[j]);
      }
      // (the lanes of a head take the same side of these branches, so the sums below
      // have all eight)
      if (w) {
        float ss = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) ss = fmaf(x[j], x[j], ss);
        ss += lane_xor<1>(ss);
        ss += lane_xor<2>(ss);
        ss += lane_xor<4>(ss);
        float eps = a.eps;
        if (!(ss <= kMostSum) || (ss < kLeastSum && eps < kLeastEps)) {
          const float up = ss < 1.0f ? 0x1p100f : 0x1p-70f;
          eps = eps * up * up;
          ss = 0.0f;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            x[j] *= up;
            ss = fmaf(x[j], x[j], ss);
          }
          ss += lane_xor<1>(ss);
          ss += lane_xor<2>(ss);
          ss += lane_xor<4>(ss);
        }
        const float rs = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + eps);
        const uint16_t* wl = w + layer * kHeadDim + 8 * cidx;
        const u32x4_t w0 = *reinterpret_cast<const u32x4_t*>(wl), w1 = *reinterpret_cast<const u32x4_t*>(wl + 64);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[2 * j] *= rs * elem_lo<T>(w0[j]);
          x[2 * j + 1] *= rs * elem_hi<T>(w0[j]);
          x[8 + 2 * j] *= rs * elem_lo<T>(w1[j]);
          x[9 + 2 * j] *= rs * elem_hi<T>(w1[j]);
        }
      }
      if (turn) {
        float y[16];
        if (a.interleaved) {
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            y[j] = x[j] * cs[j] - x[j + 1] * sn[j];
            y[j + 1] = x[j + 1] * cs[j] + x[j] * sn[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y[j] = x[j] * cs[j] - x[8 + j] * sn[j];
            y[8 + j] = x[8 + j] * cs[j] + x[j] * sn[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = y[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ylo[j] = elem_pack<T>(x[2 * j], x[2 * j + 1]);
        yhi[j] = elem_pack<T>(x[8 + 2 * j], x[9 + 2 * j]);
      }
    }
    if (dst) {
      *reinterpret_cast<u32x4_t*>(dst + 8 * cidx) = ylo;
      *reinterpret_cast<u32x4_t*>(dst + 64 + 8 * cidx) = yhi;
    }
  }
}

}  // namespace

hipError_t launch_paged_compact(const PagedCompactArgs& a, bool four, bool half, hipStream_t stream) {
  // (one work-group for the lengths where nothing is kept)
  const int64_t blocks = a.total_budget > 0 ? (a.total_budget + kRowsPerGroup - 1) / kRowsPerGroup : 1;
  const dim3 grid(uint32_t(blocks), a.c.n_units);
  if (!four) hipLaunchKernelGGL(paged_compact_kernel, grid, dim3(256), 0, stream, a);
  else if (half) hipLaunchKernelGGL((paged4_compact_kernel<_Float16>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged4_compact_kernel<__bf16>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <typename T>
static void read4(const PagedReadArgs& a, dim3 grid, hipStream_t stream) {
  const bool past = 2 * a.c.total_new * a.c.n_units * kRow4 > (int64_t(128) << 20);
  if (past) hipLaunchKernelGGL((paged_read_kernel<T, true, true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_read_kernel<T, true, false>), grid, dim3(256), 0, stream, a);
}

hipError_t launch_paged_read(const PagedReadArgs& a, bool four, bool half, hipStream_t stream) {
  const int64_t blocks = (a.c.total_new * a.c.n_kv_heads + kReadRows - 1) / kReadRows;
  const int64_t x = blocks < kMaxBlocks ? blocks : kMaxBlocks;
  const dim3 grid(uint32_t(x), a.c.n_layers, uint32_t((blocks + x - 1) / x));
  if (!four) hipLaunchKernelGGL((paged_read_kernel<__bf16, false, false>), grid, dim3(256), 0, stream, a);
  else half ? read4<_Float16>(a, grid, stream) : read4<__bf16>(a, grid, stream);
  return hipGetLastError();
}

namespace {

template <typename T, bool FOUR>
void append(const PagedAppendArgs& a, bool few, dim3 grid, hipStream_t stream) {
  if (few) hipLaunchKernelGGL((paged_append_kernel<T, 4, FOUR>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_append_kernel<T, 1, FOUR>), grid, dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, bool four, bool half, hipStream_t stream) {
  // Few (token, layer) pairs: four waves each, for their latency; else a wave each, which
  // forms the angles once.  28 query heads, a wave / four waves each: 1 pair 4.7 / 3.4 us,
  // 448 pairs 6.0 / 4.7, 1024 pairs 6.9 / 5.9, 1792 pairs 9.2 / 10.1, 4096 pairs 14.3 /
  // 16.3, 87808 pairs 303 / 317.  Over 4 bits, where a wave has more to do, 7.3
  // / 4.7, 8.4 / 6.1, 9.1 / 7.6, 12.1 / 11.3, 18.4 / 22.1, 342 / 487: the same rule, though four
  // are still ahead at 1792.
  const bool few = a.c.total_new * a.c.n_layers <= 1024;
  // A grid has less than 2^32 threads along x, which 2^26 tokens reach: the rest of them
  // along z.
  const int64_t blocks = (a.c.total_new + (few ? 0 : 3)) / (few ? 1 : 4), x = blocks < kMaxBlocks ? blocks : kMaxBlocks;
  const dim3 grid(uint32_t(x), a.c.n_layers, uint32_t((blocks + x - 1) / x));
  if (four) half ? append<_Float16, true>(a, few, grid, stream) : append<__bf16, true>(a, few, grid, stream);
  else half ? append<_Float16, false>(a, few, grid, stream) : append<__bf16, false>(a, few, grid, stream);
  return hipGetLastError();
}

}  // namespace stlite
