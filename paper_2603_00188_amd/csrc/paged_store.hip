// Rows into a paged cache: the compression's kept rows (a gather, as the dense
// compaction) and the new tokens of a serving step (norm and rotation on the way).
#include "paged.h"
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
  if (blockIdx.x == 0 && unit == 0)
    for (int32_t s = threadIdx.x; s < a.c.n_seqs; s += 256) a.c.seq_lens[s] = a.cu_budget[s + 1] - a.cu_budget[s];
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
      const int32_t at = int32_t(j - a.cu_budget[s]);
      const int32_t entry = at >> a.c.page_shift;
      const int32_t page = entry < a.c.max_pages ? a.c.page_table[int64_t(s) * a.c.max_pages + entry] : -1;
      if (page >= 0 && page < a.c.n_pages) dst[r] = page_row(a.c, unit, page) + (at & ((1 << a.c.page_shift) - 1));
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

// ---------------------------------------------------------------------------
// New tokens
// ---------------------------------------------------------------------------

constexpr int64_t kMaxBlocks = int64_t(1) << 23;  // along x

// Sums of squares that fp32 holds to its full precision.  A row outside (bf16 values above
// 2^60 or all below 2^-50) is scaled by a power of two, and eps by its square, before its
// norm; a small one only where eps does not hide it, so that the scaled eps stays finite.
// (3136 normed tokens of 28 layers take 298 us; without it 295.5, in 64 bits 310.)
constexpr float kLeastSum = 0x1p-100f, kMostSum = 0x1p120f, kLeastEps = 0x1p-80f;

// One (token, layer) by `WAVES` waves.  Eight lanes hold a head: lane c the
// dimensions 8c .. 8c+7 and 64+8c .. 64+8c+7, so both members of every pair of
// either pairing lie in one lane.  The 64 (cos, sin) of the token are formed
// once, one pair per lane, and kept in registers over the token's heads.
// Angles: position * turns in 64 bits, reduced to a fraction of a turn there;
// the sine of the reduced angle in fp32.
// HBM-bound once there are a few thousand rows: 3136 tokens of 28 layers (1.62 GB read
// and written) take 298 us, 5.4 TB/s; 64 tokens of 28 layers (44 MB) 12.3 us, 3.6 TB/s,
// where the chain of dependent loads (sequence, length, page, row) is half of it.
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int kTok = 4 / WAVES;  // tokens per work-group
  __shared__ float2 sm_cs[kTok][64];
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
    const double turn = double(a.positions[axis * c.total_new + tok]) * a.turns[lane];
    const float r = float(turn - rint(turn));
    sm_cs[tl][lane] = make_float2(cospif(2.0f * r), sinpif(2.0f * r));
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

hipError_t launch_paged_compact(const PagedCompactArgs& a, hipStream_t stream) {
  // (one work-group for the lengths where nothing is kept)
  const int64_t blocks = a.total_budget > 0 ? (a.total_budget + kRowsPerGroup - 1) / kRowsPerGroup : 1;
  hipLaunchKernelGGL(paged_compact_kernel, dim3(uint32_t(blocks), a.c.n_units), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, bool half, hipStream_t stream) {
  // Few (token, layer) pairs: four waves each, for their latency; else a wave each, which
  // forms the angles once.  28 query heads, a wave / four waves each: 1 pair 4.7 / 3.4 us,
  // 448 pairs 6.0 / 4.7, 1024 pairs 6.9 / 5.9, 1792 pairs 9.2 / 10.1, 4096 pairs 14.3 /
  // 16.3, 87808 pairs 303 / 317.
  const bool few = a.c.total_new * a.c.n_layers <= 1024;
  // A grid has less than 2^32 threads along x, which 2^26 tokens reach: the rest of them
  // along z.
  const int64_t blocks = (a.c.total_new + (few ? 0 : 3)) / (few ? 1 : 4), x = blocks < kMaxBlocks ? blocks : kMaxBlocks;
  const dim3 grid(uint32_t(x), a.c.n_layers, uint32_t((blocks + x - 1) / x));
  if (half) {
    if (few) hipLaunchKernelGGL((paged_append_kernel<_Float16, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_append_kernel<_Float16, 1>), grid, dim3(256), 0, stream, a);
  } else {
    if (few) hipLaunchKernelGGL((paged_append_kernel<__bf16, 4>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_append_kernel<__bf16, 1>), grid, dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace stlite
