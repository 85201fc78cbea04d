// Causal attention of new tokens over a paged cache (stlite_paged_attention):
//   out_t = sum_{j <= m_t} softmax_j(scale q_t . k_j) v_j,   m_t = len - n + t,
// in two forms, by the number of new tokens per sequence, and the launch that
// joins the parts of items that several work-groups share.
#include <type_traits>

#include "paged_plan.h"
#include "tile_lds.h"

namespace stlite {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// The page table of one sequence as a wave reads it: 64 entries in a register,
// one per lane, fetched by index without a memory access.
struct PageWindow {
  const int32_t* row;
  int32_t n_pages, last;  // last: index of the row's last entry
  int32_t base;           // first entry held
  int32_t held;           // this lane's entry
  uint64_t bad;           // entries out of range

  __device__ PageWindow(const PagedDev& c, int32_t seq)
      : row(c.page_table + int64_t(seq) * c.max_pages), n_pages(c.n_pages), last(c.max_pages - 1), base(-1), held(0), bad(0) {}

  // Makes the window hold `entry` (wave-uniform).
  __device__ void seek(int32_t entry) {
    if ((entry & ~63) == base) return;
    base = entry & ~63;
    const int32_t e = row[min(base + int32_t(threadIdx.x & 63), last)];
    const bool ok = e >= 0 && e < n_pages;
    held = ok ? e : 0;
    bad = __ballot(!ok);
  }
  __device__ int32_t page(int32_t entry) const { return __builtin_amdgcn_readlane(held, entry & 63); }
  __device__ bool is_bad(int32_t entry) const { return (bad >> (entry & 63)) & 1; }
};

// ---------------------------------------------------------------------------
// One new token per sequence
// ---------------------------------------------------------------------------
//
// HBM-bound: the pass streams K and V once.  Four waves take 16-key sub-tiles of
// a share in turn (a sub-tile lies in one page):
//   S^T = K Q^T   16x16x32, cached rows as the A operand read straight from HBM,
//                 the heads of the group (at most 16, zero padded) as B;
//   O += P V      v_mfma_f32_16x16x4_f32, which takes one cached row per lane and
//                 k-step: V needs no transpose and P stays fp32.
constexpr int kDecWaves = 4;
constexpr int kDecHeads = 16;

__device__ inline u32x4_t load_row16(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}

template <typename T>
__global__ __launch_bounds__(kDecWaves * 64, 2) void paged_decode_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = kDecWaves * 64;
  __shared__ float sm_m[kDecWaves][kDecHeads], sm_l[kDecWaves][kDecHeads];
  __shared__ float sm_o[kDecWaves][kDecHeads][kHeadDim];
  __shared__ typename PagedPlan<NT>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<NT> plan(a, sm_plan);
  int64_t x = int64_t(blockIdx.x) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  if (x >= y) return;
  PagedItem it = plan.find(x);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = lane & 15, quad = lane >> 4;
  const int32_t in_page = (1 << c.page_shift) - 1;
  for (bool first = true;; first = false) {
    const int unit = it.unit / a.parts, part = it.unit % a.parts;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const int32_t heads = min(c.group - part * kDecHeads, kDecHeads);
    const PagedPart span = paged_part(x, y, it.start, it.keys);
    const bool whole = span.whole;
    const int32_t k0 = span.t0 * kPagedTile, k1 = min(span.t1 * kPagedTile, max(it.cached + it.n, 0));
    const int64_t qrow = (int64_t(layer) * c.total_new + it.row0) * c.n_q_heads + int64_t(kv) * c.group + part * kDecHeads;

    x8 qb[4];
    {
      const uint16_t* p = a.q + (qrow + head) * kHeadDim;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        u32x4_t w = u32x4_t{0u, 0u, 0u, 0u};
        if (head < heads) w = *reinterpret_cast<const u32x4_t*>(p + kk * 32 + quad * 8);
        qb[kk] = __builtin_bit_cast(x8, w);
      }
    }
    float m_run = -INFINITY, l_run = 0.0f;
    f32x4_t o[8];  // O[head 4 quad + r][dim 8 (lane & 15) + db]
#pragma unroll
    for (int db = 0; db < 8; ++db) o[db] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    PageWindow pages(c, it.seq);
    u32x4_t kx[4], vx[4];
    // Keys past the end repeat the last one.
    auto load = [&](int32_t j0) {
      const int32_t entry = j0 >> c.page_shift;
      pages.seek(entry);
      const int64_t row = page_row(c, unit, pages.page(entry));
      const uint16_t* kp = c.k + row * kHeadDim;
      const uint16_t* vp = c.v + row * kHeadDim;
      const int32_t jk = min(j0 + (lane & 15), k1 - 1) & in_page;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) kx[kk] = load_row16(kp + jk * kHeadDim + kk * 32 + quad * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t jv = min(j0 + 4 * quad + i, k1 - 1) & in_page;
        vx[i] = load_row16(vp + jv * kHeadDim + (lane & 15) * 8);
      }
      return pages.is_bad(entry);
    };
    int32_t j0 = k0 + 16 * wave;
    bool bad_next = false;
    if (j0 < k1) bad_next = load(j0);
    for (; j0 < k1; j0 += 16 * kDecWaves) {
      const u32x4_t kc[4] = {kx[0], kx[1], kx[2], kx[3]};
      u32x4_t vc[4] = {vx[0], vx[1], vx[2], vx[3]};
      const bool bad = bad_next;
      if (j0 + 16 * kDecWaves < k1) bad_next = load(j0 + 16 * kDecWaves);
      if (bad) continue;
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) s = E::mfma16(__builtin_bit_cast(x8, kc[kk]), qb[kk], s);
      float xs[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xs[i] = s[i] * a.scale2;
      if (j0 + 16 > k1) {  // rows past the end: no weight, and nothing for it to meet
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j0 + 4 * quad + i >= k1) {
            xs[i] = -INFINITY;
            vc[i] = u32x4_t{0u, 0u, 0u, 0u};
          }
      }
      float mt = fmaxf(fmaxf(xs[0], xs[1]), fmaxf(xs[2], xs[3]));
      mt = fmaxf(mt, __shfl_xor(mt, 16));
      mt = fmaxf(mt, __shfl_xor(mt, 32));
      const float m_new = fmaxf(m_run, mt);
      const float m_use = m_new == -INFINITY ? 0.0f : m_new;
      if (__ballot(m_new > m_run)) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= alpha;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float ar = __shfl(alpha, 4 * quad + r);
#pragma unroll
          for (int db = 0; db < 8; ++db) o[db][r] *= ar;
        }
        m_run = m_new;
      }
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(xs[i] - m_use);
      l_run += (p[0] + p[1]) + (p[2] + p[3]);
      // k-step i pairs lane (head, quad) with key j0 + 4 quad + i
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const float b = (db & 1) ? elem_hi<T>(vc[i][db >> 1]) : elem_lo<T>(vc[i][db >> 1]);
          o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], b, o[db], 0, 0, 0);
        }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);

    // Merge the waves (one without rows has max -inf and weighs nothing).
    if (!first) __syncthreads();  // the last item's merge has read these
    if (lane < kDecHeads) {
      sm_m[wave][lane] = m_run;
      sm_l[wave][lane] = l_run;
    }
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) sm_o[wave][4 * quad + r][(lane & 15) * 8 + db] = o[db][r];
    __syncthreads();
    const int64_t slot = paged_slot(blockIdx.x, plan.share, it.start) * kDecHeads;
    for (int e = threadIdx.x; e < heads * (kHeadDim / 2); e += NT) {
      const int h = e / (kHeadDim / 2), dim = e % (kHeadDim / 2) * 2;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kDecWaves; ++w) M = fmaxf(M, sm_m[w][h]);
      float L = 0.0f, O0 = 0.0f, O1 = 0.0f;
#pragma unroll
      for (int w = 0; w < kDecWaves; ++w) {
        const float wt = sm_m[w][h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[w][h] - M);
        L += wt * sm_l[w][h];
        O0 += wt * sm_o[w][h][dim];
        O1 += wt * sm_o[w][h][dim + 1];
      }
      if (whole) {
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        *reinterpret_cast<uint32_t*>(a.out + (qrow + h) * kHeadDim + dim) = elem_pack<T>(O0 * inv, O1 * inv);
      } else {
        *reinterpret_cast<float2*>(a.po + (slot + h) * kHeadDim + dim) = make_float2(O0, O1);
        if (dim == 0) {
          a.pm[slot + h] = M;
          a.pl[slot + h] = L;
        }
      }
    }
    x = span.end;
    if (x >= y) break;
    plan.next(it);
  }
}

// ---------------------------------------------------------------------------
// Several new tokens per sequence
// ---------------------------------------------------------------------------
//
// An item's rows (token-major, all query heads of the kv head) are cut into
// blocks of 32, one per wave; the work-group streams 64-key tiles of K and V
// through a ring in LDS (direct DMA).  Everything is transposed, so that a lane
// owns one query (column lane & 31; two lanes share it, each with half the keys)
// and the softmax needs no exchange but one swap:
//   S^T = K Q^T      32x32x16, A: K rows from LDS, B: queries in registers;
//   P^T              exp2 of the accumulators, packed where they are: register
//                    order is a permutation of the keys within 16, which the V
//                    reads follow;
//   O^T += V^T P^T   A: V read transposed from LDS (ds_read_b64_tr_b16).
// The running maximum moves only when a tile exceeds it by 2^kLazy, so that the
// output is rescaled rarely.

constexpr float kLazy = 8.0f;
constexpr int kExtTile = kPagedTile;
constexpr int kTileBytes = kExtTile * kHeadDim * 2;

typedef __attribute__((address_space(3))) u32x2_t* lds_u32x2_t;

// Four keys of one dimension per lane: each group of 16 lanes reads 4 rows of 16
// elements (lane i: row i >> 2, elements 4 (i & 3) ..) and gets them transposed.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ inline u32x2_t read_transposed(uint32_t lds) {
  typedef __attribute__((address_space(3))) s16x4_t* ptr_t;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr_t)(uintptr_t)lds));
}

template <typename T, int NW>
__global__ __launch_bounds__(NW * 64, 2) void paged_extend_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = NW * 64;
  constexpr int kStages = NW == 8 ? 3 : 2;
  constexpr int kRows = NW * 32;
  constexpr int kLoads = 2 * 16 / NW;  // DMA instructions of a wave per tile
  __shared__ __align__(1024) uint16_t sm_tiles[kStages * 2 * kTileBytes / 2];  // [stage][K, V][64][128]
  __shared__ typename PagedPlan<NT>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<NT> plan(a, sm_plan);
  int64_t x = int64_t(blockIdx.x) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  if (x >= y) return;
  PagedItem it = plan.find(x);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int32_t in_page = (1 << c.page_shift) - 1;
  const uint32_t lds0 = uint32_t(reinterpret_cast<uintptr_t>(sm_tiles));
  // K: chunk (16 bytes) q of key k lies at slot q ^ (k & 15): 16 keys' reads of
  // one chunk take 16 slots.  V: at slot q ^ (4 (k & 3) + (k >> 2 & 3)): a
  // transposed read of 4 keys x 32 dimensions takes all 16 slots.
  uint32_t k_at[8], v_at[4][2];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) k_at[kk] = col * 256 + (((2 * kk + h) ^ (col & 15)) << 4);
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int i = lane & 15;
      const int chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      v_at[db][r] = kTileBytes + (8 * r + 4 * h + (i >> 2)) * 256 + ((chunk ^ (4 * (i >> 2) + 2 * r + h)) << 4) + (i & 1) * 8;
    }

  for (;;) {
    const int unit = it.unit;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const PagedPart span = paged_part(x, y, it.start, it.keys);
    const bool whole = span.whole;
    const int32_t tok0 = it.index * a.tokens, toks = min(it.n - tok0, a.tokens);
    const int32_t rows = toks * c.group;
    const int32_t seen = max(it.cached + tok0 + toks, 0);  // keys that the last token sees
    const int32_t t0 = span.t0, t1 = min(span.t1, (seen + kPagedTile - 1) / kPagedTile);
    // This lane's query (rows past the item's repeat the last one).
    const int32_t row = min(wave * 32 + col, rows - 1);
    const int32_t tok = row / c.group, head = row - tok * c.group;
    const int32_t limit = it.cached + tok0 + tok;  // last key that it sees
    const int64_t qrow = (int64_t(layer) * c.total_new + it.row0 + tok0 + tok) * c.n_q_heads + int64_t(kv) * c.group + head;
    const bool live = wave * 32 < rows;
    const int32_t limit_lo = __builtin_amdgcn_readfirstlane(limit);
    const int32_t limit_hi = __builtin_amdgcn_readlane(limit, 31);

    x8 qf[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      qf[kk] = __builtin_bit_cast(x8, *reinterpret_cast<const u32x4_t*>(a.q + qrow * kHeadDim + kk * 16 + h * 8));
    float m_ref = -INFINITY, l_run = 0.0f;
    f32x16_t o[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;

    PageWindow pages(c, it.seq);
    // Bad 16-key groups of tile t, which the window holds (bit g: keys 16 g .. 16 g + 15).
    auto bad_groups = [&](int32_t t) {
      if (pages.bad == 0) return 0u;
      uint32_t m = 0;
#pragma unroll
      for (int g = 0; g < 4; ++g) m |= uint32_t(pages.is_bad(min((t * kExtTile + 16 * g) >> c.page_shift, c.max_pages - 1))) << g;
      return m;
    };

    auto issue = [&](int32_t t, int stage) {
      const int32_t first_entry = (t * kExtTile) >> c.page_shift;
      pages.seek(first_entry);
      // this wave's keys lie in one page
      const int32_t key0 = t * kExtTile + wave * (kExtTile / NW);
      const int32_t entry = min(key0, seen - 1) >> c.page_shift;
      const int64_t base = page_row(c, unit, pages.page(entry)) * kHeadDim;
      const __amdgpu_buffer_rsrc_t kr =
          __builtin_amdgcn_make_buffer_rsrc(c.k + base, 0, (in_page + 1) * (kHeadDim * 2), kBufferFlags);
      const __amdgpu_buffer_rsrc_t vr =
          __builtin_amdgcn_make_buffer_rsrc(c.v + base, 0, (in_page + 1) * (kHeadDim * 2), kBufferFlags);
      const uint32_t dst0 = lds0 + stage * (2 * kTileBytes) + wave * (kTileBytes / NW);
#pragma unroll
      for (int g = 0; g < kLoads / 2; ++g) {
        const int32_t kl = wave * (kExtTile / NW) + 4 * g + (lane >> 4);  // key within the tile
        const uint32_t r = uint32_t(min(t * kExtTile + kl, seen - 1) & in_page) * (kHeadDim * 2);
        const uint32_t kc = uint32_t((lane & 15) ^ (kl & 15)) * 16u;
        const uint32_t vc = uint32_t((lane & 15) ^ (4 * (kl & 3) + ((kl >> 2) & 3))) * 16u;
        uint32_t kd = dst0 + g * 1024, vd = kd + kTileBytes;
        asm volatile("" : "+s"(kd), "+s"(vd));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void_t)(uintptr_t)kd, 16, r + kc, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void_t)(uintptr_t)vd, 16, r + vc, 0, 0, 0);
      }
      return bad_groups(t);
    };

    auto tile = [&](int32_t t, int stage, auto masked, uint32_t bad) {
      constexpr bool kMasked = decltype(masked)::value;
      const uint32_t base = lds0 + stage * (2 * kTileBytes);
      f32x16_t s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          const x8 kf = *reinterpret_cast<const __attribute__((address_space(3))) x8*>((uintptr_t)(base + k_at[kk] + kb * 8192));
          s[kb] = E::mfma32(kf, qf[kk], s[kb]);
        }
      }
      if (kMasked) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int32_t key = t * kExtTile + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
            if (key > limit || ((bad >> (2 * kb + (i >> 3))) & 1)) s[kb][i] = -INFINITY;
          }
      }
      float mt = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kb][i]);
      float other = mt;
      swap32(mt, other);
      mt = fmaxf(mt, other) * a.scale2;
      if (__ballot(mt > m_ref + kLazy + E::kBias)) {
        const float m_new = fmaxf(m_ref, mt - E::kBias);
        const float alpha = m_ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
        m_ref = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
      const float minus_m = m_ref == -INFINITY ? 0.0f : -m_ref;
      x8 pf[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        u32x4_t w;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kk >> 1][8 * (kk & 1) + j], a.scale2, minus_m));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kk >> 1][8 * (kk & 1) + j + 1], a.scale2, minus_m));
          l_run += p0 + p1;
          w[j >> 1] = elem_pack<T>(p0, p1);
        }
        pf[kk] = __builtin_bit_cast(x8, w);
      }
      uint32_t odd = 0;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const u32x2_t lo = read_transposed(base + v_at[db][0] + kk * 4096);
          const u32x2_t hi = read_transposed(base + v_at[db][1] + kk * 4096);
          u32x4_t w = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
          if (kMasked) {
            // 0 * infinity is no zero: what is not finite is left out here
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t nf = E::not_finite(w[j]);
              odd |= nf;
              w[j] &= ~((nf >> 15) * 0xffffu);
            }
          }
          o[db] = E::mfma32(__builtin_bit_cast(x8, w), pf[kk], o[db]);
        }
      if (kMasked && __ballot(odd != 0)) {
        // and reaches the queries that see it here: p v is v, for v infinite or NaN
#pragma unroll 1
        for (int32_t kl = 0; kl < kExtTile; ++kl) {
          const int32_t key = t * kExtTile + kl;
          if (key >= seen || ((bad >> (kl >> 4)) & 1)) continue;
          const uint32_t swz = 4 * (kl & 3) + ((kl >> 2) & 3);
#pragma unroll
          for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t dim = 32 * db + 8 * (i >> 2) + 4 * h + (i & 3);
              const uint32_t at = base + kTileBytes + kl * 256 + (((dim >> 3) ^ swz) << 4) + (dim & 7) * 2;
              const uint16_t e = *reinterpret_cast<const __attribute__((address_space(3))) uint16_t*>((uintptr_t)at);
              if (E::not_finite(e) && key <= limit) o[db][i] += elem_lo<T>(e);
            }
        }
      }
    };

    __syncthreads();  // the last item's tiles have been read
    // (stores of the last item and loads so far must not count among the DMAs)
    wait_vmcnt<0>();
    uint32_t bad[kStages - 1] = {};  // of the tiles in flight
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
      if (t0 + i < t1) bad[i] = issue(t0 + i, i);
    int stage = 0;
    for (int32_t t = t0; t < t1; ++t) {
      if (kStages == 3 && t + 1 < t1) wait_vmcnt<kLoads>();
      else wait_vmcnt<0>();
      barrier_lds();
      const uint32_t bad_now = bad[0];
#pragma unroll
      for (int i = 0; i + 1 < kStages - 1; ++i) bad[i] = bad[i + 1];
      if (t + kStages - 1 < t1) bad[kStages - 2] = issue(t + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
      if (live && t * kExtTile <= limit_hi) {
        if (bad_now || t * kExtTile + kExtTile - 1 > limit_lo) tile(t, stage, std::true_type{}, bad_now);
        else tile(t, stage, std::false_type{}, 0u);
      }
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }

    float other = l_run;
    swap32(l_run, other);
    l_run += other;
    if (wave * 32 + col < rows) {
      if (whole) {
        const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
        uint16_t* p = a.out + qrow * kHeadDim + 4 * h;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            u32x2_t w;
            w[0] = elem_pack<T>(o[db][4 * g] * inv, o[db][4 * g + 1] * inv);
            w[1] = elem_pack<T>(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv);
            *reinterpret_cast<u32x2_t*>(p + 32 * db + 8 * g) = w;
          }
      } else {
        const int64_t slot = paged_slot(blockIdx.x, plan.share, it.start) * kRows + wave * 32 + col;
        float* p = a.po + slot * kHeadDim + 4 * h;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4_t*>(p + 32 * db + 8 * g) =
                f32x4_t{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
        if (h == 0) {
          a.pm[slot] = m_ref;
          a.pl[slot] = l_run;
        }
      }
    }
    x = span.end;
    if (x >= y) break;
    plan.next(it);
  }
}

// ---------------------------------------------------------------------------
// Joining the parts
// ---------------------------------------------------------------------------
//
// Work-group (w, z) joins the rows 8 z .. 8 z + 7 of the item that the boundary
// between shares w and w + 1 cuts, if w is the first share in it: 32 lanes x 4
// dimensions per part, 8 parts at a time.
constexpr int kJoinRows = 8;

template <typename T>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  __shared__ float sm_m[8], sm_l[8];
  __shared__ f32x4_t sm_o[8][32];
  __shared__ typename PagedPlan<256>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<256> plan(a, sm_plan);
  const int64_t cut = (int64_t(blockIdx.x) + 1) * plan.share;
  if (cut >= plan.total) return;
  const PagedItem it = plan.find(cut);
  if (it.start == cut || it.start / plan.share != int64_t(blockIdx.x)) return;
  const int32_t w0 = blockIdx.x, w1 = int32_t((it.start + it.keys - 1) / plan.share);
  const int unit = it.unit / a.parts, part = it.unit % a.parts;
  const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
  const int32_t tok0 = it.index * a.tokens;
  const int32_t head0 = part * kDecHeads;  // (one part but for decode)
  const int32_t rows = a.parts > 1 ? min(c.group - head0, kDecHeads) : min(it.n - tok0, a.tokens) * c.group;
  const int grp = threadIdx.x >> 5, l32 = threadIdx.x & 31;
  for (int32_t row = blockIdx.y * kJoinRows; row < min(rows, int32_t(blockIdx.y + 1) * kJoinRows); ++row) {
    float M = -INFINITY, L = 0.0f;
    f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int32_t w = w0 + grp; w <= w1; w += 8) {
      const int64_t slot = paged_slot(w, plan.share, it.start) * a.rows + row;
      const float m = a.pm[slot];
      if (m == -INFINITY) continue;
      const float l = a.pl[slot];
      const f32x4_t o = *reinterpret_cast<const f32x4_t*>(a.po + slot * kHeadDim + 4 * l32);
      const float mx = fmaxf(M, m);
      const float f = __builtin_amdgcn_exp2f(M - mx), g = __builtin_amdgcn_exp2f(m - mx);
      L = L * f + l * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) O[i] = O[i] * f + o[i] * g;
      M = mx;
    }
    __syncthreads();
    sm_o[grp][l32] = O;
    if (l32 == 0) {
      sm_m[grp] = M;
      sm_l[grp] = L;
    }
    __syncthreads();
    if (grp == 0) {
      float mx = -INFINITY;
#pragma unroll
      for (int g = 0; g < 8; ++g) mx = fmaxf(mx, sm_m[g]);
      L = 0.0f;
      O = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const float f = sm_m[g] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[g] - mx);
        L += f * sm_l[g];
#pragma unroll
        for (int i = 0; i < 4; ++i) O[i] += f * sm_o[g][l32][i];
      }
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      const int32_t tok = row / c.group;
      const int64_t orow = a.parts > 1 ? (int64_t(layer) * c.total_new + it.row0) * c.n_q_heads + int64_t(kv) * c.group + head0 + row
                                       : (int64_t(layer) * c.total_new + it.row0 + tok0 + tok) * c.n_q_heads +
                                             int64_t(kv) * c.group + (row - tok * c.group);
      u32x2_t w;
      w[0] = elem_pack<T>(O[0] * inv, O[1] * inv);
      w[1] = elem_pack<T>(O[2] * inv, O[3] * inv);
      *reinterpret_cast<u32x2_t*>(a.out + orow * kHeadDim + 4 * l32) = w;
    }
  }
}

template <typename T>
hipError_t launch_join(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.shares < 2) return hipSuccess;
  const int32_t rows = a.parts > 1 ? kDecHeads : a.tokens * a.c.group;
  hipLaunchKernelGGL((paged_join_kernel<T>), dim3(a.shares - 1, (rows + kJoinRows - 1) / kJoinRows), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <typename T>
hipError_t decode(const PagedAttnArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((paged_decode_kernel<T>), dim3(a.shares), dim3(kDecWaves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<T>(a, stream);
}

template <typename T, int NW>
hipError_t extend(const PagedAttnArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((paged_extend_kernel<T, NW>), dim3(a.shares), dim3(NW * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<T>(a, stream);
}

}  // namespace

hipError_t launch_paged_decode(const PagedAttnArgs& a, bool half, hipStream_t stream) {
  return half ? decode<_Float16>(a, stream) : decode<__bf16>(a, stream);
}

hipError_t launch_paged_extend(const PagedAttnArgs& a, bool half, int32_t waves, hipStream_t stream) {
  if (half) return waves == 8 ? extend<_Float16, 8>(a, stream) : extend<_Float16, 4>(a, stream);
  return waves == 8 ? extend<__bf16, 8>(a, stream) : extend<__bf16, 4>(a, stream);
}

}  // namespace stlite
