// Causal attention of new tokens over a paged cache (stlite_paged_attention):
//   out_t = sum_{j <= m_t} softmax_j(scale q_t . k_j) v_j,   m_t = len - n + t,
// in two forms, by the number of new tokens per sequence, and the launch that
// joins the parts of items that several work-groups share.
#include <float.h>

#include <type_traits>

#include "paged4.h"
#include "paged_plan.h"
#include "tile_lds.h"

namespace stlite {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// A PageWindow with the entries in LDS, 64 words of this wave's own: a register held
// through a long loop is dear in the several-token kernel.
struct LdsPageWindow {
  const int32_t* row;
  int32_t n_pages, last, base;
  uint64_t bad;
  uint32_t at;

  __device__ LdsPageWindow(const PagedDev& c, int32_t seq, uint32_t lds)
      : row(c.page_table + int64_t(seq) * c.max_pages), n_pages(c.n_pages), last(c.max_pages - 1), base(-1), bad(0), at(lds) {}

  __device__ void seek(int32_t entry) {
    if ((entry & ~63) == base) return;
    base = entry & ~63;
    const int32_t lane = threadIdx.x & 63;
    const int32_t e = row[min(base + lane, last)];
    const bool ok = e >= 0 && e < n_pages;
    *reinterpret_cast<volatile __attribute__((address_space(3))) int32_t*>((uintptr_t)(at + lane * 4)) = ok ? e : 0;
    bad = __ballot(!ok);
  }
  // The page on every lane (a read that the caller need not wait for yet).
  __device__ int32_t peek(int32_t entry) const {
    return *reinterpret_cast<const volatile __attribute__((address_space(3))) int32_t*>((uintptr_t)(at + (entry & 63) * 4));
  }
  __device__ int32_t page(int32_t entry) const { return __builtin_amdgcn_readfirstlane(peek(entry)); }
  __device__ bool is_bad(int32_t entry) const { return (bad >> (entry & 63)) & 1; }
};

// ---------------------------------------------------------------------------
// One new token per sequence
// ---------------------------------------------------------------------------
//
// HBM-bound: the pass streams K and V once.  Four waves take 16-key sub-tiles of
// a share in turn (a sub-tile lies in one page), the next one's loads under this one's
// arithmetic:
//   S^T = K Q^T   16x16x32, cached rows as the A operand read straight from HBM,
//                 the heads of the group (zero padded to 16 or 32) as B;
//   O += P V      16x16x16, whose layout takes P where S^T left it (four keys of a head
//                 per lane) and V as it was read, four keys of a lane put together by
//                 byte permutes.  P stays fp32 by way of terms: three bf16 (8 bits each),
//                 or two fp16, a product each.  In fp32 products P and V took four times
//                 as long, which two blocks of heads could not hide: 20 heads of a kv
//                 head 66 us (16 at a time), now 48 with 32 at once and 64 with 16.
// 28 layers x 28 heads behind 30105 tokens 267 us (1.73 GB, 6.5 TB/s), a layer behind
// 150528 54 (308 MB, 5.7), 64 sequences of up to 8000 in 4 layers 697 (4.62 GB, 6.6).
constexpr int kDecWaves = 4;

__device__ inline u32x4_t load_row16(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}

template <typename T, int NG>  // 16 NG heads to an item
__global__ __launch_bounds__(kDecWaves * 64, 2) void paged_decode_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = kDecWaves * 64, kHeads = 16 * NG;
  __shared__ float sm_m[kDecWaves][kHeads], sm_l[kDecWaves][kHeads];
  __shared__ float sm_o[kDecWaves][kHeads][kHeadDim];
  __shared__ typename PagedPlan<NT>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<NT> plan(a, sm_plan);
  int64_t x = int64_t(blockIdx.x) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  if (x >= y) return;
  PagedItem it = plan.find(x);
  if (it.start >= y) return;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = lane & 15, quad = lane >> 4;
  const int32_t in_page = (1 << c.page_shift) - 1;
  for (bool first = true;; first = false) {
    const int unit = it.unit / a.parts, part = it.unit % a.parts;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const int32_t heads = min(c.group - part * kHeads, kHeads);
    const PagedPart span = paged_part(x, y, it.start, it.keys);
    const bool whole = span.whole;
    const int32_t k0 = span.t0 * kPagedTile, k1 = min(span.t1 * kPagedTile, max(it.cached + it.n, 0));
    const int64_t qrow = (int64_t(layer) * c.total_new + it.row0) * c.n_q_heads + int64_t(kv) * c.group + part * kHeads;

    x8 qb[NG][4];
    {
#pragma unroll
      for (int ng = 0; ng < NG; ++ng) {
        const uint16_t* p = a.q + (qrow + 16 * ng + head) * kHeadDim;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          u32x4_t w = u32x4_t{0u, 0u, 0u, 0u};
          if (16 * ng + head < heads) w = *reinterpret_cast<const u32x4_t*>(p + kk * 32 + quad * 8);
          qb[ng][kk] = __builtin_bit_cast(x8, w);
        }
      }
    }
    float m_run[NG], l_run[NG];
    f32x4_t o[NG][8];  // O[head 16 ng + 4 quad + r][dim 8 (lane & 15) + db]

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
    // The share's sub-tiles.  A term of a weight may be zero, and zero times infinity is no
    // infinity: where something came out that is not finite, once more without the values
    // that are not, which are then added (p v is v for them, whatever the weight).
    bool again = false;
    for (bool odd = false;; odd = true) {
#pragma unroll
      for (int ng = 0; ng < NG; ++ng) {
        m_run[ng] = -INFINITY;
        l_run[ng] = 0.0f;
#pragma unroll
        for (int db = 0; db < 8; ++db) o[ng][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
      int32_t j0 = k0 + 16 * wave;
      bool bad_next = false;
      if (j0 < k1) bad_next = load(j0);
      for (; j0 < k1; j0 += 16 * kDecWaves) {
        const u32x4_t kc[4] = {kx[0], kx[1], kx[2], kx[3]};
        u32x4_t vc[4] = {vx[0], vx[1], vx[2], vx[3]};
        const bool bad = bad_next;
        if (j0 + 16 * kDecWaves < k1) bad_next = load(j0 + 16 * kDecWaves);
        if (bad) continue;
        const bool ends = j0 + 16 > k1;
        if (ends) {  // rows past the end: no weight, and nothing for it to meet
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (j0 + 4 * quad + i >= k1) vc[i] = u32x4_t{0u, 0u, 0u, 0u};
        }
        if (odd) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) vc[i][j] &= ~((E::not_finite(vc[i][j]) >> 15) * 0xffffu);
        }
        u32x2_t terms[NG][E::kTerms];  // the weights of four keys
#pragma unroll
        for (int ng = 0; ng < NG; ++ng) {
          f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) s = E::mfma16(__builtin_bit_cast(x8, kc[kk]), qb[ng][kk], s);
          float xs[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) xs[i] = ends && j0 + 4 * quad + i >= k1 ? -INFINITY : base2(s[i], a.scale2);
          float mt = fmaxf(fmaxf(xs[0], xs[1]), fmaxf(xs[2], xs[3]));
          mt = fmaxf(mt, __shfl_xor(mt, 16));
          mt = fmaxf(mt, __shfl_xor(mt, 32));
          const float m_new = fmaxf(m_run[ng], mt);
          const float m_use = m_new == -INFINITY ? 0.0f : m_new;
          if (__ballot(m_new > m_run[ng])) {
            const float alpha = __builtin_amdgcn_exp2f(m_run[ng] - m_use);
            l_run[ng] *= alpha;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float ar = __shfl(alpha, 4 * quad + r);
#pragma unroll
              for (int db = 0; db < 8; ++db) o[ng][db][r] *= ar;
            }
            m_run[ng] = m_new;
          }
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(xs[i] - m_use + E::kTermsBias);
          l_run[ng] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
          for (int n = 0; n < E::kTerms; ++n) {
            terms[ng][n][0] = E::take(p[0], p[1], n == E::kTerms - 1);
            terms[ng][n][1] = E::take(p[2], p[3], n == E::kTerms - 1);
          }
        }
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const uint32_t half = (db & 1) ? 0x07060302u : 0x05040100u;
          u32x2_t b;  // dimension db of the lane's four keys
          b[0] = __builtin_amdgcn_perm(vc[1][db >> 1], vc[0][db >> 1], half);
          b[1] = __builtin_amdgcn_perm(vc[3][db >> 1], vc[2][db >> 1], half);
#pragma unroll
          for (int n = 0; n < E::kTerms; ++n)
#pragma unroll
            for (int ng = 0; ng < NG; ++ng) o[ng][db] = E::mfma16(terms[ng][n], b, o[ng][db]);
        }
      }
      if (odd) break;
      float z = 0.0f;
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
          for (int r = 0; r < 4; ++r) z = fmaf(o[ng][db][r], 0.0f, z);
      again = __ballot(z != z) != 0;
      if (!again) break;
    }
    if (again) {
#pragma unroll 1
      for (int32_t j = k0 + 16 * wave; j < k1; j += (j & 15) == 15 ? 16 * kDecWaves - 15 : 1) {
        pages.seek(j >> c.page_shift);
        if (pages.is_bad(j >> c.page_shift)) continue;
        const u32x4_t e = load_row16(c.v + (page_row(c, unit, pages.page(j >> c.page_shift)) + (j & in_page)) * kHeadDim + (lane & 15) * 8);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const uint32_t bits = e[db >> 1] >> (16 * (db & 1)) & 0xffffu;
          const float x = E::not_finite(bits) ? elem_lo<T>(bits) : 0.0f;
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[ng][db][r] += x;
        }
      }
    }
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      l_run[ng] += __shfl_xor(l_run[ng], 16);
      l_run[ng] += __shfl_xor(l_run[ng], 32);
    }

    // Merge the waves (one without rows has max -inf and weighs nothing).
    if (!first) __syncthreads();  // the last item's merge has read these
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      if (lane < 16) {
        sm_m[wave][16 * ng + lane] = m_run[ng];
        sm_l[wave][16 * ng + lane] = l_run[ng];
      }
#pragma unroll
      for (int db = 0; db < 8; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) sm_o[wave][16 * ng + 4 * quad + r][(lane & 15) * 8 + db] = o[ng][db][r];
    }
    __syncthreads();
    const int64_t slot = paged_slot(blockIdx.x, plan.share, it.start) * kHeads;
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
    if (it.start >= y) break;
  }
}

// ---------------------------------------------------------------------------
// Several new tokens per sequence
// ---------------------------------------------------------------------------
//
// An item's rows (token-major, all query heads of the kv head, at most 256) are cut
// into blocks of 32, one for each of eight waves, which stream 64-key tiles of K and V
// through rings in LDS (direct DMA); a wave without rows only fetches.  (Items of 128
// rows, two waves to a block with 32 keys each, took the same 62 us for five drafted tokens,
// and 268, not 219, for prompts.)  Everything is transposed, so that a lane owns one query
// (column lane & 31; two lanes share it, each with half the keys) and the softmax
// needs no exchange but one swap:
//   S^T = K Q^T      32x32x16, A: K rows from LDS, B: queries in registers;
//   P^T              exp2 of the accumulators, packed where they are: register
//                    order is a permutation of the keys within 16, which the V
//                    reads follow;
//   O^T += V^T P^T   A: V read transposed from LDS (ds_read_b64_tr_b16).
// The weights are rounded to the type of the call, which the matrix instructions take: half
// a step of it, as the output.  A second term of each, as for one token, would add 1024
// cycles of products to a step's 2048.
// The reference of the weights moves only when a tile exceeds it by 2^kLazy, so that the
// output is rescaled rarely.  It is the greatest logit to within 2^-15, so that the
// greatest weight, a power of two to that precision, is rounded to one (a whole number
// instead made the error against 64 bits 0.0023, not 0.0020, behind 30k tokens), and has
// 14 bits behind the point: its sum with kBias is exact up to kFar, and one fused product
// and sum gives an exponent.  Beyond kFar the logits are rounded before it is taken off
// (an instruction more for each, but there a logit's rounding would use up the headroom
// above the reference, and the bias would be lost in it).
//
// A step of a wave has two halves: its products (the logits of tile t + 1, the
// values of tile t) and its vector work (the weights of tile t + 1, and DMA).  The
// two waves of a SIMD, w and w + 4, are half a step apart, so that one's products
// run under the other's vector work; a barrier ends each half.  Waves 0 - 3 fetch K,
// 4 - 7 V, into rings of four tiles: in the vector half of its step t the first group
// fetches K(t+4) in place of K(t), the second V(t+3) in place of V(t-1), and both
// groups' products of step t - 1, the last readers, are done by then.  At the end of
// its products a wave waits for all but its last tile's DMA, so that K(t+1) and V(t)
// have landed for everybody when anyone's step t begins.
//
// A step of 256 rows x 64 keys takes 3680 cycles, 2048 of them matrix instructions on
// every SIMD; by its instructions the softmax half is the longer one, and LDS reads take
// about 1420 of a half's 1840 cycles.  3136 tokens x 28 heads behind 30105 tokens take 1.38 ms, 1.03 PFLOP/s, at
// the 1.8 GHz that the power leaves; five tokens in each of 16 sequences 60 us, where the
// cache (225 MB) comes at 5.9 TB/s once the first tiles have; prompts of 131 to 2999
// tokens 204 us, 0.73 PFLOP/s.

constexpr float kLazy = 8.0f;
constexpr float kFar = 960.0f;  // 960 + 28 has 10 bits before the point
constexpr int kExtWaves = 8;
static_assert(kExtRows == kExtWaves * 32);
constexpr int kRing = 4;
constexpr int kTileBytes = kPagedTile * kHeadDim * 2;
constexpr int kTileLoads = 4;  // DMA instructions of a wave per tile: it fetches 16 keys, which lie in one page

// Four keys of one dimension per lane: each group of 16 lanes reads 4 rows of 16
// elements (lane i: row i >> 2, elements 4 (i & 3) ..) and gets them transposed.
__device__ inline u32x2_t read_transposed(uint32_t lds) {
  typedef __attribute__((address_space(3))) s16x4_t* ptr_t;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr_t)(uintptr_t)lds));
}

// 16 bytes per lane from offset `at` + `from` of a buffer to LDS address `to` + 16
// lane.  In assembly because the compiler, which cannot tell the tiles apart, would
// wait for every load in flight before each transposed read; it has no output
// register, and wait_vmcnt counts it.  The LDS address is an operand in M0, so that the
// compiler knows what M0 holds.  (The nops: M0 is read one wait state after it is written,
// a scalar that the vector unit wrote, as a page read from LDS is, five.)
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
__device__ inline void dma16(i32x4_t rsrc, uint32_t to, uint32_t at, uint32_t from) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(at), "s"(rsrc), "s"(from), "{m0}"(to) : "memory");
}

// The same of 4 bytes; lane j lands at `to` + 4 j.
__device__ inline void dma4(i32x4_t rsrc, uint32_t to, uint32_t at, uint32_t from) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, %2 offen lds" ::"v"(at), "s"(rsrc), "s"(from), "{m0}"(to) : "memory");
}

// FOUR: over a 4-bit pool.  The tiles come as they are, by DMA, kAhead4 of them under way
// (a wave's sixteen keys of a tile are one run of codes and one of scales), and the wave
// that fetched them turns them into 16-bit tiles in the vector half of its step, a block of
// 32 values to a lane: K(t+2) in place of K(t), V(t+2) in place of V(t), so rings of two do.
constexpr int kAhead4 = 2;  // (eight, which a short item has to issue before its first product: 72, not 66 us)
constexpr int kRaw4 = 16 * kCodes4 + 256;  // a wave's part of a tile: codes, and a row's scales for each lane

template <typename T, bool FOUR>
__global__ __launch_bounds__(kExtWaves * 64, 2) void paged_extend_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = kExtWaves * 64;
  constexpr int kSlots = FOUR ? 2 : kRing;
  __shared__ __align__(1024) uint16_t sm_tiles[2 * kSlots * kTileBytes / 2];  // K, then V: [slot][64][128]
  __shared__ __align__(1024) uint8_t sm_raw[FOUR ? kExtWaves * kAhead4 * kRaw4 : 16];
  typedef PagedPlan<NT, FOUR> Plan;
  __shared__ typename Plan::Shared sm_plan;
  __shared__ int32_t sm_pages[kExtWaves][64];
  __shared__ int2 sm_odd[kExtWaves];
  const PagedDev& c = a.c;
  Plan plan(a, sm_plan);
  // Work-groups go round the eight dies; the shares of a die lie one after another, so
  // that items of one kv head read its cache through one L2 (prompts 215 to 204 us, a
  // screen behind 30k tokens 1362 to 1353).
  const int32_t per_die = a.shares / 8, at_die = blockIdx.x / 8;
  const int32_t this_share = at_die < per_die ? int32_t(blockIdx.x % 8) * per_die + at_die : int32_t(blockIdx.x);
  int64_t x = int64_t(this_share) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  PagedItem it;
  if (!plan.first(x, y, it)) return;
  const int64_t share = plan.share;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave >> 2;  // half a step apart
  const int col = lane & 31, h = lane >> 5;
  const int32_t in_page = (1 << c.page_shift) - 1;
  const uint32_t lds0 = uint32_t(reinterpret_cast<uintptr_t>(sm_tiles));
  // K: chunk (16 bytes) q of key k lies at slot q ^ (k & 15): 16 keys' reads of
  // one chunk take 16 slots.  V: at slot q ^ (4 (k & 3) + (k >> 2 & 3)): a
  // transposed read of 4 keys x 32 dimensions takes all 16 slots.  Either way the
  // chunk's number enters an address by exclusive or alone, so one address per
  // lane gives all of them.
  const uint32_t k_lane = lds0 + col * 256 + ((h ^ (col & 15)) << 4);
  uint32_t v_lane;
  {
    const int i = lane & 15, c0 = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    v_lane = lds0 + kSlots * kTileBytes + (4 * h + (i >> 2)) * 256 + ((4 * (i >> 2) + (c0 ^ h)) << 4) + (i & 1) * 8;
  }
  // DMA load g brings keys 4 g + (lane >> 4) of the wave's sixteen: a lane's row and
  // the chunk that belongs in its 16 bytes (+ 1024 g, ^ 64 g or ^ 16 g).
  const int key0 = 16 * (wave & 3);
  const uint32_t dma_lane = (lane >> 4) * 256 + (((lane & 15) ^ (group ? 4 * (lane >> 4) : lane >> 4)) << 4);
  const uint32_t dma_swizzle = group ? 16 : 64;
  const uint16_t* const pool = group ? c.v : c.k;
  const uint32_t dma_lds = lds0 + (group * kSlots * kPagedTile + key0) * (kHeadDim * 2);
  // FOUR: a lane's block, lane & 3, of key lane4 of the wave's sixteen (eight lanes write
  // two keys' chunks at once, of V two whose slots differ in more than the block), and where
  // its first chunk goes (the next ones: ^ 16, ^ 32, ^ 48).
  const int lane4 = group ? ((lane >> 2 & 3) << 2) | lane >> 4 : lane >> 2;
  const uint32_t raw_lds = uint32_t(reinterpret_cast<uintptr_t>(sm_raw)) + wave * (kAhead4 * kRaw4);
  const uint32_t write4 = dma_lds + lane4 * 256 + (((lane & 3) << 2 ^ (group ? 4 * (lane4 & 3) + (lane4 >> 2) : lane4)) << 4);

  // The token of an item's row (below 256: the product's error is less than 1 / group), and
  // where its query lies behind the item's first one.
  const uint32_t per_row = 65535u / uint32_t(c.group) + 1u;
  auto token_of = [&](int32_t row) { return int32_t(uint32_t(row) * per_row >> 16); };
  auto query_of = [&](int32_t row) { return token_of(row) * (c.n_q_heads - c.group) + row; };

  for (;;) {
    const int unit = it.unit;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const PagedPart span = plan.part(x, y, it);
    const bool whole = span.whole;
    const int32_t tok0 = it.index * a.tokens, toks = min(it.n - tok0, a.tokens);
    const int32_t rows = toks * c.group;
    // (the same on every lane, kept in scalar registers for the tiles' addresses)
    const int32_t seen = __builtin_amdgcn_readfirstlane(max(it.cached + tok0 + toks, 0));  // keys that the last token sees
    const int32_t t0 = __builtin_amdgcn_readfirstlane(span.t0);
    const int32_t t1 = __builtin_amdgcn_readfirstlane(min(span.t1, (seen + kPagedTile - 1) / kPagedTile));
    // This lane's query (a row past the item's repeats the last one).
    const int32_t row = min(wave * 32 + col, rows - 1);
    const int64_t qrow0 = (int64_t(layer) * c.total_new + it.row0 + tok0) * c.n_q_heads + int64_t(kv) * c.group;
    const int32_t limit = it.cached + tok0 + token_of(row);  // last key that it sees
    x8 qf[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      qf[kk] = __builtin_bit_cast(x8, *reinterpret_cast<const u32x4_t*>(a.q + (qrow0 + query_of(row)) * kHeadDim + kk * 16 + h * 8));
    const int32_t limit_lo = __builtin_amdgcn_readfirstlane(limit);
    // last tile of this wave; none where its rows are past the item's
    const int32_t t_last =
        wave * 32 < rows ? min(__builtin_amdgcn_readlane(limit, 31) >> 6, t1 - 1) : -1;

    float m_ref = -FLT_MAX, l_run = 0.0f;  // (finite: no difference of infinities while no key was seen)
    f32x16_t o[4];
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] = f32x16_t{};
    int32_t odd_lo = t1, odd_hi = -1;  // masked tiles whose values were not all finite

    // --- tiles into the rings ---
    LdsPageWindow pages(c, it.seq, uint32_t(reinterpret_cast<uintptr_t>(sm_pages[wave])));
    const int32_t last = t1 - 1;
    auto entry_of = [&](int32_t t, int32_t key) { return min(min(t, last) * kPagedTile + key, seen - 1) >> c.page_shift; };
    // This group's next tile t.  Behind the last tile that one is fetched again, into
    // a slot that nobody reads any more: every step then waits for the same number of
    // loads.  The page is read one tile ahead.
    int32_t ahead = 0;
    auto look = [&](int32_t t) {
      pages.seek(entry_of(t, 0));
      ahead = pages.peek(entry_of(t, key0));
    };
    auto fetch = [&](int32_t t) {  // returns the tile's bad 16-key groups
      const uint64_t from =
          uint64_t(Plan::uniform(reinterpret_cast<int64_t>(pool + page_row(c, unit, __builtin_amdgcn_readfirstlane(ahead)) * kHeadDim)));
      const i32x4_t rsrc = {int32_t(uint32_t(from)), int32_t(uint32_t(from >> 32) & 0xffffu), (in_page + 1) * (kHeadDim * 2), kBufferFlags};
      const int32_t key = min(t, last) * kPagedTile + key0;
      const uint32_t to = __builtin_amdgcn_readfirstlane(dma_lds + ((t - t0) & (kRing - 1)) * kTileBytes);
      if (t < last) {
        const uint32_t off = __builtin_amdgcn_readfirstlane(uint32_t(key & in_page) * (kHeadDim * 2));
#pragma unroll
        for (int g = 0; g < kTileLoads; ++g) dma16(rsrc, to + g * 1024, dma_lane ^ (g * dma_swizzle), off + g * 1024);
      } else {  // the last tile: keys past the end repeat the last one
#pragma unroll
        for (int g = 0; g < kTileLoads; ++g) {
          const uint32_t r = uint32_t(min(key + 4 * g + (lane >> 4), seen - 1) & in_page) * (kHeadDim * 2);
          dma16(rsrc, to + g * 1024, r + ((dma_lane ^ (g * dma_swizzle)) & 255), 0);
        }
      }
      uint32_t m = 0;
      if (pages.bad)
#pragma unroll
        for (int g = 0; g < 4; ++g) m |= uint32_t(pages.is_bad(entry_of(t, 16 * g))) << g;
      look(t + 1);
      return m;
    };

    // --- one tile's arithmetic ---
    auto full = [&](int32_t t, uint32_t b, int32_t first) { return b == 0 && t * kPagedTile + kPagedTile - 1 <= first; };
    auto slot = [&](int32_t t) { return uint32_t((t - t0) & (kSlots - 1)) * kTileBytes; };
    // FOUR: this wave's part of tile t on its way (rows past the sequence's end lie in its
    // last page, whatever they hold), and its sixteen keys' bad groups.
    auto fetch4 = [&](int32_t t) {  // returns them
      const uint64_t from = uint64_t(Plan::uniform(
          reinterpret_cast<int64_t>(reinterpret_cast<const uint8_t*>(pool) + page4(c, unit, __builtin_amdgcn_readfirstlane(ahead)))));
      const i32x4_t rsrc = {int32_t(uint32_t(from)), int32_t(uint32_t(from >> 32) & 0xffffu), (in_page + 1) * kRow4, kBufferFlags};
      const uint32_t row = __builtin_amdgcn_readfirstlane(uint32_t((min(t, last) * kPagedTile + key0) & in_page));
      const uint32_t to = __builtin_amdgcn_readfirstlane(raw_lds + ((t - t0) & (kAhead4 - 1)) * kRaw4);
      dma16(rsrc, to, lane * 16, row * kCodes4);
      dma4(rsrc, to + 16 * kCodes4, lane4 * 4, (in_page + 1) * kCodes4 + row * 4);
      uint32_t m = 0;
      if (pages.bad)
#pragma unroll
        for (int g = 0; g < 4; ++g) m |= uint32_t(pages.is_bad(entry_of(t, 16 * g))) << g;
      look(t + 1);
      return m;
    };
    // FOUR: that part, once it has landed, into the 16-bit tile.  0 * NaN is no zero: in a
    // tile where some queries do not see every key, values that are not finite are cleared,
    // and reach the queries that see them behind the last tile.
    auto convert4 = [&](int32_t t, uint32_t b) {
      wait_vmcnt<2 * (kAhead4 - 1)>();
      const uint32_t at = raw_lds + ((t - t0) & (kAhead4 - 1)) * kRaw4;
      u32x4_t e = *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t*>((uintptr_t)(at + lane4 * kCodes4 + (lane & 3) * 16));
      uint32_t byte = *reinterpret_cast<const __attribute__((address_space(3))) uint8_t*>((uintptr_t)(at + 16 * kCodes4 + lane * 4 + (lane & 3)));
      if (group && !full(t, b, it.cached + tok0)) {
        const bool odd = byte > uint32_t(Four<T>::kMost);
        if (__ballot(odd)) {
          if (odd) {
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = finite_codes<T>(e[j], byte);
            byte = byte == 255u ? Four<T>::kLeast : byte;
          }
          odd_lo = min(odd_lo, t);
          odd_hi = t;
        }
      }
      const float scale = scale_of(byte);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t x[4];
        values_of<T>(e[j], scale, x);
        *reinterpret_cast<__attribute__((address_space(3))) u32x4_t*>((uintptr_t)((write4 ^ j << 4) + slot(t))) = u32x4_t{x[0], x[1], x[2], x[3]};
      }
    };
    // (the 32-key blocks in turn: a product does not wait for the one before it)
    auto read_k = [&](uint32_t at, int i) {  // keys 32 (i & 1) .., dimensions 16 (i >> 1) .. (at: k_lane + slot)
      return *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t*>((uintptr_t)((at ^ (i >> 1 << 5)) + (i & 1) * 8192));
    };
    auto read_v = [&](uint32_t at, int i) {  // keys 16 (i / 4) .., dimensions 32 (i % 4) .. (at: v_lane + slot)
      const u32x2_t lo = read_transposed((at ^ (i % 4 << 6)) + i / 4 * 4096);
      const u32x2_t hi = read_transposed((at ^ (i % 4 << 6) ^ 32) + i / 4 * 4096 + 2048);
      return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    };
    f32x16_t s[2];     // logits of the tile ahead
    float mt = 0.0f;   // their maximum
    u32x4_t w[4];      // weights of the tile: eight keys of this lane to each 16
    auto product = [&](int i, u32x4_t kf) {
      s[i & 1] = E::mfma32(__builtin_bit_cast(x8, kf), qf[i >> 1], i < 2 ? f32x16_t{} : s[i & 1]);
    };
    auto add = [&](int i, u32x4_t vf) {
      o[i & 3] = E::mfma32(__builtin_bit_cast(x8, vf), __builtin_bit_cast(x8, w[i >> 2]), o[i & 3]);
    };
    constexpr int kSteps = 16;  // products of the logits, and of the values
    constexpr int kAhead = 3;   // reads run that many products ahead

    // The products of step t.  (Behind the wave's last tile the logits are of
    // whatever lies in the slot; nobody looks at them.)
    auto products = [&](int32_t t) {
      const uint32_t k_at = k_lane + slot(t + 1), v_at = v_lane + slot(t);
      u32x4_t f[kAhead + 1];
#pragma unroll
      for (int i = -kAhead; i < 2 * kSteps; ++i) {
        const int n = i + kAhead;
        if (n < kSteps) f[n % (kAhead + 1)] = read_k(k_at, n);
        else if (n < 2 * kSteps) f[n % (kAhead + 1)] = read_v(v_at, n - kSteps);
        if (i < 0) continue;
        if (i < kSteps) product(i, f[i % (kAhead + 1)]);
        else add(i - kSteps, f[i % (kAhead + 1)]);
        if (i >= kSteps + 2) {  // the logits' maximum, two or four to a product (in the vector half it cost 0.4 to 2 %)
          const int v = i - (kSteps + 2);
#pragma unroll
          for (int k = 16 * v / 14; k < 16 * (v + 1) / 14; ++k) {
            const float pair0 = s[k >> 3][2 * k & 15], pair1 = s[k >> 3][(2 * k & 15) + 1];
            mt = k == 0 ? fmaxf(pair0, pair1) : fmaxf(fmaxf(mt, pair0), pair1);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // 0 * infinity is no zero: in a tile where some queries do not see every key,
    // values that are not finite are cleared as soon as they have landed, by the wave
    // that fetched them, and reach the queries that see them behind the last tile.
    auto clean_values = [&](int32_t t) {
#pragma unroll
      for (int g = 0; g < kTileLoads; ++g) {
        auto* p = reinterpret_cast<__attribute__((address_space(3))) u32x4_t*>((uintptr_t)(dma_lds + slot(t) + g * 1024 + lane * 16));
        u32x4_t e = *p;
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t nf = E::not_finite(e[j]);
          odd |= nf;
          e[j] &= ~((nf >> 15) * 0xffffu);
        }
        if (__ballot(odd != 0)) {
          *p = e;
          odd_lo = min(odd_lo, t);
          odd_hi = t;
        }
      }
    };
    // The weights of tile t from its logits.
    auto weigh = [&](int32_t t, uint32_t b) {
      if (!full(t, b, limit_lo)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int32_t in_tile = kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
            if (t * kPagedTile + in_tile > limit || ((b >> (2 * kb + (i >> 3))) & 1)) s[kb][i] = -INFINITY;
          }
        mt = fmaxf(s[0][0], s[0][1]);
#pragma unroll
        for (int i = 2; i < 32; i += 2) mt = fmaxf(fmaxf(mt, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
      }
      float other = mt;
      swap32(mt, other);
      const float top = base2(fmaxf(mt, other), a.scale2);
      if (__ballot(top - m_ref > kLazy)) {
        const float m_new = fmaxf(m_ref, fabsf(top) > kFar ? top : rintf(top * 0x1p14f) * 0x1p-14f);
        const float alpha = __builtin_amdgcn_exp2f(m_ref - m_new);
        m_ref = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
      float scale2 = a.scale2, shift = E::kBias - m_ref;
      if (__ballot(fabsf(m_ref) > kFar && m_ref > -FLT_MAX)) {
#pragma unroll
        for (int n = 0; n < 32; ++n) s[n >> 4][n & 15] = base2(s[n >> 4][n & 15], a.scale2) - m_ref;
        scale2 = 1.0f;
        shift = E::kBias;
      }
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[n >> 3][2 * n & 15], scale2, shift));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[n >> 3][(2 * n & 15) + 1], scale2, shift));
        sum[0] += p0;
        sum[1] += p1;
        w[n >> 2][n & 3] = elem_pack<T>(p0, p1);
      }
      l_run += sum[0] + sum[1];
    };

    barrier_lds();  // the last item's outputs are out of the tiles' memory (its stores may be under way)
    if (t0 < t1) {
      look(t0);
      // (the queries have come with the page: no later wait for them drains the DMA)
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qf[kk]));
      // K(t0), K(t0+1), K(t0+2) and V(t0), V(t0+1); then a step fetches one of each
      uint32_t bad = 0;  // bad 16-key groups of tiles t, t + 1, ..: four bits each
      if constexpr (FOUR) {
#pragma unroll
        for (int i = 0; i < kAhead4; ++i) bad |= fetch4(t0 + i) << (4 * (i + 1));
        convert4(t0, (bad >> 4) & 15);
        bad |= fetch4(t0 + kAhead4) << (4 * (kAhead4 + 1));
      } else {
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i)
          if (i < kRing - 1 - group) bad |= fetch(t0 + i) << (4 * (i + 1));
        wait_vmcnt<2 * kTileLoads>();
      }
      barrier_lds();
      if (group) barrier_lds();
      // What ends the products of step t: this wave's part of the tiles of step t + 1.
      auto landed = [&](int32_t t) {
        if constexpr (!FOUR) {
          wait_vmcnt<kTileLoads>();
          if (group && t + 1 < t1 && !full(t + 1, (bad >> 4) & 15, it.cached + tok0)) clean_values(t + 1);
        }
        barrier_lds();
      };
      auto vector_half = [&](int32_t t) {
        if (t < t_last) weigh(t + 1, (bad >> 4) & 15);
        if constexpr (FOUR) {
          convert4(t + 2, (bad >> 8) & 15);
          bad = (bad | (fetch4(t + 2 + kAhead4) << (4 * (kAhead4 + 2)))) >> 4;
        } else {
          bad = (bad | (fetch(t + kRing - group) << (4 * (kRing - group)))) >> 4;
        }
        barrier_lds();
      };
      if (t0 <= t_last) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) product(i, read_k(k_lane, i));
        mt = fmaxf(s[0][0], s[0][1]);
#pragma unroll
        for (int i = 2; i < 32; i += 2) mt = fmaxf(fmaxf(mt, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
      }
      landed(t0 - 1);
      vector_half(t0 - 1);
      for (int32_t t = t0; t < t1; ++t) {
        if (t <= t_last) products(t);
        landed(t);
        vector_half(t);
      }
      if (!group) barrier_lds();
      wait_vmcnt<0>();  // no DMA may outlive the tiles that it writes
    }
    // All waves learn which tiles had values cleared.
    if (lane == 0) sm_odd[wave] = make_int2(odd_lo, odd_hi);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kExtWaves; ++i) {
      odd_lo = min(odd_lo, __builtin_amdgcn_readfirstlane(sm_odd[i].x));
      odd_hi = max(odd_hi, __builtin_amdgcn_readfirstlane(sm_odd[i].y));
    }
    // The values that were cleared: p v is v for them, whatever the weight, and what
    // is infinite or NaN already stays so.
#pragma unroll 1
    for (int32_t key = odd_lo * kPagedTile; key < min((odd_hi + 1) * kPagedTile, seen); ++key) {
      pages.seek(key >> c.page_shift);
      if (pages.is_bad(key >> c.page_shift)) continue;
      if constexpr (FOUR) {
        const uint8_t* p = reinterpret_cast<const uint8_t*>(c.v) + page4(c, unit, pages.page(key >> c.page_shift));
        const uint32_t scales = *reinterpret_cast<const uint32_t*>(p + (in_page + 1) * kCodes4 + (key & in_page) * 4);
        p += (key & in_page) * kCodes4;
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const uint32_t byte = scales >> (8 * db) & 255u;
          if (byte <= uint32_t(Four<T>::kMost)) continue;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint32_t codes = *reinterpret_cast<const uint16_t*>(p + 16 * db + 4 * g + 2 * h);
            const uint32_t w[2] = {Four<T>::template values<0>(codes, scale_of(byte)), Four<T>::template values<1>(codes, scale_of(byte))};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t bits = w[j >> 1] >> (16 * (j & 1)) & 0xffffu;
              o[db][4 * g + j] += E::not_finite(bits) && key <= limit ? elem_lo<T>(bits) : 0.0f;
            }
          }
        }
        continue;
      }
      const uint16_t* vr = c.v + (page_row(c, unit, pages.page(key >> c.page_shift)) + (key & in_page)) * kHeadDim + 4 * h;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x2_t e = *reinterpret_cast<const u32x2_t*>(vr + 32 * db + 8 * g);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t bits = e[j >> 1] >> (16 * (j & 1)) & 0xffffu;
            o[db][4 * g + j] += E::not_finite(bits) && key <= limit ? elem_lo<T>(bits) : 0.0f;
          }
        }
    }

    float other = l_run;
    swap32(l_run, other);
    l_run += other;
    // Rows of 256 bytes through this wave's part of the tiles, which nobody reads any more,
    // so that a store takes four whole rows, not 16 bytes of each of 32 (28 layers x 28 heads,
    // 256 tokens: 72 to 64 us): chunk q of row r at slot q ^ (r & 15).
    int out_lane = lane;  // (addresses from here on are not kept in registers across the loop)
    asm volatile("" : "+v"(out_lane));
    const uint32_t out_lds = lds0 + wave * (32 * 256);
    const uint32_t to = out_lds + (out_lane & 31) * 256, swizzle = (out_lane & 15) << 4;
    const int r0 = out_lane >> 4, chunk = out_lane & 15;
    auto row_out = [&](int j) {  // chunk `chunk` of row 4 j + r0
      return *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t*>((uintptr_t)(out_lds + (4 * j + r0) * 256 + ((chunk ^ ((4 * j + r0) & 15)) << 4)));
    };
    const int left = rows - wave * 32;
    if (left > 0) {
      if (whole) {
        const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            u32x2_t e;
            e[0] = elem_pack<T>(o[db][4 * g] * inv, o[db][4 * g + 1] * inv);
            e[1] = elem_pack<T>(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv);
            *reinterpret_cast<__attribute__((address_space(3))) u32x2_t*>((uintptr_t)(to + ((4 * db + g) << 4 ^ swizzle) + (out_lane >> 5) * 8)) = e;
          }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int32_t at = query_of(wave * 32 + 4 * j + r0);
          const u32x4_t e = row_out(j);
          if (4 * j + r0 < left) *reinterpret_cast<u32x4_t*>(a.out + (qrow0 + at) * kHeadDim + chunk * 8) = e;
        }
      } else {
        const int64_t at = paged_slot(this_share, share, it.start) * kExtRows + wave * 32;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
          for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
              *reinterpret_cast<__attribute__((address_space(3))) f32x4_t*>((uintptr_t)(to + ((8 * db + 2 * g) << 4 ^ (out_lane >> 5 << 4) ^ swizzle))) =
                  f32x4_t{o[2 * p + db][4 * g], o[2 * p + db][4 * g + 1], o[2 * p + db][4 * g + 2], o[2 * p + db][4 * g + 3]};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const u32x4_t e = row_out(j);
            if (4 * j + r0 < left)
              *reinterpret_cast<u32x4_t*>(a.po + (at + 4 * j + r0) * kHeadDim + p * 64 + chunk * 4) = e;
          }
        }
        if (h == 0 && col < left) {
          a.pm[at + col] = m_ref;
          a.pl[at + col] = l_run;
        }
      }
    }
    x = span.end;
    if (x >= y) break;
    plan.next(it);
    if (!plan.ours(it, y)) break;
  }
}

// ---------------------------------------------------------------------------
// Joining the parts
// ---------------------------------------------------------------------------
//
// A work-group joins up to join_rows rows of an item: the item that the boundary
// between shares x and x + 1 cuts, if x is the first share in it, or with join_items
// (few items in many parts) item x.  32 lanes x 4 dimensions hold a row;
// its parts (two mostly, up to all shares for one token over a long cache) are spread
// over the groups of lanes (8 or 32) that the rows leave, kBatch loads at once, and merged
// through LDS.  Bound by latency for one token (6 us for 11 parts of a layer, 8 us for
// 128 parts of 32k keys, 9 us for the 512 shares of 28 layers), by the partials' bytes
// for several (68 MB of 255 cut items: 19 us, 3.5 TB/s).
constexpr int kBatch = 4;

struct Joined {
  float m = -FLT_MAX, l = 0.0f;
  f32x4_t o = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // (A part without a key has maximum -inf and weighs nothing.  So has one whose logits are
  // all NaN, but its sums are NaN, and make what they are added to NaN with any factor.)
  __device__ void add(float pm, float pl, f32x4_t po) {
    const float mx = fmaxf(m, pm);
    const float f = __builtin_amdgcn_exp2f(m - mx), g = __builtin_amdgcn_exp2f(pm - mx);
    l = l * f + pl * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * f + po[i] * g;
    m = mx;
  }
};

template <typename T, int GROUPS>
__global__ __launch_bounds__(GROUPS * 32) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int NT = GROUPS * 32;
  __shared__ float sm_m[GROUPS], sm_l[GROUPS];
  __shared__ f32x4_t sm_o[GROUPS][32];
  __shared__ typename PagedPlan<NT>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<NT> plan(a, sm_plan);
  PagedItem it;
  if (a.join_items) {
    it = plan.item(blockIdx.x);
  } else {
    const int64_t cut = (int64_t(blockIdx.x) + 1) * plan.share;
    if (cut >= plan.total) return;
    it = plan.find(cut);
    if (it.start >= cut || it.start / plan.share != int64_t(blockIdx.x)) return;
  }
  const int32_t w0 = int32_t(it.start / plan.share), w1 = int32_t((it.start + it.keys - 1) / plan.share);
  if (w0 == w1 || it.keys <= a.keep) return;
  const int unit = it.unit / a.parts, part = it.unit % a.parts;
  const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
  const int32_t tok0 = it.index * a.tokens;
  const int32_t head0 = part * a.rows;  // (one part but for decode)
  const int32_t rows = a.parts > 1 ? min(c.group - head0, a.rows) : min(it.n - tok0, a.tokens) * c.group;
  const int grp = threadIdx.x >> 5, l32 = threadIdx.x & 31;
  const int32_t first = blockIdx.y * a.join_rows, end = min(rows, first + a.join_rows);
  auto load = [&](int32_t w, int32_t row, float& m, float& l, f32x4_t& o) {
    const int64_t slot = paged_slot(w, plan.share, it.start) * a.rows + row;
    m = a.pm[slot];
    l = a.pl[slot];
    o = *reinterpret_cast<const f32x4_t*>(a.po + slot * kHeadDim + 4 * l32);
  };
  auto store = [&](int32_t row, const Joined& r) {
    const float inv = r.l == 0.0f ? 0.0f : 1.0f / r.l;
    const int32_t tok = row / c.group;  // (decode: 0 with one part; with more, row is a head)
    const int64_t orow = a.parts > 1 ? (int64_t(layer) * c.total_new + it.row0) * c.n_q_heads + int64_t(kv) * c.group + head0 + row
                                     : (int64_t(layer) * c.total_new + it.row0 + tok0 + tok) * c.n_q_heads +
                                           int64_t(kv) * c.group + (row - tok * c.group);
    u32x2_t e;
    e[0] = elem_pack<T>(r.o[0] * inv, r.o[1] * inv);
    e[1] = elem_pack<T>(r.o[2] * inv, r.o[3] * inv);
    *reinterpret_cast<u32x2_t*>(a.out + orow * kHeadDim + 4 * l32) = e;
  };
  if (w1 - w0 == 1) {  // two parts: a row per group (through the loop below prompts took 218 us, not 211)
    for (int32_t row = first + grp; row < end; row += GROUPS) {
      float m[2], l[2];
      f32x4_t o[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) load(w0 + i, row, m[i], l[i], o[i]);
      Joined r;
#pragma unroll
      for (int i = 0; i < 2; ++i) r.add(m[i], l[i], o[i]);
      store(row, r);
    }
    return;
  }
  for (int32_t row0 = first; row0 < end; row0 += GROUPS) {
    const int32_t here = min(end - row0, GROUPS);
    // groups per row: none without parts
    const int per_row = min(GROUPS / here, (w1 - w0 + kBatch) / kBatch);
    const int32_t row = row0 + grp / per_row;
    Joined r;
    if (row < row0 + here)
      for (int32_t w = w0 + grp % per_row; w <= w1; w += kBatch * per_row) {
        float m[kBatch], l[kBatch];
        f32x4_t o[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)  // (past the last: that one again, left out)
          load(min(w + i * per_row, w1), row, m[i], l[i], o[i]);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const bool there = w + i * per_row <= w1;
          r.add(there ? m[i] : -FLT_MAX, there ? l[i] : 0.0f, there ? o[i] : f32x4_t{0.f, 0.f, 0.f, 0.f});
        }
      }
    if (per_row > 1) {
      __syncthreads();
      sm_o[grp][l32] = r.o;
      if (l32 == 0) {
        sm_m[grp] = r.m;
        sm_l[grp] = r.l;
      }
      __syncthreads();
      if (grp % per_row == 0 && row < row0 + here) {
        r = Joined();
        for (int g = 0; g < per_row; ++g) r.m = fmaxf(r.m, sm_m[grp + g]);
#pragma unroll 4
        for (int g = 0; g < per_row; ++g) {
          const float f = __builtin_amdgcn_exp2f(sm_m[grp + g] - r.m);
          r.l += sm_l[grp + g] * f;
#pragma unroll
          for (int i = 0; i < 4; ++i) r.o[i] += sm_o[grp + g][l32][i] * f;
        }
      }
    }
    if (grp % per_row == 0 && row < row0 + here) store(row, r);
  }
}

template <typename T>
hipError_t launch_join(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.shares < 2 || !a.joins) return hipSuccess;
  const dim3 grid(a.join_items ? a.join_items : a.shares - 1, a.join_split);
  if (a.join_groups == 8) hipLaunchKernelGGL((paged_join_kernel<T, 8>), grid, dim3(8 * 32), 0, stream, a);
  else hipLaunchKernelGGL((paged_join_kernel<T, 32>), grid, dim3(32 * 32), 0, stream, a);
  return hipGetLastError();
}

template <typename T>
hipError_t decode(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.rows == 16) hipLaunchKernelGGL((paged_decode_kernel<T, 1>), dim3(a.shares), dim3(kDecWaves * 64), 0, stream, a);
  else hipLaunchKernelGGL((paged_decode_kernel<T, 2>), dim3(a.shares), dim3(kDecWaves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<T>(a, stream);
}

template <typename T, bool FOUR>
hipError_t extend(const PagedAttnArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((paged_extend_kernel<T, FOUR>), dim3(a.shares), dim3(kExtWaves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<T>(a, stream);
}

}  // namespace

hipError_t launch_paged_decode(const PagedAttnArgs& a, bool half, hipStream_t stream) {
  return half ? decode<_Float16>(a, stream) : decode<__bf16>(a, stream);
}

hipError_t launch_paged_extend(const PagedAttnArgs& a, bool four, bool half, hipStream_t stream) {
  if (four) return half ? extend<_Float16, true>(a, stream) : extend<__bf16, true>(a, stream);
  return half ? extend<_Float16, false>(a, stream) : extend<__bf16, false>(a, stream);
}

hipError_t launch_paged_join(const PagedAttnArgs& a, bool half, hipStream_t stream) {
  return half ? launch_join<_Float16>(a, stream) : launch_join<__bf16>(a, stream);
}

}  // namespace stlite
