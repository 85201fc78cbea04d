// Attention of one or a few new tokens per sequence over a 4-bit pool
// (stlite_paged_attention with STLITE_KV4): the formula, the shares and the joining launch
// of paged_attention.hip.
#include <float.h>

#include "paged4.h"
#include "paged_plan.h"
#include "tile_lds.h"

namespace stlite {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// HBM-bound: 136 bytes of a key, read once, its codes turned into 16 bits in registers.
// Four waves take 64-key tiles of a share in turn (four runs of 16, each in one page):
//   S^T = K Q^T   16x16x32, cached rows as A, run by run.  A lane reads a whole block of its
//                 key, dimensions 32 (lane / 16) .., so that it needs one scale; the
//                 queries, B, are laid out to match: a dot product does not mind their order.
//   O += P V      16x16x32 for two runs at once, P where S^T left it (four keys of each run
//                 to a lane); V is read as eight values of each of those keys, put together
//                 by byte permutes behind the conversion.  The weights' sums are one
//                 product more, with ones.
// A column of S^T is a row of the item: with one token a head of the group, or of a part
// of it; with a few tokens, which all read the same keys, token-major rows of all heads.
// The weights are rounded to the type of the call (half a step of it, as the output;
// what a value lost to 4 bits is fifty times that), which leaves one product per 32 keys
// and 16 dimensions where the 16-bit pool's three terms would take three.  Their reference
// moves and is kept as in the kernel of several tokens; a lane looks at its own logits
// alone to find that it need not.
//
// What bounds it beside HBM is the vector unit, two conversions and a permute to four
// values being half of its instructions: tiles come as they are stored, by DMA into a ring
// of the wave's own, at addresses that a lane forms itself, codes past the caches (through
// them 96 us, not 84, for 459 MB).  Loads into registers, 32 keys ahead, took 255 vector
// and 104 scalar instructions to 32 keys, this takes 170 and 32: 64 sequences of up to 8000
// in 4 layers (1.23 GB) 240 and 214 us.
// 28 layers x 28 heads behind 30105 tokens 80 us (459 MB, 6.2 TB/s without the joining
// launch), a layer behind 150528 26, five drafted tokens in each of 16 sequences of up to
// 8000 in 2 layers, 32 heads over 8 (190 MB) 54.
constexpr int kWaves = 4;
constexpr int kRuns = 4;           // of 16 keys to a tile
constexpr int kKeys = 16 * kRuns;  // of a tile
// A tile's slot: four parts, of four rows (4 d ..) of each run, which four DMA instructions
// bring; with 16 (K) or 64 (V) bytes between them, so that sixteen rows' reads of one
// chunk, or four rows' 4 apart, take all banks.  Then the scales, run by run.
constexpr int kKPart = 1024 + 16, kVPart = 1024 + 64;
constexpr int kVAt = 4 * kKPart, kScalesAt = kVAt + 4 * kVPart, kSlot = kScalesAt + 2 * kKeys * 4;
constexpr float kLazy = 8.0f, kFar = 960.0f;

// 16 or 4 bytes per lane, each from an address of its own, to LDS address `to` + 16 lane or
// + 4 lane.  (As dma16.)
__device__ inline void dma16_each(const uint8_t* from, uint32_t to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "{m0}"(to) : "memory");
}
__device__ inline void dma4_each(const uint8_t* from, uint32_t to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(from), "{m0}"(to) : "memory");
}

template <typename V>
__device__ inline V lds_read(uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>((uintptr_t)at);
}

// 16 NG HALVES rows to an item.  Of more than 32 rows the sums and queries take more
// registers than two waves of a SIMD have: with HALVES = 2 the two waves of a SIMD, w and
// w + 4, take half of the rows each of the same tiles, one of them fetching K and the other
// V.  (One wave with all of them, products and vector work in turn, took 134 us where this
// takes 106.)  One tile is under way while another is worked on: with three 81 us became 91
// for 16 rows, 106 became 109 for 64.
template <typename T, int NG, int HALVES>
__global__ __launch_bounds__(kWaves * 64 * HALVES, 2) void paged4_few_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = kWaves * 64 * HALVES, kRows = 16 * NG * HALVES, kDepth = 2;
  constexpr int kDmas = HALVES == 1 ? 10 : 5;        // instructions of a wave to a tile
  constexpr int kWindow = HALVES == 1 ? 512 : 256;  // entries of the page table that a wave holds
  __shared__ float sm_m[kWaves][kRows], sm_l[kWaves][kRows];
  __shared__ __align__(1024) uint8_t sm_ring[kWaves][kDepth][kSlot];  // (the waves' sums, once an item is done)
  __shared__ int32_t sm_pages[kWaves * HALVES][kWindow];
  typedef PagedPlan<NT, true> Plan;
  __shared__ typename Plan::Shared sm_plan;
  const PagedDev& c = a.c;
  Plan plan(a, sm_plan);
  int64_t x = int64_t(blockIdx.x) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  PagedItem it;
  if (!plan.first(x, y, it)) return;

  const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = wave8 % kWaves, half = HALVES == 1 ? 0 : wave8 / kWaves;
  const int col = lane & 15, quad = lane >> 4;
  const int32_t in_page = (1 << c.page_shift) - 1, scales_at = (in_page + 1) * kCodes4;
  const uint32_t page_bytes = uint32_t(in_page + 1) * kRow4;
  const uint32_t ring = uint32_t(reinterpret_cast<uintptr_t>(sm_ring[wave]));
  const uint32_t window = uint32_t(reinterpret_cast<uintptr_t>(sm_pages[wave8]));
  const int64_t v_off = reinterpret_cast<int64_t>(c.v) - reinterpret_cast<int64_t>(c.k);
  // DMA: lane l has run l / 16, row 4 d + l / 4 % 4 of it and chunk l % 4, or its scales' row l % 16.
  const uint32_t codes_from = uint32_t((16 * quad & in_page) + (lane >> 2 & 3)) * kCodes4 + (lane & 3) * 16;
  const uint32_t scales_from = uint32_t(scales_at + ((16 * quad & in_page) + col) * 4);
  const uint32_t entry_from = uint32_t(16 * quad >> c.page_shift);
  const uint32_t k_read = (col >> 2) * kKPart + (col & 3) * kCodes4 + quad * 16;
  const uint32_t v_read = kVAt + quad * kVPart + col * 4;
  const uint32_t scale_turn = (8 * (col >> 2) + 9) & 31;  // rotates block col / 4's byte into a float's exponent
  const x8 ones = __builtin_bit_cast(x8, u32x4_t{elem_pack<T>(1.f, 1.f), elem_pack<T>(1.f, 1.f), elem_pack<T>(1.f, 1.f), elem_pack<T>(1.f, 1.f)});

  for (;;) {
    const int unit = it.unit / a.parts, part = it.unit % a.parts;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const int32_t tok0 = it.index * a.tokens, toks = min(it.n - tok0, a.tokens);
    const int32_t rows = a.parts > 1 ? min(c.group - part * kRows, kRows) : toks * c.group;
    const PagedPart span = plan.part(x, y, it);
    const bool whole = span.whole;
    const int32_t sees_first = __builtin_amdgcn_readfirstlane(max(it.cached + tok0 + 1, 0));  // keys that every row sees
    const int32_t k0 = span.t0 * kPagedTile;
    const int32_t k1 = __builtin_amdgcn_readfirstlane(min(span.t1 * kPagedTile, max(it.cached + tok0 + toks, 0)));
    // Row r's place among the queries and outputs.
    auto place = [&](int32_t r) {
      const int32_t tok = a.parts > 1 ? 0 : r / c.group;
      return (int64_t(layer) * c.total_new + it.row0 + tok0 + tok) * c.n_q_heads + int64_t(kv) * c.group + part * kRows +
             (r - tok * c.group);
    };
    const int32_t first = __builtin_amdgcn_readfirstlane(k0 + kKeys * wave);  // this wave's first key
    const int32_t steps = first < k1 ? (k1 - first + kKeys * kWaves - 1) / (kKeys * kWaves) : 0;
    // (the waves of HALVES = 2 go in step)
    const int32_t rounds = HALVES == 1 ? steps : __builtin_amdgcn_readfirstlane(max((k1 - k0 + kKeys * kWaves - 1) / (kKeys * kWaves), 0));

    // --- tiles into the ring ---
    int32_t held = -kWindow;  // first entry in the window
    const int32_t* const table = c.page_table + int64_t(it.seq) * c.max_pages;
    const uint8_t* const unit_at = reinterpret_cast<const uint8_t*>(
        Plan::uniform(reinterpret_cast<int64_t>(reinterpret_cast<const uint8_t*>(c.k) + page4(c, unit, 0))));
    bool bad = false;  // a page was none
    // Tile i.  Where a page is none, what page 0 holds is read, and left out; rows past the
    // sequence's end lie in its last page, whatever they hold, or in what the table has behind it.
    auto fetch = [&](int32_t i) {
      const int32_t j0 = first + i * (kKeys * kWaves), entry = j0 >> c.page_shift;
      if (entry < held || entry >= held + kWindow) {
        held = entry & ~(kWindow - 1);
        int32_t e[kWindow / 64];
#pragma unroll
        for (int n = 0; n < kWindow / 64; ++n) e[n] = table[min(held + n * 64 + lane, c.max_pages - 1)];
#pragma unroll
        for (int n = 0; n < kWindow / 64; ++n)
          *reinterpret_cast<volatile __attribute__((address_space(3))) int32_t*>((uintptr_t)(window + (n * 64 + lane) * 4)) = e[n];
      }
      const uint32_t to = ring + (i & (kDepth - 1)) * kSlot;
      uint32_t page = *reinterpret_cast<const volatile __attribute__((address_space(3))) uint32_t*>(
          (uintptr_t)(window + ((uint32_t(entry) & (kWindow - 1)) + entry_from) * 4));
      bad |= __ballot(page >= uint32_t(c.n_pages)) != 0;
      page = page < uint32_t(c.n_pages) ? page : 0;
      const uint8_t* const at = unit_at + uint64_t(page) * page_bytes;
      const uint8_t* const codes = at + (uint32_t(j0 & in_page) * kCodes4 + codes_from);
      const uint8_t* const scales = at + (uint32_t(j0 & in_page) * 4 + scales_from);
      if (HALVES == 1 || half == 0) {
#pragma unroll
        for (int d = 0; d < 4; ++d) dma16_each(codes + d * 4 * kCodes4, to + d * kKPart);
        dma4_each(scales, to + kScalesAt);
      }
      if (HALVES == 1 || half == 1) {
#pragma unroll
        for (int d = 0; d < 4; ++d) dma16_each(codes + v_off + d * 4 * kCodes4, to + kVAt + d * kVPart);
        dma4_each(scales + v_off, to + kScalesAt + kKeys * 4);
      }
    };
#pragma unroll 1
    for (int i = 0; i < min(steps, kDepth - 1); ++i) fetch(i);

    x8 qb[NG][4];     // dimensions 32 quad + 8 kk ..
    int32_t sees[NG];  // keys that this lane's rows see
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const int32_t r = min(16 * (NG * half + ng) + col, rows - 1);
      const uint16_t* p = a.q + place(r) * kHeadDim;
      sees[ng] = it.cached + tok0 + 1 + (a.parts > 1 ? 0 : r / c.group);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qb[ng][kk] = __builtin_bit_cast(x8, *reinterpret_cast<const u32x4_t*>(p + quad * 32 + kk * 8));
    }
    float m_ref[NG];
    f32x4_t l[NG];     // sums of the weights of rows 4 quad + r, on every column
    f32x4_t o[NG][8];  // O[row 16 (NG half + ng) + 4 quad + r][dimension 8 col + db]
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      m_ref[ng] = -FLT_MAX;  // (finite: no difference of infinities while no key was seen)
      l[ng] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int db = 0; db < 8; ++db) o[ng][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    bool odd = false;  // keys that some rows do not see had values that are not finite

    auto step = [&](int32_t j0, uint32_t at) {
      uint64_t none = 0;  // lanes whose run's page is none
      if (bad) none = __ballot(uint32_t(table[min((j0 >> c.page_shift) + int32_t(entry_from), c.max_pages - 1)]) >= uint32_t(c.n_pages));
      const bool ends = none != 0 || j0 + kKeys > min(k1, sees_first);  // keys are left out, for some rows or all
      // Key i of run r, of the four of this lane, and the first that is left out for all rows.
      auto key = [&](int r, int i) { return j0 + 16 * r + 4 * quad + i; };
      auto end = [&](int r) { return none >> (16 * r) & 1 ? 0 : k1; };
      u32x4_t kc[kRuns];
      uint32_t ks[kRuns];
#pragma unroll
      for (int r = 0; r < kRuns; ++r) {
        kc[r] = lds_read<u32x4_t>(at + k_read + r * 4 * kCodes4);
        ks[r] = lds_read<uint8_t>(at + col * 4 + quad + (kScalesAt + r * 64));
      }
      f32x4_t s[NG][kRuns];
#pragma unroll
      for (int r = 0; r < kRuns; ++r) {
        const float scale = scale_of(ks[r]);
#pragma unroll
        for (int ng = 0; ng < NG; ++ng) s[ng][r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t w[4];
          values_of<T>(kc[r][kk], scale, w);
          const x8 kf = __builtin_bit_cast(x8, u32x4_t{w[0], w[1], w[2], w[3]});
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) s[ng][r] = E::mfma16(kf, qb[ng][kk], s[ng][r]);
        }
      }
      u32x4_t w[NG][kRuns / 2];  // the weights of eight keys each
#pragma unroll
      for (int ng = 0; ng < NG; ++ng) {
        if (ends) {
          asm volatile("");  // (a branch: rarely taken)
#pragma unroll
          for (int r = 0; r < kRuns; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key(r, i) >= min(end(r), sees[ng])) s[ng][r][i] = -INFINITY;
        }
        float mt = fmaxf(s[ng][0][0], s[ng][0][1]);
#pragma unroll
        for (int i = 2; i < 4 * kRuns; i += 2) mt = fmaxf(fmaxf(mt, s[ng][i >> 2][i & 3]), s[ng][i >> 2][(i & 3) + 1]);
        if (__ballot(base2(mt, a.scale2) - m_ref[ng] > kLazy)) {
          float other = mt;
          swap16(mt, other);
          mt = other = fmaxf(mt, other);
          swap32(mt, other);
          const float top = base2(fmaxf(mt, other), a.scale2);
          const float m_new = fmaxf(m_ref[ng], fabsf(top) > kFar ? top : rintf(top * 0x1p14f) * 0x1p-14f);
          const float alpha = __builtin_amdgcn_exp2f(m_ref[ng] - m_new);
          m_ref[ng] = m_new;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float ar = __shfl(alpha, 4 * quad + r);
            l[ng][r] *= ar;
#pragma unroll
            for (int db = 0; db < 8; ++db) o[ng][db][r] *= ar;
          }
        }
        float scale2 = a.scale2, shift = E::kBias - m_ref[ng];
        if (__ballot(fabsf(m_ref[ng]) > kFar && m_ref[ng] > -FLT_MAX)) {
#pragma unroll
          for (int i = 0; i < 4 * kRuns; ++i) s[ng][i >> 2][i & 3] = base2(s[ng][i >> 2][i & 3], a.scale2) - m_ref[ng];
          scale2 = 1.0f;
          shift = E::kBias;
        }
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[ng][r][i], scale2, shift));
          w[ng][r >> 1][2 * (r & 1)] = elem_pack<T>(p[0], p[1]);
          w[ng][r >> 1][2 * (r & 1) + 1] = elem_pack<T>(p[2], p[3]);
        }
      }
#pragma unroll
      for (int h = 0; h < kRuns / 2; ++h) {
        uint32_t vc[8];
        u32x4_t vs[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
          for (int i = 0; i < 4; ++i) vc[4 * r + i] = lds_read<uint32_t>(at + v_read + (4 * (2 * h + r) + i) * kCodes4);
          vs[r] = lds_read<u32x4_t>(at + quad * 16 + (kScalesAt + kKeys * 4 + (2 * h + r) * 64));
        }
        // (The conversion takes a scale's exponent alone.)
        float vscale[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          vscale[i] = __builtin_bit_cast(float, __builtin_amdgcn_alignbit(vs[i >> 2][i & 3], vs[i >> 2][i & 3], scale_turn));
        // Keys that are left out: no weight, and no NaN or infinity for it to meet.  Where
        // some rows see a key and others do not, what is not finite reaches the former
        // behind the last tile.
        if (ends) {
          asm volatile("");
          auto byte = [&](int i) { return vs[i >> 2][i & 3] >> (8 * (col >> 2)) & 255u; };
          uint32_t most = 0;  // scale byte of keys that some rows see
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int32_t j = key(2 * h + (i >> 2), i & 3);
            if (j >= end(2 * h + (i >> 2))) vscale[i] = 1.0f;
            else if (j >= sees_first) most = max(most, byte(i));
          }
          if (__ballot(most > uint32_t(Four<T>::kMost))) {
            odd = true;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int32_t j = key(2 * h + (i >> 2), i & 3);
              if (j < end(2 * h + (i >> 2)) && j >= sees_first) {
                vc[i] = finite_codes<T>(vc[i], byte(i));
                if (byte(i) == 255u) vscale[i] = 1.0f;
              }
            }
          }
        }
#pragma unroll
        for (int ng = 0; ng < NG; ++ng) l[ng] = E::mfma16(__builtin_bit_cast(x8, w[ng][h]), ones, l[ng]);
        auto add = [&](int d, const uint32_t (&u)[8]) {  // dimensions 2 d and 2 d + 1 of the lane's eight
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint32_t pick = b ? 0x07060302u : 0x05040100u;
            u32x4_t f;
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], pick);
#pragma unroll
            for (int ng = 0; ng < NG; ++ng)
              o[ng][2 * d + b] = E::mfma16(__builtin_bit_cast(x8, w[ng][h]), __builtin_bit_cast(x8, f), o[ng][2 * d + b]);
          }
        };
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<0>(vc[i], vscale[i]);
        add(0, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<1>(vc[i], vscale[i]);
        add(1, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<2>(vc[i], vscale[i]);
        add(2, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<3>(vc[i], vscale[i]);
        add(3, u);
      }
    };
    // (the queries have come: no later wait for them drains the DMA)
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qb[ng][kk]));
    for (int32_t i = 0; i < rounds; ++i) {
      // this wave's part of tile i has landed: all but the kDepth - 2 behind it (near the end: all)
      if (i + kDepth - 1 <= steps) wait_vmcnt<kDmas * (kDepth - 2)>();
      else wait_vmcnt<0>();
      if (HALVES == 2) barrier_lds();  // and the other wave's, which is done with tile i - 1
      if (HALVES == 2 && i >= steps) continue;
      if (i + kDepth - 1 < steps) fetch(i + kDepth - 1);  // in place of tile i - 1, whose values have been used
      step(first + i * (kKeys * kWaves), ring + (i & (kDepth - 1)) * kSlot);
    }
    if (odd) {
      for (int32_t j = max(k0, sees_first); j < k1; ++j) {
        if ((j - k0) / kKeys % kWaves != wave) continue;
        const int32_t page = table[j >> c.page_shift];
        if (uint32_t(page) >= uint32_t(c.n_pages)) continue;
        const uint8_t* const at = unit_at + v_off + uint64_t(page) * page_bytes;
        const uint32_t byte = (at + scales_at + (j & in_page) * 4)[col >> 2];
        uint32_t w[4];
        values_of<T>(*reinterpret_cast<const uint32_t*>(at + (j & in_page) * kCodes4 + col * 4), scale_of(byte), w);
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] &= (E::not_finite(w[d]) >> 15) * 0xffffu;  // the others count already
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t seen = j < __shfl(sees[ng], 4 * quad + r) ? ~0u : 0u;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              o[ng][2 * d][r] += elem_lo<T>(w[d] & seen);
              o[ng][2 * d + 1][r] += elem_hi<T>(w[d] & seen);
            }
          }
      }
    }
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const int row = 16 * (NG * half + ng);
      if (lane < 16) sm_m[wave][row + lane] = m_ref[ng];
      if (col == 0)
#pragma unroll
        for (int r = 0; r < 4; ++r) sm_l[wave][row + 4 * quad + r] = l[ng][r];
    }

    // Merge the waves, as many rows at a time as their rings hold (a wave that saw no key has
    // weights of 0).
    constexpr int kAtOnce = 16 * (NG * HALVES < 2 ? 1 : 2);
    static_assert(sizeof(sm_ring[0]) >= sizeof(float) * kAtOnce * kHeadDim && sizeof(sm_ring[0]) % sizeof(float) == 0);
    const auto sum_at = [&](int w, int row, int dim) -> float& {
      return *reinterpret_cast<float*>(&sm_ring[w][0][0] + (row * kHeadDim + dim) * int(sizeof(float)));
    };
    const int64_t slot = paged_slot(blockIdx.x, plan.share, it.start) * kRows;
#pragma unroll
    for (int row0 = 0; row0 < kRows; row0 += kAtOnce) {
      if (row0 >= rows) break;
      __syncthreads();  // the rings, or the last rows' sums, have been read
      if (half == row0 / (16 * NG))
#pragma unroll
        for (int ng = 0; ng < kAtOnce / 16; ++ng)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int db = 0; db < 8; db += 4)
              *reinterpret_cast<f32x4_t*>(&sum_at(wave, 16 * ng + 4 * quad + r, col * 8 + db)) =
                  f32x4_t{o[ng][db][r], o[ng][db + 1][r], o[ng][db + 2][r], o[ng][db + 3][r]};
      __syncthreads();
      for (int e = threadIdx.x; e < min(rows - row0, kAtOnce) * (kHeadDim / 2); e += NT) {
        const int h = e / (kHeadDim / 2), dim = e % (kHeadDim / 2) * 2, row = row0 + h;
        float M = -FLT_MAX;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w][row]);
        float L = 0.0f, O0 = 0.0f, O1 = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float wt = __builtin_amdgcn_exp2f(sm_m[w][row] - M);
          const float2 part = *reinterpret_cast<const float2*>(&sum_at(w, h, dim));
          L += wt * sm_l[w][row];
          O0 += wt * part.x;
          O1 += wt * part.y;
        }
        if (whole) {
          const float inv = L == 0.0f ? 0.0f : 1.0f / L;
          *reinterpret_cast<uint32_t*>(a.out + place(row) * kHeadDim + dim) = elem_pack<T>(O0 * inv, O1 * inv);
        } else {
          *reinterpret_cast<float2*>(a.po + (slot + row) * kHeadDim + dim) = make_float2(O0, O1);
          if (dim == 0) {
            a.pm[slot + row] = M;
            a.pl[slot + row] = L;
          }
        }
      }
    }
    x = span.end;
    if (x >= y) break;
    plan.next(it);
    if (!plan.ours(it, y)) break;
    __syncthreads();  // the sums have been read
  }
}

template <typename T>
hipError_t few(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.rows == 16) hipLaunchKernelGGL((paged4_few_kernel<T, 1, 1>), dim3(a.shares), dim3(kWaves * 64), 0, stream, a);
  else if (a.rows == 32) hipLaunchKernelGGL((paged4_few_kernel<T, 2, 1>), dim3(a.shares), dim3(kWaves * 64), 0, stream, a);
  else hipLaunchKernelGGL((paged4_few_kernel<T, 2, 2>), dim3(a.shares), dim3(kWaves * 128), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged4_few(const PagedAttnArgs& a, bool half, hipStream_t stream) {
  const hipError_t e = half ? few<_Float16>(a, stream) : few<__bf16>(a, stream);
  return e != hipSuccess ? e : launch_paged_join(a, half, stream);
}

}  // namespace stlite
