// Attention of one or a few new tokens per sequence over a 4-bit pool
// (stlite_paged_attention with STLITE_KV4): the formula, the shares and the joining launch
// of paged_attention.hip.
#include "paged4.h"
#include "paged_plan.h"
#include "tile_lds.h"

namespace stlite {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// HBM-bound: 136 bytes of a key, read once, its codes turned into 16 bits in registers.
// Four waves take 32-key sub-tiles of a share in turn (two runs of 16, each in one page),
// the next one's loads under this one's arithmetic:
//   S^T = K Q^T   16x16x32 twice, cached rows as A.  A lane reads a whole block of its key,
//                 dimensions 32 (lane / 16) .., so that it needs one scale; the queries,
//                 B, are laid out to match: a dot product does not mind their order.
//   O += P V      16x16x32, P where S^T left it (four keys of each run to a lane); V is
//                 read as eight values of each of those keys, put together by byte
//                 permutes behind the conversion.
// A column of S^T is a row of the item: with one token a head of the group, or of a part
// of it; with a few tokens, which all read the same keys, token-major rows of all heads.
// The weights are rounded to the type of the call (half a step of it, as the output;
// what a value lost to 4 bits is fifty times that), which leaves one product per 32 keys
// and 16 dimensions where the 16-bit pool's three terms would take three.
constexpr int kWaves = 4;
constexpr int kKeys = 32;  // of a sub-tile

template <typename V>
__device__ inline V load_once(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
}

template <typename T, int NG>  // 16 NG rows to an item
__global__ __launch_bounds__(kWaves * 64, 2) void paged4_few_kernel(PagedAttnArgs a) {
  typedef Elem<T> E;
  typedef typename E::x8 x8;
  constexpr int NT = kWaves * 64, kRows = 16 * NG;
  __shared__ float sm_m[kWaves][kRows], sm_l[kWaves][kRows];
  __shared__ float sm_o[kWaves][kRows][kHeadDim];
  __shared__ typename PagedPlan<NT>::Shared sm_plan;
  const PagedDev& c = a.c;
  PagedPlan<NT> plan(a, sm_plan);
  int64_t x = int64_t(blockIdx.x) * plan.share;
  const int64_t y = min(x + plan.share, plan.total);
  if (x >= y) return;
  PagedItem it = plan.find(x);
  if (it.start >= y) return;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int32_t in_page = (1 << c.page_shift) - 1, scales_at = (in_page + 1) * kCodes4;
  const uint8_t* const k_pool = reinterpret_cast<const uint8_t*>(c.k);
  const uint8_t* const v_pool = reinterpret_cast<const uint8_t*>(c.v);
  for (bool first = true;; first = false) {
    const int unit = it.unit / a.parts, part = it.unit % a.parts;
    const int layer = unit / c.n_kv_heads, kv = unit % c.n_kv_heads;
    const int32_t tok0 = it.index * a.tokens, toks = min(it.n - tok0, a.tokens);
    const int32_t rows = a.parts > 1 ? min(c.group - part * kRows, kRows) : toks * c.group;
    const PagedPart span = paged_part(x, y, it.start, it.keys);
    const bool whole = span.whole;
    const int32_t sees_first = max(it.cached + tok0 + 1, 0);  // keys that every row sees
    const int32_t k0 = span.t0 * kPagedTile, k1 = min(span.t1 * kPagedTile, max(it.cached + tok0 + toks, 0));
    // Row r's place among the queries and outputs.
    auto place = [&](int32_t r) {
      const int32_t tok = a.parts > 1 ? 0 : r / c.group;
      return (int64_t(layer) * c.total_new + it.row0 + tok0 + tok) * c.n_q_heads + int64_t(kv) * c.group + part * kRows +
             (r - tok * c.group);
    };

    x8 qb[NG][4];     // dimensions 32 quad + 8 kk ..
    int32_t sees[NG];  // keys that this lane's rows see
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const int32_t r = min(16 * ng + col, rows - 1);
      const uint16_t* p = a.q + place(r) * kHeadDim;
      sees[ng] = it.cached + tok0 + 1 + (a.parts > 1 ? 0 : r / c.group);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qb[ng][kk] = __builtin_bit_cast(x8, *reinterpret_cast<const u32x4_t*>(p + quad * 32 + kk * 8));
    }
    float m_run[NG], l_run[NG];
    f32x4_t o[NG][8];  // O[row 16 ng + 4 quad + r][dimension 8 col + db]
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      m_run[ng] = -INFINITY;
      l_run[ng] = 0.0f;
#pragma unroll
      for (int db = 0; db < 8; ++db) o[ng][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    // A sub-tile as it is stored.  Rows past the share's end, or of a page that is none,
    // are read where they would lie in a page that is one, and left out by `end`.
    struct Raw {
      u32x4_t k[2];     // a block of key 16 r + col
      uint32_t ks[2];   // its scale byte
      uint32_t v[8];    // eight values of key 16 (i / 4) + 4 quad + i % 4
      u32x4_t vs[2];    // those four keys' scales
      int32_t end[2];   // first key of run r that is left out
    };
    PageWindow pages(c, it.seq);
    auto load = [&](int32_t j0, Raw& n) {
      pages.seek(j0 >> c.page_shift);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int32_t j = j0 + 16 * r, entry = j >> c.page_shift, row = j & in_page;
        const int64_t at = page4(c, unit, pages.page(entry));
        n.end[r] = pages.is_bad(entry) ? j : min(k1, j + 16);
        const uint8_t* kp = k_pool + at;
        const uint8_t* vp = v_pool + at;
        n.k[r] = load_once<u32x4_t>(kp + row * kCodes4 + (col * kCodes4 + quad * 16));
        n.ks[r] = (kp + scales_at + row * 4)[col * 4 + quad];
#pragma unroll
        for (int i = 0; i < 4; ++i) n.v[4 * r + i] = load_once<uint32_t>(vp + row * kCodes4 + (4 * quad + i) * kCodes4 + col * 4);
        n.vs[r] = *reinterpret_cast<const u32x4_t*>(vp + scales_at + row * 4 + quad * 16);
      }
    };
    bool odd = false;  // blocks that some rows do not see were NaN
    int32_t j0 = k0 + kKeys * wave;
    Raw next;
    if (j0 < k1) load(j0, next);
    for (; j0 < k1; j0 += kKeys * kWaves) {
      const Raw now = next;
      if (j0 + kKeys * kWaves < k1) load(j0 + kKeys * kWaves, next);
      const bool ends = now.end[0] < j0 + 16 || now.end[1] < j0 + 32 || sees_first < j0 + 32;
      f32x4_t s[NG][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float scale = scale_of(now.ks[r]);
#pragma unroll
        for (int ng = 0; ng < NG; ++ng) s[ng][r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t w[4];
          values_of<T>(now.k[r][kk], scale, w);
          const x8 kf = __builtin_bit_cast(x8, u32x4_t{w[0], w[1], w[2], w[3]});
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) s[ng][r] = E::mfma16(kf, qb[ng][kk], s[ng][r]);
        }
      }
      u32x4_t w[NG];  // the weights of eight keys
#pragma unroll
      for (int ng = 0; ng < NG; ++ng) {
        float xs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) xs[i] = base2(s[ng][i >> 2][i & 3], a.scale2);
        if (ends) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (j0 + 16 * (i >> 2) + 4 * quad + (i & 3) >= min(now.end[i >> 2], sees[ng])) xs[i] = -INFINITY;
        }
        float mt = xs[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mt = fmaxf(mt, xs[i]);
        float other = mt;
        swap16(mt, other);
        mt = other = fmaxf(mt, other);
        swap32(mt, other);
        const float m_new = fmaxf(m_run[ng], fmaxf(mt, other));
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
        float p[8], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(xs[i] - m_use + E::kTermsBias);
          sum += p[i];
        }
        l_run[ng] += sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[ng][i] = elem_pack<T>(p[2 * i], p[2 * i + 1]);
      }
      // (Keys that are left out: no weight, and no NaN or infinity for it to meet.  Where
      // some rows see a key and others do not, what is not finite reaches the former behind
      // the last tile.)
      float vscale[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t byte = now.vs[i >> 2][i & 3] >> (8 * (col >> 2)) & 255u;
        vscale[i] = scale_of(byte);
        if (ends) {
          const int32_t j = j0 + 16 * (i >> 2) + 4 * quad + (i & 3);
          const bool in = j < now.end[i >> 2], partly = j >= sees_first && byte > uint32_t(Four<T>::kMost);
          odd |= in && partly;
          if (!in || partly) vscale[i] = 1.0f;
        }
      }
      auto add = [&](int d, const uint32_t (&u)[8]) {  // dimensions 2 d and 2 d + 1 of the lane's eight
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t pick = b ? 0x07060302u : 0x05040100u;
          u32x4_t f;
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], pick);
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
            o[ng][2 * d + b] = E::mfma16(__builtin_bit_cast(x8, w[ng]), __builtin_bit_cast(x8, f), o[ng][2 * d + b]);
        }
      };
      uint32_t u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<0>(now.v[i], vscale[i]);
      add(0, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<1>(now.v[i], vscale[i]);
      add(1, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<2>(now.v[i], vscale[i]);
      add(2, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = Four<T>::template values<3>(now.v[i], vscale[i]);
      add(3, u);
    }
    if (__ballot(odd)) {
      for (int32_t j = max(k0, sees_first); j < k1; ++j) {
        if ((j - k0) / kKeys % kWaves != wave) continue;
        pages.seek(j >> c.page_shift);
        if (pages.is_bad(j >> c.page_shift)) continue;
        const uint32_t byte = (v_pool + page4(c, unit, pages.page(j >> c.page_shift)) + scales_at + (j & in_page) * 4)[col >> 2];
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t seen = __shfl(sees[ng], 4 * quad + r);
            const float e = byte > uint32_t(Four<T>::kMost) && j < seen ? __builtin_nanf("") : 0.0f;
#pragma unroll
            for (int db = 0; db < 8; ++db) o[ng][db][r] += e;
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
        for (int r = 0; r < 4; ++r) sm_o[wave][16 * ng + 4 * quad + r][col * 8 + db] = o[ng][db][r];
    }
    __syncthreads();
    const int64_t slot = paged_slot(blockIdx.x, plan.share, it.start) * kRows;
    for (int e = threadIdx.x; e < rows * (kHeadDim / 2); e += NT) {
      const int h = e / (kHeadDim / 2), dim = e % (kHeadDim / 2) * 2;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm_m[w][h]);
      float L = 0.0f, O0 = 0.0f, O1 = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float wt = sm_m[w][h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_m[w][h] - M);
        L += wt * sm_l[w][h];
        O0 += wt * sm_o[w][h][dim];
        O1 += wt * sm_o[w][h][dim + 1];
      }
      if (whole) {
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        *reinterpret_cast<uint32_t*>(a.out + place(h) * kHeadDim + dim) = elem_pack<T>(O0 * inv, O1 * inv);
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

template <typename T>
hipError_t few(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.rows == 16) hipLaunchKernelGGL((paged4_few_kernel<T, 1>), dim3(a.shares), dim3(kWaves * 64), 0, stream, a);
  else hipLaunchKernelGGL((paged4_few_kernel<T, 2>), dim3(a.shares), dim3(kWaves * 64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged4_few(const PagedAttnArgs& a, bool half, hipStream_t stream) {
  const hipError_t e = half ? few<_Float16>(a, stream) : few<__bf16>(a, stream);
  return e != hipSuccess ? e : launch_paged_join(a, half, stream);
}

}  // namespace stlite
