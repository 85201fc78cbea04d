// The flat range of a paged attention call (PagedAttnArgs) as a
// work-group finds its way in it.
#pragma once

#include "paged.h"
#include "paged_cuts.h"

namespace stlite {

// A run of whole tokens' queries of one (unit, head group, sequence).
struct PagedItem {
  int32_t unit, seq, index;  // unit = (layer, kv head, head group)
  int32_t n, cached, row0;   // new tokens, tokens before them (negative: too short), first new token
  int64_t start, keys;       // place of its first key in the flat range
};

template <int NT>  // threads of the work-group, a multiple of 64
struct PagedPlan {
  struct Shared {
    int64_t wave[NT / 64];
    int64_t base;
    int32_t seq, index;
  };
  const PagedAttnArgs& a;
  Shared& sh;
  int64_t per_unit, total, share;
  int64_t mine, before;  // this thread's sequences' places, and those of the threads before it
  int32_t s0, s1;        // this thread's sequences

  __device__ int32_t items_of(int32_t s) const { return paged_items(a.c.cu_new[s + 1] - a.c.cu_new[s], a.tokens); }
  __device__ int64_t range_of(int32_t s) const {
    const int32_t n = a.c.cu_new[s + 1] - a.c.cu_new[s];
    return paged_range(n, paged_len(a.c, s) - n, a.tokens, a.item_cost);
  }

  // The sum of v over the threads before this one, and over all.
  __device__ int64_t scan(int64_t v, int64_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    if (lane == 63) sh.wave[wave] = sum;
    __syncthreads();
    sum -= v;
    all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) sum += sh.wave[w];
      all += sh.wave[w];
    }
    all = uniform(all);
    return sum;
  }

  __device__ PagedPlan(const PagedAttnArgs& args, Shared& shared) : a(args), sh(shared) {
    if (a.c.n_seqs == 1) {  // one trajectory: nothing to search
      s0 = 0;
      s1 = 1;
      before = 0;
      mine = per_unit = uniform(range_of(0));
    } else {
      const int32_t per = (a.c.n_seqs + NT - 1) / NT;
      s0 = min(int32_t(threadIdx.x) * per, a.c.n_seqs);
      s1 = min(s0 + per, a.c.n_seqs);
      mine = 0;
      for (int32_t s = s0; s < s1; ++s) mine += range_of(s);
      before = scan(mine, per_unit);
    }
    total = per_unit * a.c.n_units * a.parts;
    share = paged_share(total, a.shares, a.min_share);
  }

  __device__ static int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(uint64_t(v) >> 32));
    return int64_t((uint64_t(hi) << 32) | lo);
  }

  // The item that place x of the range lies in (0 <= x < total; the whole
  // work-group calls).
  __device__ PagedItem find(int64_t x) {
    const int64_t unit = x / per_unit, rem = x - unit * per_unit;
    PagedItem it;
    it.unit = int32_t(unit);
    if (a.c.n_seqs == 1) {
      it.seq = 0;
      load_seq(it);
      it.index = paged_item_of(rem, it.n, it.cached, a.tokens, a.item_cost);
      it.start = unit * per_unit + paged_prefix(it.index, it.cached, a.tokens, a.item_cost) + a.item_cost;
      set_keys(it);
      return it;
    }
    __syncthreads();
    if (mine > 0 && rem >= before && rem < before + mine) {
      int64_t b = before;
      int32_t s = s0;
      for (; s + 1 < s1; ++s) {
        const int64_t k = range_of(s);
        if (rem < b + k) break;
        b += k;
      }
      sh.seq = s;
      sh.base = b;
    }
    __syncthreads();
    it.seq = __builtin_amdgcn_readfirstlane(sh.seq);
    const int64_t base = uniform(sh.base), in = rem - base;
    load_seq(it);
    it.index = paged_item_of(in, it.n, it.cached, a.tokens, a.item_cost);
    it.start = unit * per_unit + base + paged_prefix(it.index, it.cached, a.tokens, a.item_cost) + a.item_cost;
    set_keys(it);
    return it;
  }

  // Item i of the call's join_items (the whole work-group calls).
  __device__ PagedItem item(int32_t i) {
    const int32_t per = a.join_items / (a.c.n_units * a.parts);
    PagedItem it;
    it.unit = i / per;
    it.index = i % per;
    it.seq = 0;
    int64_t base = 0;
    if (a.c.n_seqs > 1) {
      int32_t count = 0;
      for (int32_t s = s0; s < s1; ++s) count += items_of(s);
      __syncthreads();  // (the last scan's sums have been read)
      int64_t all;
      int32_t at = it.index - int32_t(scan(count, all));
      if (at >= 0 && at < count) {
        int64_t b = before;
        int32_t s = s0;
        for (; at >= items_of(s); ++s) {
          at -= items_of(s);
          b += range_of(s);
        }
        sh.seq = s;
        sh.index = at;
        sh.base = b;
      }
      __syncthreads();
      it.seq = __builtin_amdgcn_readfirstlane(sh.seq);
      it.index = __builtin_amdgcn_readfirstlane(sh.index);
      base = uniform(sh.base);
    }
    load_seq(it);
    it.start = it.unit * per_unit + base + paged_prefix(it.index, it.cached, a.tokens, a.item_cost) + a.item_cost;
    set_keys(it);
    return it;
  }

  // The item behind `it` (it is not the last one of the range).
  __device__ void next(PagedItem& it) const {
    it.start += it.keys + a.item_cost;
    if (++it.index < paged_items(it.n, a.tokens)) return set_keys(it);
    it.index = 0;
    do {
      if (++it.seq == a.c.n_seqs) {
        it.seq = 0;
        ++it.unit;
      }
      load_seq(it);
    } while (it.n == 0);
    set_keys(it);
  }

  __device__ void load_seq(PagedItem& it) const {
    it.row0 = a.c.cu_new[it.seq];
    it.n = a.c.cu_new[it.seq + 1] - it.row0;
    it.cached = paged_len(a.c, it.seq) - it.n;
  }
  __device__ void set_keys(PagedItem& it) const {
    it.keys = paged_item_keys(it.index, it.n, it.cached, a.tokens);
  }
};

}  // namespace stlite
