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

// NT: threads of the work-group, a multiple of 64; KEEPS: items of up to a.keep keys are
// not cut, but whole in the share that their middle lies in.
template <int NT, bool KEEPS = false>
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

  // The first item of the share [x, y), if it has one (the whole work-group calls).
  __device__ bool first(int64_t& x, int64_t y, PagedItem& it) {
    if (x >= y) return false;
    it = find(x);
    if (kept(it) && middle2(it) <= 2 * x) {  // the share before has it
      x = it.start + it.keys;
      if (x >= y) return false;
      next(it);
    }
    return ours(it, y);
  }
  // Whether the item, not one of an earlier share, is this one's, which ends at y.
  __device__ bool ours(const PagedItem& it, int64_t y) const { return kept(it) ? middle2(it) <= 2 * y : it.start < y; }
  __device__ PagedPart part(int64_t x, int64_t y, const PagedItem& it) const {
    return kept(it) ? paged_part(it.start, it.start + it.keys, it.start, it.keys) : paged_part(x, y, it.start, it.keys);
  }
  __device__ bool kept(const PagedItem& it) const { return KEEPS && it.keys <= a.keep; }
  __device__ int64_t middle2(const PagedItem& it) const { return 2 * it.start + it.keys - a.item_cost; }

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

}  // namespace stlite
