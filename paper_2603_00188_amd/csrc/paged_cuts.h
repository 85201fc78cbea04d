// How a paged attention call is cut: a flat range of places (PagedAttnArgs) into
// equal shares, and where an item lies in it.  Integer arithmetic shared by the
// attention kernels and the joining launch, which must agree on every cut, with
// nothing of HIP in it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define STLITE_BOTH __host__ __device__ inline
#else
#define STLITE_BOTH inline
#endif

namespace stlite {

constexpr int32_t kPagedTile = 64;  // keys of a step

// Items of a sequence with n new tokens, `tokens` each; what the first i of them
// take of the range (not the last one) and what all of them take, with `cached`
// tokens before the new ones.  An item takes `cost` places, what beginning one costs
// in keys' time, and then one for each of its keys.  A sequence too short for its new
// tokens (cached < 0) counts as if nothing were cached: every item has a key of the
// range, so that every output is written.
STLITE_BOTH int32_t paged_items(int32_t n, int32_t tokens) { return int32_t((int64_t(n) + tokens - 1) / tokens); }
STLITE_BOTH int64_t paged_prefix(int64_t i, int32_t cached, int32_t tokens, int32_t cost) {
  return i * (int64_t(cached > 0 ? cached : 0) + cost) + int64_t(tokens) * (i * (i + 1) / 2);
}
STLITE_BOTH int64_t paged_item_keys(int32_t index, int32_t n, int32_t cached, int32_t tokens) {
  const int64_t own = (int64_t(index) + 1) * tokens;
  return (cached > 0 ? cached : 0) + (own < n ? own : n);
}
STLITE_BOTH int64_t paged_range(int32_t n, int32_t cached, int32_t tokens, int32_t cost) {
  const int32_t items = paged_items(n, tokens);
  return items == 0 ? 0 : paged_prefix(items - 1, cached, tokens, cost) + cost + paged_item_keys(items - 1, n, cached, tokens);
}
// The item that place `in` of the sequence lies in.
STLITE_BOTH int32_t paged_item_of(int64_t in, int32_t n, int32_t cached, int32_t tokens, int32_t cost) {
  int32_t lo = 0, hi = paged_items(n, tokens);
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (paged_prefix(mid, cached, tokens, cost) <= in) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Places of a share.
STLITE_BOTH int64_t paged_share(int64_t total, int32_t shares, int32_t min_share) {
  const int64_t even = (total + shares - 1) / shares;
  return even > min_share ? even : min_share;
}

// What the places [x, y) take of the item whose first key is at `start` < y: the
// 64-key tiles [t0, t1).  Neighbouring shares round the same key up, so that every
// tile is in one share.
struct PagedPart {
  int64_t end;  // of the part in the range
  int32_t t0, t1;
  bool whole;
};
STLITE_BOTH PagedPart paged_part(int64_t x, int64_t y, int64_t start, int64_t keys) {
  const int64_t xr = x > start ? x - start : 0, yr = y - start < keys ? y - start : keys;
  PagedPart p;
  p.end = start + yr;
  p.t0 = int32_t((xr + kPagedTile - 1) / kPagedTile);
  p.t1 = int32_t((yr + kPagedTile - 1) / kPagedTile);
  p.whole = xr == 0 && yr == keys;
  return p;
}

// Where share w keeps its part of the item at `start`: a share cuts at most its
// first item (slot 0) and its last one (slot 1).
STLITE_BOTH int64_t paged_slot(int64_t w, int64_t share, int64_t start) { return 2 * w + (w * share >= start ? 0 : 1); }

}  // namespace stlite
