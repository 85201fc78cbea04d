// Host layer of the paged cache (include/stlite_paged.h): argument validation,
// workspace sizing and launch configuration.
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "paged.h"
#include "stlite.h"
#include "stlite_paged.h"

namespace stlite {
stlite_status report_error(stlite_status st, const char* msg);  // stlite_abi.hip
}

using namespace stlite;

namespace {

stlite_status fail(stlite_status st, const char* fmt, ...) {
  char msg[384];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  return report_error(st, msg);
}

stlite_status ok() { return report_error(STLITE_OK, ""); }

stlite_status hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(STLITE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr int32_t kMaxGroup = 128;
constexpr int64_t kMaxLen = int64_t(1) << 28;
constexpr int64_t kIntRows = (int64_t(1) << 31) - 1;

// The pool and its tables; `batch`: the new tokens too.
stlite_status check_cache(const stlite_paged* c, bool batch) {
  if (!c) return fail(STLITE_ERR_INVALID_ARG, "the cache is NULL");
  if (c->n_layers < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1)
    return fail(STLITE_ERR_INVALID_ARG, "n_layers, n_q_heads and n_kv_heads must be >= 1");
  if (c->n_q_heads % c->n_kv_heads != 0)
    return fail(STLITE_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", c->n_q_heads,
                c->n_kv_heads);
  if (c->head_dim != kHeadDim)
    return fail(STLITE_ERR_UNSUPPORTED, "head_dim %d: only %d is implemented", c->head_dim, kHeadDim);
  if (c->n_q_heads / c->n_kv_heads > kMaxGroup)
    return fail(STLITE_ERR_UNSUPPORTED, "%d query heads per kv head: at most %d", c->n_q_heads / c->n_kv_heads,
                kMaxGroup);
  if (c->dtype != STLITE_BF16 && c->dtype != STLITE_FP16)
    return fail(STLITE_ERR_INVALID_ARG, "dtype must be STLITE_BF16 or STLITE_FP16 (got %d)", c->dtype);
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
    return fail(STLITE_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256 (got %d)", c->page_size);
  if (c->n_pages < 1) return fail(STLITE_ERR_INVALID_ARG, "n_pages must be >= 1");
  if (int64_t(c->n_pages) * c->page_size > kIntRows)
    return fail(STLITE_ERR_UNSUPPORTED, "n_pages * page_size = %lld: at most 2^31 - 1 rows",
                (long long)(int64_t(c->n_pages) * c->page_size));
  if (c->n_seqs < 1) return fail(STLITE_ERR_INVALID_ARG, "n_seqs must be >= 1");
  if (c->n_seqs > 65535) return fail(STLITE_ERR_UNSUPPORTED, "n_seqs %d: at most 65535 sequences", c->n_seqs);
  if (int64_t(c->n_layers) * c->n_kv_heads > 65535)
    return fail(STLITE_ERR_UNSUPPORTED, "more than 65535 (layer, kv head) units");
  if (c->max_pages < 1) return fail(STLITE_ERR_INVALID_ARG, "max_pages must be >= 1");
  if (c->max_len < 1 || c->max_len > int64_t(c->max_pages) * c->page_size)
    return fail(STLITE_ERR_INVALID_ARG, "max_len %d outside [1, max_pages * page_size = %lld]", c->max_len,
                (long long)(int64_t(c->max_pages) * c->page_size));
  if (c->max_len > kMaxLen) return fail(STLITE_ERR_UNSUPPORTED, "max_len %d: at most 2^28", c->max_len);
  if (!c->k || !c->v || !c->page_table) return fail(STLITE_ERR_INVALID_ARG, "k, v and page_table must be non-NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(STLITE_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (!batch) return STLITE_OK;
  if (!c->seq_lens || !c->cu_new || !c->h_cu_new)
    return fail(STLITE_ERR_INVALID_ARG, "seq_lens, cu_new and h_cu_new must be non-NULL");
  if (c->h_cu_new[0] != 0) return fail(STLITE_ERR_INVALID_ARG, "cu_new[0] must be 0");
  for (int32_t s = 0; s < c->n_seqs; ++s) {
    const int64_t n = int64_t(c->h_cu_new[s + 1]) - c->h_cu_new[s];
    if (n < 0 || n > c->max_len)
      return fail(STLITE_ERR_INVALID_ARG, "sequence %d has %lld new tokens, outside [0, max_len = %d]", s, (long long)n,
                  c->max_len);
  }
  if (c->total_new != c->h_cu_new[c->n_seqs])
    return fail(STLITE_ERR_INVALID_ARG, "total_new %lld != cu_new[n_seqs] %d", (long long)c->total_new,
                c->h_cu_new[c->n_seqs]);
  return STLITE_OK;
}

PagedDev device_view(const stlite_paged* c) {
  PagedDev d;
  d.k = static_cast<uint16_t*>(c->k);
  d.v = static_cast<uint16_t*>(c->v);
  d.page_table = c->page_table;
  d.seq_lens = c->seq_lens;
  d.cu_new = c->cu_new;
  d.n_layers = c->n_layers;
  d.n_q_heads = c->n_q_heads;
  d.n_kv_heads = c->n_kv_heads;
  d.n_units = c->n_layers * c->n_kv_heads;
  d.group = c->n_q_heads / c->n_kv_heads;
  d.n_seqs = c->n_seqs;
  d.n_pages = c->n_pages;
  d.max_pages = c->max_pages;
  d.max_len = c->max_len;
  d.page_shift = 0;
  while ((1 << d.page_shift) < c->page_size) ++d.page_shift;
  d.total_new = c->total_new;
  return d;
}

// How an attention call runs, from what the host knows (not the lengths).
//
// item_cost: a work-group's queries, first page and tiles, unequal limits and output
// take it as long as six tiles of several tokens, or four sub-tiles of one.  Counted
// as none / as here, and flat within 1 % from half to twice that: 5 prompts of 131 to
// 2999 tokens 324 / 219 us, 5 drafted tokens in each of 16 sequences 69.6 / 64, one
// token of one layer 17 / 14.4; a screen behind 30k tokens and a step's decoding alike.
// min_share: five tokens behind 678 took 17.6 us with 128, 19 with 256, 24 with 512; one
// token 11.3 with 64, 14.2 with 128.  Shares: one work-group of several tokens per CU
// (its rings fill the LDS), two of one token (256 / 512 / 1024: a ragged batch 742 / 729
// / 743 us, a step 265 / 270 / 274, a long cache 64.6 / 63.8 / 67.5).  One token by the
// several-token kernel: 18 us for 11, 72 for 64, 309 for 270, 806 for 729.
struct AttnPlan {
  bool decode;
  int32_t parts, tokens, rows, shares, min_share, item_cost, join_items, join_rows, join_groups, join_split;
  size_t bytes;
};

AttnPlan attn_plan(const stlite_paged* c) {
  AttnPlan p;
  const int64_t group = c->n_q_heads / c->n_kv_heads;
  int64_t most = 0, live = 0;  // new tokens of a sequence; sequences with any
  for (int32_t s = 0; s < c->n_seqs; ++s) {
    const int64_t n = int64_t(c->h_cu_new[s + 1]) - c->h_cu_new[s];
    most = std::max(most, n);
    live += n > 0;
  }
  p.decode = most <= 1;
  int64_t items = int64_t(c->n_layers) * c->n_kv_heads;
  if (p.decode) {
    p.rows = group <= 16 ? 16 : 32;
    p.parts = int32_t(ceil_div(group, p.rows));
    p.tokens = 1;
    p.shares = 512;
    p.min_share = 64;
    p.item_cost = 64;
    items *= p.parts * live;
  } else {
    p.parts = 1;
    p.rows = kExtRows;
    p.tokens = int32_t(p.rows / group);
    p.shares = 256;
    p.min_share = 128;
    p.item_cost = 384;
    int64_t blocks = 0;
    for (int32_t s = 0; s < c->n_seqs; ++s) blocks += ceil_div(int64_t(c->h_cu_new[s + 1]) - c->h_cu_new[s], p.tokens);
    items *= blocks;
  }
  if (items == 1) p.item_cost = 0;  // nothing to balance
  // (no more shares than the longest possible range fills)
  const double range = double(items) * (double(c->max_len) + p.item_cost);
  p.shares = int32_t(std::max(1.0, std::min(double(p.shares), std::ceil(range / p.min_share))));
  // Joining by boundary gives every cut item to one work-group (with a quarter of its
  // rows each, and four times the work-groups, prompts of 131 to 2999 tokens took 220 us,
  // with all of them 216).  Where that is more than a round of its loads on average (rows
  // times parts over 32 groups of lanes, four loads each), one round of work-groups (two
  // per CU) shares out the items' rows, which costs a second scan of the lengths.  By
  // boundary / by item: one token behind 3 sequences of up to 79079 in 2 units 63.8 / 45.6
  // us, 4 of up to 6000 in 4 units 28.0 / 21.4, two layers of one behind 8000 24.2 / 18.4;
  // 16 of up to 1000 in 4 units 19.0 / 24.0, five drafted tokens in 16 in 8 62 / 65.
  const int64_t item_rows = p.decode ? std::min<int64_t>(group, p.rows) : std::min<int64_t>(p.tokens, most) * group;
  p.join_items = items < p.shares && item_rows * p.shares >= 128 * items ? int32_t(items) : 0;
  p.join_rows = p.join_items ? int32_t(ceil_div(items * item_rows, 512)) : int32_t(item_rows);
  // A boundary's work-group has 256 threads where that is few rounds of loads too, so that
  // the 511 of one token run at once, else 1024.  256 / 1024 threads: 8 sequences of up to
  // 1000 16.6 / 20.2 us, 64 of up to 150 in 8 layers 41 / 44, a step 263 / 266; the 255
  // of several tokens gain less, five drafted ones in 16 sequences 64 / 62.
  p.join_groups = !p.join_items && item_rows * (items + p.shares) <= (p.decode ? 128 : 64) * items ? 8 : 32;
  p.join_split = int32_t(ceil_div(item_rows, p.join_rows));
  const size_t slots = size_t(p.shares) * 2 * p.rows;
  p.bytes = p.shares == 1 ? 0 : 2 * align_up(slots * sizeof(float)) + align_up(slots * kHeadDim * sizeof(float));
  return p;
}

stlite_status check_rows(const stlite_rows* r, int64_t heads, const char* name) {
  if (!r || !r->data) return fail(STLITE_ERR_INVALID_ARG, "%s must be non-NULL", name);
  if (!aligned16(r->data) || r->token_stride % 8 != 0 || r->layer_stride % 8 != 0)
    return fail(STLITE_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned, strides multiples of 8", name);
  if (r->token_stride < heads * kHeadDim || r->layer_stride < 0)
    return fail(STLITE_ERR_INVALID_ARG, "%s: token_stride %lld is less than a token's %lld elements, or layer_stride < 0",
                name, (long long)r->token_stride, (long long)(heads * kHeadDim));
  return STLITE_OK;
}

bool meet(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + b_bytes && y < x + a_bytes;
}
size_t pool_bytes(const stlite_paged* c) {
  return size_t(c->n_layers) * c->n_kv_heads * c->n_pages * c->page_size * kHeadDim * sizeof(uint16_t);
}
size_t query_bytes(const stlite_paged* c) {
  return size_t(c->n_layers) * c->total_new * c->n_q_heads * kHeadDim * sizeof(uint16_t);
}
bool meets_pool(const stlite_paged* c, const void* p, size_t bytes) {
  return meet(p, bytes, c->k, pool_bytes(c)) || meet(p, bytes, c->v, pool_bytes(c));
}

// Whether rows of `heads` heads share an element with the `bytes` bytes at p; what lies
// between two tokens' rows or two layers' is another's.
bool rows_meet(const stlite_paged* c, const stlite_rows* r, int64_t heads, const void* p, size_t bytes) {
  const int64_t own = heads * kHeadDim * int64_t(sizeof(uint16_t)), step = r->token_stride * int64_t(sizeof(uint16_t));
  for (int64_t l = 0; l < c->n_layers; ++l) {
    const int64_t from = int64_t(reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(r->data + l * r->layer_stride));
    const int64_t t = from < own ? 0 : (from - own) / step + 1;  // the first token that ends behind p
    if (t < c->total_new && t * step < from + int64_t(bytes)) return true;
  }
  return false;
}

RowsIn rows_in(const stlite_rows* r) {
  return r ? RowsIn{r->data, r->token_stride, r->layer_stride} : RowsIn{nullptr, 0, 0};
}

}  // namespace

extern "C" {

stlite_status stlite_paged_validate(const stlite_paged* c, const int32_t* h_page_table, const int32_t* h_seq_lens) {
  const stlite_status st = check_cache(c, true);
  if (st != STLITE_OK) return st;
  if (!h_seq_lens) return ok();
  for (int32_t s = 0; s < c->n_seqs; ++s) {
    const int32_t n = c->h_cu_new[s + 1] - c->h_cu_new[s];
    if (h_seq_lens[s] < n || h_seq_lens[s] > c->max_len)
      return fail(STLITE_ERR_INVALID_ARG, "sequence %d has length %d, outside [%d new tokens, max_len = %d]", s,
                  h_seq_lens[s], n, c->max_len);
  }
  if (!h_page_table) return ok();
  std::vector<int32_t> holders;
  try {
    holders.assign(size_t(c->n_pages), 0);
  } catch (const std::bad_alloc&) {
    return fail(STLITE_ERR_INVALID_ARG, "no host memory for %d pages", c->n_pages);
  }
  for (int32_t s = 0; s < c->n_seqs; ++s) {
    const int32_t used = int32_t(ceil_div(h_seq_lens[s], c->page_size));
    for (int32_t e = 0; e < used; ++e) {
      const int32_t page = h_page_table[int64_t(s) * c->max_pages + e];
      if (page < 0 || page >= c->n_pages)
        return fail(STLITE_ERR_INVALID_ARG, "sequence %d: page_table entry %d is %d, outside [0, %d)", s, e, page,
                    c->n_pages);
      ++holders[size_t(page)];
    }
  }
  for (int32_t s = 0; s < c->n_seqs; ++s) {
    const int32_t n = c->h_cu_new[s + 1] - c->h_cu_new[s];
    if (n == 0) continue;
    const int32_t first = (h_seq_lens[s] - n) / c->page_size, used = int32_t(ceil_div(h_seq_lens[s], c->page_size));
    for (int32_t e = first; e < used; ++e)
      if (holders[size_t(h_page_table[int64_t(s) * c->max_pages + e])] > 1)
        return fail(STLITE_ERR_INVALID_ARG, "sequence %d stores new tokens in page %d, which the table holds twice", s,
                    h_page_table[int64_t(s) * c->max_pages + e]);
  }
  return ok();
}

stlite_status stlite_paged_workspace_size(const stlite_paged* c, size_t* bytes) {
  if (!bytes) return fail(STLITE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = 0;
  const stlite_status st = check_cache(c, true);
  if (st != STLITE_OK) return st;
  if (c->total_new > 0) *bytes = attn_plan(c).bytes;
  return ok();
}

stlite_status stlite_paged_compact(const stlite_problem* p, const stlite_paged* c, const uint16_t* k,
                                   const uint16_t* v, const int32_t* kept, int32_t per_layer, void* stream) {
  stlite_status st = stlite_validate(p);
  if (st != STLITE_OK) return st;
  st = check_cache(c, false);
  if (st != STLITE_OK) return st;
  if (p->n_layers != c->n_layers || p->n_kv_heads != c->n_kv_heads || p->n_seqs != c->n_seqs)
    return fail(STLITE_ERR_INVALID_ARG, "the problem has %d layers, %d kv heads, %d sequences; the cache %d, %d, %d",
                p->n_layers, p->n_kv_heads, p->n_seqs, c->n_layers, c->n_kv_heads, c->n_seqs);
  for (int32_t s = 0; s < p->n_seqs; ++s)
    if (p->h_cu_budget[s + 1] - p->h_cu_budget[s] > c->max_len)
      return fail(STLITE_ERR_INVALID_ARG, "sequence %d keeps %d rows, more than max_len = %d", s,
                  p->h_cu_budget[s + 1] - p->h_cu_budget[s], c->max_len);
  if (!c->seq_lens) return fail(STLITE_ERR_INVALID_ARG, "seq_lens must be non-NULL");
  if (p->total_budget > 0 && (!k || !v || !kept)) return fail(STLITE_ERR_INVALID_ARG, "k, v and kept must be non-NULL");
  if (!aligned16(k) || !aligned16(v)) return fail(STLITE_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  const size_t rows_bytes = size_t(p->n_layers) * p->n_kv_heads * p->total_tokens * kHeadDim * sizeof(uint16_t);
  if (p->total_budget > 0 && (meets_pool(c, k, rows_bytes) || meets_pool(c, v, rows_bytes)))
    return fail(STLITE_ERR_INVALID_ARG, "k and v must not alias the pool: rows are not moved in place");
  PagedCompactArgs a;
  a.c = device_view(c);
  a.cu_budget = p->cu_budget;
  a.total_tokens = p->total_tokens;
  a.total_budget = p->total_budget;
  a.k = k;
  a.v = v;
  a.kept = kept;
  a.kept_per_layer = per_layer != 0;
  return hip_status(launch_paged_compact(a, static_cast<hipStream_t>(stream)), "paged_compact launch");
}

stlite_status stlite_paged_append(const stlite_paged* c, const stlite_rope* rope, const int32_t* positions,
                                  const stlite_rows* q, const stlite_rows* k, const stlite_rows* v,
                                  const uint16_t* q_norm, const uint16_t* k_norm, float eps, uint16_t* q_out,
                                  void* stream) {
  stlite_status st = check_cache(c, true);
  if (st != STLITE_OK) return st;
  PagedAppendArgs a{};
  if ((rope == nullptr) != (positions == nullptr))
    return fail(STLITE_ERR_INVALID_ARG, "rope and positions must be both given or both NULL");
  if (rope) {
    if (!std::isfinite(rope->theta) || rope->theta < 1.0)
      return fail(STLITE_ERR_INVALID_ARG, "theta must be finite and >= 1");
    if (rope->interleaved != 0 && rope->interleaved != 1)
      return fail(STLITE_ERR_INVALID_ARG, "interleaved must be 0 or 1 (got %d)", rope->interleaved);
    if (rope->reserved != 0) return fail(STLITE_ERR_INVALID_ARG, "reserved field must be 0");
    if (rope->n_axes != 1 && rope->n_axes != 3)
      return fail(STLITE_ERR_INVALID_ARG, "n_axes must be 1 or 3 (got %d)", rope->n_axes);
    a.axis1 = a.axis2 = 64;
    if (rope->n_axes == 3) {
      const int32_t* s = rope->sections;
      if (s[0] < 0 || s[1] < 0 || s[2] < 0 || int64_t(s[0]) + s[1] + s[2] != 64)
        return fail(STLITE_ERR_INVALID_ARG, "sections %d + %d + %d must be >= 0 and add up to 64", s[0], s[1], s[2]);
      a.axis1 = s[0];
      a.axis2 = s[0] + s[1];
    }
    a.interleaved = rope->interleaved;
    double coarse[8], fine[8];  // (16 powers instead of 64: a microsecond of the host's)
    for (int i = 0; i < 8; ++i) {
      coarse[i] = std::pow(rope->theta, -i / 8.0) / (2.0 * M_PI);
      fine[i] = std::pow(rope->theta, -i / 64.0);
    }
    for (int i = 0; i < 64; ++i) a.turns[i] = coarse[i / 8] * fine[i % 8];
  }
  if (c->total_new == 0) return ok();
  st = check_rows(k, c->n_kv_heads, "k");
  if (st == STLITE_OK) st = check_rows(v, c->n_kv_heads, "v");
  const bool queries = q && q->data;
  if (st == STLITE_OK && queries) st = check_rows(q, c->n_q_heads, "q");
  if (st != STLITE_OK) return st;
  if (queries != (q_out != nullptr)) return fail(STLITE_ERR_INVALID_ARG, "q and q_out must be both given or both NULL");
  if (!aligned16(q_out) || !aligned16(q_norm) || !aligned16(k_norm))
    return fail(STLITE_ERR_INVALID_ARG, "q_out, q_norm and k_norm must be 16-byte aligned");
  if ((q_norm || k_norm) && !(eps >= 0.0f && std::isfinite(eps)))
    return fail(STLITE_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (queries) {
    const size_t bytes = query_bytes(c);
    if (rows_meet(c, q, c->n_q_heads, q_out, bytes) || rows_meet(c, k, c->n_kv_heads, q_out, bytes) ||
        rows_meet(c, v, c->n_kv_heads, q_out, bytes) || meets_pool(c, q_out, bytes))
      return fail(STLITE_ERR_INVALID_ARG, "q_out must not alias an input or the pool");
  }
  a.c = device_view(c);
  a.q = rows_in(queries ? q : nullptr);
  a.k = rows_in(k);
  a.v = rows_in(v);
  a.q_out = q_out;
  a.q_norm = q_norm;
  a.k_norm = k_norm;
  a.eps = eps;
  a.positions = positions;
  return hip_status(launch_paged_append(a, c->dtype == STLITE_FP16, static_cast<hipStream_t>(stream)),
                    "paged_append launch");
}

stlite_status stlite_paged_attention(const stlite_paged* c, const uint16_t* q, float scale, uint16_t* out, void* ws,
                                     size_t ws_bytes, void* stream) {
  const stlite_status st = check_cache(c, true);
  if (st != STLITE_OK) return st;
  if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e))
    return fail(STLITE_ERR_INVALID_ARG, "scale must be > 0 and at most 2^127");
  if (c->total_new == 0) return ok();
  const AttnPlan p = attn_plan(c);
  if (p.bytes > 0 && !ws) return fail(STLITE_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", p.bytes);
  if (ws_bytes < p.bytes) return fail(STLITE_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, p.bytes);
  if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return fail(STLITE_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (!q || !out) return fail(STLITE_ERR_INVALID_ARG, "q and out must be non-NULL");
  const size_t bytes = query_bytes(c);
  if (meet(q, bytes, out, bytes) || meets_pool(c, out, bytes))
    return fail(STLITE_ERR_INVALID_ARG, "out must not alias q or the pool");
  if (!aligned16(q) || !aligned16(out)) return fail(STLITE_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (p.bytes > 0 && (meet(ws, p.bytes, q, bytes) || meet(ws, p.bytes, out, bytes) || meets_pool(c, ws, p.bytes)))
    return fail(STLITE_ERR_WORKSPACE, "the workspace must not alias q, out or the pool");
  PagedAttnArgs a;
  a.c = device_view(c);
  a.q = q;
  a.out = out;
  a.scale2 = scale * kLog2e;
  a.parts = p.parts;
  a.tokens = p.tokens;
  a.rows = p.rows;
  a.shares = p.shares;
  a.min_share = p.min_share;
  a.item_cost = p.item_cost;
  a.join_items = p.join_items;
  a.join_rows = p.join_rows;
  a.join_groups = p.join_groups;
  a.join_split = p.join_split;
  const size_t slots = size_t(p.shares) * 2 * p.rows;
  a.pm = static_cast<float*>(ws);
  a.pl = a.pm + align_up(slots * sizeof(float)) / sizeof(float);
  a.po = a.pl + align_up(slots * sizeof(float)) / sizeof(float);
  const bool half = c->dtype == STLITE_FP16;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(p.decode ? launch_paged_decode(a, half, s) : launch_paged_extend(a, half, s),
                    "paged_attention launch");
}

}  // extern "C"
