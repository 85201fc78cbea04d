// Pages for growing sequences (stlite_paged_grow) and back (stlite_paged_release): page
// table, lengths and places of the next new tokens, out of a list of free pages.
#include "paged.h"

namespace stlite {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
// Places up to which the growing work-group writes them itself.
constexpr int64_t kOwnSlots = 4096;

// The sum of v over the threads before this one, and over all.
__device__ inline int64_t scan(int64_t v, int64_t (&sm)[kWaves], int64_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  __syncthreads();  // (the last scan's sums have been read)
  if (lane == 63) sm[wave] = sum;
  __syncthreads();
  sum -= v;
  all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) sum += sm[w];
    all += sm[w];
  }
  return sum;
}

// The thread whose pages entry f of the chunk's flat list belongs to: the last one with
// before[t] <= f (one without pages has the next one's).
__device__ inline int owner(const int64_t (&before)[kThreads], int64_t f) {
  int lo = 0, hi = kThreads;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= f) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ inline int32_t pages_of(const PagedDev& c, int64_t len) {
  return int32_t((len + (int64_t(1) << c.page_shift) - 1) >> c.page_shift);
}

__device__ inline int32_t slot_of(const PagedDev& c, int32_t s, int64_t i) {
  const int32_t len = c.seq_lens[s];
  const int64_t at = int64_t(len) - c.cu_new[s + 1] + i;
  if (len < 0 || len > c.max_len || at < 0) return -1;
  const int32_t page = c.page_table[int64_t(s) * c.max_pages + (at >> c.page_shift)];
  return page >= 0 && page < c.n_pages ? (page << c.page_shift) + int32_t(at & ((1 << c.page_shift) - 1)) : -1;
}

__device__ inline int32_t seq_of(const int32_t* cu, int32_t n, int64_t j) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (cu[mid] <= j) lo = mid;
    else hi = mid;
  }
  return lo;
}

// One work-group, since every sequence's pages lie behind those of the sequences before
// it: a scan of what 1024 sequences at a time need, then their pages as one flat list, a
// thread each.  Latency-bound: three loads, a scan, a load and a store one after another.
__global__ __launch_bounds__(kThreads) void paged_grow_kernel(PagedPagesArgs a) {
  __shared__ int64_t sm_wave[kWaves], sm_before[kThreads];
  __shared__ int32_t sm_held[kThreads];
  const PagedDev& c = a.c;
  const int32_t n_free = min(max(*a.n_free, 0), c.n_pages);
  int64_t carry = 0;  // pages that the sequences before this chunk need
  int64_t taken = 0;  // pages given out
  for (int32_t base = 0; base < c.n_seqs; base += kThreads) {
    const int32_t s = base + int32_t(threadIdx.x);
    int32_t len = 0, held = 0;
    int64_t grown = 0, need = 0;
    bool fits = false;
    if (s < c.n_seqs) {
      const int32_t now = c.seq_lens[s], n = c.cu_new[s + 1] - c.cu_new[s];
      held = min(max(a.held[s], 0), c.max_pages);
      len = now < 0 ? now : min(now, c.max_len);
      grown = int64_t(len) + n;
      fits = len >= 0 && grown <= c.max_len;
      if (fits) need = max(pages_of(c, grown) - held, 0);
    }
    int64_t all;
    const int64_t before = scan(need, sm_wave, all);
    const bool granted = fits && (need == 0 || carry + before + need <= n_free);
    sm_before[threadIdx.x] = before;
    sm_held[threadIdx.x] = held;
    if (s < c.n_seqs) {
      c.seq_lens[s] = granted ? int32_t(grown) : len < 0 ? len : ~len;
      if (granted) a.held[s] = held + int32_t(need);
    }
    int64_t here;  // what this chunk takes: the needs of a first part of its sequences
    scan(granted ? need : 0, sm_wave, here);
    __syncthreads();
    for (int64_t f = threadIdx.x; f < here; f += kThreads) {
      const int t = owner(sm_before, f);
      c.page_table[int64_t(base + t) * c.max_pages + sm_held[t] + (f - sm_before[t])] = a.free_pages[n_free - 1 - (carry + f)];
    }
    carry += all;
    taken += here;
  }
  __syncthreads();
  if (threadIdx.x == 0) *a.n_free = n_free - int32_t(taken);
  if (a.slots && c.total_new <= kOwnSlots)
    for (int64_t i = threadIdx.x; i < c.total_new; i += kThreads) a.slots[i] = slot_of(c, seq_of(c.cu_new, c.n_seqs, i), i);
}

__global__ __launch_bounds__(256) void paged_slots_kernel(PagedPagesArgs a) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i < a.c.total_new) a.slots[i] = slot_of(a.c, seq_of(a.c.cu_new, a.c.n_seqs, i), i);
}

// The pages behind every sequence's new end, as one flat list (sequences in turn, entries
// in turn) whose last page lies where the free ones ended: growing again takes the same
// pages in the same places.
__global__ __launch_bounds__(kThreads) void paged_release_kernel(PagedPagesArgs a) {
  __shared__ int64_t sm_wave[kWaves], sm_before[kThreads];
  __shared__ int32_t sm_kept[kThreads];
  const PagedDev& c = a.c;
  const int32_t n_free = min(max(*a.n_free, 0), c.n_pages);
  // What sequence s keeps of its tokens, its pages then, and those that it gives back.
  auto give = [&](int32_t s, int32_t& len, int32_t& kept) {
    const int32_t now = c.seq_lens[s], full = min(now < 0 ? ~now : now, c.max_len), held = min(max(a.held[s], 0), c.max_pages);
    const int32_t want = a.lens ? a.lens[s] : -1;
    len = want < 0 ? now : min(want, full);
    kept = min(held, pages_of(c, want < 0 ? full : len));
    return held - kept;
  };
  int64_t total = 0;
  {
    int64_t mine = 0;
    int32_t len, kept;
    for (int32_t s = threadIdx.x; s < c.n_seqs; s += kThreads) mine += give(s, len, kept);
    scan(mine, sm_wave, total);
  }
  int64_t carry = 0;
  for (int32_t base = 0; base < c.n_seqs; base += kThreads) {
    const int32_t s = base + int32_t(threadIdx.x);
    int32_t len = 0, kept = 0, count = 0;
    if (s < c.n_seqs) count = give(s, len, kept);
    int64_t all;
    sm_before[threadIdx.x] = scan(count, sm_wave, all);
    sm_kept[threadIdx.x] = kept;
    if (s < c.n_seqs) {
      c.seq_lens[s] = len;
      a.held[s] = kept;
    }
    __syncthreads();
    for (int64_t f = threadIdx.x; f < all; f += kThreads) {
      const int t = owner(sm_before, f);
      int32_t* entry = c.page_table + int64_t(base + t) * c.max_pages + sm_kept[t] + (f - sm_before[t]);
      const int64_t to = n_free + total - 1 - (carry + f);
      if (to < c.n_pages) a.free_pages[to] = *entry;  // (more than there are pages: the list is full)
      *entry = -1;
    }
    carry += all;
    __syncthreads();  // the lists have been read
  }
  if (threadIdx.x == 0) *a.n_free = int32_t(min(n_free + total, int64_t(c.n_pages)));
}

}  // namespace

hipError_t launch_paged_grow(const PagedPagesArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(paged_grow_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  if (a.slots && a.c.total_new > kOwnSlots)
    hipLaunchKernelGGL(paged_slots_kernel, dim3(uint32_t((a.c.total_new + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_paged_release(const PagedPagesArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(paged_release_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace stlite
