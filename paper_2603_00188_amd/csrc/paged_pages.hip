// Pages for growing sequences (stlite_paged_grow) and back (stlite_paged_release): page
// table, lengths and places of the next new tokens, out of a list of free pages.
#include "paged.h"

namespace stlite {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

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

// The thread whose entries entry f of the chunk's flat list is among: the last one with
// before[t] <= f (one without entries has the next one's).
template <typename I>
__device__ inline int owner(const I (&before)[kThreads], I f) {
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

// One work-group, since every sequence's pages lie behind those of the sequences before
// it: a scan of what 1024 sequences at a time need, then their pages as one flat list and
// their new tokens as another, a thread each.  With many of those, kLists writes them by
// many work-groups, each with the scan of its own, and a second launch of one, kState, what
// the scans read.  Latency-bound: three loads, a scan, a load and a store one after another.
enum { kAll, kLists, kState };
template <int PART>
__global__ __launch_bounds__(kThreads) void paged_grow_kernel(PagedPagesArgs a) {
  __shared__ int64_t sm_wave[kWaves], sm_before[kThreads];
  __shared__ int32_t sm_held[kThreads], sm_len[kThreads], sm_cu[kThreads];
  const PagedDev& c = a.c;
  const int64_t first = int64_t(blockIdx.x) * kThreads + threadIdx.x, stride = int64_t(gridDim.x) * kThreads;
  const int32_t n_free = min(max(*a.n_free, 0), c.n_pages);
  int64_t carry = 0;  // pages that the sequences before this chunk need
  int64_t taken = 0;  // pages given out
  for (int32_t base = 0; base < c.n_seqs; base += kThreads) {
    const int32_t s = base + int32_t(threadIdx.x);
    int32_t len = 0, held = 0, cu = INT32_MAX;
    int64_t grown = 0, need = 0;
    bool fits = false;
    if (s < c.n_seqs) {
      const int32_t now = c.seq_lens[s];
      cu = c.cu_new[s];
      held = min(max(a.held[s], 0), c.max_pages);
      len = now < 0 ? now : min(now, c.max_len);
      grown = int64_t(len) + (c.cu_new[s + 1] - cu);
      fits = len >= 0 && grown <= c.max_len;
      if (fits) need = max(pages_of(c, grown) - held, 0);
    }
    int64_t all;
    const int64_t before = scan(need, sm_wave, all);
    const bool granted = fits && (need == 0 || carry + before + need <= n_free);
    if (PART != kLists && s < c.n_seqs) {
      c.seq_lens[s] = granted ? int32_t(grown) : len < 0 ? len : ~len;
      if (granted) a.held[s] = held + int32_t(need);
      else if (len == 0 && held > 0 && held < c.max_pages) a.page_table[int64_t(s) * c.max_pages + held] = kPagesEnd;
    }
    int64_t here;  // what this chunk takes: the needs of a first part of its sequences
    scan(granted ? need : 0, sm_wave, here);
    if (PART != kState) {
      sm_before[threadIdx.x] = before;
      sm_held[threadIdx.x] = held;
      sm_len[threadIdx.x] = granted ? len : -1;
      sm_cu[threadIdx.x] = cu;
      __syncthreads();
      for (int64_t f = first; f < here; f += stride) {
        const int t = owner(sm_before, f);
        a.page_table[int64_t(base + t) * c.max_pages + sm_held[t] + (f - sm_before[t])] = a.free_pages[n_free - 1 - (carry + f)];
      }
      if (a.slots) {
        const int32_t end = c.cu_new[min(base + kThreads, c.n_seqs)];
        for (int64_t i = sm_cu[0] + first; i < end; i += stride) {
          const int t = owner(sm_cu, int32_t(i));
          const int64_t at = int64_t(sm_len[t]) + (i - sm_cu[t]);
          const int32_t entry = int32_t(at >> c.page_shift), more = entry - sm_held[t];
          int32_t page = -1;
          if (sm_len[t] >= 0)
            page = more < 0 ? a.page_table[int64_t(base + t) * c.max_pages + entry]
                            : a.free_pages[n_free - 1 - (carry + sm_before[t] + more)];
          a.slots[i] = page >= 0 && page < c.n_pages ? (page << c.page_shift) + int32_t(at & ((1 << c.page_shift) - 1)) : -1;
        }
      }
      __syncthreads();  // the lists have been read
    }
    carry += all;
    taken += here;
  }
  if (PART != kLists) {
    __syncthreads();
    if (threadIdx.x == 0) *a.n_free = n_free - int32_t(taken);
  }
}

// The pages behind every sequence's new end, as one flat list (sequences in turn, entries
// in turn) whose last page lies where the free ones ended: growing again takes the same
// pages in the same places.  One work-group, or as growing where there may be many pages.
template <int PART>
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
    if (PART != kLists && s < c.n_seqs) {
      c.seq_lens[s] = len;
      a.held[s] = kept;
    }
    if (PART == kState) continue;
    int64_t all;
    sm_before[threadIdx.x] = scan(count, sm_wave, all);
    sm_kept[threadIdx.x] = kept;
    __syncthreads();
    for (int64_t f = int64_t(blockIdx.x) * kThreads + threadIdx.x; f < all; f += int64_t(gridDim.x) * kThreads) {
      const int t = owner(sm_before, f);
      int32_t* entry = a.page_table + int64_t(base + t) * c.max_pages + sm_kept[t] + (f - sm_before[t]);
      const int64_t to = n_free + total - 1 - (carry + f);
      if (to < c.n_pages) a.free_pages[to] = *entry;  // (more than there are pages: the list is full)
      *entry = -1;
    }
    carry += all;
    __syncthreads();  // the lists have been read
  }
  if (PART != kLists && threadIdx.x == 0) *a.n_free = int32_t(min(n_free + total, int64_t(c.n_pages)));
}

}  // namespace

hipError_t launch_paged_grow(const PagedPagesArgs& a, hipStream_t stream) {
  // 1000 sequences of up to 2999 new tokens (90000 pages, 1.5 million places) take 19 us by
  // 256 work-groups and a second launch (14 and 6), 61 by one and a launch for the places;
  // 64 of one token 6 us by one.
  if (a.c.total_new <= 4096) {
    hipLaunchKernelGGL((paged_grow_kernel<kAll>), dim3(1), dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((paged_grow_kernel<kLists>), dim3(256), dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_grow_kernel<kState>), dim3(1), dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_paged_release(const PagedPagesArgs& a, hipStream_t stream) {
  // How many there are, the host does not know, only that a small pool has not many: 90000
  // pages of 1000 sequences take 54 us by one work-group, 10 by 256 and a second launch (7
  // and 3); a page or two of 64 sequences 4.5 by one.
  if (a.c.n_pages <= 65536) {
    hipLaunchKernelGGL((paged_release_kernel<kAll>), dim3(1), dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((paged_release_kernel<kLists>), dim3(256), dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_release_kernel<kState>), dim3(1), dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace stlite
