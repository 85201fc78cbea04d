// Drafted tokens against the target's probabilities (stlite_verify_drafts).
//
// A sequence's run of drafted tokens ends at the first that is not accepted, or behind the
// last.  One row of each side's probabilities decides the next token then, and only that
// row is read whole: of the others the drafted token's entry.
//   weights   w_j = max(p_j - q_j, 0) where a token was refused (all but the token's p_j
//             where the draft's distribution is not given), p_j behind the last one
//   token     the least j with w_0 + .. + w_j > pick (w_0 + .. + w_{V-1})
// Sums are formed in 64 bits: a row has up to 2^24 entries, and where the threshold falls
// between two tokens must not turn on their order.
#include <float.h>

#include "verify.h"

namespace stlite {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <typename T>
struct Probs {
  static constexpr int kPer = 16 / sizeof(T);
  // (rows of any vocabulary: aligned to an entry only)
  typedef T vec __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
};

// What is negative, infinite or NaN counts as 0.
__device__ inline float weight(float x) { return x > 0.0f && x <= FLT_MAX ? x : 0.0f; }

// The row that decides sequence s's next token.
template <typename T>
struct Row {
  const T* p;
  const T* q;     // nullptr: none, or `without` stands for it
  int32_t without;  // the refused token where the draft's distribution is not given, else -1

  __device__ Row(const VerifyArgs& a, int32_t row0, int32_t n, int32_t stop) {
    const int64_t row = int64_t(row0) + stop;
    const bool refused = stop < n - 1;
    p = static_cast<const T*>(a.target) + row * a.target_stride;
    q = refused && a.draft ? static_cast<const T*>(a.draft) + row * a.draft_stride : nullptr;
    without = refused && !a.draft ? a.tokens[row] : -1;
  }
  __device__ static double rest(float p, float q) { return fmax(double(weight(p)) - double(weight(q)), 0.0); }
  __device__ double rest_at(int32_t j) const {
    return q ? rest(float(p[j]), float(q[j])) : j == without ? 0.0 : double(weight(float(p[j])));
  }
};

// The sum of v over the threads before this one, and over all, in the threads' order.
__device__ inline double scan(double v, double (&sm)[kWaves], double& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  __syncthreads();
  if (lane == 63) sm[wave] = sum;
  const double mine = __shfl_up(sum, 1);
  __syncthreads();
  double before = lane ? mine : 0.0;
  all = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sm[w];
    all += sm[w];
  }
  return before;
}

// The first drafted token of the sequence that is not accepted, n - 1 if all are.  The
// comparison is of exact numbers: a product of two 24-bit ones fits in 64 bits.
template <typename T>
__device__ inline int32_t stop_of(const VerifyArgs& a, int32_t row0, int32_t n, int32_t& sm_stop) {
  if (threadIdx.x == 0) sm_stop = n - 1;
  __syncthreads();
  for (int32_t t = threadIdx.x; t < n - 1; t += kThreads) {
    const int64_t row = int64_t(row0) + t;
    const int32_t x = a.tokens[row];
    bool good = false;
    if (x >= 0 && x < a.vocab) {
      const double p = weight(float(static_cast<const T*>(a.target)[row * a.target_stride + x]));
      const double q = a.draft ? weight(float(static_cast<const T*>(a.draft)[row * a.draft_stride + x])) : 1.0f;
      good = double(a.accept[row]) * q < p;
    }
    if (!good) atomicMin(&sm_stop, t);
  }
  __syncthreads();
  return sm_stop;
}

// One chunk of one sequence's deciding row, a piece of it to each wave: the sums of its
// weights and of its p.  HBM-bound: 64 rows of 131072 fp32 of both sides (67 MB) take 10 us,
// 6.5 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sum_kernel(VerifyArgs a) {
  __shared__ int32_t sm_stop;
  const int32_t s = blockIdx.y, row0 = a.cu_new[s], n = a.cu_new[s + 1] - row0;
  if (n <= 0 || (a.seq_lens && a.seq_lens[s] < 0)) return;
  const int32_t stop = stop_of<T>(a, row0, n, sm_stop);
  const Row<T> row(a, row0, n, stop);
  typedef typename Probs<T>::vec vec;
  constexpr int kPer = Probs<T>::kPer;
  const int lane = threadIdx.x & 63;
  const int32_t piece = int32_t(blockIdx.x) * kWaves + int32_t(threadIdx.x >> 6), j0 = piece * a.piece;
  const int32_t j1 = min(j0 + a.piece, a.vocab);
  double rest = 0.0, full = 0.0;
#pragma unroll 4
  for (int32_t j = j0 + lane * kPer; j < j1; j += 64 * kPer) {
    if (j + kPer <= j1) {
      const vec p = *reinterpret_cast<const vec*>(row.p + j);
      vec q = {};
      if (row.q) q = *reinterpret_cast<const vec*>(row.q + j);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float w = weight(float(p[i]));
        full += double(w);
        rest += row.q ? Row<T>::rest(float(p[i]), float(q[i])) : j + i == row.without ? 0.0 : double(w);
      }
    } else {
      for (int32_t i = j; i < j1; ++i) {
        full += double(weight(float(row.p[i])));
        rest += row.rest_at(i);
      }
    }
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    rest += __shfl_xor(rest, d);
    full += __shfl_xor(full, d);
  }
  if (lane == 0) a.sums[int64_t(s) * a.pieces + piece] = make_double2(rest, full);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.stop[s] = stop;
}

// A sequence's next token: the piece that the threshold falls into, and the entry in it.
// Where rounding, or a number that is not below one, leaves no entry behind the threshold,
// the last one with any weight.  Latency-bound: the sums, a scan, a piece's entries, another.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a) {
  constexpr int kEach = kVerifyMaxPiece / kThreads;  // entries of a thread
  __shared__ double sm[2][kWaves], sm_before;
  __shared__ int32_t sm_first[2][kWaves], sm_last[2][kWaves];
  const int32_t s = blockIdx.x, row0 = a.cu_new[s], n = a.cu_new[s + 1] - row0;
  if (n <= 0 || (a.seq_lens && a.seq_lens[s] < 0)) {  // idle
    for (int32_t t = threadIdx.x; t < n; t += kThreads) a.out[int64_t(row0) + t] = -1;
    if (threadIdx.x == 0) a.n_out[s] = 0;
    return;
  }
  const int32_t stop = a.stop[s];
  const Row<T> row(a, row0, n, stop);
  const double2* sums = a.sums + int64_t(s) * a.pieces;
  const int32_t per = (a.pieces + kThreads - 1) / kThreads;
  const int32_t c0 = min(int32_t(threadIdx.x) * per, a.pieces), c1 = min(c0 + per, a.pieces);
  double rest = 0.0, full = 0.0, total;
  for (int32_t i = c0; i < c1; ++i) {
    rest += sums[i].x;
    full += sums[i].y;
  }
  double before = scan(rest, sm[0], total);
  const bool some = total > 0.0;
  if (!some) before = scan(full, sm[1], total);  // nothing is left over: p itself decides
  const double threshold = double(a.pick[s]) * total;
  // One entry (a piece, then a token) of weight w behind `sum`: of this thread's, which lie
  // in order, the first that passes the threshold and the last with any weight.
  int32_t first = INT32_MAX, last = -1;
  auto walk = [&](int32_t at, double w, double& sum) {
    if (!(w > 0.0)) return;
    last = at;
    sum += w;
    if (sum > threshold) first = min(first, at);
  };
  // Of all threads', in their order, the first that passes, else the last; -1: no weight.
  auto found = [&](int k) {
    const uint64_t f = __ballot(first != INT32_MAX), l = __ballot(last >= 0);
    const int32_t lo = __shfl(first, f ? __builtin_ctzll(f) : 0), hi = __shfl(last, l ? 63 - __builtin_clzll(l) : 0);
    if ((threadIdx.x & 63) == 0) {
      sm_first[k][threadIdx.x >> 6] = lo;
      sm_last[k][threadIdx.x >> 6] = hi;
    }
    __syncthreads();
    int32_t at = INT32_MAX, end = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      at = min(at, sm_first[k][w]);
      end = max(end, sm_last[k][w]);
    }
    first = INT32_MAX;
    last = -1;
    return min(at, end);
  };
  double sum = before;
  for (int32_t i = c0; i < c1; ++i) walk(i, some ? sums[i].x : sums[i].y, sum);
  const int32_t piece = found(0);
  int32_t token = -1;
  if (piece >= 0) {
    const int32_t each = a.piece / kThreads, j0 = piece * a.piece + int32_t(threadIdx.x) * each;
    double w[kEach], mine = 0.0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      w[i] = 0.0;
      if (i < each && j0 + i < a.vocab) w[i] = some ? row.rest_at(j0 + i) : double(weight(float(row.p[j0 + i])));
    }
    sum = before;
    for (int32_t i = c0; i < c1 && i <= piece; ++i) {
      if (i == piece) sm_before = sum;
      sum += some ? sums[i].x : sums[i].y;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += w[i];
    sum = scan(mine, sm[0], all) + sm_before;
#pragma unroll
    for (int i = 0; i < kEach; ++i) walk(j0 + i, w[i], sum);
    token = found(1);
  }
  for (int32_t t = threadIdx.x; t < n; t += kThreads)
    a.out[int64_t(row0) + t] = t < stop ? a.tokens[int64_t(row0) + t] : t == stop ? token : -1;
  if (threadIdx.x == 0) {
    a.n_out[s] = stop + 1;
    if (a.seq_lens) a.seq_lens[s] = max(a.seq_lens[s] - (n - 1 - stop), 0);
  }
}

template <typename T>
hipError_t verify(const VerifyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((verify_sum_kernel<T>), dim3(a.pieces / kWaves, a.n_seqs), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((verify_pick_kernel<T>), dim3(a.n_seqs), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, int type, hipStream_t stream) {
  return type == 0 ? verify<__bf16>(a, stream) : type == 1 ? verify<_Float16>(a, stream) : verify<float>(a, stream);
}

}  // namespace stlite
