// Sequences of packed rows as a kernel walks them (causal_conv.hip, selective_scan*.hip).
#pragma once
#include "common.h"

namespace {

// Rows are counted in the direction of the walk: row r of it lies at r, or at n - 1 - r when it runs backwards; sequence j of the walk is then the
// caller's sequence n_seq - 1 - j.  Offsets are held within the rows, whatever they say.
struct Walk {
  const int32_t* offsets;
  int32_t n_seq, n, backwards;
  __device__ __forceinline__ Walk(const int32_t* off, int32_t seqs, int32_t capacity, int32_t back) : offsets(off), n_seq(seqs), backwards(back) {
    const int32_t rows = off[seqs];
    n = rows < 0 ? 0 : rows < capacity ? rows : capacity;
  }
  __device__ __forceinline__ int64_t row(int32_t r) const { return backwards ? n - 1 - r : r; }
  __device__ __forceinline__ int32_t number(int32_t j) const { return backwards ? n_seq - 1 - j : j; }
  __device__ __forceinline__ int32_t start(int32_t j) const {   // j in [0, n_seq]
    const int32_t o = offsets[backwards ? n_seq - j : j];
    const int32_t in = o < 0 ? 0 : o < n ? o : n;
    return backwards ? n - in : in;
  }
  // The sequence of row r in [0, n): the last one that starts at r or before it, by the whole wave (r the same in all lanes).
  __device__ __forceinline__ int32_t find(int32_t r, int lane) const {
    int32_t lo = 0, hi = n_seq;          // it is in [lo, hi); every turn leaves at most a 64th of that, rounded up
    while (hi - lo > 64) {
      const int32_t step = (hi - lo + 63) / 64;
      const int64_t at = lo + (int64_t)(lane + 1) * step;
      const int c = __popcll(__ballot(at < hi && start((int32_t)at) <= r));
      lo += c * step;
      hi = hi - lo < step ? hi : lo + step;
    }
    const int32_t at = lo + 1 + lane;
    return lo + __popcll(__ballot(at < hi && start(at) <= r));
  }
  // The same by one lane, which knows that it is in [lo, hi].
  __device__ __forceinline__ int32_t find_between(int32_t r, int32_t lo, int32_t hi) const {
    while (lo < hi) {
      const int32_t mid = lo + (hi - lo + 1) / 2;
      if (start(mid) <= r) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  }
};

// More rows than the buffers hold are left out and reported.
__device__ __forceinline__ void report_rows(const int32_t* offsets, int32_t n_seq, int32_t capacity, int32_t* flags) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && offsets[n_seq] > capacity) atomicOr(flags, EMC2_DEVFLAG_CAPACITY);
}

}  // namespace
