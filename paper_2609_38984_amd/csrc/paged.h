// The sequence that a row of a chunk belongs to, for the kernels that write and read a
// paged cache.
#pragma once
#include "launchers.h"

namespace swam {

typedef __attribute__((address_space(4))) const int32_t const_i32;

// the rows [a, e) of sequence s, clamped to [0, n)
__device__ __forceinline__ void chunk_of(const Paged& p, int s, int n, int& a, int& e) {
  e = p.cu ? min(max(p.cu[s + 1], 0), n) : n;
  a = p.cu ? min(max(p.cu[s], 0), e) : 0;
}

// tokens that sequence s holds before the chunk
__device__ __forceinline__ int held(const Paged& p, int s) {
  return min(max(p.length[s], 0), p.max_pages << p.lg_page);
}

// The first sequence that ends behind row r (n_seqs - 1 at most), which is the one that holds r, if one does, unless
// offsets fall: two rounds of 64 probes find it among 1,024 sequences in two latencies.
__device__ __forceinline__ int seq_of(const Paged& p, int64_t r) {
  if (p.cu == nullptr || p.n_seqs == 1) return 0;
  const int lane = threadIdx.x & 63, step = (p.n_seqs + 63) >> 6;
  int at = 0;
  if (step > 1) {
    const uint64_t past = __ballot(p.cu[min((lane + 1) * step, p.n_seqs)] > r);
    at = past ? (__ffsll((unsigned long long)past) - 1) * step : 63 * step;
  }
  const uint64_t past = __ballot(lane < step || step == 1 ? p.cu[min(at + lane + 1, p.n_seqs)] > r : false);
  at += past ? __ffsll((unsigned long long)past) - 1 : 0;
  return __builtin_amdgcn_readfirstlane(min(at, p.n_seqs - 1));
}

// The sequence that holds row r, or -1: a look at all, for where the one above does not.
__device__ __forceinline__ int seq_that_holds(const Paged& p, int64_t r) {
  const int lane = threadIdx.x & 63;
  if (p.cu == nullptr) return -1;
#pragma unroll 1
  for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
    const int s = min(s0 + lane, p.n_seqs - 1);
    const uint64_t holds = __ballot(p.cu[s] <= r && r < p.cu[s + 1]);
    if (holds) return __builtin_amdgcn_readfirstlane(s0 + __ffsll((unsigned long long)holds) - 1);
  }
  return -1;
}

}  // namespace swam
