// What the attention kernels share: which rows a sequence has, and where a cache keeps a token.
#pragma once
#include <cuda_runtime.h>

#include "../../include/dragon.h"

namespace dragon {

// The rows of `count` sequences: equal parts of the rows, or starts[s] .. starts[s + 1] - 1 (device, may be null).  Starts that
// are out of order or range are cut to it, so that no row number leaves the tensors.
struct Sequences {
  const int* starts;
  int count, rows, each;      // each: rows of every sequence where starts is null
  __device__ __forceinline__ void rows_of(int s, int* a, int* b) const {
    if (!starts) { *a = s * each; *b = *a + each; return; }
    *a = min(max(__ldg(starts + s), 0), rows);
    *b = min(max(__ldg(starts + s + 1), *a), rows);
  }
  // the sequence that row r lies in, -1 for a row of none
  __device__ __forceinline__ int of_row(int r) const {
    if (!starts) return r / each;
    int lo = 0, hi = count;             // the last s with starts[s] <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(starts + mid) <= r) lo = mid; else hi = mid;
    }
    int a, b;
    rows_of(lo, &a, &b);
    return r >= a && r < b ? lo : -1;
  }
  // whether starts[t], t = threadIdx.x + k * blockDim.x, are in range and in order; for one CTA, which reports
  __device__ __forceinline__ bool in_order() const {
    bool ok = true;
    for (int s = threadIdx.x; starts && s < count; s += blockDim.x) {
      const int a = __ldg(starts + s), b = __ldg(starts + s + 1);
      ok &= a >= 0 && b >= a && b <= rows;
    }
    return ok;
  }
};

constexpr int kMostTokens = 0x7fffff00;      // of a sequence: positions, and the end of their last tile, stay within 32 bits

// The pages of a cache: token p of sequence s is row pages[s][p / page] * page + p % page
struct Pages {
  const int* pages;           // [sequences][most]
  const int* lengths;         // tokens of every sequence
  int most, shift, pool;      // page = 1 << shift rows; pool: pages there are
  // tokens that the table has room for (and positions in 32 bits), of those that sequence s says it has
  __device__ __forceinline__ int tokens(int s, bool* fits) const {
    const int n = max(__ldg(lengths + s), 0);
    const long long room = min((long long)most << shift, (long long)kMostTokens);
    *fits = n <= room;
    return (int)min((long long)n, room);
  }
  __device__ __forceinline__ int page_of(int s, int p) const { return __ldg(pages + (size_t)s * most + (p >> shift)); }
  __device__ __forceinline__ bool in_pool(int page) const { return page >= 0 && page < pool; }
};

// whether a sequence of n new rows has at most `few` of them times the heads of a group (the product itself may pass 32 bits)
__device__ __forceinline__ bool has_few_rows(int n, int group, int few) { return (long long)n * group <= few; }

__device__ __forceinline__ void report(int* status, int code) { atomicExch(status, code); }

}  // namespace dragon
