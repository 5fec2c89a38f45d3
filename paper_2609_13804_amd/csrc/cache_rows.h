// The rows and runs of a batch over the paged cache, as the kernels of
// cache.hip and attend.hip read them.
#pragma once

#include "sp_internal.h"

namespace sp {
namespace {

// The last i in [0, count) with key(i) <= value, for ascending keys; 0 if none.
// The whole wave searches, 64 places a step: one load for 64 keys, two for 4096.
template <typename Key, typename V>
__device__ __forceinline__ int wave_find_last(int count, V value, Key key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = count;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int64_t at = (int64_t)lane * step;
    const bool below = at < n && key(lo + (int)at) <= value;
    int c = __popcll(__ballot(below));
    if (c < 1) c = 1;
    lo += (c - 1) * step;
    n -= (c - 1) * step;
    if (n > step) n = step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Sequence s's first row.
__device__ __forceinline__ int64_t first_row(const CacheRows& r, int s) {
  return r.padded ? (int64_t)s * r.rows_per_seq : r.info[s];
}

// Sequence s's rows [first, first + n): SP_DEV_OK, or the error of its entries.
__device__ __forceinline__ int rows_of(const CacheRows& r, int s, int64_t& first, int& n) {
  if (r.padded) {
    first = (int64_t)s * r.rows_per_seq;
    n = r.info[s];
  } else {
    const int a = r.info[s], b = r.info[s + 1];
    first = a;
    if (a < 0 || b < a || b > r.rows) return SP_DEV_BAD_OFFSETS;
    n = b - a;
  }
  if (n < 0) return SP_DEV_BAD_OFFSETS;
  return n > r.max_rows ? SP_DEV_GROUP_TOO_LARGE : SP_DEV_OK;
}

// A run's tokens: SP_DEV_OK, or the error of its entry.
__device__ __forceinline__ int tokens_of(const CacheRuns& r, int i, int& len) {
  len = r.len[i];
  return len < 0 ? SP_DEV_BAD_OFFSETS : len > r.max_len ? SP_DEV_GROUP_TOO_LARGE : SP_DEV_OK;
}

}  // namespace
}  // namespace sp
