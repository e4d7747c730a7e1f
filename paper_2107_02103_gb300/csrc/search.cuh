// Binary search in sorted keys, for kernels and, as plain C++, for tests on the host.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define DP_SEARCH __host__ __device__ __forceinline__
#else
#define DP_SEARCH inline
#endif

namespace dpc {

// The first of n keys (any n that an int holds) that is at least v; key(i) is the i-th.
template <typename Key>
DP_SEARCH int lower_bound(const Key &key, int n, uint32_t v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + ((hi - lo) >> 1);  // lo + hi may pass 2^31
    if (key(mid) < v) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

}  // namespace dpc
