// Rows of f64, f32, bf16 or f16 for the expert-block operators (routing, 8-bit product, norms): what an
// element accumulates in, packs of 1 to 16 bytes, and the pack width a set of arrays allows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>
#include <type_traits>

#include "dp_common.cuh"

namespace dpc {
namespace {

// Sums of 16-bit and f32 elements are held in f32, those of f64 in f64; weights have the sums' type.
template <typename T>
struct Acc {
  using type = float;
};
template <>
struct Acc<double> {
  using type = double;
};
template <typename T>
using acc_t = typename Acc<T>::type;

__device__ __forceinline__ double to_acc(double x) { return x; }
__device__ __forceinline__ float to_acc(float x) { return x; }
__device__ __forceinline__ float to_acc(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_acc(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_acc(acc_t<T> x) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
  } else {
    return x;
  }
}

// V elements moved by one load or store (V sizeof(T) = 1 .. 16 bytes, the address a multiple of that).
template <typename T, int V>
struct alignas(V * sizeof(T)) Pack {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
  return *reinterpret_cast<const Pack<T, V> *>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &x) {
  *reinterpret_cast<Pack<T, V> *>(p) = x;
}

// The 16 bytes at p, whatever its alignment to them (p aligned to its elements), from the two aligned words that
// hold them; near the ends lo, hi of its array, or past them (then zero), element by element.  A row of odd length
// costs two loads for 16 bytes this way, the second from L1, against a load for each element.
template <typename T>
__device__ __forceinline__ Pack<T, 16 / (int)sizeof(T)> load_any(const T *p, const T *lo, const T *hi) {
  constexpr int V = 16 / (int)sizeof(T);
  const uint32_t off = (uint32_t)((uintptr_t)p & 15);
  const char *a = reinterpret_cast<const char *>(p) - off;
  Pack<T, V> out;
  if (off == 0 && p >= lo && p + V <= hi) return load_pack<T, V>(p);
  if (a >= reinterpret_cast<const char *>(lo) && a + 32 <= reinterpret_cast<const char *>(hi)) {
    const uint4 x = __ldg(reinterpret_cast<const uint4 *>(a)), y = __ldg(reinterpret_cast<const uint4 *>(a) + 1);
    const uint32_t sh = (off & 3) * 8;
    uint4 r;
    switch (off >> 2) {  // the same for a whole row
      case 0:
        r = make_uint4(__funnelshift_r(x.x, x.y, sh), __funnelshift_r(x.y, x.z, sh), __funnelshift_r(x.z, x.w, sh),
                       __funnelshift_r(x.w, y.x, sh));
        break;
      case 1:
        r = make_uint4(__funnelshift_r(x.y, x.z, sh), __funnelshift_r(x.z, x.w, sh), __funnelshift_r(x.w, y.x, sh),
                       __funnelshift_r(y.x, y.y, sh));
        break;
      case 2:
        r = make_uint4(__funnelshift_r(x.z, x.w, sh), __funnelshift_r(x.w, y.x, sh), __funnelshift_r(y.x, y.y, sh),
                       __funnelshift_r(y.y, y.z, sh));
        break;
      default:
        r = make_uint4(__funnelshift_r(x.w, y.x, sh), __funnelshift_r(y.x, y.y, sh), __funnelshift_r(y.y, y.z, sh),
                       __funnelshift_r(y.z, y.w, sh));
    }
    memcpy(&out, &r, 16);
  } else {
    T zero;
    memset(&zero, 0, sizeof zero);
#pragma unroll
    for (int l = 0; l < V; ++l) out.v[l] = p + l >= lo && p + l < hi ? p[l] : zero;
  }
  return out;
}

// Waits on an mbarrier give up after kPolls tries or when `stop`, looked at now and then, says so.  A block whose
// wait gave up waits once more for its own copies in flight, leaves NaN and adds one to g_wait_timeouts.
constexpr int kWaitPolls = 1 << 18;  // a try takes up to 4.5 us: about a second
__device__ unsigned int g_wait_timeouts;  // of this translation unit's kernels

template <int kPolls = kWaitPolls, typename Stop>
__device__ __forceinline__ bool bounded_wait(uint32_t bar, uint32_t parity, Stop stop) {
  uint32_t done = 0;
  for (int it = 0; it < kPolls && !done; ++it) {
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done)
                 : "r"(bar), "r"(parity)
                 : "memory");
    if (!done && (it & 63) == 63 && stop()) return false;
  }
  return done != 0;
}

// The count, read after a device synchronisation, then cleared.
[[maybe_unused]] int take_unit_timeouts(unsigned int *count) {
  unsigned int v = 0, zero = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&v, g_wait_timeouts, sizeof v);
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_wait_timeouts, &zero, sizeof zero);
  if (e != cudaSuccess) return set_error(DP_ERR_CUDA, "dp_tc_wait_timeouts: %s", cudaGetErrorString(e));
  *count += v;
  return DP_OK;
}

// Whether every array begins at a multiple of its element's size (NULL does).
template <typename... E>
bool at_elements(const E *...p) {
  return (... && !((uintptr_t)p & (sizeof(E) - 1)));
}
[[maybe_unused]] int misaligned(const char *who) {
  return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
}

// The widest pack (in elements) that rows of H elements at these addresses allow: 16 bytes down to one element.
template <typename T, typename... P>
int pack_width(int64_t H, P... ptrs) {
  uintptr_t bits = 16 | (uintptr_t)(H * (int64_t)sizeof(T));
  const uintptr_t all[] = {(uintptr_t)ptrs...};
  for (uintptr_t p : all) bits |= p;
  const uintptr_t bytes = bits & (~bits + 1);  // the lowest set bit
  return bytes < sizeof(T) ? 0 : (int)(bytes / sizeof(T));  // 0: not even aligned to an element
}

}  // namespace
}  // namespace dpc
