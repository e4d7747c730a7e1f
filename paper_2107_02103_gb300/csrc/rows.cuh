// Rows of f64, f32, bf16 or f16 for the expert-block operators (routing, 8-bit product, norms): what an
// element accumulates in, packs of 1 to 16 bytes, and the pack width a set of arrays allows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

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
