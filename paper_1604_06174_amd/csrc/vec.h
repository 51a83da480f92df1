// Vectors of V consecutive elements of a bf16 or fp32 tensor, as one load or
// store (two for eight fp32), for kernels templated on the element type.  They
// may lie at any element: global accesses need no wider alignment here, so a row
// of odd pitch or a slice that starts anywhere takes them too.
#pragma once

#include <hip/hip_runtime.h>

namespace ckpt {

template <typename T, int V>
struct Vec;
template <>
struct Vec<__bf16, 8> {
  typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2)));
  type v;
};
template <>
struct Vec<float, 8> {
  typedef float type __attribute__((ext_vector_type(8), aligned(4)));
  type v;
};
template <>
struct Vec<__bf16, 1> {
  typedef __bf16 type __attribute__((ext_vector_type(1)));
  type v;
};
template <>
struct Vec<float, 1> {
  typedef float type __attribute__((ext_vector_type(1)));
  type v;
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p) {
  Vec<T, V> r;
  r.v = *reinterpret_cast<const typename Vec<T, V>::type *>(p);
  return r;
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float v[V]) {
  typename Vec<T, V>::type r;
#pragma unroll
  for (int k = 0; k < V; ++k) r[k] = (T)v[k];
  *reinterpret_cast<typename Vec<T, V>::type *>(p) = r;
}

}  // namespace ckpt
