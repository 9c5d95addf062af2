// units.hpp -- rows read and written 16 bytes a lane, in 32- or 16-bit floats, at any alignment that
// the type itself has (gfx950 loads and stores 16 bytes at an address of any element).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svmx.h"

namespace svmx {

// Values of a unit: 16 bytes of T.
template <class T>
constexpr int UNIT = 16 / sizeof(T);

template <class T, int N>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// N values as they were read (converted where they are used, so that several loads can be under way).
template <int N, class T>
struct Raw {
  static constexpr int M = N < UNIT<T> ? N : UNIT<T>;
  typename VecOf<T, M>::type v[N / M];
  __device__ __forceinline__ float at(int e) const { return (float)v[e / M][e % M]; }
};

template <int N, class T>
__device__ __forceinline__ Raw<N, T> load_whole(const T *__restrict__ p) {
  Raw<N, T> r;
#pragma unroll
  for (int q = 0; q < N / Raw<N, T>::M; ++q)
    r.v[q] = *reinterpret_cast<const typename VecOf<T, Raw<N, T>::M>::type *>(p + q * Raw<N, T>::M);
  return r;
}

// N values that nothing else on this card reads soon: they take no room in the caches.
template <int N, class T>
__device__ __forceinline__ Raw<N, T> load_once(const T *__restrict__ p) {
  Raw<N, T> r;
#pragma unroll
  for (int q = 0; q < N / Raw<N, T>::M; ++q)
    r.v[q] = __builtin_nontemporal_load(reinterpret_cast<const typename VecOf<T, Raw<N, T>::M>::type *>(p + q * Raw<N, T>::M));
  return r;
}

// Of which `left` are in the row; the others come as 0.
template <int N, class T>
__device__ __forceinline__ Raw<N, T> load_raw(const T *__restrict__ p, int64_t left) {
  if (left >= N) return load_whole<N>(p);
  Raw<N, T> r;
#pragma unroll
  for (int e = 0; e < N; ++e) r.v[e / Raw<N, T>::M][e % Raw<N, T>::M] = e < left ? p[e] : (T)0.f;
  return r;
}

// N values at p, of which `left` are in the row; the others come as 0.
template <int N, class T>
__device__ __forceinline__ void load_n(const T *__restrict__ p, int64_t left, float (&v)[N]) {
  if (left >= N) {
    constexpr int M = N < UNIT<T> ? N : UNIT<T>;
#pragma unroll
    for (int q = 0; q < N; q += M) {
      const typename VecOf<T, M>::type u = *reinterpret_cast<const typename VecOf<T, M>::type *>(p + q);
#pragma unroll
      for (int e = 0; e < M; ++e) v[q + e] = (float)u[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < left ? (float)p[e] : 0.f;
  }
}

// One rounding to T, to nearest even.
template <int N, class T>
__device__ __forceinline__ void store_n(T *__restrict__ p, int64_t left, const float (&v)[N]) {
  if (left >= N) {
    constexpr int M = N < UNIT<T> ? N : UNIT<T>;
#pragma unroll
    for (int q = 0; q < N; q += M) {
      typename VecOf<T, M>::type u;
#pragma unroll
      for (int e = 0; e < M; ++e) u[e] = (T)v[q + e];
      *reinterpret_cast<typename VecOf<T, M>::type *>(p + q) = u;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) p[e] = (T)v[e];
  }
}

// N values, all of them in the row, that nothing reads soon.
template <int N, class T>
__device__ __forceinline__ void store_once(T *__restrict__ p, const float (&v)[N]) {
  constexpr int M = N < UNIT<T> ? N : UNIT<T>;
#pragma unroll
  for (int q = 0; q < N; q += M) {
    typename VecOf<T, M>::type u;
#pragma unroll
    for (int e = 0; e < M; ++e) u[e] = (T)v[q + e];
    __builtin_nontemporal_store(u, reinterpret_cast<typename VecOf<T, M>::type *>(p + q));
  }
}

// The same with the type known at run time (uniform over the launch): what a kernel reads once, or
// where it waits for memory anyway.
template <int N>
__device__ __forceinline__ void load_any(const void *p, int32_t type, int64_t at, int64_t left, float (&v)[N]) {
  if (type == SVM_F32)
    load_n<N>(static_cast<const float *>(p) + at, left, v);
  else if (type == SVM_BF16)
    load_n<N>(static_cast<const __bf16 *>(p) + at, left, v);
  else
    load_n<N>(static_cast<const _Float16 *>(p) + at, left, v);
}

template <int N>
__device__ __forceinline__ void store_any(void *p, int32_t type, int64_t at, int64_t left, const float (&v)[N]) {
  if (type == SVM_F32)
    store_n<N>(static_cast<float *>(p) + at, left, v);
  else if (type == SVM_BF16)
    store_n<N>(static_cast<__bf16 *>(p) + at, left, v);
  else
    store_n<N>(static_cast<_Float16 *>(p) + at, left, v);
}

}  // namespace svmx
