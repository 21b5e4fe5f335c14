// Rows of arrays in vectors of 16 bytes, and sums over the threads that share a row.
#pragma once
#include "common.h"

namespace prism {

// N consecutive entries.  Aligned as one entry is: the card's 16-byte loads and stores of global memory need no more, so rows of any width, stride and
// start go the same way.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  typedef float type __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Vec<__bf16> {
  static constexpr int N = 8;
  typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2)));
};

// Entries at .. at + N - 1 of a row of `width`; those past its end are `rest`
template <typename T> __device__ inline typename Vec<T>::type load_vector(const T* row, int at, int width, float rest = 0.0f) {
  typename Vec<T>::type v;
  if (at + Vec<T>::N <= width) return *(const typename Vec<T>::type*)(row + at);
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) v[e] = at + e < width ? row[at + e] : (T)rest;
  return v;
}
template <typename T> __device__ inline void store_vector(T* row, int at, int width, const typename Vec<T>::type& v) {
  if (at + Vec<T>::N <= width) {
    *(typename Vec<T>::type*)(row + at) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e)
    if (at + e < width) row[at + e] = v[e];
}

// Sum over the THREADS (a power of two) neighbours that share a row, the same value in each; more than 64 are the whole workgroup and use one of the
// two halves of `memory` (THREADS / 32 floats), by turns, so that one barrier a sum is enough.
template <int THREADS> __device__ inline float row_sum(float v, float* memory, int turn) {
#pragma unroll
  for (int d = 1; d < (THREADS < 64 ? THREADS : 64); d *= 2) v += __shfl_xor(v, d);
  if constexpr (THREADS > 64) {
    float* part = memory + (turn & 1) * (THREADS / 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) v += part[i];
  }
  return v;
}

}  // namespace prism
