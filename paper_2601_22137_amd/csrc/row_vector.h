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

// Rounded, two at a time where the type has an instruction for it
template <typename T> __device__ inline typename Vec<T>::type rounded(const float (&f)[Vec<T>::N]) {
  typedef float floats __attribute__((ext_vector_type(Vec<T>::N)));
  floats x;
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) x[e] = f[e];
  return __builtin_convertvector(x, typename Vec<T>::type);
}

// Keeps the compiler from holding what was computed from a vector before (its entries in 32 bits, twice the registers) until it is used again
template <typename T> __device__ inline void as_loaded(typename Vec<T>::type& v) {
  typedef unsigned words __attribute__((ext_vector_type(4)));
  words w = __builtin_bit_cast(words, v);
  asm("" : "+v"(w));
  v = __builtin_bit_cast(typename Vec<T>::type, w);
}

// Entries at .. at + N - 1 of a row of `width`; those past its end are `rest`.  PAST: past the caches, for arrays that are gone through once.
template <typename T, bool PAST = false> __device__ inline typename Vec<T>::type load_vector(const T* row, int at, int width, float rest = 0.0f) {
  using V = typename Vec<T>::type;
  constexpr int N = Vec<T>::N;
  auto load = [](const T* p) { return PAST ? __builtin_nontemporal_load((const V*)p) : *(const V*)p; };
  if (at + N <= width) return load(row + at);
  V v;
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = (T)rest;
  if (at >= width) return v;
  if (width >= N) {            // the row's last vector, moved to its place
    const int bits = (at + N - width) * (128 / N);
    const unsigned __int128 x = __builtin_bit_cast(unsigned __int128, load(row + width - N)), r = __builtin_bit_cast(unsigned __int128, v);
    return __builtin_bit_cast(V, (x >> bits) | (r << (128 - bits)));
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (at + e < width) v[e] = row[at + e];
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

// ... past the caches
template <typename T> __device__ inline void stream_vector_to(T* row, int at, int width, const typename Vec<T>::type& v) {
  if (at + Vec<T>::N <= width) __builtin_nontemporal_store(v, (typename Vec<T>::type*)(row + at));
  else store_vector(row, at, width, v);
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
