// Dropout whose mask is a function of (seed, offset, element) and is never stored: y = residual + x [u >= limit] / keep, with the
// gradient the same call on dy.  u is a half word of Philox4x32-10 with key = seed and counter = (group of eight elements in two
// words, offset, tag): one generator call gives the numbers of eight elements, the 16 bits make a probability exact to 2^-17.
//
// Bound by memory: a thread takes eight elements, 16 bytes of bf16 at a time; the generator's ten rounds run beside the loads.  65536 x 768 bf16 with a
// residual: 55 us, 5.5 TB/s read and written, the rate of a large copy; 12345677 elements of fp32: 16 us.  256 to 8192 workgroups of 256; a call of 257 x 768 takes
// 2.4 us on the card and 7 with its launch.  One rounding, of the sum with the residual.
#include "layer.h"
#include "philox.h"

namespace prism {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr unsigned DROPOUT_TAG = 7;   // fourth counter word; the sketches have the function ids 1 .. 6 there

template <typename T> struct Eight;   // eight consecutive elements as 16-byte words
template <> struct Eight<float> {
  f32x4 a, b;
  __device__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ void set(int i, float v) { if (i < 4) a[i] = v; else b[i - 4] = v; }
};
template <> struct Eight<__bf16> {
  bf16x8 a;
  __device__ float get(int i) const { return (float)a[i]; }
  __device__ void set(int i, float v) { a[i] = (__bf16)v; }
};

template <typename T>
__device__ inline Eight<T> load8(const T* p, int count, bool whole) {
  if (whole) return *reinterpret_cast<const Eight<T>*>(p);
  Eight<T> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.set(i, i < count ? (float)p[i] : 0.0f);
  return r;
}

template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, const T* residual, T* y, long long n, unsigned limit, float scale, unsigned k0,
                                                      unsigned k1, unsigned offset, bool aligned) {
  const long long groups = (n + 7) >> 3;
  for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; g < groups; g += (long long)gridDim.x * 256) {
    const long long e0 = g << 3;
    const int count = (int)(n - e0 < 8 ? n - e0 : 8);
    const bool whole = aligned && count == 8;
    const Eight<T> xv = load8(x + e0, count, whole);
    Eight<T> rv;
    if constexpr (RES) rv = load8(residual + e0, count, whole);
    U4 c;
    c.x = (unsigned)g; c.y = (unsigned)(g >> 32); c.z = offset; c.w = DROPOUT_TAG;
    const U4 w = philox4x32_10(c, k0, k1);
    Eight<T> out;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned word = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
      const unsigned u = (i & 1) ? word >> 16 : word & 0xFFFFu;
      const float v = u >= limit ? xv.get(i) * scale : 0.0f;   // selected, not multiplied: a dropped infinity is 0
      out.set(i, RES ? v + rv.get(i) : v);
    }
    if (whole) *reinterpret_cast<Eight<T>*>(y + e0) = out;
    else
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) y[e0 + i] = (T)out.get(i);
  }
}

template <typename T>
void launch(const void* x, const void* residual, void* y, long long n, unsigned limit, uint64_t seed, uint32_t offset, hipStream_t s) {
  const long long groups = (n + 7) >> 3, blocks = (groups + 255) / 256;
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
  const float scale = 65536.0f / (float)(65536u - limit);
  const bool aligned = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & 15) == 0;
  const unsigned k0 = (unsigned)(seed & 0xFFFFFFFFull), k1 = (unsigned)(seed >> 32);
  if (residual)
    hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, s, (const T*)x, (const T*)residual, (T*)y, n, limit, scale, k0, k1, offset, aligned);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, s, (const T*)x, (const T*)nullptr, (T*)y, n, limit, scale, k0, k1, offset, aligned);
}

}  // namespace

int launch_dropout(const void* x, const void* residual, void* y, long long n, int dt, unsigned limit, uint64_t seed, uint32_t offset, hipStream_t s) {
  ProfScope prof(PK_DROPOUT, s);
  if (dt == PRISM_F32) launch<float>(x, residual, y, n, limit, seed, offset, s);
  else launch<__bf16>(x, residual, y, n, limit, seed, offset, s);
  return PRISM_OK;
}

}  // namespace prism
