// Norm of rows of the residual stream, with the sum that makes them (layer_norm_rows.h has the formulas).  The variance is taken from the differences to the mean, sums are in 32 bits.
#include "layer_norm_rows.h"

namespace prism {
namespace {

template <typename T, int THREADS, int NV, int MODE, bool RES>
__global__ void __launch_bounds__(threads_of(THREADS)) layer_norm_kernel(LayerNorm p) {
  using R = Row<T, THREADS, NV, MODE>;
  using V = typename Vec<T>::type;
  using C = Columns<T, THREADS, NV, MODE>;
  constexpr int N = R::N, PER = threads_of(THREADS) / THREADS;
  __shared__ float memory[THREADS > 64 ? THREADS / 32 : 1], columns[2][C::FLOATS];
  const C w(p.w, p.width, 1.0f, columns[0]), b(p.b, p.width, 0.0f, columns[1]);
  int turn = 0;
  for (long long first = (long long)blockIdx.x * PER; first < p.rows; first += (long long)gridDim.x * PER) {
    const long long row = first + threadIdx.x / THREADS;
    const bool there = row < p.rows;
    const int width = there ? p.width : 0;
    const T* x = (const T*)p.x + (there ? row : 0) * p.xs;
    V v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = R::load(x, j, width);
    if constexpr (RES) {
      const T* res = (const T*)p.residual + (there ? row : 0) * p.rs;
      T* total = (T*)p.total + (there ? row : 0) * p.ts;
      V r[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) r[j] = R::load(res, j, width);
      R::settle(v, width);
      R::settle(r, width);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float o[N];
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = (float)v[j][e] + (float)r[j][e];
        v[j] = rounded<T>(o);
        R::store(total, j, width, v[j]);
      }
    } else {
      R::settle(v, width);
    }
    float mean = 0.0f;
    if (p.center) {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) sum += (float)v[j][e];
      mean = row_sum<THREADS>(sum, memory, turn++) / (float)p.width;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) as_loaded<T>(v[j]);
    float square = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = R::inside(j, e, width) ? (float)v[j][e] - mean : 0.0f;
        square += d * d;
      }
    const float r = 1.0f / sqrtf(row_sum<THREADS>(square, memory, turn++) / (float)p.width + p.eps);
    if (there && p.stats && threadIdx.x % THREADS == 0) p.stats[row] = make_float2(mean, r);
#pragma unroll
    for (int j = 0; j < NV; ++j) as_loaded<T>(v[j]);
    T* y = (T*)p.y + (there ? row : 0) * p.ys;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = ((float)v[j][e] - mean) * r * w.get(j, e) + b.get(j, e);
      R::store(y, j, width, rounded<T>(o));
    }
  }
}

template <typename T, int THREADS, int NV, int MODE> struct Forward {
  static void launch(const LayerNorm& p, int blocks, hipStream_t s) {
    hipLaunchKernelGGL((p.residual ? layer_norm_kernel<T, THREADS, NV, MODE, true> : layer_norm_kernel<T, THREADS, NV, MODE, false>), dim3(blocks), dim3(threads_of(THREADS)), 0, s, p);
  }
};

}  // namespace

int launch_layer_norm(const void* x, const void* residual, const float* weight, const float* bias, void* y, void* total, float* stats, int dt,
                      const prism_layer_norm_desc& d, hipStream_t s) {
  ProfScope prof(PK_LAYER_NORM, s);
  LayerNorm p = layer_norm_common(d);
  p.x = x; p.xs = d.x; p.residual = residual; p.rs = d.residual; p.total = total; p.ts = d.total; p.y = y; p.ys = d.y;
  p.w = weight; p.b = bias; p.stats = (float2*)stats;
  const Shape h = shape_of(d.width, dt, d.rows, residual ? 4 : 2);
  by_type<Forward>(dt, h, p, blocks_of(d.rows, h, 2048), s);
  return PRISM_OK;
}

}  // namespace prism
