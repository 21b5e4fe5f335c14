// Norm of rows of the residual stream, with the sum that makes them, and its gradients.
//
//   h = x + residual, mean = sum h / width (0 where it is not taken off), r = (mean (h - mean)^2 + eps)^(-1/2), y = (h - mean) r w + b
//   g = dy w, n = (h - mean) r:  dx = r (g - mean g - n mean (g n)) + dtotal (without mean g where the mean is not taken off), dw = sum dy n, db = sum dy
//
// THREADS threads share a row and keep it in registers, NV vectors of 16 bytes each: one pass over memory, the variance from the differences to the mean.  Sums are in 32
// bits.  Statistics are of h as it is stored (rounded), so the gradients meet the same numbers.
#include "layer.h"
#include "row_vector.h"

namespace prism {
namespace {

struct LayerNorm {
  const void *x, *residual, *dy, *dtotal;
  void *total, *y;                       // backward: y is dx, x the sum
  const float *w, *b;
  float2* stats;
  float* part;                           // backward: [workgroup][dw, db][width]
  long long xs, rs, ds, gs, ts, ys, rows;
  int width;
  float eps;
  bool center, bias;
};

constexpr int threads_of(int THREADS) { return THREADS < 256 ? 256 : THREADS; }

template <typename T, int THREADS, int NV> struct Row {
  static constexpr int N = Vec<T>::N;
  // lane l of the row has vectors l, l + THREADS, ...
  static __device__ int at(int j) { return ((int)(threadIdx.x % THREADS) + j * THREADS) * N; }
  static __device__ void weights(const float* w, int width, float none, float (&to)[NV * N]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) to[j * N + e] = w && at(j) + e < width ? w[at(j) + e] : none;
  }
};

template <typename T, int THREADS, int NV, bool RES>
__global__ void __launch_bounds__(threads_of(THREADS)) layer_norm_kernel(LayerNorm p) {
  using R = Row<T, THREADS, NV>;
  using V = typename Vec<T>::type;
  constexpr int N = R::N, PER = threads_of(THREADS) / THREADS;
  __shared__ float memory[THREADS > 64 ? THREADS / 32 : 1];
  float w[NV * N], b[NV * N];
  R::weights(p.w, p.width, 1.0f, w);
  R::weights(p.b, p.width, 0.0f, b);
  int turn = 0;
  for (long long first = (long long)blockIdx.x * PER; first < p.rows; first += (long long)gridDim.x * PER) {
    const long long row = first + threadIdx.x / THREADS;
    const bool there = row < p.rows;
    const int width = there ? p.width : 0;
    const T* x = (const T*)p.x + (there ? row : 0) * p.xs;
    V v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vector(x, R::at(j), width);
    if constexpr (RES) {
      const T* res = (const T*)p.residual + (there ? row : 0) * p.rs;
      T* total = (T*)p.total + (there ? row : 0) * p.ts;
      V r[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) r[j] = load_vector(res, R::at(j), width);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[j][e] = (T)((float)v[j][e] + (float)r[j][e]);
        store_vector(total, R::at(j), width, v[j]);
      }
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
    float square = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = R::at(j) + e < width ? (float)v[j][e] - mean : 0.0f;
        square += d * d;
      }
    const float r = 1.0f / sqrtf(row_sum<THREADS>(square, memory, turn++) / (float)p.width + p.eps);
    if (there && p.stats && threadIdx.x % THREADS == 0) p.stats[row] = make_float2(mean, r);
    T* y = (T*)p.y + (there ? row : 0) * p.ys;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      V o;
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = (T)(((float)v[j][e] - mean) * r * w[j * N + e] + b[j * N + e]);
      store_vector(y, R::at(j), width, o);
    }
  }
}

template <typename T, int THREADS, int NV, bool TOTAL>
__global__ void __launch_bounds__(threads_of(THREADS)) layer_norm_backward_kernel(LayerNorm p) {
  using R = Row<T, THREADS, NV>;
  using V = typename Vec<T>::type;
  constexpr int N = R::N, PER = threads_of(THREADS) / THREADS;
  __shared__ float memory[THREADS > 64 ? THREADS / 32 : 1];
  float w[NV * N], dw[NV * N] = {}, db[NV * N] = {};
  R::weights(p.w, p.width, 1.0f, w);
  int turn = 0;
  for (long long first = (long long)blockIdx.x * PER; first < p.rows; first += (long long)gridDim.x * PER) {
    const long long row = first + threadIdx.x / THREADS;
    const bool there = row < p.rows;
    const int width = there ? p.width : 0;
    const long long at = there ? row : 0;
    V h[NV], d[NV], t[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) d[j] = load_vector((const T*)p.dy + at * p.ds, R::at(j), width);
#pragma unroll
    for (int j = 0; j < NV; ++j) h[j] = load_vector((const T*)p.x + at * p.xs, R::at(j), width);
    if constexpr (TOTAL) {
#pragma unroll
      for (int j = 0; j < NV; ++j) t[j] = load_vector((const T*)p.dtotal + at * p.gs, R::at(j), width);
    }
    const float2 stats = p.stats[at];
    float sum = 0.0f, product = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float dy = (float)d[j][e], n = ((float)h[j][e] - stats.x) * stats.y, g = dy * w[j * N + e];
        sum += g;
        product += g * n;
        dw[j * N + e] += dy * n;
        db[j * N + e] += dy;
      }
    product = row_sum<THREADS>(product, memory, turn++) / (float)p.width;
    sum = p.center ? row_sum<THREADS>(sum, memory, turn++) / (float)p.width : 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      V o;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float n = ((float)h[j][e] - stats.x) * stats.y;
        float dx = stats.y * ((float)d[j][e] * w[j * N + e] - sum - n * product);
        if constexpr (TOTAL) dx += (float)t[j][e];
        o[e] = (T)dx;
      }
      store_vector((T*)p.y + at * p.ys, R::at(j), width, o);
    }
  }
  if (!p.part) return;
  // the rows of a workgroup in a fixed order, so that the same call gives the same bits
  float* part = p.part + (size_t)blockIdx.x * 2 * p.width;
  __shared__ float sums[PER > 1 ? PER : 1][PER > 1 ? THREADS * N + 1 : 1];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which && !p.bias) break;
    float (&mine)[NV * N] = which ? db : dw;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (PER > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) sums[threadIdx.x / THREADS][threadIdx.x % THREADS * N + e] = mine[j * N + e];
        __syncthreads();
        for (int c = threadIdx.x; c < THREADS * N; c += threads_of(THREADS)) {
          double v = 0.0;
          for (int i = 0; i < PER; ++i) v += sums[i][c];
          if (j * THREADS * N + c < p.width) part[which * p.width + j * THREADS * N + c] = (float)v;
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (R::at(j) + e < p.width) part[which * p.width + R::at(j) + e] = mine[j * N + e];
      }
    }
  }
}

// dw and db = the sums of the workgroups' partial sums, 16 columns a workgroup, in 64 bits: their terms cancel
__global__ void __launch_bounds__(1024) layer_norm_join_kernel(const float* part, float* dw, float* db, int blocks, int width) {
  const int column = blockIdx.x * 16 + (threadIdx.x & 15);
  float* to = blockIdx.y ? db : dw;
  if (!to) return;
  __shared__ double sums[64][17];
  double v = 0.0;
  if (column < width) {
#pragma unroll 8
    for (int r = threadIdx.x >> 4; r < blocks; r += 64) v += part[((size_t)r * 2 + blockIdx.y) * width + column];
  }
  sums[threadIdx.x >> 4][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x >= 16 || column >= width) return;
  v = 0.0;
#pragma unroll
  for (int r = 0; r < 64; ++r) v += sums[r][threadIdx.x];
  to[column] = (float)v;
}

struct Shape { int threads, nv; };
// The fewest threads a row that hold it in a few vectors each
Shape shape_of(int width, int dt) {
  const int n = dt == PRISM_F32 ? 4 : 8, vectors = (width + n - 1) / n;
  constexpr Shape all[] = {{16, 1}, {32, 1}, {32, 2}, {32, 3}, {64, 2}, {64, 3}, {64, 4}, {256, 2}, {256, 3}, {256, 4}, {1024, 2}, {1024, 4}};
  for (const Shape& s : all)
    if (s.threads * s.nv >= vectors) return s;
  return all[11];
}
int rows_per_block(const Shape& s) { return threads_of(s.threads) / s.threads; }
int blocks_of(long long rows, int width, int dt, int most) {
  const Shape s = shape_of(width, dt);
  const long long need = (rows + rows_per_block(s) - 1) / rows_per_block(s);
  return (int)(need < most ? need : most);
}
constexpr int FORWARD_BLOCKS = 2048, BACKWARD_BLOCKS = 1024;

template <typename T, int THREADS, int NV> void launch(const LayerNorm& p, int blocks, bool back, hipStream_t s) {
  void (*kernel)(LayerNorm) = nullptr;
  if (back) kernel = p.dtotal ? layer_norm_backward_kernel<T, THREADS, NV, true> : layer_norm_backward_kernel<T, THREADS, NV, false>;
  else kernel = p.residual ? layer_norm_kernel<T, THREADS, NV, true> : layer_norm_kernel<T, THREADS, NV, false>;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads_of(THREADS)), 0, s, p);
}
template <typename T> void by_shape(const LayerNorm& p, Shape h, int blocks, bool back, hipStream_t s) {
  switch (h.threads * 8 + h.nv) {
    case 16 * 8 + 1: return launch<T, 16, 1>(p, blocks, back, s);
    case 32 * 8 + 1: return launch<T, 32, 1>(p, blocks, back, s);
    case 32 * 8 + 2: return launch<T, 32, 2>(p, blocks, back, s);
    case 32 * 8 + 3: return launch<T, 32, 3>(p, blocks, back, s);
    case 64 * 8 + 2: return launch<T, 64, 2>(p, blocks, back, s);
    case 64 * 8 + 3: return launch<T, 64, 3>(p, blocks, back, s);
    case 64 * 8 + 4: return launch<T, 64, 4>(p, blocks, back, s);
    case 256 * 8 + 2: return launch<T, 256, 2>(p, blocks, back, s);
    case 256 * 8 + 3: return launch<T, 256, 3>(p, blocks, back, s);
    case 256 * 8 + 4: return launch<T, 256, 4>(p, blocks, back, s);
    case 1024 * 8 + 2: return launch<T, 1024, 2>(p, blocks, back, s);
    default: return launch<T, 1024, 4>(p, blocks, back, s);
  }
}
void by_type(const LayerNorm& p, int dt, int blocks, bool back, hipStream_t s) {
  if (dt == PRISM_F32) by_shape<float>(p, shape_of(p.width, dt), blocks, back, s);
  else by_shape<__bf16>(p, shape_of(p.width, dt), blocks, back, s);
}

LayerNorm common(const prism_layer_norm_desc& d) {
  LayerNorm p = {};
  p.rows = d.rows; p.width = d.width; p.eps = d.eps; p.center = d.center;
  return p;
}

}  // namespace

int launch_layer_norm(const void* x, const void* residual, const float* weight, const float* bias, void* y, void* total, float* stats, int dt,
                      const prism_layer_norm_desc& d, hipStream_t s) {
  ProfScope prof(PK_LAYER_NORM, s);
  LayerNorm p = common(d);
  p.x = x; p.xs = d.x; p.residual = residual; p.rs = d.residual; p.total = total; p.ts = d.total; p.y = y; p.ys = d.y;
  p.w = weight; p.b = bias; p.stats = (float2*)stats;
  by_type(p, dt, blocks_of(d.rows, d.width, dt, FORWARD_BLOCKS), false, s);
  return PRISM_OK;
}

size_t layer_norm_backward_bytes(const prism_layer_norm_desc& d, int dt) {
  return (size_t)blocks_of(d.rows, d.width, dt, BACKWARD_BLOCKS) * 2 * d.width * sizeof(float);
}

int launch_layer_norm_backward(const void* dy, const void* total, const float* stats, const float* weight, const void* dtotal, void* dx, float* dweight,
                               float* dbias, int dt, const prism_layer_norm_desc& d, float* part, hipStream_t s) {
  ProfScope prof(PK_LAYER_NORM_BACKWARD, s);
  LayerNorm p = common(d);
  p.dy = dy; p.ds = d.dy; p.x = total; p.xs = d.total; p.dtotal = dtotal; p.gs = d.dtotal; p.y = dx; p.ys = d.dx;
  p.w = weight; p.stats = (float2*)stats; p.part = part; p.bias = dbias != nullptr;
  const int blocks = blocks_of(d.rows, d.width, dt, BACKWARD_BLOCKS);
  if (blocks) by_type(p, dt, blocks, true, s);
  if (part) hipLaunchKernelGGL(layer_norm_join_kernel, dim3((d.width + 15) / 16, dbias ? 2 : 1), dim3(1024), 0, s, part, dweight, dbias, blocks, d.width);
  return PRISM_OK;
}

}  // namespace prism
