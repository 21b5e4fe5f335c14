// Gradients of the norm of rows (layer_norm_rows.h has the formulas).  A workgroup goes through many rows and keeps its share of dw and db in registers; the shares are joined by a
// second launch in a fixed order.  The sums of 24 columns a lane, their weights and three rows leave room for two waves a SIMD (65536 x 768 bf16: 67 us, memory); rows of 16384 entries spill a
// few registers (4096 of them 169 us, 3.2 TB/s).
#include "layer_norm_rows.h"

namespace prism {
namespace {

template <typename T, int THREADS, int NV, int MODE, bool TOTAL>
__global__ void __launch_bounds__(threads_of(THREADS)) layer_norm_backward_kernel(LayerNorm p) {
  using R = Row<T, THREADS, NV, MODE>;
  using V = typename Vec<T>::type;
  using C = Columns<T, THREADS, NV, MODE>;
  constexpr int N = R::N, PER = threads_of(THREADS) / THREADS;
  __shared__ float memory[THREADS > 64 ? THREADS / 32 : 1], columns[C::FLOATS];
  const C w(p.w, p.width, 1.0f, columns);
  float dw[NV * N] = {}, db[NV * N] = {};
  int turn = 0;
  for (long long first = (long long)blockIdx.x * PER; first < p.rows; first += (long long)gridDim.x * PER) {
    const long long row = first + threadIdx.x / THREADS;
    const bool there = row < p.rows;
    const int width = there ? p.width : 0;
    const long long at = there ? row : 0;
    V h[NV], d[NV], t[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) d[j] = R::load((const T*)p.dy + at * p.ds, j, width);
#pragma unroll
    for (int j = 0; j < NV; ++j) h[j] = R::load((const T*)p.x + at * p.xs, j, width);
    auto load_dtotal = [&]() {
#pragma unroll
      for (int j = 0; j < NV; ++j) t[j] = R::load((const T*)p.dtotal + at * p.gs, j, width);
    };
    if constexpr (TOTAL && THREADS < 1024) load_dtotal();
    const float2 stats = p.stats[at];
    R::settle(d, width);
    R::settle(h, width);
    if constexpr (TOTAL && THREADS < 1024) R::settle(t, width);
    float sum = 0.0f, product = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float dy = (float)d[j][e], n = ((float)h[j][e] - stats.x) * stats.y, g = dy * w.get(j, e);
        sum += g;
        product += g * n;
        dw[j * N + e] += dy * n;
        db[j * N + e] += dy;
      }
    if constexpr (TOTAL && THREADS == 1024) {                        // (registers)
      load_dtotal();
      R::settle(t, width);
    }
    product = row_sum<THREADS>(product, memory, turn++) / (float)p.width;
    sum = p.center ? row_sum<THREADS>(sum, memory, turn++) / (float)p.width : 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      as_loaded<T>(d[j]);
      as_loaded<T>(h[j]);
      float o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float n = ((float)h[j][e] - stats.x) * stats.y;
        float dx = stats.y * ((float)d[j][e] * w.get(j, e) - sum - n * product);
        if constexpr (TOTAL) dx += (float)t[j][e];
        o[e] = dx;
      }
      // past the caches where the call's arrays do not fit them: 65536 x 768 bf16 with the forward pass 137 us among others (145 through them), 153 alone (150)
      R::template store<true>((T*)p.y + at * p.ys, j, width, rounded<T>(o));
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

// dw and db = the sums of the workgroups' partial sums, 32 columns a workgroup, in 64 bits: their terms cancel
__global__ void __launch_bounds__(1024) layer_norm_join_kernel(const float* part, float* dw, float* db, int blocks, int width) {
  const int column = blockIdx.x * 32 + (threadIdx.x & 31);
  float* to = blockIdx.y ? db : dw;
  if (!to) return;
  __shared__ double sums[32][33];
  double v = 0.0;
  if (column < width) {
#pragma unroll 8
    for (int r = threadIdx.x >> 5; r < blocks; r += 32) v += part[((size_t)r * 2 + blockIdx.y) * width + column];
  }
  sums[threadIdx.x >> 5][threadIdx.x & 31] = v;
  __syncthreads();
  if (threadIdx.x >= 32 || column >= width) return;
  v = 0.0;
#pragma unroll
  for (int r = 0; r < 32; ++r) v += sums[r][threadIdx.x];
  to[column] = (float)v;
}

template <typename T, int THREADS, int NV, int MODE> struct Backward {
  static void launch(const LayerNorm& p, int blocks, hipStream_t s) {
    hipLaunchKernelGGL((p.dtotal ? layer_norm_backward_kernel<T, THREADS, NV, MODE, true> : layer_norm_backward_kernel<T, THREADS, NV, MODE, false>), dim3(blocks),
                       dim3(threads_of(THREADS)), 0, s, p);
  }
};

// Workgroups: as many as run at once.  More of them write more partial sums (16384 x 4096 bf16: 512 of them 109 us, 1024 137 us), fewer leave the chip idle.
int backward_blocks(const Shape& h, const prism_layer_norm_desc& d, int dt) {
  const int entries = h.nv * (dt == PRISM_F32 ? 4 : 8);
  return blocks_of(d.rows, h, h.threads == 1024 ? 256 : entries <= 8 ? 1024 : 512);
}

}  // namespace

size_t layer_norm_backward_bytes(const prism_layer_norm_desc& d, int dt) {
  return (size_t)backward_blocks(shape_of(d.width, dt, d.rows, 4), d, dt) * 2 * d.width * sizeof(float);
}

int launch_layer_norm_backward(const void* dy, const void* total, const float* stats, const float* weight, const void* dtotal, void* dx, float* dweight,
                               float* dbias, int dt, const prism_layer_norm_desc& d, float* part, hipStream_t s) {
  ProfScope prof(PK_LAYER_NORM_BACKWARD, s);
  LayerNorm p = layer_norm_common(d);
  p.dy = dy; p.ds = d.dy; p.x = total; p.xs = d.total; p.dtotal = dtotal; p.gs = d.dtotal; p.y = dx; p.ys = d.dx;
  p.w = weight; p.stats = (float2*)stats; p.part = part; p.bias = dbias != nullptr;
  const Shape h = shape_of(d.width, dt, d.rows, dtotal ? 4 : 3);
  const int blocks = backward_blocks(h, d, dt);
  if (blocks) by_type<Backward>(dt, h, p, blocks, s);
  if (part) hipLaunchKernelGGL(layer_norm_join_kernel, dim3((d.width + 31) / 32, dbias ? 2 : 1), dim3(1024), 0, s, part, dweight, dbias, blocks, d.width);
  return PRISM_OK;
}

}  // namespace prism
