// Rows of the residual stream in registers: what the norm and its gradients share.
//
//   h = x + residual, mean = sum h / width (0 where it is not taken off), r = (mean (h - mean)^2 + eps)^(-1/2), y = (h - mean) r w + b
//   g = dy w, n = (h - mean) r:  dx = r (g - mean g - n mean (g n)) + dtotal (without mean g where the mean is not taken off), dw = sum dy n, db = sum dy
//
// THREADS threads share a row, NV vectors of 16 bytes each: one pass over memory, at the rate of a large copy and above: 65536 x 768 bf16 with a residual 63 us (403 MB, 6.4 TB/s), gradients
// 67 + 5 us; 16384 x 4096 88 and 97; 65536 x 771 80 and 93 (part of a vector in every row).  Statistics are of h as it is stored (rounded), so that the gradients meet the same numbers.
#pragma once
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

// How rows are read.  WHOLE: they end with a whole vector (no code for part of one, which costs registers); ODD: they do not, TINY: they have not even one; ..PAST: past the caches.
enum { TINY, ODD, ODD_PAST, WHOLE, WHOLE_PAST };
constexpr bool whole_rows(int mode) { return mode >= WHOLE; }

// Lane l of a row's THREADS has its vectors l, l + THREADS, ...: NV at most
template <typename T, int THREADS, int NV, int MODE> struct Row {
  static constexpr int N = Vec<T>::N;
  using V = typename Vec<T>::type;
  static __device__ int at(int j) { return ((int)(threadIdx.x % THREADS) + j * THREADS) * N; }
  static __device__ bool inside(int j, int e, int width) { return whole_rows(MODE) ? at(j) < width : at(j) + e < width; }
  // A row's last vector is read so that it ends with the row, and put in its place by settle(): all the loads of a row first, as a wave waits for what it settles.  Entries past the
  // end are 0 then.
  static __device__ V load(const T* row, int j, int width) {
    if constexpr (MODE == TINY) return load_vector(row, at(j), width);
    V v = {};
    if (at(j) < width) {
      const V* from = (const V*)(row + (whole_rows(MODE) || at(j) + N <= width ? at(j) : width - N));
      v = MODE == ODD_PAST || MODE == WHOLE_PAST ? __builtin_nontemporal_load(from) : *from;
    }
    return v;
  }
  static __device__ void settle(V (&v)[NV], int width) {
    if constexpr (MODE == ODD || MODE == ODD_PAST) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (at(j) < width && at(j) + N > width) v[j] = __builtin_bit_cast(V, __builtin_bit_cast(unsigned __int128, v[j]) >> ((at(j) + N - width) * (128 / N)));
    }
  }
  template <bool OVER = false> static __device__ void store(T* row, int j, int width, const V& v) {     // OVER: past the caches in the ..PAST modes
    if constexpr (MODE == ODD_PAST && OVER) return stream_vector_to(row, at(j), width, v);
    if constexpr (!whole_rows(MODE)) return store_vector(row, at(j), width, v);
    if (at(j) >= width) return;
    if constexpr (MODE == WHOLE_PAST && OVER) __builtin_nontemporal_store(v, (V*)(row + at(j)));
    else *(V*)(row + at(j)) = v;
  }
};

// fp32 of every column, `none` where there is no array: in registers, or, where a row fills the workgroup's, in LDS
template <typename T, int THREADS, int NV, int MODE> struct Columns {
  using R = Row<T, THREADS, NV, MODE>;
  static constexpr int N = R::N;
  static constexpr bool LDS = THREADS == 1024;
  float held[LDS ? 1 : NV * N];
  float* memory;
  static constexpr int FLOATS = LDS ? THREADS * NV * N : 1;
  __device__ Columns(const float* w, int width, float none, float* lds) : memory(lds) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        Vec<float>::type v = {none, none, none, none};
        if (w) {
          if constexpr (whole_rows(MODE)) { if (R::at(j) < width) v = *(const Vec<float>::type*)(w + R::at(j) + q); }
          else v = load_vector(w, R::at(j) + q, width);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (LDS) memory[place(j, q + e)] = v[e];
          else held[j * N + q + e] = v[e];
        }
      }
  }
  // entries of a vector lie THREADS apart: a lane reads and writes its own only, without conflicts
  static __device__ int place(int j, int e) { return (j * N + e) * THREADS + (int)(threadIdx.x % THREADS); }
  __device__ float get(int j, int e) const {
    if constexpr (LDS) return memory[place(j, e)];
    else return held[j * N + e];
  }
};

// Rows of `width` entries: the fewest threads that hold one in a few vectors each.  past: the call's `arrays` do not fit the card's last cache (256 MB); 65536 x 768 bf16 with a residual then
// takes 138 us with its gradients, 160 through the caches, while 8192 x 768 takes 9.2 us (10.9 past them).  More than three vectors a lane cost the gradients a wave of each SIMD: 65536
// x 1111 bf16 120 us in three, 250 in four.
struct Shape { int threads, nv, mode = TINY; };
inline Shape shape_of(int width, int dt, long long rows, int arrays) {
  const int n = dt == PRISM_F32 ? 4 : 8, vectors = (width + n - 1) / n;
  constexpr Shape whole[] = {{16, 1}, {32, 1}, {32, 3}, {64, 2}, {64, 3}, {256, 1}, {256, 2}, {256, 3}, {1024, 1}, {1024, 2}, {1024, 4}};
  constexpr Shape odd[] = {{32, 1}, {32, 3}, {64, 2}, {64, 3}, {256, 1}, {256, 2}, {256, 3}, {1024, 2}, {1024, 4}};
  const bool past = rows * width * (16 / n) * arrays > (256ll << 20);
  if (width < n) return {32, 1, TINY};
  Shape r = {1024, 4, width % n ? past ? ODD_PAST : ODD : past ? WHOLE_PAST : WHOLE};
  auto find = [&](const Shape* all, int count) {
    for (int i = count - 1; i >= 0; --i)
      if (all[i].threads * all[i].nv >= vectors) { r.threads = all[i].threads; r.nv = all[i].nv; }
  };
  if (!whole_rows(r.mode)) find(odd, 9);
  else find(whole, 11);
  return r;
}
inline int rows_per_block(const Shape& s) { return threads_of(s.threads) / s.threads; }
inline int blocks_of(long long rows, const Shape& s, int most) {
  const long long need = (rows + rows_per_block(s) - 1) / rows_per_block(s);
  return (int)(need < most ? need : most);
}

// launch<T, threads, nv, mode>() of L for a shape
template <typename T, template <typename, int, int, int> class L, int MODE, typename... A> void by_shape(const Shape& h, const A&... a) {
  constexpr int MOST = Vec<T>::N == 4 ? 4 : 2;      // four vectors of 1024 threads: rows over 8192 entries of fp32 only
  const int shape = h.threads * 8 + h.nv;
  if constexpr (MODE == TINY) {
    return L<T, 32, 1, MODE>::launch(a...);
  } else if constexpr (!whole_rows(MODE)) {
    switch (shape) {
      case 32 * 8 + 1: return L<T, 32, 1, MODE>::launch(a...);
      case 32 * 8 + 3: return L<T, 32, 3, MODE>::launch(a...);
      case 64 * 8 + 2: return L<T, 64, 2, MODE>::launch(a...);
      case 64 * 8 + 3: return L<T, 64, 3, MODE>::launch(a...);
      case 256 * 8 + 1: return L<T, 256, 1, MODE>::launch(a...);
      case 256 * 8 + 2: return L<T, 256, 2, MODE>::launch(a...);
      case 256 * 8 + 3: return L<T, 256, 3, MODE>::launch(a...);
      case 1024 * 8 + 2: return L<T, 1024, 2, MODE>::launch(a...);
      default: return L<T, 1024, MOST, MODE>::launch(a...);
    }
  } else {
    switch (shape) {
      case 16 * 8 + 1: return L<T, 16, 1, MODE>::launch(a...);
      case 32 * 8 + 1: return L<T, 32, 1, MODE>::launch(a...);
      case 32 * 8 + 3: return L<T, 32, 3, MODE>::launch(a...);
      case 64 * 8 + 2: return L<T, 64, 2, MODE>::launch(a...);
      case 64 * 8 + 3: return L<T, 64, 3, MODE>::launch(a...);
      case 256 * 8 + 1: return L<T, 256, 1, MODE>::launch(a...);
      case 256 * 8 + 2: return L<T, 256, 2, MODE>::launch(a...);
      case 256 * 8 + 3: return L<T, 256, 3, MODE>::launch(a...);
      case 1024 * 8 + 1: return L<T, 1024, 1, MODE>::launch(a...);
      case 1024 * 8 + 2: return L<T, 1024, 2, MODE>::launch(a...);
      default: return L<T, 1024, MOST, MODE>::launch(a...);
    }
  }
}
template <typename T, template <typename, int, int, int> class L, typename... A> void by_mode(const Shape& h, const A&... a) {
  if (h.mode == TINY) by_shape<T, L, TINY>(h, a...);
  else if (h.mode == ODD) by_shape<T, L, ODD>(h, a...);
  else if (h.mode == ODD_PAST) by_shape<T, L, ODD_PAST>(h, a...);
  else if (h.mode == WHOLE) by_shape<T, L, WHOLE>(h, a...);
  else by_shape<T, L, WHOLE_PAST>(h, a...);
}
template <template <typename, int, int, int> class L, typename... A> void by_type(int dt, const Shape& h, const A&... a) {
  if (dt == PRISM_F32) by_mode<float, L>(h, a...);
  else by_mode<__bf16, L>(h, a...);
}

inline LayerNorm layer_norm_common(const prism_layer_norm_desc& d) {
  LayerNorm p = {};
  p.rows = d.rows; p.width = d.width; p.eps = d.eps; p.center = d.center;
  return p;
}

}  // namespace
}  // namespace prism
