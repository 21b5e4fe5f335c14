// RMS norm of every head of the queries and keys and their rotation by position, in one pass over them, and its gradient.
//
//   n = x r w, r = (mean x^2 + eps)^(-1/2);  pair (a, b) of n at position t: scale (a cos - b sin, b cos + a sin), angle = t inv_freq
//   dn = R^T dy,  dw = sum dn x r,  dx = r (dn w - x r mean(dn w x r))
//
// A head is cut into units of eight pairs, a lane takes one: two vectors of eight elements, from the two halves of the rotated part or next to each
// other, so the partner of an element is always in the same lane.  2, 4, 8 or 16 lanes make a head and share the sum of squares.  The angle is taken in
// turns in 64 bits (32 would lose 0.004 rad at position 10^5); a lane computes its eight sines and cosines once and uses them for HS heads of its token.
//
// Bound by memory: every entry is read and written once (gradients: two read, one written), sums and statistics are in 32 bits, results are rounded once.  4 x 4096 tokens,
// 32 + 8 heads of 128, bf16: 78 us (335 MB, 4.3 TB/s) and gradients 104 + 7 us (503 MB, 4.8 TB/s; vector units 60 and 69 % busy); a large copy runs at 4.6 to 5.4.
#include "layer.h"

namespace prism {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct NormRope {
  const void *x[2], *dy[2];      // queries, keys; dy: the gradient of the results
  void* out[2];                  // results (or the gradient of x)
  long long xs[2][3], ds[2][3], os[2][3];   // strides of batch, token, head
  const float* w[2];
  const int* pos;
  const float* inv_freq;
  float* part[2];                // partial sums of dw: [workgroup][16 lanes]
  int heads[2], groups[2];       // groups of HS heads
  int len, dim, rot, start;
  unsigned items[2];             // tokens x groups
  int blocks_q;                  // backward: the first blocks_q workgroups take queries
  float eps, scale;
  bool norm, interleaved;
};

// Eight entries as they lie in memory
template <typename T> struct Eight;
template <> struct Eight<float> {
  f32x4 lo, hi;
  __device__ float get(int e) const { return e < 4 ? lo[e & 3] : hi[e & 3]; }
  __device__ void set(int e, float x) { if (e < 4) lo[e & 3] = x; else hi[e & 3] = x; }
};
template <> struct Eight<__bf16> {
  bf16x8 v;
  __device__ float get(int e) const { return (float)v[e]; }
  __device__ void set(int e, float x) { v[e] = (__bf16)x; }
};

// Where a unit's elements lie: pair e of unit u holds slots 16 u + 2 e and the next; slots 2 p and 2 p + 1 below rot are pair p.
// VEC: every unit is two whole vectors.
template <typename T, bool VEC> struct Unit {
  int u, dim, rot;
  bool split;                            // the partners of a pair lie rot / 2 apart
  struct Raw { Eight<T> a, b; };
  __device__ bool halves() const { return split && 16 * u < rot; }
  __device__ int element(int slot) const { return (!split || slot >= rot) ? slot : (slot & 1) ? (slot >> 1) + rot / 2 : slot >> 1; }
  __device__ int second() const { return halves() ? rot / 2 + 8 * u : 16 * u + 8; }

  __device__ void load(const T* row, Raw& r) const {
    if constexpr (VEC) {
      const int f = halves() ? 8 * u : 16 * u, s = second();
      r = Raw{};
      if (f < dim) r.a = *(const Eight<T>*)(row + f);
      if (s < dim) r.b = *(const Eight<T>*)(row + s);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {       // each half of the pairs by itself
      const int s = 16 * u + 2 * e;
      r.a.set(e, s < dim ? (float)row[element(s)] : 0.0f);
      r.b.set(e, s + 1 < dim ? (float)row[element(s + 1)] : 0.0f);
    }
  }
  __device__ void pairs(const Raw& r, float (&a)[8], float (&b)[8]) const {
    if (!VEC || halves()) {
#pragma unroll
      for (int e = 0; e < 8; ++e) { a[e] = r.a.get(e); b[e] = r.b.get(e); }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = r.a.get(2 * e); b[e] = r.a.get(2 * e + 1);
        a[4 + e] = r.b.get(2 * e); b[4 + e] = r.b.get(2 * e + 1);
      }
    }
  }
  __device__ void store(T* row, const float (&a)[8], const float (&b)[8]) const {
    if constexpr (VEC) {
      Raw r;
      if (halves()) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { r.a.set(e, a[e]); r.b.set(e, b[e]); }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r.a.set(2 * e, a[e]); r.a.set(2 * e + 1, b[e]);
          r.b.set(2 * e, a[4 + e]); r.b.set(2 * e + 1, b[4 + e]);
        }
      }
      const int f = halves() ? 8 * u : 16 * u, s = second();
      if (f < dim) *(Eight<T>*)(row + f) = r.a;
      if (s < dim) *(Eight<T>*)(row + s) = r.b;
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * u + 2 * e;
      if (s < dim) row[element(s)] = (T)a[e];
      if (s + 1 < dim) row[element(s + 1)] = (T)b[e];
    }
  }
};

// cos and sin (times scale) of the unit's pairs at a position; pairs past the rotated part stay as they are.  The instructions take turns and are off by 1.3e-7 at most
// on half a turn to either side.  (Series on an eighth of a turn: results of fp32 7.4e-8 -> 6.5e-8 from 64 bits in the mean, 38 -> 40 us for 3 x 777 tokens, 24 heads of 80.)
template <bool VEC> __device__ inline void angles(const NormRope& p, int u, int position, float (&c)[8], float (&s)[8]) {
  float f[8];
  if (VEC && 16 * u + 16 <= p.rot) {
    const Eight<float> x = *(const Eight<float>*)(p.inv_freq + 8 * u);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = x.get(e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 16 * u + 2 * e < p.rot ? p.inv_freq[8 * u + e] : 0.0f;
  }
  const double per_turn = (double)position * 0.15915494309189535;   // 1 / (2 pi)
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double turns = per_turn * (double)f[e];
    const float x = (float)(turns - rint(turns)), by = 16 * u + 2 * e < p.rot ? p.scale : 1.0f;
    c[e] = __builtin_amdgcn_cosf(x) * by;
    s[e] = __builtin_amdgcn_sinf(x) * by;
  }
}

template <int L> __device__ inline float over_lanes(float v) {
#pragma unroll
  for (int m = 1; m < L; m *= 2) v += __shfl_xor(v, m);
  return v;
}

template <bool VEC> __device__ inline void weights(const NormRope& p, int u, int kind, float (&wa)[8], float (&wb)[8]) {
  const Unit<float, VEC> un = {u, p.dim, p.rot, !p.interleaved};
  if (p.w[kind]) {
    typename Unit<float, VEC>::Raw r;
    un.load(p.w[kind], r);
    un.pairs(r, wa, wb);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) wa[e] = wb[e] = 1.0f;
  }
}

template <typename T, bool VEC, int L, int HS>
__global__ void __launch_bounds__(256) norm_rope_kernel(NormRope p) {
  unsigned it = blockIdx.x * (256 / L) + threadIdx.x / L;
  const int kind = it >= p.items[0];
  if (kind) it -= p.items[0];
  if (it >= p.items[kind]) return;             // whole heads leave: the sum below is over the lanes of one
  const Unit<T, VEC> un = {(int)threadIdx.x % L, p.dim, p.rot, !p.interleaved};
  const unsigned token = it / p.groups[kind];
  const int h0 = (it - token * p.groups[kind]) * HS, b = token / p.len, i = token - b * p.len;
  const T* x = (const T*)p.x[kind] + b * p.xs[kind][0] + i * p.xs[kind][1];
  T* out = (T*)p.out[kind] + b * p.os[kind][0] + i * p.os[kind][1];
  typename Unit<T, VEC>::Raw raw[HS];
  float c[8], s[8], wa[8], wb[8];
#pragma unroll
  for (int h = 0; h < HS; ++h)
    if (h0 + h < p.heads[kind]) un.load(x + (h0 + h) * p.xs[kind][2], raw[h]);
  angles<VEC>(p, un.u, p.pos ? p.pos[token] : p.start + i, c, s);
  weights<VEC>(p, un.u, kind, wa, wb);
#pragma unroll
  for (int h = 0; h < HS; ++h) {
    if (h0 + h >= p.heads[kind]) continue;
    float a[8], bb[8];
    un.pairs(raw[h], a, bb);
    if (p.norm) {
      float q = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) q += a[e] * a[e] + bb[e] * bb[e];
      const float r = 1.0f / sqrtf(over_lanes<L>(q) / (float)p.dim + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) { a[e] *= r * wa[e]; bb[e] *= r * wb[e]; }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = a[e] * c[e] - bb[e] * s[e];
      bb[e] = bb[e] * c[e] + a[e] * s[e];
      a[e] = t;
    }
    un.store(out + (h0 + h) * p.os[kind][2], a, bb);
  }
}

template <typename T, bool VEC, int L, int HS>
__global__ void __launch_bounds__(256) norm_rope_backward_kernel(NormRope p) {
  const int kind = (int)blockIdx.x >= p.blocks_q, block = blockIdx.x - (kind ? p.blocks_q : 0), nblocks = kind ? gridDim.x - p.blocks_q : p.blocks_q;
  const Unit<T, VEC> un = {(int)threadIdx.x % L, p.dim, p.rot, !p.interleaved};
  float ga[8] = {}, gb[8] = {}, wa[8], wb[8];
  weights<VEC>(p, un.u, kind, wa, wb);
  for (unsigned it = block * (256 / L) + threadIdx.x / L; it < p.items[kind]; it += nblocks * (256 / L)) {
    const unsigned token = it / p.groups[kind];
    const int h0 = (it - token * p.groups[kind]) * HS, b = token / p.len, i = token - b * p.len;
    const T* x = (const T*)p.x[kind] + b * p.xs[kind][0] + i * p.xs[kind][1];
    const T* dy = (const T*)p.dy[kind] + b * p.ds[kind][0] + i * p.ds[kind][1];
    T* out = (T*)p.out[kind] + b * p.os[kind][0] + i * p.os[kind][1];
    typename Unit<T, VEC>::Raw xr[HS], dr[HS];
    float c[8], s[8];
#pragma unroll
    for (int h = 0; h < HS; ++h)
      if (h0 + h < p.heads[kind]) {
        un.load(dy + (h0 + h) * p.ds[kind][2], dr[h]);
        if (p.norm) un.load(x + (h0 + h) * p.xs[kind][2], xr[h]);
      }
    angles<VEC>(p, un.u, p.pos ? p.pos[token] : p.start + i, c, s);
#pragma unroll
    for (int h = 0; h < HS; ++h) {
      if (h0 + h >= p.heads[kind]) continue;
      float a[8], bb[8];
      un.pairs(dr[h], a, bb);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = a[e] * c[e] + bb[e] * s[e];
        bb[e] = bb[e] * c[e] - a[e] * s[e];
        a[e] = t;
      }
      if (p.norm) {
        float xa[8], xb[8];
        un.pairs(xr[h], xa, xb);
        float q = 0.0f, d = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q += xa[e] * xa[e] + xb[e] * xb[e];
          d += a[e] * wa[e] * xa[e] + bb[e] * wb[e] * xb[e];
        }
        const float r = 1.0f / sqrtf(over_lanes<L>(q) / (float)p.dim + p.eps);
        const float m = over_lanes<L>(d) / (float)p.dim * r * r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ga[e] += a[e] * xa[e] * r;
          gb[e] += bb[e] * xb[e] * r;
          a[e] = r * (a[e] * wa[e] - xa[e] * m);
          bb[e] = r * (bb[e] * wb[e] - xb[e] * m);
        }
      }
      un.store(out + (h0 + h) * p.os[kind][2], a, bb);
    }
  }
  if (!p.norm || !p.part[kind]) return;
  // the heads of a workgroup in a fixed order, so that the same call gives the same bits; in 64 bits, as the sums of the join: the terms of dw cancel
  __shared__ float sums[256 / L][16 * L + 1];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sums[threadIdx.x / L][16 * un.u + 2 * e] = ga[e];
    sums[threadIdx.x / L][16 * un.u + 2 * e + 1] = gb[e];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * L; t += 256) {
    double v = 0.0;
    for (int r = 0; r < 256 / L; ++r) v += sums[r][t];
    p.part[kind][(size_t)block * (16 * L) + t] = (float)v;
  }
}

// dw = the sum of the workgroups' partial sums; a workgroup takes 16 slots of the queries' (blockIdx.y = 0) or keys' weights
__global__ void __launch_bounds__(1024) norm_rope_join_kernel(NormRope p, float* dqw, float* dkw, int blocks_k, int width) {
  const int kind = blockIdx.y, col = blockIdx.x * 16 + (threadIdx.x & 15), blocks = kind ? blocks_k : p.blocks_q;
  float* to = kind ? dkw : dqw;
  if (!to) return;
  __shared__ double sums[64][17];
  double v = 0.0;
#pragma unroll 8
  for (int r = threadIdx.x >> 4; r < blocks; r += 64) v += p.part[kind][(size_t)r * width + col];
  sums[threadIdx.x >> 4][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x >= 16 || col >= p.dim) return;
  v = 0.0;
#pragma unroll
  for (int r = 0; r < 64; ++r) v += sums[r][threadIdx.x];
  const Unit<float, false> un = {0, p.dim, p.rot, !p.interleaved};
  to[un.element(col)] = (float)v;
}

void strides(long long (&to)[3], const prism_strides& s) { to[0] = s.batch; to[1] = s.token; to[2] = s.head; }

// whether rows of this array may be read as whole vectors of 16 bytes
bool whole_vectors(const void* p, const prism_strides& s, int size) {
  return (((uintptr_t)p | (uintptr_t)(s.batch * size) | (uintptr_t)(s.token * size) | (uintptr_t)(s.head * size)) & 15) == 0;
}

int lanes_of(int dim) { return dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16; }

NormRope common(const void* q, const void* k, const prism_norm_rope_desc& d) {
  NormRope p = {};
  p.x[0] = q; p.x[1] = k;
  strides(p.xs[0], d.q); strides(p.xs[1], d.k);
  p.w[0] = d.q_weight; p.w[1] = d.k_weight;
  p.pos = d.positions; p.inv_freq = d.inv_freq;
  p.heads[0] = d.q_heads; p.heads[1] = d.k_heads;
  p.len = d.len; p.dim = d.head_dim; p.rot = d.rot_dim; p.start = d.start;
  p.eps = d.eps; p.scale = d.scale;
  p.norm = d.norm; p.interleaved = d.interleaved;
  return p;
}

bool fits_vectors(const prism_norm_rope_desc& d) {
  return d.head_dim % 8 == 0 && (d.interleaved || d.rot_dim % 16 == 0) && (((uintptr_t)d.inv_freq | (uintptr_t)d.q_weight | (uintptr_t)d.k_weight) & 15) == 0;
}

// Heads per lane share the sines of their token: four (gradients: two, whose operands fill as many registers) where that leaves the chip four waves per SIMD.
// 4 x 4096 tokens, 32 + 8 heads of 128: one head a lane 114 us and gradients 111, shared 84 and 106; 2048 tokens: 13.9 and 23.2, shared 12.4 and 21.3 (always two: 22.5).
int heads_per_lane(const prism_norm_rope_desc& d, int L, int most) {
  const long long waves = (long long)d.batch * d.len * (d.q_heads + d.k_heads) * L / 64;
  while (most > 1 && waves < most * 4096ll) most /= 2;
  return most;
}

void set_items(NormRope& p, const prism_norm_rope_desc& d, int HS) {
  for (int kind = 0; kind < 2; ++kind) {
    p.groups[kind] = p.heads[kind] ? (p.heads[kind] + HS - 1) / HS : 1;
    p.items[kind] = p.heads[kind] ? (unsigned)(d.batch * d.len) * (unsigned)p.groups[kind] : 0u;
  }
}

template <typename T, bool VEC, int L> void launch(NormRope& p, int HS, int blocks_k, bool back, hipStream_t s) {
  const dim3 grid(back ? p.blocks_q + blocks_k : (unsigned)(((unsigned long long)p.items[0] + p.items[1] + 256 / L - 1) / (256 / L)));
  void (*kernel)(NormRope) = back ? norm_rope_backward_kernel<T, VEC, L, 1> : norm_rope_kernel<T, VEC, L, 1>;
  if constexpr (VEC) {
    if (HS == 2) kernel = back ? norm_rope_backward_kernel<T, VEC, L, 2> : norm_rope_kernel<T, VEC, L, 2>;
    else if (HS == 4) kernel = norm_rope_kernel<T, VEC, L, 4>;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p);
}
template <typename T, bool VEC> void by_lanes(NormRope& p, int L, int HS, int blocks_k, bool back, hipStream_t s) {
  if (L == 2) launch<T, VEC, 2>(p, HS, blocks_k, back, s);
  else if (L == 4) launch<T, VEC, 4>(p, HS, blocks_k, back, s);
  else if (L == 8) launch<T, VEC, 8>(p, HS, blocks_k, back, s);
  else launch<T, VEC, 16>(p, HS, blocks_k, back, s);
}
void by_type(NormRope& p, int dt, bool vec, int L, int HS, int blocks_k, bool back, hipStream_t s) {
  if (dt == PRISM_F32) vec ? by_lanes<float, true>(p, L, HS, blocks_k, back, s) : by_lanes<float, false>(p, L, HS, blocks_k, back, s);
  else vec ? by_lanes<__bf16, true>(p, L, HS, blocks_k, back, s) : by_lanes<__bf16, false>(p, L, HS, blocks_k, back, s);
}

}  // namespace

int launch_norm_rope(const void* q, const void* k, void* qo, void* ko, int dt, const prism_norm_rope_desc& d, hipStream_t s) {
  ProfScope prof(PK_NORM_ROPE, s);
  NormRope p = common(q, k, d);
  const int size = dt == PRISM_F32 ? 4 : 2, L = lanes_of(d.head_dim);
  p.out[0] = qo; p.out[1] = ko;
  strides(p.os[0], d.q_out); strides(p.os[1], d.k_out);
  const bool vec = fits_vectors(d) && (!d.q_heads || (whole_vectors(q, d.q, size) && whole_vectors(qo, d.q_out, size))) &&
          (!d.k_heads || (whole_vectors(k, d.k, size) && whole_vectors(ko, d.k_out, size)));
  const int HS = vec ? heads_per_lane(d, L, 4) : 1;
  set_items(p, d, HS);
  if (((unsigned long long)p.items[0] + p.items[1]) * L > 0xFFFFFF00ull) {
    set_last_error("a launch takes fewer than 2^32 work-items, one for 16 entries of a head");
    return PRISM_EUNSUPPORTED;
  }
  by_type(p, dt, vec, L, HS, 0, false, s);
  return PRISM_OK;
}

size_t norm_rope_backward_bytes(const prism_norm_rope_desc& d) {
  return d.norm ? (size_t)2 * NR_MAX_BLOCKS * 16 * lanes_of(d.head_dim) * sizeof(float) : 0;
}

int launch_norm_rope_backward(const void* dqo, const void* dko, const void* q, const void* k, void* dq, void* dk, float* dqw, float* dkw, int dt,
                              const prism_norm_rope_desc& d, float* part, hipStream_t s) {
  ProfScope prof(PK_NORM_ROPE_BACKWARD, s);
  NormRope p = common(q, k, d);
  const int size = dt == PRISM_F32 ? 4 : 2, L = lanes_of(d.head_dim);
  p.dy[0] = dqo; p.dy[1] = dko;
  strides(p.ds[0], d.q_out); strides(p.ds[1], d.k_out);
  p.out[0] = dq; p.out[1] = dk;
  strides(p.os[0], d.dq); strides(p.os[1], d.dk);
  const bool vec = fits_vectors(d) &&
          (!d.q_heads || ((!d.norm || whole_vectors(q, d.q, size)) && whole_vectors(dqo, d.q_out, size) && whole_vectors(dq, d.dq, size))) &&
          (!d.k_heads || ((!d.norm || whole_vectors(k, d.k, size)) && whole_vectors(dko, d.k_out, size) && whole_vectors(dk, d.dk, size)));
  const int HS = vec ? heads_per_lane(d, L, 2) : 1;
  set_items(p, d, HS);
  // workgroups in proportion to the work of queries and keys
  const long long slots = 256 / L, all = (long long)p.items[0] + p.items[1];
  auto blocks = [&](int kind) {
    const long long need = (p.items[kind] + slots - 1) / slots, share = all ? (NR_MAX_BLOCKS * (long long)p.items[kind] + all - 1) / all : 0;
    return (int)(need < share ? need : share);
  };
  p.blocks_q = blocks(0);
  const int blocks_k = blocks(1), width = 16 * L;
  if (d.norm) {
    p.part[0] = dqw ? part : nullptr;
    p.part[1] = dkw ? part + (size_t)NR_MAX_BLOCKS * width : nullptr;
  }
  by_type(p, dt, vec, L, HS, blocks_k, true, s);
  if (d.norm && (dqw || dkw)) hipLaunchKernelGGL(norm_rope_join_kernel, dim3(L, 2), dim3(1024), 0, s, p, dqw, dkw, blocks_k, width);
  return PRISM_OK;
}

}  // namespace prism
