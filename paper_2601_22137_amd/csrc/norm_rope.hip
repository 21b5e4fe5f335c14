// RMS norm of every head of the queries and keys and their rotation by position, in one pass over them, and its gradient.
//
//   n = x r w, r = (mean x^2 + eps)^(-1/2);  pair (a, b) of n at position t: scale (a cos - b sin, b cos + a sin), angle = t inv_freq
//   dn = R^T dy,  dw = sum dn x r,  dx = r (dn w - x r mean(dn w x r))
//
// A head is cut into units of eight pairs, a lane takes one: two vectors of eight elements, from the two halves of the rotated part or next to each
// other, so the partner of an element is always in the same lane.  2, 4, 8 or 16 lanes make a head and share the sum of squares.  The angle is taken in
// turns in 64 bits (32 would lose 0.004 rad at position 10^5); a lane computes its eight sines and cosines once and uses them for HS heads of its token.
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
  bool norm, interleaved, vec;
};

template <typename T> __device__ inline void load8(const T* p, float (&v)[8]);
template <> __device__ inline void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}
template <> __device__ inline void load8<__bf16>(const __bf16* p, float (&v)[8]) {
  const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
}
template <typename T> __device__ inline void store8(T* p, const float (&v)[8]);
template <> __device__ inline void store8<float>(float* p, const float (&v)[8]) {
  f32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) { a[e] = v[e]; b[e] = v[4 + e]; }
  *(f32x4*)p = a;
  *(f32x4*)(p + 4) = b;
}
template <> __device__ inline void store8<__bf16>(__bf16* p, const float (&v)[8]) {
  bf16x8 a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = (__bf16)v[e];
  *(bf16x8*)p = a;
}

// Where a unit's elements lie: pair e of unit u holds slots 16 u + 2 e and the next; slots 2 p and 2 p + 1 below rot are pair p.
struct Unit {
  int u, dim, rot;
  bool split, vec;                       // split: the partners of a pair lie rot / 2 apart
  __device__ bool halves() const { return split && 16 * u < rot; }
  __device__ int element(int slot) const { return (!split || slot >= rot) ? slot : (slot & 1) ? (slot >> 1) + rot / 2 : slot >> 1; }

  template <typename T> __device__ void load(const T* row, float (&a)[8], float (&b)[8]) const {
    if (vec) {
      if (halves()) {
        load8(row + 8 * u, a);
        load8(row + rot / 2 + 8 * u, b);
        return;
      }
      float v[2][8] = {};
      if (16 * u < dim) load8(row + 16 * u, v[0]);
      if (16 * u + 8 < dim) load8(row + 16 * u + 8, v[1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) { a[e] = v[e >> 2][2 * (e & 3)]; b[e] = v[e >> 2][2 * (e & 3) + 1]; }
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * u + 2 * e;
      a[e] = s < dim ? (float)row[element(s)] : 0.0f;
      b[e] = s + 1 < dim ? (float)row[element(s + 1)] : 0.0f;
    }
  }
  template <typename T> __device__ void store(T* row, const float (&a)[8], const float (&b)[8]) const {
    if (vec) {
      if (halves()) {
        store8(row + 8 * u, a);
        store8(row + rot / 2 + 8 * u, b);
        return;
      }
      float v[2][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[e >> 2][2 * (e & 3)] = a[e]; v[e >> 2][2 * (e & 3) + 1] = b[e]; }
      if (16 * u < dim) store8(row + 16 * u, v[0]);
      if (16 * u + 8 < dim) store8(row + 16 * u + 8, v[1]);
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

// cos and sin (times scale) of the unit's pairs at a position; pairs past the rotated part stay as they are
__device__ inline void angles(const NormRope& p, int u, int position, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c[e] = 1.0f;
    s[e] = 0.0f;
    if (16 * u + 2 * e < p.rot) {
      const double turns = (double)position * (double)p.inv_freq[8 * u + e] * 0.15915494309189535;   // 1 / (2 pi)
      float sn, cs;
      sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
      c[e] = cs * p.scale;
      s[e] = sn * p.scale;
    }
  }
}

template <int L> __device__ inline float over_lanes(float v) {
#pragma unroll
  for (int m = 1; m < L; m *= 2) v += __shfl_xor(v, m);
  return v;
}

__device__ inline void weights(const NormRope& p, const Unit& un, int kind, float (&wa)[8], float (&wb)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int s = 16 * un.u + 2 * e;
    wa[e] = p.w[kind] && s < p.dim ? p.w[kind][un.element(s)] : 1.0f;
    wb[e] = p.w[kind] && s + 1 < p.dim ? p.w[kind][un.element(s + 1)] : 1.0f;
  }
}

template <typename T, int L, int HS>
__global__ void __launch_bounds__(256) norm_rope_kernel(NormRope p) {
  unsigned it = blockIdx.x * (256 / L) + threadIdx.x / L;
  const int kind = it >= p.items[0];
  if (kind) it -= p.items[0];
  if (it >= p.items[kind]) return;             // whole heads leave: the sum below is over the lanes of one
  const Unit un = {(int)threadIdx.x % L, p.dim, p.rot, !p.interleaved, p.vec};
  const unsigned token = it / p.groups[kind];
  const int h0 = (it - token * p.groups[kind]) * HS, b = token / p.len, i = token - b * p.len;
  const T* x = (const T*)p.x[kind] + b * p.xs[kind][0] + i * p.xs[kind][1];
  T* out = (T*)p.out[kind] + b * p.os[kind][0] + i * p.os[kind][1];
  float va[HS][8], vb[HS][8], c[8], s[8], wa[8], wb[8];
#pragma unroll
  for (int h = 0; h < HS; ++h)
    if (h0 + h < p.heads[kind]) un.load(x + (h0 + h) * p.xs[kind][2], va[h], vb[h]);
  angles(p, un.u, p.pos ? p.pos[token] : p.start + i, c, s);
  weights(p, un, kind, wa, wb);
#pragma unroll
  for (int h = 0; h < HS; ++h) {
    if (h0 + h >= p.heads[kind]) break;
    float (&a)[8] = va[h], (&bb)[8] = vb[h];
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

template <typename T, int L, int HS>
__global__ void __launch_bounds__(256) norm_rope_backward_kernel(NormRope p) {
  const int kind = (int)blockIdx.x >= p.blocks_q, block = blockIdx.x - (kind ? p.blocks_q : 0), nblocks = kind ? gridDim.x - p.blocks_q : p.blocks_q;
  const Unit un = {(int)threadIdx.x % L, p.dim, p.rot, !p.interleaved, p.vec};
  float ga[8] = {}, gb[8] = {}, wa[8], wb[8];
  weights(p, un, kind, wa, wb);
  for (unsigned it = block * (256 / L) + threadIdx.x / L; it < p.items[kind]; it += nblocks * (256 / L)) {
    const unsigned token = it / p.groups[kind];
    const int h0 = (it - token * p.groups[kind]) * HS, b = token / p.len, i = token - b * p.len;
    const T* x = (const T*)p.x[kind] + b * p.xs[kind][0] + i * p.xs[kind][1];
    const T* dy = (const T*)p.dy[kind] + b * p.ds[kind][0] + i * p.ds[kind][1];
    T* out = (T*)p.out[kind] + b * p.os[kind][0] + i * p.os[kind][1];
    float xa[HS][8], xb[HS][8], da[HS][8], db[HS][8], c[8], s[8];
#pragma unroll
    for (int h = 0; h < HS; ++h)
      if (h0 + h < p.heads[kind]) {
        un.load(dy + (h0 + h) * p.ds[kind][2], da[h], db[h]);
        if (p.norm) un.load(x + (h0 + h) * p.xs[kind][2], xa[h], xb[h]);
      }
    angles(p, un.u, p.pos ? p.pos[token] : p.start + i, c, s);
#pragma unroll
    for (int h = 0; h < HS; ++h) {
      if (h0 + h >= p.heads[kind]) break;
      float (&a)[8] = da[h], (&bb)[8] = db[h];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = a[e] * c[e] + bb[e] * s[e];
        bb[e] = bb[e] * c[e] - a[e] * s[e];
        a[e] = t;
      }
      if (p.norm) {
        float q = 0.0f, d = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q += xa[h][e] * xa[h][e] + xb[h][e] * xb[h][e];
          d += a[e] * wa[e] * xa[h][e] + bb[e] * wb[e] * xb[h][e];
        }
        const float r = 1.0f / sqrtf(over_lanes<L>(q) / (float)p.dim + p.eps);
        const float m = over_lanes<L>(d) / (float)p.dim * r * r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ga[e] += a[e] * xa[h][e] * r;
          gb[e] += bb[e] * xb[h][e] * r;
          a[e] = r * (a[e] * wa[e] - xa[h][e] * m);
          bb[e] = r * (bb[e] * wb[e] - xb[h][e] * m);
        }
      }
      un.store(out + (h0 + h) * p.os[kind][2], a, bb);
    }
  }
  if (!p.norm || !p.part[kind]) return;
  // the heads of a workgroup in a fixed order, so that the same call gives the same bits
  __shared__ float sums[256 / L][16 * L + 1];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sums[threadIdx.x / L][16 * un.u + 2 * e] = ga[e];
    sums[threadIdx.x / L][16 * un.u + 2 * e + 1] = gb[e];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * L; t += 256) {
    float v = 0.0f;
    for (int r = 0; r < 256 / L; ++r) v += sums[r][t];
    p.part[kind][(size_t)block * (16 * L) + t] = v;
  }
}

// dw = the sum of the workgroups' partial sums; a workgroup takes 16 slots of the queries' (blockIdx.y = 0) or keys' weights
__global__ void __launch_bounds__(256) norm_rope_join_kernel(NormRope p, float* dqw, float* dkw, int blocks_k, int width) {
  const int kind = blockIdx.y, col = blockIdx.x * 16 + (threadIdx.x & 15), blocks = kind ? blocks_k : p.blocks_q;
  float* to = kind ? dkw : dqw;
  if (!to) return;
  __shared__ float sums[16][17];
  float v = 0.0f;
  for (int r = threadIdx.x >> 4; r < blocks; r += 16) v += p.part[kind][(size_t)r * width + col];
  sums[threadIdx.x >> 4][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x >= 16 || col >= p.dim) return;
  v = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) v += sums[r][threadIdx.x];
  const Unit un = {0, p.dim, p.rot, !p.interleaved, p.vec};
  to[un.element(col)] = v;
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

bool sizes_fit_vectors(const prism_norm_rope_desc& d) { return d.head_dim % 8 == 0 && (d.interleaved || d.rot_dim % 16 == 0); }

// Heads per lane: four share the sines of their token where that leaves the chip two waves per SIMD at least.
int heads_per_lane(const prism_norm_rope_desc& d, int L) {
  const long long waves = (long long)d.batch * d.len * (d.q_heads + d.k_heads) * L / 64;
  return waves >= 4 * 2048 ? 4 : 1;
}

void set_items(NormRope& p, const prism_norm_rope_desc& d, int HS) {
  for (int kind = 0; kind < 2; ++kind) {
    p.groups[kind] = p.heads[kind] ? (p.heads[kind] + HS - 1) / HS : 1;
    p.items[kind] = p.heads[kind] ? (unsigned)(d.batch * d.len) * (unsigned)p.groups[kind] : 0u;
  }
}

template <typename T, int L> void forward(NormRope& p, int HS, hipStream_t s) {
  const dim3 grid((unsigned)(((unsigned long long)p.items[0] + p.items[1] + 256 / L - 1) / (256 / L)));
  if (HS == 4) hipLaunchKernelGGL((norm_rope_kernel<T, L, 4>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((norm_rope_kernel<T, L, 1>), grid, dim3(256), 0, s, p);
}
template <typename T, int L> void backward(NormRope& p, int HS, int blocks_k, hipStream_t s) {
  const dim3 grid(p.blocks_q + blocks_k);
  if (HS == 4) hipLaunchKernelGGL((norm_rope_backward_kernel<T, L, 4>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((norm_rope_backward_kernel<T, L, 1>), grid, dim3(256), 0, s, p);
}
template <typename T> void by_lanes(NormRope& p, int L, int HS, int blocks_k, bool back, hipStream_t s) {
  if (L == 2) back ? backward<T, 2>(p, HS, blocks_k, s) : forward<T, 2>(p, HS, s);
  else if (L == 4) back ? backward<T, 4>(p, HS, blocks_k, s) : forward<T, 4>(p, HS, s);
  else if (L == 8) back ? backward<T, 8>(p, HS, blocks_k, s) : forward<T, 8>(p, HS, s);
  else back ? backward<T, 16>(p, HS, blocks_k, s) : forward<T, 16>(p, HS, s);
}

}  // namespace

int launch_norm_rope(const void* q, const void* k, void* qo, void* ko, int dt, const prism_norm_rope_desc& d, hipStream_t s) {
  ProfScope prof(PK_NORM_ROPE, s);
  NormRope p = common(q, k, d);
  const int size = dt == PRISM_F32 ? 4 : 2, L = lanes_of(d.head_dim), HS = heads_per_lane(d, L);
  p.out[0] = qo; p.out[1] = ko;
  strides(p.os[0], d.q_out); strides(p.os[1], d.k_out);
  p.vec = sizes_fit_vectors(d) && (!d.q_heads || (whole_vectors(q, d.q, size) && whole_vectors(qo, d.q_out, size))) &&
          (!d.k_heads || (whole_vectors(k, d.k, size) && whole_vectors(ko, d.k_out, size)));
  set_items(p, d, HS);
  if (dt == PRISM_F32) by_lanes<float>(p, L, HS, 0, false, s);
  else by_lanes<__bf16>(p, L, HS, 0, false, s);
  return PRISM_OK;
}

size_t norm_rope_backward_bytes(const prism_norm_rope_desc& d) {
  return d.norm ? (size_t)2 * NR_MAX_BLOCKS * 16 * lanes_of(d.head_dim) * sizeof(float) : 0;
}

int launch_norm_rope_backward(const void* dqo, const void* dko, const void* q, const void* k, void* dq, void* dk, float* dqw, float* dkw, int dt,
                              const prism_norm_rope_desc& d, float* part, hipStream_t s) {
  ProfScope prof(PK_NORM_ROPE_BACKWARD, s);
  NormRope p = common(q, k, d);
  const int size = dt == PRISM_F32 ? 4 : 2, L = lanes_of(d.head_dim), HS = heads_per_lane(d, L);
  p.dy[0] = dqo; p.dy[1] = dko;
  strides(p.ds[0], d.q_out); strides(p.ds[1], d.k_out);
  p.out[0] = dq; p.out[1] = dk;
  strides(p.os[0], d.dq); strides(p.os[1], d.dk);
  p.vec = sizes_fit_vectors(d) &&
          (!d.q_heads || ((!d.norm || whole_vectors(q, d.q, size)) && whole_vectors(dqo, d.q_out, size) && whole_vectors(dq, d.dq, size))) &&
          (!d.k_heads || ((!d.norm || whole_vectors(k, d.k, size)) && whole_vectors(dko, d.k_out, size) && whole_vectors(dk, d.dk, size)));
  set_items(p, d, HS);
  auto blocks = [&](int kind) {
    const long long n = ((long long)p.items[kind] + 256 / L - 1) / (256 / L);
    return (int)(n < NR_MAX_BLOCKS ? n : NR_MAX_BLOCKS);
  };
  p.blocks_q = blocks(0);
  const int blocks_k = blocks(1), width = 16 * L;
  if (d.norm) {
    p.part[0] = dqw ? part : nullptr;
    p.part[1] = dkw ? part + (size_t)NR_MAX_BLOCKS * width : nullptr;
  }
  if (dt == PRISM_F32) by_lanes<float>(p, L, HS, blocks_k, true, s);
  else by_lanes<__bf16>(p, L, HS, blocks_k, true, s);
  if (d.norm && (dqw || dkw)) hipLaunchKernelGGL(norm_rope_join_kernel, dim3(L, 2), dim3(256), 0, s, p, dqw, dkw, blocks_k, width);
  return PRISM_OK;
}

}  // namespace prism
