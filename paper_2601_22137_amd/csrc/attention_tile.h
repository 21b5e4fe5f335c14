// What the attention kernels share: tiles of rows in LDS, products of tiles in the layout of the matrix instructions, and the masks.
//
// Rows.  The query heads that share a key head are taken together: row r of a (sequence, key head) pair is token r / G of query head r % G of the
// group.  A wave has 32 of them (or 32 keys) and the 32 x 32 products put them on its lanes: register r of lane (n, h) = (l % 32, l / 32) holds
// entry (8 (r / 4) + 4 h + r % 4, n).  A score matrix computed that way is at once the second operand of the product that follows: the sum over its first index
// may run in any order, so the eight registers 8 s .. 8 s + 7 are taken as they lie, and the first operand is read to match.
#pragma once
#include "layer.h"
#include "tile_rows.h"

namespace prism {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef const void __attribute__((address_space(1)))* gptr_t;
typedef void __attribute__((address_space(3)))* lptr_t;

constexpr int NW = 4, NT = 64 * NW;       // waves and threads of a workgroup
constexpr float LOG2E = 1.4426950408889634f;

struct Attn {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  float* lse;                       // [batch][q_heads][q_len], natural logarithm
  const float* lse_in;
  long long qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];   // strides of batch, token, head
  int batch, n, m, hq, hk, G, dim;  // n queries, m keys
  int R, row_tiles;                 // rows of a pair: G n
  float scale, cap;
  int causal;
  const float* slopes;
  const int *prefix, *lens, *qdoc, *kdoc;
  const int4 *qrange, *krange;      // of the documents of 64 tokens: lowest, highest, whether a token without one is among them
  int nsplit;                       // parts of the keys of a row tile (forward, dq)
  int chunk, parts, items;          // dk, dv: see AttnPlan
  float *part, *part_ml;            // results of the parts
  bool direct;                      // rows are whole vectors of 16 bytes
  bool whole;                       // ... and the offsets within a tile fit 31 bits (dk, dv: of queries and dout)
  bool whole_keys;                  // backward: the same of keys and values
};

__device__ const unsigned zero_page[4] = {0, 0, 0, 0};

// f(0) .. f(D - 1), the numbers as types; in place whatever its size: its operands are registers
template <int D, typename F> __device__ __forceinline__ void steps(F&& f) {
  if constexpr (D > 0) {
    steps<D - 1>(f);
    f(std::integral_constant<int, D - 1>{});
  }
}

// f(e) for step x's share of TOTAL entries that are spread over N steps
template <int N, int TOTAL, int X, typename F> __device__ __forceinline__ void share(std::integral_constant<int, X>, F&& f) {
  constexpr int from = X * TOTAL / N, to = (X + 1) * TOTAL / N;
  steps<to - from>([&](auto e) __attribute__((always_inline)) { f(std::integral_constant<int, from + decltype(e)::value>{}); });
}

// The same value, computed again where it is used: what the rare branches of a loop derive from it is not kept in registers across the loop.
__device__ inline int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The value is there at this point of the program: a sum is not put off to where it is used.
__device__ inline void keep(float& a) { asm volatile("" : "+v"(a)); }

// Tiles of rows in LDS, of 64 or 128 elements, of which products take the first DP (the head size rounded up to 64, 96 or 128, fp32 also 32; entries past
// the head are zero), in chunks of 16 bytes.  2 x 4096 x 8 heads of 80, causal, bf16: 103 us and gradients 349 with products of 128 entries, 91 and 297 with 96.  Chunk c of row r lies at c ^ swizzle(r):
// the reads of 16 rows at one chunk (the operand as it is), of 4 rows at four chunks (the transposed one, bf16) and of two rows four apart (fp32) then fall on different banks.
template <typename T, int DP> struct Lds {
  static constexpr int RB = (DP > 64 ? 128 : 64) * (int)sizeof(T), CPR = RB / 16, EPC = 16 / (int)sizeof(T), STEPS = DP / EPC / 2;
  __device__ static int swizzle(int r) {
    if constexpr (CPR == 8) return ((r >> 2) & 3) | ((r >> 1) & 1) << 2;
    else if constexpr (sizeof(T) == 2) return ((r >> 2) & 3) | (r & 3) << 2;
    else return (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3;
  }
};

// A row in a lane's registers: chunk 2 s + h for step s
template <typename T, int DP> using Frag = u32x4[Lds<T, DP>::STEPS];

// ROWS rows into LDS; row(r) is the address of a row's first element, or null for a row of zeros.  `direct`: without passing through registers; the
// caller waits for vmcnt before the barrier.
template <typename T, int DP, int ROWS, typename F>
__device__ inline void load_tile(char* lds, bool direct, int dim, int tid, F&& row) {
  using L = Lds<T, DP>;
  tid = here(tid);
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int u = 0; u < ROWS * L::CPR / NT; ++u) {
    const int at = u * NT + tid, r = at / L::CPR, c = (at % L::CPR) ^ L::swizzle(r);
    const T* p = row(r);
    if (direct) {
      const void* src = p && c * L::EPC < dim ? (const void*)(p + c * L::EPC) : (const void*)zero_page;
      __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)(lds + (u * NW + wave) * 1024), 16, 0, 0);
    } else {
      union { T e[L::EPC]; u32x4 v; } x;
      x.v = (u32x4){0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < L::EPC; ++e)
        if (p && c * L::EPC + e < dim) x.e[e] = p[c * L::EPC + e];
      *(u32x4*)(lds + at * 16) = x.v;
    }
  }
}

template <int BYTES> __device__ inline void zero_tiles(char* lds, int tid) {
  for (int x = tid * 16; x < BYTES; x += NT * 16) *(u32x4*)(lds + x) = (u32x4){0, 0, 0, 0};
  __syncthreads();
}

// The same for whole tiles of rows.  The chunks of a thread lie a fixed number of rows apart: one offset and uniform steps (tile_rows.h) where the swizzle repeats at that
// distance, two offsets in turn for rows of 512 bytes (8 apart).  GROUPS: rows are heads of tokens; else every row is a token of its own.
template <typename T, int DP, int ROWS, bool GROUPS = false> struct Chunks {
  static constexpr int APART = NT / Lds<T, DP>::CPR, N = ROWS / APART, KINDS = APART < 16 ? 2 : 1;
  static_assert(N <= 4, "row_steps");
  unsigned at[KINDS];
  RowSteps steps;      // bytes
  bool any[KINDS];   // a chunk past the head's entries stays as zero_tiles has left it
  // row x is token x / G, head x % G (G divides 32) of the first row's token
  __device__ void set(int tid, int G, long long token, long long head, int dim) {
    using L = Lds<T, DP>;
    const int r = tid / L::CPR;
#pragma unroll
    for (int k = 0; k < KINDS; ++k) {
      const int c = (tid % L::CPR) ^ L::swizzle(r + k * APART);
      any[k] = c * L::EPC < dim;
      at[k] = (unsigned)row_offset(r, G, token, head) * (unsigned)sizeof(T) + (c << 4);
    }
    steps = row_steps(APART, G, token * (long long)sizeof(T), head * (long long)sizeof(T));
  }
  __device__ void load(char* lds, const char* base, int wave) const {
#pragma unroll
    for (int k = 0; k < KINDS; ++k) {
      // uniform address plus 32-bit offset: added by the load itself, not kept as an address per lane
      const unsigned off = (unsigned)here((int)at[k]);
      if (any[k])
#pragma unroll
        for (int u = k; u < N; u += KINDS) {
          const __attribute__((address_space(1))) char* from = (const __attribute__((address_space(1))) char*)(base + (GROUPS && N > 2 ? steps.to(u) : u * steps.one));
          __builtin_amdgcn_global_load_lds((gptr_t)(from + off), (lptr_t)(lds + (u * NW + wave) * 1024), 16, 0, 0);
        }
    }
  }
};

typedef const u32x4 __attribute__((address_space(3)))* lds16_t;
__device__ inline u32x4 lds_read16(unsigned a) { return *(lds16_t)a; }
__device__ inline unsigned lds_address(const char* p) { return (unsigned)(size_t)(const __attribute__((address_space(3))) char*)p; }

// The chunks of columns_by in bf16 at their LDS addresses: 8 + 8 rows of four columns' neighbours, transposed
__device__ inline bf16x8 lds_read_columns(unsigned a0, unsigned a1) {
  union { s16x4 q[2]; bf16x8 v; } a;
  a.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a0);
  a.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a1);
  return a.v;
}

// The documents of 64 tokens from `at` on, by one wave
__device__ inline void load_ids(int* lds, const int* doc, int at, int len, int lane) {
  if (at + 64 <= len) {
    const __attribute__((address_space(1))) char* from = (const __attribute__((address_space(1))) char*)(doc + at);
    __builtin_amdgcn_global_load_lds((gptr_t)(from + (unsigned)here(lane) * 4), (lptr_t)lds, 4, 0, 0);
  } else {
    lds[lane] = at + lane < len ? doc[at + lane] : -1;
  }
}

// One row as a lane's operand
template <typename T, int DP>
__device__ inline void load_row(Frag<T, DP>& f, bool direct, int dim, int h, const T* p) {
  using L = Lds<T, DP>;
#pragma unroll
  for (int s = 0; s < L::STEPS; ++s) {
    const int c = 2 * s + h;
    if (direct) {
      f[s] = (u32x4){0, 0, 0, 0};
      if (p && c * L::EPC < dim) f[s] = *(const u32x4*)(p + c * L::EPC);
    } else {
      union { T e[L::EPC]; u32x4 v; } x;
      x.v = (u32x4){0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < L::EPC; ++e)
        if (p && c * L::EPC + e < dim) x.e[e] = p[c * L::EPC + e];
      f[s] = x.v;
    }
  }
}

// c += A B over one chunk of each operand: 16 products of the sum in bf16, 8 in fp32
template <typename T> __device__ inline f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
    return c;
  }
}

// (32 rows of the tile from row0 on) x (the rows held as f): register r of lane (n, h) gets row 8 (r / 4) + 4 h + r % 4 against row n of f
template <typename T, int DP>
__device__ inline f32x16 rows_by_rows(const char* lds, int row0, const Frag<T, DP>& f, int lane) {
  using L = Lds<T, DP>;
  const int r = lane & 31, h = lane >> 5;
  f32x16 c = {};
#pragma unroll
  for (int s = 0; s < L::STEPS; ++s) {
    const u32x4 a = *(const u32x4*)(lds + (row0 + r) * L::RB + (((2 * s + h) ^ L::swizzle(r)) << 4));
    c = mma<T>(a, f[s], c);
  }
  return c;
}

// acc[t] += (columns 32 t .. of 32 rows of the tile, transposed) x p: entry (d, n) gets sum over the rows of tile[row][d] p[row][n].  p is rounded to the
// tile's type: in bf16 its relative error of 2^-9 is that of the results themselves.
template <typename T, int DP>
__device__ inline void columns_by(f32x16 (&acc)[DP / 32], const char* lds, int row0, const f32x16& p, int lane) {
  using L = Lds<T, DP>;
  const int h = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int i = lane & 15, mb = (lane >> 4) & 1;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 b;
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = (__bf16)p[8 * s + e];
      const int r0 = 4 * h + (i >> 2), r1 = r0 + 8;              // of 16 rows
#pragma unroll
      for (int t = 0; t < DP / 32; ++t) {
        const int c = 4 * t + 2 * mb + ((i & 3) >> 1);
        const char* a0 = lds + (row0 + 16 * s + r0) * L::RB + ((c ^ L::swizzle(r0)) << 4) + 8 * (i & 1);
        const char* a1 = lds + (row0 + 16 * s + r1) * L::RB + ((c ^ L::swizzle(r1)) << 4) + 8 * (i & 1);
        union { s16x4 q[2]; bf16x8 v; } a;
        a.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a0);
        a.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a1);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b, acc[t], 0, 0, 0);
      }
    }
  } else {
    const int n = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r >> 2) + 4 * h + (r & 3);
#pragma unroll
      for (int t = 0; t < DP / 32; ++t) {
        const float a = *(const float*)(lds + (row0 + row) * L::RB + (((8 * t + (n >> 2)) ^ L::swizzle(row)) << 4) + 4 * (n & 3));
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[r], acc[t], 0, 0, 0);
      }
    }
  }
}

// The largest (NaN if one is): the one instruction that needs no quieting of its operands first
__device__ inline float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float max_of(float a, float b, float c) { return max_of(max_of(a, b), c); }

__device__ inline float other_half(float x) {   // the value of lane l ^ 32
  return __shfl_xor(x, 32);
}

// 1 - 2 / (1 + e^2x): an absolute error of 1e-7, of a score the cap times that.  SERIES: near zero the odd series (to x^13: 2e-9 at 0.3), so that the error is some units of
// the score itself whatever the cap: in fp32 always, in bf16 above caps of CAP_SERIES (up to it, 1e-7 of the cap is a sixteenth of the weights' own rounding at most).
// bf16, 2 x 4096 tokens, 16 heads of 128 on 4, causal: forward 214 us without and 236 with the series, gradients 715 and 1552 (dk and dv then spill 228 bytes a work-item).
constexpr float CAP_SERIES = 1024.0f;
template <bool SERIES> __device__ inline float tanh_of(float x) {
  const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * (2.0f * LOG2E)));
  if constexpr (!SERIES) return t;
  const float y = x * x;
  float s = 21844.0f / 6081075.0f;
  s = s * y - 1382.0f / 155925.0f;
  s = s * y + 62.0f / 2835.0f;
  s = s * y - 17.0f / 315.0f;
  s = s * y + 2.0f / 15.0f;
  s = s * y - 1.0f / 3.0f;
  return fabsf(x) < 0.3f ? x + x * y * s : t;
}

// What a query sees: keys up to `last` (causal, prefix and length in one number) of its own document.
struct Row {
  int at;      // its place among the keys
  int last;    // the last key that it may see, -1: none
  int doc;     // its document; without documents 0
  float slope; // log2(e) times that of its head
};

// 0 for rows there are not, before the first one too: a key tile without rows asks for the one before its range
__device__ inline int doc_of_row(const Attn& p, int b, int r) { return p.qdoc && r >= 0 && r < p.R ? p.qdoc[(long long)b * p.n + r / p.G] : 0; }

__device__ inline Row row_of(const Attn& p, int b, int kh, int r, int keys, int doc) {
  Row w;
  w.at = 0; w.last = -1; w.doc = -2; w.slope = 0.0f;
  if (r < p.R) {
    const int i = r / p.G, g = r - i * p.G;
    w.at = i + keys - p.n;
    int last = keys - 1;
    if (p.causal) {
      last = min(last, w.at);
      if (p.prefix) last = max(last, min(p.prefix[b], keys) - 1);
    }
    w.last = max(last, -1);
    w.doc = doc;
    if (doc < 0) { w.doc = -2; w.last = -1; }
    if (p.slopes) w.slope = p.slopes[kh * p.G + g] * LOG2E;
  }
  return w;
}

__device__ inline Row row_of(const Attn& p, int b, int kh, int r, int keys) { return row_of(p, b, kh, r, keys, doc_of_row(p, b, r)); }

__device__ inline int keys_of(const Attn& p, int b) { return p.lens ? min(max(p.lens[b], 0), p.m) : p.m; }

// Workgroups of one pair are neighbours on one XCD (workgroup id modulo 8), whose L2 then holds the pair's keys and values for all of them.
__device__ inline int place(int id, int total) {
  const int xcd = id & 7, q = total >> 3, rem = total & 7;
  return xcd * q + min(xcd, rem) + (id >> 3);
}

template <typename T> __device__ inline void store4(T* p, f32x4 v, bool whole, int count) {
  if constexpr (sizeof(T) == 2) {
    bf16x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (__bf16)v[e];
    if (whole) { *(bf16x4*)p = x; return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) p[e] = x[e];
  } else {
    if (whole) { *(f32x4*)p = v; return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) p[e] = v[e];
  }
}

// acc[t] register r of lane (n, h) is entry 32 t + 8 (r / 4) + 4 h + r % 4 of the row that starts at `to`
template <typename T, int DP>
__device__ inline void store_row(T* to, const f32x16 (&acc)[DP / 32], float factor, int dim, bool direct, int h) {
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * t + 8 * g + 4 * h;
      if (d >= dim) continue;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[t][4 * g + e] * factor;
      store4<T>(to + d, v, direct, dim - d);
    }
}

inline void set_strides(long long (&to)[3], const prism_strides& s) { to[0] = s.batch; to[1] = s.token; to[2] = s.head; }

// keys (forward, dq) or rows (dk, dv) of a tile in LDS
template <typename T> constexpr int key_tile() { return sizeof(T) == 2 ? 64 : 32; }

// What the rows of a wave see, and of its workgroup
struct Limits {
  int last, first;           // the largest and (of the rows there are) the smallest last key
  int lo, hi;                // lowest and highest document
  bool mixed;                // whether the rows are of more than one document, or of none
};

__device__ inline Limits limits_of(const Attn& p, const Row& w, int b, int kh, int r, int keys) {
  Limits x;
  if (!p.qdoc) {     // what a row sees grows with its token: the wave's first and last row say it all
    const int r0 = __builtin_amdgcn_readfirstlane(r);
    x.first = r0 < p.R ? row_of(p, b, kh, r0, keys, 0).last : 0x7FFFFFFF;
    x.last = r0 < p.R ? row_of(p, b, kh, min(r0 + 31, p.R - 1), keys, 0).last : -1;
    x.lo = x.hi = 0;
    x.mixed = false;
    return x;
  }
  x.last = w.last;
  x.first = r < p.R ? w.last : 0x7FFFFFFF;
  x.lo = r < p.R && w.doc >= 0 ? w.doc : 0x7FFFFFFF;
  x.hi = r < p.R ? w.doc : -2;
  int none = r < p.R && w.doc < 0;
#pragma unroll
  for (int m = 1; m < 32; m *= 2) {
    x.last = max(x.last, __shfl_xor(x.last, m));
    x.first = min(x.first, __shfl_xor(x.first, m));
    x.lo = min(x.lo, __shfl_xor(x.lo, m));
    x.hi = max(x.hi, __shfl_xor(x.hi, m));
    none |= __shfl_xor(none, m);
  }
  x.last = __builtin_amdgcn_readfirstlane(x.last);
  x.first = __builtin_amdgcn_readfirstlane(x.first);
  x.lo = __builtin_amdgcn_readfirstlane(x.lo);
  x.hi = __builtin_amdgcn_readfirstlane(x.hi);
  x.mixed = __builtin_amdgcn_readfirstlane(none) || x.lo != x.hi;
  return x;
}

// The key tiles [all0, all1) that the rows of row tile `tile` see, and [t0, t1), part `split` of them; all threads call it
template <int KT>
__device__ inline void key_range(const Attn& p, const Limits& lim, int b, int kh, int tile, int keys, int split, int* sh, int& all0, int& all1, int& t0, int& t1) {
  int first_tile = 0, end_tile = 0;
  if (!p.kdoc) {
    end_tile = (row_of(p, b, kh, min(tile * 128 + 127, p.R - 1), keys, 0).last + KT) / KT;
  } else {           // from the first to the last block of 64 keys with one of the workgroup's documents
    if (threadIdx.x < 5) sh[threadIdx.x] = threadIdx.x == 1 || threadIdx.x == 3 ? 0x7FFFFFFF : -1;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      atomicMax(&sh[0], lim.last);
      atomicMin(&sh[1], lim.lo);
      atomicMax(&sh[2], lim.hi);
    }
    __syncthreads();
    const int last = sh[0], lo = sh[1], hi = sh[2];
    const int blocks = (p.m + 63) / 64, upto = last < 0 ? -1 : last / 64;
    int f = 0x7FFFFFFF, e = -1;
    for (int x = threadIdx.x; x <= upto; x += NT) {
      const int4 k = p.krange[(long long)b * blocks + x];
      if (k.x <= hi && k.y >= lo) { f = min(f, x); e = max(e, x); }
    }
    if (e >= 0) { atomicMin(&sh[3], f); atomicMax(&sh[4], e); }
    __syncthreads();
    if (sh[4] >= 0) {
      first_tile = sh[3] * 64 / KT;
      end_tile = min(last / KT + 1, (sh[4] + 1) * 64 / KT);
    }
  }
  all0 = __builtin_amdgcn_readfirstlane(first_tile);
  all1 = __builtin_amdgcn_readfirstlane(max(end_tile, first_tile));
  const int per = (all1 - all0 + p.nsplit - 1) / p.nsplit;
  t0 = min(all0 + split * per, all1);
  t1 = min(all0 + (split + 1) * per, all1);
}

// Documents of a block of 64 tokens: lowest, highest, whether one of none is among them.  Read through the scalar cache: a vector load would have to wait for the
// tiles on their way.
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef const i32x4 __attribute__((address_space(4)))* range_ptr;
__device__ inline int4 range_of(const int4* ranges, long long block) {
  const i32x4 x = *(range_ptr)(ranges + block);
  return make_int4(x[0], x[1], x[2], x[3]);
}
template <int KT> __device__ inline int4 key_docs(const Attn& p, int b, int t) {
  return p.kdoc ? range_of(p.krange, (long long)b * ((p.m + 63) / 64) + t * KT / 64) : make_int4(0, 0, 0, 0);
}

// Whether the wave's rows see any key of tile t, whose documents are k, and whether its scores have to be masked
template <int KT> __device__ inline bool tile_seen(const Attn& p, const Limits& lim, const int4& k, int t, bool& need) {
  need = t * KT + KT - 1 > lim.first;
  if (t * KT > lim.last) return false;
  if (p.kdoc) {
    if (k.x > lim.hi || k.y < lim.lo) return false;
    need = need || lim.mixed || k.z || k.x != k.y || k.x != lim.lo;
  }
  return true;
}

// Products q.k to what the exponent takes: without cap and bias they stay (the factor is applied with the exponent), else times log2(e), capped, biased.
// Register r is key j + 8 (r / 4) + r % 4.
template <bool SERIES>
__device__ inline void scores(const Attn& p, f32x16& s, const Row& w, int j, bool cap, bool bias, float in, float out) {
  if (cap) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = out * tanh_of<SERIES>(s[e] * in);
  } else if (bias) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] *= in;
  }
  if (bias) {
    const float far = (float)(w.at - j);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] -= w.slope * fabsf(far - (float)(8 * (e >> 2) + (e & 3)));
  }
}

// Rows that may see one of the 128 keys of a tile, at most; and the parts that they are cut into, alike up to a tile
__host__ __device__ inline long long rows_of_key_tile(bool causal, bool prefix, int n, int m, int G, int tile) {
  const long long hidden = causal && !prefix ? tile * 128ll - m + n : 0;
  return G * (hidden < 0 ? n : hidden > n ? 0 : n - hidden);
}
__host__ __device__ inline int parts_of(long long rows, int chunk) { return chunk && rows > chunk ? (int)((rows + chunk - 1) / chunk) : 1; }

// ---- host

inline bool rows_are_vectors(const void* p, const prism_strides& s, int dt) {
  const int size = dt == PRISM_F32 ? 4 : 2;
  return (((uintptr_t)p | (uintptr_t)(s.batch * size) | (uintptr_t)(s.token * size) | (uintptr_t)(s.head * size)) & 15) == 0;
}

inline Attn attn_common(const void* q, const void* k, const void* v, int dt, const prism_attention_desc& d, char* ws) {
  Attn p = {};
  p.q = q; p.k = k; p.v = v;
  set_strides(p.qs, d.q); set_strides(p.ks, d.k); set_strides(p.vs, d.v);
  p.batch = d.batch; p.n = d.q_len; p.m = d.k_len; p.hq = d.q_heads; p.hk = d.k_heads; p.G = d.q_heads / d.k_heads; p.dim = d.head_dim;
  p.R = p.G * p.n;
  p.row_tiles = (p.R + 127) / 128;
  p.scale = d.scale; p.cap = d.softcap; p.causal = d.causal;
  p.slopes = d.slopes; p.prefix = d.prefix; p.lens = d.k_lens; p.qdoc = d.q_doc; p.kdoc = d.k_doc;
  p.qrange = (const int4*)ws;
  p.krange = p.qrange + (long long)d.batch * ((d.q_len + 63) / 64);
  p.direct = d.head_dim * (dt == PRISM_F32 ? 4 : 2) % 16 == 0 && rows_are_vectors(q, d.q, dt) && rows_are_vectors(k, d.k, dt) && rows_are_vectors(v, d.v, dt);
  const long long widest = d.k.token > d.v.token ? d.k.token : d.v.token;
  p.whole = p.direct && widest < (1ll << 22);
  return p;
}

}  // namespace
}  // namespace prism
