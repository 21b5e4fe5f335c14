// Gradients of attention (attention.hip): with p = exp(score - lse), dp = dout.v and the row sums D = sum dout out
//
//   ds = p (dp - D) (1 - tanh^2) scale,   dq = ds k,   dk = ds^T q,   dv = p^T dout
//
// Two kernels that both compute the scores again: one walks the keys for 128 rows (dq), one the rows for 128 keys (dk, dv; all heads of the group, so
// shared heads need no sum afterwards).  Seven products instead of five, but no sum across workgroups whose order could change the bits of dq.
//
// Scores, dp, D and all sums are held in 32 bits; p and ds are rounded to the operands' type for the products that follow, as results are.  2 x 4096 tokens, 16 heads of 128 on 4, causal,
// capped, bf16: dq 310 us (three transcendental instructions a score, exp2 and rcp for the tanh, exp2 for the weight: vector units busy 76 % of the cycles, matrix units 37), dk and dv 480
// and 25 for the sum of their parts (matrix units 33 %, vector units 53; the waves wait for data or a barrier 36 % of their cycles); 2 x 1111, 8 heads of 80 with prefix and bias in fp32:
// 117 and 164 (matrix units 53 and 48 %, one wave per SIMD).
#include "attention_tile.h"

namespace prism {
namespace {

// 1 - tanh^2 from a capped score (times log2 e, before its bias)
__device__ inline float slope_of_cap(float capped, float per) {
  const float t = capped * per;
  return 1.0f - t * t;
}

__device__ inline float lse2_of(const Attn& p, int b, int i, int head, int r) {
  if (r >= p.R) return INFINITY;
  const float lse = p.lse_in[((long long)b * p.hq + head) * p.n + i];
  return lse == -INFINITY ? INFINITY : lse * LOG2E;
}

// A row that sees nothing has no gradient whatever its query and its dout hold
template <typename T, int DP> __device__ inline void clear_unseeing(Frag<T, DP>& f, float lse2) {
#pragma unroll
  for (int s = 0; s < Lds<T, DP>::STEPS; ++s)
    if (lse2 == INFINITY) f[s] = (u32x4){0, 0, 0, 0};
}

// ... and its token's block of documents is marked as one with a query of none, for dk and dv (every workgroup that writes there writes the same)
__device__ inline void mark_unseeing(const Attn& p, float lse2, int b, int i) {
  if (p.qdoc && lse2 == INFINITY) ((int*)(p.qrange + (long long)b * ((p.n + 63) / 64) + i / 64))[2] = 1;
}

// A lane's share of the product of two rows
template <typename T, int DP> __device__ inline float product_with_row(const Frag<T, DP>& f, const Attn& p, const T* row, int h) {
  using L = Lds<T, DP>;
  Frag<T, DP> o;
  load_row<T, DP>(o, p.direct, p.dim, h, row);
  float d = 0.0f;
#pragma unroll
  for (int s = 0; s < L::STEPS; ++s) {
    union { u32x4 v; T e[L::EPC]; } x, y;
    x.v = o[s];
    y.v = f[s];
#pragma unroll
    for (int e = 0; e < L::EPC; ++e) d += (float)x.e[e] * (float)y.e[e];
  }
  return d;
}

// Also, by the first part of a row tile's keys: stat[pair][0][r] = log2 of the row's sum of weights, +inf where the row sees nothing (its weights are then 0
// everywhere), and stat[pair][1][r] = D, for dk and dv.  (fp32)  Two waves per SIMD where that needs no spill: heads up to 64; with heads of 80 to 96 252 bytes of scratch made both
// gradients of 2 x 2048 x 8 heads of 80 545 -> 764 us.
template <typename T, int DP>
__global__ void __launch_bounds__(NT, DP <= 64 ? 2 : 1) attention_dq_kernel(Attn p, float* stat) {
  using L = Lds<T, DP>;
  constexpr int KT = key_tile<T>(), KB = KT / 32, TB = KT * L::RB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // keys and values, two tiles of each
  __shared__ __attribute__((aligned(16))) int kd[2][KT];
  __shared__ int shared_range[5];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  int id = place(blockIdx.x, gridDim.x);
  const int split = id % p.nsplit;
  id /= p.nsplit;
  const int tile = p.row_tiles - 1 - id % p.row_tiles, pair = id / p.row_tiles, b = pair / p.hk, kh = pair - b * p.hk;
  const int keys = keys_of(p, b), r = tile * 128 + wave * 32 + (lane & 31);
  const Row w = row_of(p, b, kh, r, keys);
  const Limits lim = limits_of(p, w, b, kh, r, keys);
  int all0, all1, t0, t1;
  key_range<KT>(p, lim, b, kh, tile, keys, split, shared_range, all0, all1, t0, t1);
  const int i = r / p.G, head = kh * p.G + r - i * p.G;
  const bool any = w.last >= 0;
  Frag<T, DP> qf, dof;
  load_row<T, DP>(dof, p.direct, p.dim, h, any ? (const T*)p.dout + b * p.dos[0] + i * p.dos[1] + head * p.dos[2] : nullptr);
  stat += (long long)pair * 2 * p.R;
  const float lse2 = lse2_of(p, b, i, head, r);
  float delta = product_with_row<T, DP>(dof, p, any ? (const T*)p.o + b * p.os[0] + i * p.os[1] + head * p.os[2] : nullptr, h);
  delta += other_half(delta);
  if (lse2 == INFINITY) delta = 0.0f;
  if (split == 0 && h == 0 && r < p.R) {
    stat[r] = lse2;
    stat[p.R + r] = delta;
    mark_unseeing(p, lse2, b, i);
  }
  load_row<T, DP>(qf, p.direct, p.dim, h, any ? (const T*)p.q + b * p.qs[0] + i * p.qs[1] + head * p.qs[2] : nullptr);
  clear_unseeing<T, DP>(dof, lse2);
  clear_unseeing<T, DP>(qf, lse2);
  const T* kbase = (const T*)p.k + b * p.ks[0] + kh * p.ks[2];
  const T* vbase = (const T*)p.v + b * p.vs[0] + kh * p.vs[2];
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  auto seen = [&](int j) { return j < keys && !(kdoc && kdoc[j] < 0); };
  Chunks<T, DP, KT> kat, vat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole_keys) {
    kat.set(tid, 1, p.ks[1], 0, p.dim);
    vat.set(tid, 1, p.vs[1], 0, p.dim);
  }
  auto issue = [&](int t, int buf) {
    if (p.whole_keys && !kdoc && (t + 1) * KT <= keys) {
      kat.load(smem + buf * TB, (const char*)(kbase + (long long)t * KT * p.ks[1]), wave);
      vat.load(smem + (2 + buf) * TB, (const char*)(vbase + (long long)t * KT * p.vs[1]), wave);
      return;
    }
    load_tile<T, DP, KT>(smem + buf * TB, p.direct, p.dim, tid, [&](int x) { const int j = t * KT + x; return seen(j) ? kbase + j * p.ks[1] : nullptr; });
    load_tile<T, DP, KT>(smem + (2 + buf) * TB, p.direct, p.dim, tid, [&](int x) { const int j = t * KT + x; return seen(j) ? vbase + j * p.vs[1] : nullptr; });
    if (kdoc && tid < KT) kd[buf][tid] = t * KT + tid < keys ? kdoc[t * KT + tid] : -1;
  };
  f32x16 acc[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) acc[t] = (f32x16){};
  const bool cap = p.cap > 0.0f, bias = p.slopes != nullptr;
  const float mul = cap || bias ? 1.0f : p.scale * LOG2E, in = cap ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E, per = cap ? 1.0f / out : 0.0f;
  if (t0 < t1) issue(t0, 0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1, j0 = t * KT;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
    if (t + 1 < t1) issue(t + 1, buf ^ 1);
    bool need;
    if (!tile_seen<KT>(p, lim, key_docs<KT>(p, b, t), t, need)) continue;
    const char *kt = smem + buf * TB, *vt = smem + (2 + buf) * TB;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 s = rows_by_rows<T, DP>(kt, 32 * kb, qf, lane);
      f32x16 ds = rows_by_rows<T, DP>(vt, 32 * kb, dof, lane);
      if (cap) scores<true>(p, s, w, 0, true, false, in, out);
      f32x16 f = s;                                          // capped, not yet biased
      if (bias) scores<true>(p, s, w, j0 + 32 * kb + 4 * h, false, true, cap ? 1.0f : in, out);
      if (need) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int j = 8 * g + 4 * h + 32 * kb;
          int4 d = make_int4(w.doc, w.doc, w.doc, w.doc);
          if (kdoc) d = *(const int4*)&kd[buf][j];
          const int dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * g + e] = j0 + j + e <= w.last && dd[e] == w.doc ? s[4 * g + e] : -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ds[e] = __builtin_amdgcn_exp2f(s[e] * mul - lse2) * (ds[e] - delta);
        if (cap) ds[e] *= slope_of_cap(f[e], per);
      }
      columns_by<T, DP>(acc, kt, 32 * kb, ds, lane);
    }
  }
  if (r >= p.R) return;
  if (p.nsplit == 1)
    store_row<T, DP>((T*)p.dq + b * p.dqs[0] + i * p.dqs[1] + head * p.dqs[2], acc, p.scale, p.dim, p.direct, h);
  else
    store_row<float, DP>(p.part + (((long long)split * p.batch * p.hk + pair) * p.R + r) * p.dim, acc, p.scale, p.dim, p.direct, h);
}

// The same in bf16.  A tile of 64 keys is taken as two blocks: scores K Q^T and dp = V dO^T of the first, with its exponentials beside the latter; the scores of the second beside
// ds of the first; dq; and so on.  D from the rounded `out` is off by 2^-9 of it, which shows where a row sees few keys (elsewhere in the mean over the keys it does not): a
// workgroup that sees eight tiles at most takes D = sum p dp, in a walk of its own through them.  (Packed documents of 8 x 1024, 12 heads of 64: 45 us, in two launches 54.)
template <int DP, bool CAP, bool BIAS, bool SERIES>
__global__ void __launch_bounds__(NT, 2) attention_dq_bf16_kernel(Attn p, float* stat) {
  typedef __bf16 T;
  using L = Lds<T, DP>;
  constexpr int KT = 64, TB = KT * L::RB, TD = DP / 32, STEPS = L::STEPS, AHEAD = 4;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // keys and values, two tiles of each
  __shared__ __attribute__((aligned(16))) int kd[2][KT];
  __shared__ int shared_range[5];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  int id = place(blockIdx.x, gridDim.x);
  const int split = id % p.nsplit;
  id /= p.nsplit;
  const int tile = p.row_tiles - 1 - id % p.row_tiles, pair = id / p.row_tiles, b = pair / p.hk, kh = pair - b * p.hk;
  const int keys = keys_of(p, b), r = tile * 128 + wave * 32 + (lane & 31);
  const Row w = row_of(p, b, kh, r, keys);
  const Limits lim = limits_of(p, w, b, kh, r, keys);
  int all0, all1, t0, t1;
  key_range<KT>(p, lim, b, kh, tile, keys, split, shared_range, all0, all1, t0, t1);
  const int i = r / p.G, head = kh * p.G + r - i * p.G;
  const bool any = w.last >= 0;
  Frag<T, DP> qf, dof;
  load_row<T, DP>(dof, p.direct, p.dim, h, any ? (const T*)p.dout + b * p.dos[0] + i * p.dos[1] + head * p.dos[2] : nullptr);
  stat += (long long)pair * 2 * p.R;
  const float lse2 = lse2_of(p, b, i, head, r);
  float delta = 0.0f;
  const bool exact = all1 - all0 <= 8;
  if (!exact) delta = product_with_row<T, DP>(dof, p, any ? (const T*)p.o + b * p.os[0] + i * p.os[1] + head * p.os[2] : nullptr, h);
  load_row<T, DP>(qf, p.direct, p.dim, h, any ? (const T*)p.q + b * p.qs[0] + i * p.qs[1] + head * p.qs[2] : nullptr);
  clear_unseeing<T, DP>(dof, lse2);
  clear_unseeing<T, DP>(qf, lse2);
  const T* kbase = (const T*)p.k + b * p.ks[0] + kh * p.ks[2];
  const T* vbase = (const T*)p.v + b * p.vs[0] + kh * p.vs[2];
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  Chunks<T, DP, KT> kat, vat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole_keys) {
    kat.set(tid, 1, p.ks[1], 0, p.dim);
    vat.set(tid, 1, p.vs[1], 0, p.dim);
  }
  auto issue = [&](int t, bool hidden, int buf) __attribute__((always_inline)) {
    auto seen = [&](int j) { return j < keys && !(kdoc && kdoc[j] < 0); };
    if (p.whole_keys && !hidden && (t + 1) * KT <= keys) {
      kat.load(smem + buf * TB, (const char*)(kbase + (long long)t * KT * p.ks[1]), wave);
      vat.load(smem + (2 + buf) * TB, (const char*)(vbase + (long long)t * KT * p.vs[1]), wave);
    } else {
      load_tile<T, DP, KT>(smem + buf * TB, p.direct, p.dim, tid, [&](int x) { const int j = t * KT + x; return seen(j) ? kbase + j * p.ks[1] : nullptr; });
      load_tile<T, DP, KT>(smem + (2 + buf) * TB, p.direct, p.dim, tid, [&](int x) { const int j = t * KT + x; return seen(j) ? vbase + j * p.vs[1] : nullptr; });
    }
    if (kdoc && wave == 0) load_ids(kd[buf], kdoc, t * KT, p.m, lane);
  };
  f32x16 acc[TD];
#pragma unroll
  for (int t = 0; t < TD; ++t) acc[t] = (f32x16){};
  const float in = CAP ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E;
  const unsigned lds0 = lds_address(smem), ka = lds0 + (lane & 31) * L::RB + ((h ^ L::swizzle(lane & 31)) << 4);
  const int cr = 4 * h + ((lane & 15) >> 2), cc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const unsigned ca = lds0 + cr * L::RB + ((cc ^ L::swizzle(cr)) << 4) + 8 * (lane & 1);
  // walk through tiles [t0, t1), for D or for dq
  auto walk = [&](auto for_delta, int t0, int t1) {
    constexpr bool DELTA = decltype(for_delta)::value;
    constexpr int NC = DELTA ? 0 : 2 * TD;
    int4 docs = make_int4(0, 0, 0, 0);
    if (t0 < t1) {
      docs = key_docs<KT>(p, b, t0);
      issue(t0, docs.z, 0);
    }
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1, j0 = t * KT;
      const int4 after = key_docs<KT>(p, b, min(t + 1, t1 - 1));
      __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
      __syncthreads();
      if (t + 1 < t1) issue(t + 1, after.z, buf ^ 1);
      bool need;
      const bool some = tile_seen<KT>(p, lim, docs, t, need);
      docs = after;
      if (!some) continue;
      const unsigned at = buf * TB;
      // operands in the order of their use: rows of K and of V of the first block, rows of K of the second, columns of K of the first, rows of V and columns of K of the second
      auto read = [&](auto xt) -> u32x4 {
        constexpr int x = decltype(xt)::value, S = STEPS;
        if constexpr (x < S) return lds_read16((ka ^ (x << 5)) + at);
        else if constexpr (x < 2 * S) return lds_read16((ka ^ ((x - S) << 5)) + at + 2 * TB);
        else if constexpr (x < 3 * S) return lds_read16((ka ^ ((x - 2 * S) << 5)) + at + 32 * L::RB);
        else if constexpr (x >= 3 * S + NC && x < 4 * S + NC) return lds_read16((ka ^ ((x - 3 * S - NC) << 5)) + at + 2 * TB + 32 * L::RB);
        else {
          constexpr bool second = x >= 4 * S + NC;
          constexpr int y = second ? x - 4 * S - NC : x - 3 * S, z = (y / TD * 16 + (second ? 32 : 0)) * L::RB;
          return __builtin_bit_cast(u32x4, lds_read_columns((ca ^ (y % TD << 6)) + at + z, (ca ^ (y % TD << 6) ^ 32) + at + z + 8 * L::RB));
        }
      };
      constexpr int N = 4 * STEPS + 2 * NC;
      u32x4 op[N];
      auto next = [&](auto xt) {
        constexpr int x = decltype(xt)::value;
        if constexpr (x + AHEAD < N) op[x + AHEAD] = read(std::integral_constant<int, x + AHEAD>{});
        return op[x];
      };
      steps<AHEAD>([&](auto x) { op[decltype(x)::value] = read(x); });
      f32x16 s[2] = {}, dp[2] = {};
      bf16x8 grads[2];
      auto mask = [&](auto kbt) {
        constexpr int kb = decltype(kbt)::value;
        if (!need) return;
        const int hh = here(h);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int j = 8 * g + 4 * hh + 32 * kb;
          int4 d = make_int4(w.doc, w.doc, w.doc, w.doc);
          if (kdoc) d = *(const int4*)&kd[buf][j];
          const int dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[kb][4 * g + e] = j0 + j + e <= w.last && dd[e] == w.doc ? s[kb][4 * g + e] : -INFINITY;
        }
      };
      auto weigh = [&](auto kbt, auto et) {      // s becomes the weight
        constexpr int kb = decltype(kbt)::value, e = decltype(et)::value;
        float a = s[kb][e] * in, t2 = 0.0f;
        if constexpr (CAP) {
          t2 = tanh_of<SERIES>(a);
          a = t2 * out;
        }
        if constexpr (BIAS) a -= w.slope * fabsf((float)(w.at - j0 - 4 * h) - (float)(32 * kb + 8 * (e >> 2) + (e & 3)));
        if constexpr (CAP) a = s[kb][e] > -INFINITY ? a : -INFINITY;      // the cap has taken a masked score back up
        s[kb][e] = __builtin_amdgcn_exp2f(a - lse2);
        if constexpr (DELTA) return;
        if constexpr (CAP) s[kb][e] *= 1.0f - t2 * t2;
      };
      auto grad = [&](auto kbt, auto et) {
        constexpr int kb = decltype(kbt)::value, e = decltype(et)::value;
        grads[e >> 3][e & 7] = (__bf16)(s[kb][e] * (dp[kb][e] - delta));
      };
      // product of rows, with EACH entries of work beside every step
      auto rows = [&](f32x16& c, const Frag<T, DP>& f, auto first, auto&& work) {
        steps<STEPS>([&](auto xt) {
          constexpr int x = decltype(xt)::value;
          c = mma<T>(next(std::integral_constant<int, decltype(first)::value + x>{}), f[x], c);
          share<STEPS, 16>(xt, work);
          __builtin_amdgcn_sched_barrier(0);
        });
      };
      auto columns = [&](auto first) {
        steps<NC>([&](auto xt) {
          constexpr int x = decltype(xt)::value;
          acc[x % TD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, next(std::integral_constant<int, decltype(first)::value + x>{})), grads[x / TD], acc[x % TD], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        });
      };
      std::integral_constant<int, 0> b0;
      std::integral_constant<int, 1> b1;
      auto nothing = [](auto) {};
      rows(s[0], qf, std::integral_constant<int, 0>{}, nothing);
      mask(b0);
      rows(dp[0], dof, std::integral_constant<int, STEPS>{}, [&](auto e) { weigh(b0, e); });
      rows(s[1], qf, std::integral_constant<int, 2 * STEPS>{}, [&](auto e) {
        if constexpr (DELTA) { delta += s[0][decltype(e)::value] * dp[0][decltype(e)::value]; keep(delta); }
        else grad(b0, e);
      });
      columns(std::integral_constant<int, 3 * STEPS>{});
      mask(b1);
      rows(dp[1], dof, std::integral_constant<int, 3 * STEPS + NC>{}, [&](auto e) { weigh(b1, e); });
      steps<16>([&](auto e) {
        if constexpr (DELTA) delta += s[1][decltype(e)::value] * dp[1][decltype(e)::value];
        else grad(b1, e);
      });
      columns(std::integral_constant<int, 4 * STEPS + NC>{});
    }
  };
  if (exact) {
    walk(std::true_type{}, all0, all1);
    __syncthreads();   // the tiles are filled again
  }
  delta += other_half(delta);
  if (lse2 == INFINITY) delta = 0.0f;
  if (split == 0 && h == 0 && r < p.R) {
    stat[r] = lse2;
    stat[p.R + r] = delta;
    mark_unseeing(p, lse2, b, i);
  }
  walk(std::false_type{}, t0, t1);
  const int re = tile * 128 + wave * 32 + (here(lane) & 31), ie = re / p.G;   // (again, rather than kept)
  if (re >= p.R) return;
  if (p.nsplit == 1)
    store_row<T, DP>((T*)p.dq + b * p.dqs[0] + ie * p.dqs[1] + (kh * p.G + re - ie * p.G) * p.dqs[2], acc, p.scale, p.dim, p.direct, h);
  else
    store_row<float, DP>(p.part + (((long long)split * p.batch * p.hk + pair) * p.R + re) * p.dim, acc, p.scale, p.dim, p.direct, h);
}

// The row tiles [t0, t1) that may see one of the workgroup's keys, and the lowest and highest document of the wave's keys; all threads call it.
// The workgroups of a pair walk their tiles from the last one down, a part every so many-th: whatever their keys, they then read the same rows at about the
// same time, from the XCD's L2.
template <int RT>
__device__ inline void row_range(const Attn& p, int b, int tile, int keys, int mydoc, int* sh, int& t0, int& t1, int& dlo, int& dhi) {
  const int tid = threadIdx.x;
  int i0 = 0, i1 = p.n;
  if (p.causal && !(p.prefix && min(p.prefix[b], keys) > tile * 128)) i0 = max(0, tile * 128 - keys + p.n);
  if (tile * 128 >= keys) i1 = 0;
  dlo = dhi = 0;
  if (p.kdoc) {
    dlo = mydoc < 0 ? 0x7FFFFFFF : mydoc;
    dhi = mydoc;
    int lo = 0x7FFFFFFF, hi = -1;
    const int kblocks = (p.m + 63) / 64, qblocks = (p.n + 63) / 64;
    for (int x = 2 * tile; x < min(2 * tile + 2, kblocks); ++x) {
      const int4 k = p.krange[(long long)b * kblocks + x];
      lo = min(lo, k.x);
      hi = max(hi, k.y);
    }
    // the first and last block of 64 queries with one of them
    if (tid == 0) { sh[0] = 0x7FFFFFFF; sh[1] = -1; }
    __syncthreads();
    int f = 0x7FFFFFFF, e = -1;
    for (int x = i0 / 64 + tid; x < qblocks; x += NT) {
      const int4 k = p.qrange[(long long)b * qblocks + x];
      if (k.x <= hi && k.y >= lo) { f = min(f, x); e = max(e, x); }
    }
    if (e >= 0) { atomicMin(&sh[0], f); atomicMax(&sh[1], e); }
    __syncthreads();
    if (sh[1] < 0) i1 = 0;
    else {
      i0 = max(i0, sh[0] * 64);
      i1 = min(i1, (sh[1] + 1) * 64);
    }
    __syncthreads();
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
      dlo = min(dlo, __shfl_xor(dlo, m));
      dhi = max(dhi, __shfl_xor(dhi, m));
    }
    dlo = __builtin_amdgcn_readfirstlane(dlo);
    dhi = __builtin_amdgcn_readfirstlane(dhi);
  }
  const int first_tile = i0 * p.G / RT, end_tile = i0 < i1 ? (i1 * p.G + RT - 1) / RT : first_tile;
  t0 = __builtin_amdgcn_readfirstlane(first_tile);
  t1 = __builtin_amdgcn_readfirstlane(end_tile);
}

// Rows from the first one on that see nothing, of those without documents
__device__ inline int unseeing_rows(const Attn& p, int b, int keys) {
  return __builtin_amdgcn_readfirstlane(p.causal && !(p.prefix && min(p.prefix[b], keys) > 0) ? max(p.n - keys, 0) * p.G : 0);
}

// Key tile, part (of how many) and pair of a workgroup; the key tiles with the most rows come first
__device__ inline void key_tile_of(const Attn& p, int& tile, int& part, int& parts, int& pair) {
  const int id = place(blockIdx.x, gridDim.x);
  pair = id / p.items;
  part = id - pair * p.items;
  tile = 0;
  parts = 1;
  if (!p.chunk) {
    tile = part;
    part = 0;
    return;
  }
  for (;; ++tile) {
    parts = parts_of(rows_of_key_tile(p.causal, p.prefix, p.n, p.m, p.G, tile), p.chunk);
    if (part < parts) return;
    part -= parts;
  }
}

template <typename T, int DP>
__device__ inline void store_dkv(const Attn& p, const f32x16 (&dk)[DP / 32], const f32x16 (&dv)[DP / 32], int part, int pair, int b, int kh, int j, int h) {
  if (j >= p.m) return;
  if (p.parts == 1) {
    store_row<T, DP>((T*)p.dk + b * p.dks[0] + j * p.dks[1] + kh * p.dks[2], dk, p.scale, p.dim, p.direct, h);
    store_row<T, DP>((T*)p.dv + b * p.dvs[0] + j * p.dvs[1] + kh * p.dvs[2], dv, 1.0f, p.dim, p.direct, h);
  } else {
    const long long pairs = (long long)p.batch * p.hk, row = ((long long)part * pairs + pair) * p.m + j;
    store_row<float, DP>(p.part + row * p.dim, dk, p.scale, p.dim, p.direct, h);
    store_row<float, DP>(p.part + (p.parts * pairs * p.m + row) * p.dim, dv, 1.0f, p.dim, p.direct, h);
  }
}

// dk and dv in fp32.  One wave per SIMD above heads of 32: at two, heads of 64 spilled 312 bytes and took 532 us in place of 402 (both gradients, 2 x 2048 x 8 heads).
template <typename T, int DP>
__global__ void __launch_bounds__(NT, DP <= 32 ? 2 : 1) attention_dkv_kernel(Attn p, const float* stat) {
  using L = Lds<T, DP>;
  constexpr int RT = key_tile<T>(), RBK = RT / 32, TB = RT * L::RB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // queries and dout, two tiles of each
  __shared__ __attribute__((aligned(16))) float lse2[2][RT], delta[2][RT], slope[2][RT];
  __shared__ __attribute__((aligned(16))) int last[2][RT], doc[2][RT], place_of[2][RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  int tile, part, parts, pair;
  key_tile_of(p, tile, part, parts, pair);
  const int b = pair / p.hk, kh = pair - b * p.hk;
  const int keys = keys_of(p, b), j = tile * 128 + wave * 32 + (lane & 31), wave_j1 = tile * 128 + wave * 32 + 31;
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  int mydoc = j < keys ? 0 : -1;
  if (kdoc && j < keys) mydoc = max(kdoc[j], -1);
  int t0, t1, dlo, dhi;
  row_range<RT>(p, b, tile, keys, mydoc, &last[0][0], t0, t1, dlo, dhi);
  const bool keys_mixed = kdoc && (dlo != dhi || __any(mydoc < 0));
  Frag<T, DP> kf, vf;
  load_row<T, DP>(kf, p.direct, p.dim, h, mydoc < 0 ? nullptr : (const T*)p.k + b * p.ks[0] + j * p.ks[1] + kh * p.ks[2]);
  load_row<T, DP>(vf, p.direct, p.dim, h, mydoc < 0 ? nullptr : (const T*)p.v + b * p.vs[0] + j * p.vs[1] + kh * p.vs[2]);
  const T* qbase = (const T*)p.q + b * p.qs[0] + kh * p.G * p.qs[2];
  const T* dobase = (const T*)p.dout + b * p.dos[0] + kh * p.G * p.dos[2];
  const float* st = stat + (long long)pair * 2 * p.R;
  const int unseeing = unseeing_rows(p, b, keys);
  Chunks<T, DP, RT, true> qat, doat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole) {
    qat.set(tid, p.G, p.qs[1], p.qs[2], p.dim);
    doat.set(tid, p.G, p.dos[1], p.dos[2], p.dim);
  }
  auto issue = [&](int t, int buf) {
    if (p.whole && !kdoc && (t + 1) * RT <= p.R && t * RT >= unseeing) {
      const long long token = (long long)t * RT / p.G;
      qat.load(smem + buf * TB, (const char*)(qbase + token * p.qs[1]), wave);
      doat.load(smem + (2 + buf) * TB, (const char*)(dobase + token * p.dos[1]), wave);
    } else {
      auto at = [&](int x, const T* base, const long long (&s)[3]) -> const T* {
        const int r = t * RT + x, i = r / p.G, g = r - i * p.G;
        return r < p.R && st[r] != INFINITY ? base + i * s[1] + g * s[2] : nullptr;
      };
      load_tile<T, DP, RT>(smem + buf * TB, p.direct, p.dim, tid, [&](int x) { return at(x, qbase, p.qs); });
      load_tile<T, DP, RT>(smem + (2 + buf) * TB, p.direct, p.dim, tid, [&](int x) { return at(x, dobase, p.dos); });
    }
    if (tid < RT) {
      const int r = t * RT + tid;
      const Row w = row_of(p, b, kh, r, keys);
      lse2[buf][tid] = r < p.R ? st[r] : INFINITY;
      delta[buf][tid] = r < p.R ? st[p.R + r] : 0.0f;
      last[buf][tid] = w.last;
      doc[buf][tid] = w.doc;
      place_of[buf][tid] = w.at;
      slope[buf][tid] = w.slope;
    }
  };
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) { dk[t] = (f32x16){}; dv[t] = (f32x16){}; }
  const bool cap = p.cap > 0.0f, bias = p.slopes != nullptr;
  const float mul = cap || bias ? 1.0f : p.scale * LOG2E, in = cap ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E, per_cap = cap ? 1.0f / out : 0.0f;
  if (t1 - 1 - part >= t0) issue(t1 - 1 - part, 0);
  for (int t = t1 - 1 - part, buf = 0; t >= t0; t -= parts, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
    if (t - parts >= t0) issue(t - parts, buf ^ 1);
    // Rows that see nothing have lse2 = +inf and need no mask.  The keys that a row sees grow with its token: the tile's first row says whether all see all.
    const Row first = row_of(p, b, kh, t * RT, keys);
    bool need = kdoc || first.last < wave_j1;
    if (kdoc && !keys_mixed && first.last >= wave_j1) {
      const int qblocks = (p.n + 63) / 64, x0 = t * RT / p.G / 64, x1 = min(t * RT + RT - 1, p.R - 1) / p.G / 64;
      const int4 a = p.qrange[(long long)b * qblocks + x0], c = p.qrange[(long long)b * qblocks + x1];
      need = !(a.x == dlo && a.y == dlo && c.x == dlo && c.y == dlo);
    }
    const char *qt = smem + buf * TB, *dot = smem + (2 + buf) * TB;
#pragma unroll
    for (int rb = 0; rb < RBK; ++rb) {
      f32x16 s = rows_by_rows<T, DP>(qt, 32 * rb, kf, lane);
      f32x16 f;
      if (cap) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[e] = out * tanh_of<true>(s[e] * in);
          f[e] = slope_of_cap(s[e], per_cap);
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int x = 32 * rb + 8 * g + 4 * h;
        const f32x4 ls = *(const f32x4*)&lse2[buf][x];
        if (bias) {
          const f32x4 sl = *(const f32x4*)&slope[buf][x];
          const int4 pl = *(const int4*)&place_of[buf][x];
          const int pp[4] = {pl.x, pl.y, pl.z, pl.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * g + e] = s[4 * g + e] * (cap ? 1.0f : in) - sl[e] * fabsf((float)(pp[e] - j));
        }
        if (need) {
          const int4 la = *(const int4*)&last[buf][x], d4 = *(const int4*)&doc[buf][x];
          const int ll[4] = {la.x, la.y, la.z, la.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * g + e] = j <= ll[e] && dd[e] == mydoc ? s[4 * g + e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * g + e] = __builtin_amdgcn_exp2f(s[4 * g + e] * mul - ls[e]);
      }
      columns_by<T, DP>(dv, dot, 32 * rb, s, lane);
      f32x16 dp = rows_by_rows<T, DP>(dot, 32 * rb, vf, lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 de = *(const f32x4*)&delta[buf][32 * rb + 8 * g + 4 * h];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dp[4 * g + e] = s[4 * g + e] * (dp[4 * g + e] - de[e]);
          if (cap) dp[4 * g + e] *= f[4 * g + e];
        }
      }
      columns_by<T, DP>(dk, qt, 32 * rb, dp, lane);
    }
  }
  store_dkv<T, DP>(p, dk, dv, part, pair, b, kh, j, h);
}

template <int STEPS, int NC, int AHEAD> constexpr int read_by(int x) {
  const int ahead = x < STEPS || x >= 2 * STEPS + NC ? 5 : AHEAD, n = 2 * STEPS + 2 * NC;
  int to = x + 1 + ahead;
  if (x < STEPS && to > STEPS + AHEAD) to = STEPS + AHEAD;   // the second product's are read no further ahead than its own
  return to < n ? to : n;
}

// dk and dv in bf16.  Per block of 32 rows: scores Q K^T, then dp = dO V^T while the exponentials are taken, then dv while ds is, then dk; the operands of every product are read from LDS a few products ahead.
// Two waves per SIMD have 256 registers each: 128 of them are sums at DP = 128, so V stays in LDS there (its rows are read again for every block), and
// tiles of 32 rows leave room for two workgroups per CU.
template <int DP, bool CAP, bool BIAS, bool SERIES>
__global__ void __launch_bounds__(NT, 2) attention_dkv_bf16_kernel(Attn p, const float* stat) {
  typedef __bf16 T;
  using L = Lds<T, DP>;
  constexpr bool V_IN_LDS = DP > 64;
  constexpr int RT = DP > 64 ? 32 : 64, TB = RT * L::RB, TD = DP / 32, STEPS = L::STEPS, NC = 2 * TD, AHEAD = DP > 64 ? 2 : 3;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // queries and dout, two tiles of each; the values of the workgroup's keys
  __shared__ __attribute__((aligned(16))) float lse2[2][64], delta[2][64], slope[2][RT];
  __shared__ __attribute__((aligned(16))) int last[2][RT], doc[2][RT], place_of[2][RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  int tile, part, parts, pair;
  key_tile_of(p, tile, part, parts, pair);
  const int b = pair / p.hk, kh = pair - b * p.hk;
  const int keys = keys_of(p, b), j = tile * 128 + wave * 32 + (lane & 31), wave_j1 = tile * 128 + wave * 32 + 31;
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  int mydoc = j < keys ? 0 : -1;
  if (kdoc && j < keys) mydoc = max(kdoc[j], -1);
  int t0, t1, dlo, dhi;
  row_range<RT>(p, b, tile, keys, mydoc, &last[0][0], t0, t1, dlo, dhi);
  const bool keys_mixed = kdoc && (dlo != dhi || __any(mydoc < 0));
  const T* krow = mydoc < 0 ? nullptr : (const T*)p.k + b * p.ks[0] + j * p.ks[1] + kh * p.ks[2];
  const T* vrow = mydoc < 0 ? nullptr : (const T*)p.v + b * p.vs[0] + j * p.vs[1] + kh * p.vs[2];
  Frag<T, DP> kf, vf;
  load_row<T, DP>(kf, p.direct, p.dim, h, krow);
  load_row<T, DP>(vf, p.direct, p.dim, h, vrow);
  const unsigned lds0 = lds_address(smem), row_at = (lane & 31) * L::RB + ((h ^ L::swizzle(lane & 31)) << 4);
  const unsigned va = lds0 + 4 * TB + wave * 32 * L::RB + row_at;
  if constexpr (V_IN_LDS) {   // read by the wave that writes it
#pragma unroll
    for (int s = 0; s < STEPS; ++s) *(__attribute__((address_space(3))) u32x4*)(va ^ (s << 5)) = vf[s];
  }
  const T* qbase = (const T*)p.q + b * p.qs[0] + kh * p.G * p.qs[2];
  const T* dobase = (const T*)p.dout + b * p.dos[0] + kh * p.G * p.dos[2];
  const float* st = stat + (long long)pair * 2 * p.R;
  const int unseeing = unseeing_rows(p, b, keys);
  // Where the group divides 32, a tile's rows lie alike in every tile
  Chunks<T, DP, RT, true> qat, doat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole) {
    qat.set(tid, p.G, p.qs[1], p.qs[2], p.dim);
    doat.set(tid, p.G, p.dos[1], p.dos[2], p.dim);
  }
  // documents of the 64-token blocks of a tile's first and last row
  auto docs_of = [&](int t, int4& x, int4& y) {
    const int qblocks = (p.n + 63) / 64;
    x = range_of(p.qrange, (long long)b * qblocks + t * RT / p.G / 64);
    y = range_of(p.qrange, (long long)b * qblocks + min(t * RT + RT - 1, p.R - 1) / p.G / 64);
  };
  int row_doc = doc_of_row(p, b, (t1 - 1 - part) * RT + tid);   // of the tile that is issued next, read while the one before is on its way
  auto issue = [&](int t, int buf) __attribute__((always_inline)) {
    int4 dx = make_int4(0, 0, 0, 0), dy = dx;
    if (p.qdoc) docs_of(t, dx, dy);
    const bool hidden = p.qdoc ? dx.z || dy.z : t * RT < unseeing;
    if (p.whole && !hidden && (t + 1) * RT <= p.R) {
      const long long token = (long long)t * RT / p.G;
      qat.load(smem + buf * TB, (const char*)(qbase + token * p.qs[1]), wave);
      doat.load(smem + (2 + buf) * TB, (const char*)(dobase + token * p.dos[1]), wave);
    } else {
      auto at = [&](int x, const T* base, const long long (&s)[3]) -> const T* {
        const int r = t * RT + x, i = r / p.G, g = r - i * p.G;
        return r < p.R && !(hidden && st[r] == INFINITY) ? base + i * s[1] + g * s[2] : nullptr;
      };
      load_tile<T, DP, RT>(smem + buf * TB, p.direct, p.dim, tid, [&](int x) { return at(x, qbase, p.qs); });
      load_tile<T, DP, RT>(smem + (2 + buf) * TB, p.direct, p.dim, tid, [&](int x) { return at(x, dobase, p.dos); });
    }
    if ((t + 1) * RT > p.R) {
      if (tid < RT) {
        lse2[buf][tid] = t * RT + tid < p.R ? st[t * RT + tid] : INFINITY;
        delta[buf][tid] = t * RT + tid < p.R ? st[p.R + t * RT + tid] : 0.0f;
      }
    } else if (wave == 0) {   // 64 of them; what lies past a tile of 32 (or the last pair, in the pad of the workspace) is not used
      const __attribute__((address_space(1))) char *x = (const __attribute__((address_space(1))) char*)(st + t * RT), *y = x + (size_t)p.R * sizeof(float);
      const unsigned at = here(lane) * 4;
      asm volatile("" : "+s"(x), "+s"(y));
      __builtin_amdgcn_global_load_lds((gptr_t)(x + at), (lptr_t)lse2[buf], 4, 0, 0);
      __builtin_amdgcn_global_load_lds((gptr_t)(y + at), (lptr_t)delta[buf], 4, 0, 0);
    }
    if (BIAS || kdoc || (t + 1) * RT > p.R || row_of(p, b, kh, t * RT, keys, 0).last < tile * 128 + 127) {
      const int x = here(tid);
      if (x < RT) {
        const Row w = row_of(p, b, kh, t * RT + x, keys, row_doc);
        last[buf][x] = w.last;
        doc[buf][x] = w.doc;
        place_of[buf][x] = w.at;
        slope[buf][x] = w.slope;
      }
      if (tid < RT && t >= parts) row_doc = doc_of_row(p, b, (t - parts) * RT + tid);
    }
  };
  f32x16 dk[TD], dv[TD];
#pragma unroll
  for (int t = 0; t < TD; ++t) { dk[t] = (f32x16){}; dv[t] = (f32x16){}; }
  const float in = CAP ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E;
  const unsigned qa = lds0 + row_at;
  const int cr = 4 * h + ((lane & 15) >> 2), cc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const unsigned ca = lds0 + cr * L::RB + ((cc ^ L::swizzle(cr)) << 4) + 8 * (lane & 1);
  if (t1 - 1 - part >= t0) issue(t1 - 1 - part, 0);
  for (int t = t1 - 1 - part, buf = 0; t >= t0; t -= parts, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
    if (t - parts >= t0) issue(t - parts, buf ^ 1);
    // Rows that see nothing have lse2 = +inf and need no mask.  The keys that a row sees grow with its token: the tile's first row says whether all see all.
    const Row first = row_of(p, b, kh, t * RT, keys, 0);
    bool need = kdoc || first.last < wave_j1 || (t + 1) * RT > p.R;
    if (kdoc && !keys_mixed && first.last >= wave_j1 && (t + 1) * RT <= p.R) {
      int4 x, y;
      docs_of(t, x, y);
      need = !(x.x == dlo && x.y == dlo && y.x == dlo && y.y == dlo);
    }
#pragma unroll
    for (int rb = 0; rb < RT / 32; ++rb) {
      const unsigned at = buf * TB + rb * 32 * L::RB;
      // operand x of the block: rows of Q, rows of dO, columns of dO, columns of Q
      auto read = [&](auto xt) -> u32x4 {
        constexpr int x = decltype(xt)::value;
        if constexpr (x < STEPS) return lds_read16((qa ^ (x << 5)) + at);
        else if constexpr (x < 2 * STEPS) return lds_read16((qa ^ ((x - STEPS) << 5)) + at + 2 * TB);
        else {
          constexpr int y = (x - 2 * STEPS) % NC, z = y / TD * 16 * L::RB + (x - 2 * STEPS < NC ? 2 * TB : 0);
          return __builtin_bit_cast(u32x4, lds_read_columns((ca ^ (y % TD << 6)) + at + z, (ca ^ (y % TD << 6) ^ 32) + at + z + 8 * L::RB));
        }
      };
      // how many operands have been read when product x is taken: more ahead in the first and last product, whose sums leave the registers for it
      constexpr int N = 2 * STEPS + 2 * NC;
      u32x4 op[N], vop[2];
      auto next = [&](auto xt) {
        constexpr int x = decltype(xt)::value, from = x == 0 ? 0 : read_by<STEPS, NC, AHEAD>(x - 1), to = read_by<STEPS, NC, AHEAD>(x);
        steps<to - from>([&](auto y) { op[from + decltype(y)::value] = read(std::integral_constant<int, from + decltype(y)::value>{}); });
        return op[x];
      };
      f32x16 s = {}, dp = {};
      steps<STEPS>([&](auto xt) {
        constexpr int x = decltype(xt)::value;
        s = mma<T>(next(xt), kf[x], s);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (V_IN_LDS) vop[0] = lds_read16(va);
      if (need) {
        const int hh = here(h);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int x = 32 * rb + 8 * g + 4 * hh;
          const int4 la = *(const int4*)&last[buf][x], d4 = *(const int4*)&doc[buf][x];
          const int ll[4] = {la.x, la.y, la.z, la.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * g + e] = j <= ll[e] && dd[e] == mydoc ? s[4 * g + e] : -INFINITY;
        }
      }
      bf16x8 weights[2], grads[2];
      f32x4 row4, slope4;
      int4 place4;
      steps<STEPS>([&](auto xt) {
        constexpr int x = decltype(xt)::value;
        u32x4 v;
        if constexpr (V_IN_LDS) {
          if constexpr (x + 1 < STEPS) vop[(x + 1) & 1] = lds_read16(va ^ ((x + 1) << 5));
          v = vop[x & 1];
        } else {
          v = vf[x];
        }
        dp = mma<T>(next(std::integral_constant<int, STEPS + x>{}), v, dp);
        share<STEPS, 16>(xt, [&](auto et) {
          constexpr int e = decltype(et)::value;
          if constexpr (e % 4 == 0) {
            constexpr int r4 = 8 * (e / 4);
            row4 = *(const f32x4*)&lse2[buf][32 * rb + r4 + 4 * h];
            if constexpr (BIAS) {
              slope4 = *(const f32x4*)&slope[buf][32 * rb + r4 + 4 * h];
              place4 = *(const int4*)&place_of[buf][32 * rb + r4 + 4 * h];
            }
          }
          float a = s[e] * in, t2 = 0.0f;
          if constexpr (CAP) {
            t2 = tanh_of<SERIES>(a);
            a = t2 * out;
          }
          if constexpr (BIAS) a -= slope4[e & 3] * fabsf((float)((e & 3) == 0 ? place4.x - j : (e & 3) == 1 ? place4.y - j : (e & 3) == 2 ? place4.z - j : place4.w - j));
          if constexpr (CAP) a = s[e] > -INFINITY ? a : -INFINITY;      // the cap has taken a masked score back up
          s[e] = __builtin_amdgcn_exp2f(a - row4[e & 3]);
          weights[e >> 3][e & 7] = (__bf16)s[e];
          if constexpr (CAP) s[e] *= 1.0f - t2 * t2;
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      steps<NC>([&](auto xt) {
        constexpr int x = decltype(xt)::value;
        dv[x % TD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, next(std::integral_constant<int, 2 * STEPS + x>{})), weights[x / TD], dv[x % TD], 0, 0, 0);
        share<NC, 16>(xt, [&](auto et) {
          constexpr int e = decltype(et)::value;
          if constexpr (e % 4 == 0) row4 = *(const f32x4*)&delta[buf][32 * rb + 8 * (e / 4) + 4 * h];
          grads[e >> 3][e & 7] = (__bf16)(s[e] * (dp[e] - row4[e & 3]));
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      steps<NC>([&](auto xt) {
        constexpr int x = decltype(xt)::value;
        dk[x % TD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, next(std::integral_constant<int, 2 * STEPS + NC + x>{})), grads[x / TD], dk[x % TD], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  }
  store_dkv<T, DP>(p, dk, dv, part, pair, b, kh, j, h);
}

// to[pair][row] = the sum of the parts, in their order; row -> (token, head) as row / G and row % G.  KEYS: dk and dv (blockIdx.y), whose key tiles have their own
// numbers of parts.  A thread takes E entries: four where rows are whole vectors.
template <typename T, bool KEYS, int E> __global__ void __launch_bounds__(256) attention_sum_kernel(Attn p, T* to0, T* to1) {
  const int R = KEYS ? p.m : p.R, G = KEYS ? 1 : p.G;
  const long long total = (long long)p.batch * p.hk * R * p.dim, at = ((long long)blockIdx.x * 256 + threadIdx.x) * E;
  if (at >= total) return;
  const long long row = at / p.dim;
  const int d = (int)(at - row * p.dim), pair = (int)(row / R), r = (int)(row - (long long)pair * R), b = pair / p.hk, kh = pair - b * p.hk, i = r / G;
  const int n = KEYS ? parts_of(rows_of_key_tile(p.causal, p.prefix, p.n, p.m, p.G, r / 128), p.chunk) : p.nsplit;
  const float* part = p.part + (KEYS && blockIdx.y ? p.parts * total : 0) + at;
  const long long (&st)[3] = !KEYS ? p.dqs : blockIdx.y ? p.dvs : p.dks;
  T* to = (blockIdx.y ? to1 : to0) + b * st[0] + i * st[1] + (kh * G + r - i * G) * st[2] + d;
  if constexpr (E == 4) {
    f32x4 v = {};
#pragma unroll 4
    for (int s = 0; s < n; ++s) v += *(const f32x4*)(part + s * total);
    store4<T>(to, v, true, 4);
  } else {
    float v = 0.0f;
    for (int s = 0; s < n; ++s) v += part[s * total];
    *to = (T)v;
  }
}

template <typename T, bool KEYS> void sum_parts(const Attn& p, void* to0, void* to1, hipStream_t s) {
  ProfScope prof(PK_ATTENTION_JOIN, s);
  const long long total = (long long)p.batch * p.hk * (KEYS ? p.m : p.R) * p.dim, threads = p.direct ? total / 4 : total;
  const dim3 grid((unsigned)((threads + 255) / 256), to1 ? 2 : 1);
  if (p.direct) hipLaunchKernelGGL((attention_sum_kernel<T, KEYS, 4>), grid, dim3(256), 0, s, p, (T*)to0, (T*)to1);
  else hipLaunchKernelGGL((attention_sum_kernel<T, KEYS, 1>), grid, dim3(256), 0, s, p, (T*)to0, (T*)to1);
}

template <typename T, int DP> int launch(Attn& p, const AttnPlan& plan, float* stat, hipStream_t s) {
  constexpr int bytes = 4 * key_tile<T>() * Lds<T, DP>::RB;
  void (*dkv)(Attn, const float*);
  void (*dq)(Attn, float*);
  int dkv_bytes = bytes;
  if constexpr (sizeof(T) == 4) {
    dq = attention_dq_kernel<T, DP>;
    dkv = attention_dkv_kernel<T, DP>;
  } else {
    auto pick = [&](auto cap, auto bias, auto series) {
      constexpr bool C = decltype(cap)::value, B = decltype(bias)::value, S = decltype(series)::value;
      dq = attention_dq_bf16_kernel<DP, C, B, S>;
      dkv = attention_dkv_bf16_kernel<DP, C, B, S>;
    };
    std::true_type yes;
    std::false_type no;
    if (p.cap > CAP_SERIES) pick(yes, yes, yes);   // (without slopes they are 0)
    else p.cap > 0.0f ? (p.slopes ? pick(yes, yes, no) : pick(yes, no, no)) : (p.slopes ? pick(no, yes, no) : pick(no, no, no));
    dkv_bytes = DP > 64 ? (4 * 32 + 128) * Lds<T, DP>::RB : 4 * 64 * Lds<T, DP>::RB;
  }
  int rc = allow_dynamic_lds((const void*)dq, bytes);
  if (rc == PRISM_OK) rc = allow_dynamic_lds((const void*)dkv, dkv_bytes);
  if (rc != PRISM_OK) return rc;
  const unsigned pairs = (unsigned)p.batch * p.hk;
  p.nsplit = plan.split;
  if (p.R > 0) {
    ProfScope prof(PK_ATTENTION_DQ, s);
    hipLaunchKernelGGL(dq, dim3(pairs * p.row_tiles * p.nsplit), dim3(NT), bytes, s, p, stat);
  }
  if (p.nsplit > 1 && p.R > 0) sum_parts<T, false>(p, p.dq, nullptr, s);
  if (p.m == 0) return PRISM_OK;
  p.chunk = plan.chunk;
  p.parts = plan.parts;
  p.items = plan.items;
  {
    ProfScope prof(PK_ATTENTION_DKV, s);
    hipLaunchKernelGGL(dkv, dim3(pairs * p.items), dim3(NT), dkv_bytes, s, p, (const float*)stat);
  }
  if (p.parts > 1) sum_parts<T, true>(p, p.dk, p.dv, s);
  return PRISM_OK;
}

}  // namespace

int launch_attention_backward(const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk,
                              void* dv, int dt, const prism_attention_desc& d, char* ws, hipStream_t s) {
  const AttnPlan plan = attention_plan(d, dt, true);
  Attn p = attn_common(q, k, v, dt, d, ws);
  launch_doc_ranges(d, (int4*)ws, s);
  p.o = out; p.dout = dout; p.lse_in = lse;
  p.dq = dq; p.dk = dk; p.dv = dv;
  set_strides(p.os, d.out); set_strides(p.dos, d.dout);
  set_strides(p.dqs, d.dq); set_strides(p.dks, d.dk); set_strides(p.dvs, d.dv);
  p.part = (float*)(ws + plan.o_part);
  p.direct = p.direct && rows_are_vectors(out, d.out, dt) && rows_are_vectors(dout, d.dout, dt) && rows_are_vectors(dq, d.dq, dt) &&
             rows_are_vectors(dk, d.dk, dt) && rows_are_vectors(dv, d.dv, dt);
  // the rows of a tile lie alike in all tiles, their offsets within one fit 31 bits
  const long long G = d.q_heads / d.k_heads;
  p.whole_keys = p.whole;
  p.whole = p.whole && p.direct && 32 % G == 0;
  for (const prism_strides& x : {d.q, d.dout}) p.whole = p.whole && x.token * (32 / G) + x.head * G < (1ll << 28);
  float* stat = (float*)(ws + plan.o_stat);
  if (dt == PRISM_F32)
    return d.head_dim <= 32 ? launch<float, 32>(p, plan, stat, s) : d.head_dim <= 64 ? launch<float, 64>(p, plan, stat, s) : d.head_dim <= 96 ? launch<float, 96>(p, plan, stat, s) : launch<float, 128>(p, plan, stat, s);
  return d.head_dim <= 64 ? launch<__bf16, 64>(p, plan, stat, s) : d.head_dim <= 96 ? launch<__bf16, 96>(p, plan, stat, s) : launch<__bf16, 128>(p, plan, stat, s);
}

}  // namespace prism
