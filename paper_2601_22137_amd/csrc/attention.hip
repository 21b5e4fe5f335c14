// Attention: out = softmax(scores) v over the keys that a query sees, in one pass over the keys with the running maximum and sum of every row.
//
//   score(i, j) = cap tanh(scale q_i.k_j / cap) - slope |at_i - j|,  at_i = i + keys - n
//
// A workgroup takes 128 rows (32 per wave, on the lanes) of a pair and walks the keys in tiles that all four waves share in LDS, two of them in
// flight.  Scores come out of the product K Q^T with a row per lane, so a row's maximum and sum are plain arithmetic in its own two lanes, and the
// weights go from the registers straight into V^T P^T (attention_tile.h).
//
// Scores, maxima, sums and results are held in 32 bits; the weights are rounded to the type of the values for the second product.  Long prompts in bf16, 8192 tokens, 32 heads of 128
// on 8, causal: 535 us, 1.03 PFLOP/s of the 1.32 that a large product of the vendor library reaches (555 to 660 in runs of these calls alone).  The matrix units are busy 59 % of
// the cycles, the vector units 50, LDS 30 without conflicts; the waves wait for data or a barrier 28 % of theirs; and the clock is down to 1.6 GHz, the power limit.  Twice the rows per wave
// halve the reads of LDS, but leave one wave per SIMD: 614 us against 518 when it was tried.  Capped scores (2 x 4096 tokens, 16 heads of 128 on 4: 245 us) are bound by the vector units, 68 % busy
// beside matrix units at 31: three transcendental instructions a score (exp2 and rcp for the tanh, exp2 for the weight), the tanh with no product beside it.
#include "attention_tile.h"

namespace prism {
namespace {

// Documents of every block of 64 tokens: queries', then keys'
__global__ void __launch_bounds__(256) doc_range_kernel(const int* qdoc, const int* kdoc, int4* range, int n, int m, int batch) {
  const int bq = (n + 63) / 64, bk = (m + 63) / 64;
  const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), queries = (long long)bq * batch;
  if (w >= queries + (long long)bk * batch) return;
  const bool key = w >= queries;
  const long long x = key ? w - queries : w;
  const int blocks = key ? bk : bq, len = key ? m : n, b = (int)(x / blocks), i = (int)(x % blocks) * 64 + (threadIdx.x & 63);
  const int d = i < len ? (key ? kdoc : qdoc)[(long long)b * len + i] : -1;
  int lo = d < 0 ? 0x7FFFFFFF : d, hi = d, none = d < 0;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    lo = min(lo, __shfl_xor(lo, s));
    hi = max(hi, __shfl_xor(hi, s));
    none |= __shfl_xor(none, s);
  }
  if ((threadIdx.x & 63) == 0) range[w] = make_int4(lo, hi, none, 0);
}

// The row's result, or what this part of its keys has of it
template <typename T, int DP>
__device__ inline void finish(const Attn& p, const f32x16 (&acc)[DP / 32], float m, float l, int split, int pair, int b, int i, int head, int r, int h) {
  if (r >= p.R) return;
  if (p.nsplit == 1) {
    store_row<T, DP>((T*)p.out + b * p.os[0] + i * p.os[1] + head * p.os[2], acc, l == 0.0f ? 0.0f : 1.0f / l, p.dim, p.direct, h);
    if (p.lse && h == 0) p.lse[((long long)b * p.hq + head) * p.n + i] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (1.0f / LOG2E);
  } else {
    const long long row = ((long long)split * p.batch * p.hk + pair) * p.R + r;
    if (l != 0.0f) store_row<float, DP>(p.part + row * p.dim, acc, 1.0f, p.dim, p.direct, h);
    if (h == 0) { p.part_ml[2 * row] = m; p.part_ml[2 * row + 1] = l; }
  }
}

// (fp32) Bound by the matrix units (2 x 1111 tokens, 8 heads of 80: busy 53 % of the cycles, the waves wait to issue half of theirs) and, in short calls, by how evenly the parts fill the chip: 2 x 2048 x 8 heads of 128, causal: 199 us, 86 TFLOP/s of the
// pairs that are seen; 2 x 4096, all seen, 1094 us, 126 of 154.
template <typename T, int DP>
__global__ void __launch_bounds__(NT, 2) attention_kernel(Attn p) {
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
  Frag<T, DP> qf;
  const int i = r / p.G, head = kh * p.G + r - i * p.G;
  load_row<T, DP>(qf, p.direct, p.dim, h, w.last < 0 ? nullptr : (const T*)p.q + b * p.qs[0] + i * p.qs[1] + head * p.qs[2]);
  const T* kbase = (const T*)p.k + b * p.ks[0] + kh * p.ks[2];
  const T* vbase = (const T*)p.v + b * p.vs[0] + kh * p.vs[2];
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  auto seen = [&](int j) { return j < keys && !(kdoc && kdoc[j] < 0); };
  Chunks<T, DP, KT> kat, vat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole) {
    kat.set(tid, 1, p.ks[1], 0, p.dim);
    vat.set(tid, 1, p.vs[1], 0, p.dim);
  }
  auto issue = [&](int t, int buf) {
    if (p.whole && !kdoc && (t + 1) * KT <= keys) {
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
  float m = -3.4e38f, l = 0.0f;   // the reference of the exponents, at most 8 below the row's maximum so far, and the lane's share of the sum
  const bool cap = p.cap > 0.0f, bias = p.slopes != nullptr;
  const float mul = cap || bias ? 1.0f : p.scale * LOG2E, in = cap ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E;
  if (t0 < t1) issue(t0, 0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1, j0 = t * KT;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
    if (t + 1 < t1) issue(t + 1, buf ^ 1);
    bool need;
    if (!tile_seen<KT>(p, lim, key_docs<KT>(p, b, t), t, need)) continue;
    const char *kt = smem + buf * TB, *vt = smem + (2 + buf) * TB;
    f32x16 s[KB];
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = rows_by_rows<T, DP>(kt, 32 * kb, qf, lane);
      scores<true>(p, s[kb], w, j0 + 32 * kb + 4 * h, cap, bias, in, out);
      if (need) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int j = 8 * g + 4 * prism::here(h) + 32 * kb;
          int4 d = make_int4(w.doc, w.doc, w.doc, w.doc);
          if (kdoc) d = *(const int4*)&kd[buf][j];
          const int dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) s[kb][4 * g + e] = j0 + j + e <= w.last && dd[e] == w.doc ? s[kb][4 * g + e] : -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max_of(top, s[kb][e]);
    }
    top *= mul;
    if (__any(top > m + 8.0f)) {
      const float to = fmaxf(m, fmaxf(top, other_half(top))), f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t2][e] *= f;
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(s[kb][e] * mul - m);
        l += s[kb][e];
      }
      columns_by<T, DP>(acc, vt, 32 * kb, s[kb], lane);
    }
  }
  l += other_half(l);
  finish<T, DP>(p, acc, m, l, split, pair, b, i, head, r, h);
}

// The same for bf16, with the work of neighbouring tiles interleaved: while the matrix units take K Q^T of tile t + 1, the vector units take the exponentials of
// tile t, and while those take V^T P^T of tile t, these the exponentials that are left and the maximum of tile t + 1.  The keys run one tile ahead of the
// values in LDS.  MOD: scores with a cap or a bias; SERIES: of a large cap.
template <int DP, bool MOD, bool SERIES>
__global__ void __launch_bounds__(NT, DP > 64 ? 2 : 3) attention_bf16_kernel(Attn p) {
  typedef __bf16 T;
  using L = Lds<T, DP>;
  constexpr int KT = 64, TB = KT * L::RB, TD = DP / 32, STEPS = L::STEPS;
  constexpr int NK = 2 * STEPS, NP = 4 * TD, AHEAD = 3;   // products of a tile: K Q^T, V^T P^T; operands are read AHEAD of them
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
  Frag<T, DP> qf;
  const int i = r / p.G, head = kh * p.G + r - i * p.G;
  load_row<T, DP>(qf, p.direct, p.dim, h, w.last < 0 ? nullptr : (const T*)p.q + b * p.qs[0] + i * p.qs[1] + head * p.qs[2]);
  const T* kbase = (const T*)p.k + b * p.ks[0] + kh * p.ks[2];
  const T* vbase = (const T*)p.v + b * p.vs[0] + kh * p.vs[2];
  const int* kdoc = p.kdoc ? p.kdoc + (long long)b * p.m : nullptr;
  Chunks<T, DP, KT> kat, vat;
  if (p.dim < DP) zero_tiles<4 * TB>(smem, tid);
  if (p.whole) {
    kat.set(tid, 1, p.ks[1], 0, p.dim);
    vat.set(tid, 1, p.vs[1], 0, p.dim);
  }
  auto seen = [&](int j) { return j < keys && !(kdoc && kdoc[j] < 0); };
  auto issue = [&](const T* base, long long stride, const Chunks<T, DP, KT>& at, int t, bool hidden, char* to) __attribute__((always_inline)) {
    if (p.whole && !hidden && (t + 1) * KT <= keys) at.load(to, (const char*)(base + (long long)t * KT * stride), wave);
    else load_tile<T, DP, KT>(to, p.direct, p.dim, tid, [&](int x) { const int j = t * KT + x; return seen(j) ? base + j * stride : nullptr; });
  };
  // hidden: a key of no document is among the tile's
  auto issue_k = [&](int t, bool hidden, int buf) {
    issue(kbase, p.ks[1], kat, t, hidden, smem + buf * TB);
    if (kdoc && wave == 0) load_ids(kd[buf], kdoc, t * KT, p.m, lane);
  };
  auto issue_v = [&](int t, bool hidden, int buf) { issue(vbase, p.vs[1], vat, t, hidden, smem + (2 + buf) * TB); };

  // addresses of a lane's operands: chunk 2 s + h of row l % 32, and the columns of columns_by; steps and columns are exclusive ors of their low bits
  const unsigned lds0 = lds_address(smem);
  const unsigned ka = lds0 + (lane & 31) * L::RB + ((h ^ L::swizzle(lane & 31)) << 4);
  const int vr = 4 * h + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const unsigned va = lds0 + 2 * TB + vr * L::RB + ((vc ^ L::swizzle(vr)) << 4) + 8 * (lane & 1);
  auto read_k = [&](int buf, int x) { return lds_read16((ka ^ ((x % STEPS) << 5)) + buf * TB + x / STEPS * 32 * L::RB); };
  auto read_v = [&](int buf, int x) {
    const unsigned at = buf * TB + x / TD * 16 * L::RB;
    return lds_read_columns((va ^ (x % TD << 6)) + at, (va ^ (x % TD << 6) ^ 32) + at + 8 * L::RB);
  };

  f32x16 acc[TD], sa[2], sb[2];
#pragma unroll
  for (int t = 0; t < TD; ++t) acc[t] = (f32x16){};
  float m = -3.4e38f, l[2] = {0.0f, 0.0f};   // the reference of the exponents, at most 8 below the row's maximum so far, and the lane's share of the sum
  const bool cap = MOD && p.cap > 0.0f, bias = MOD && p.slopes != nullptr;
  const float mul = MOD ? 1.0f : p.scale * LOG2E, in = cap ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E;
  // Scores of the next tile into n and / or the weights of this one, whose scores s holds, into acc; returns the largest product of n
  auto products = [&](auto has_next, auto has_this, int buf, f32x16 (&s)[2], f32x16 (&n)[2]) __attribute__((always_inline)) {
    constexpr bool NEXT = decltype(has_next)::value, THIS = decltype(has_this)::value;
    float top = -INFINITY;
    u32x4 kf[AHEAD + 1];
    bf16x8 vf[AHEAD + 1], weights = {};
    auto weigh = [&](int e) __attribute__((always_inline)) {
      s[e >> 4][e & 15] = __builtin_amdgcn_exp2f(s[e >> 4][e & 15] * mul - m);
      l[e & 1] += s[e >> 4][e & 15];
    };
    if constexpr (NEXT) {
      n[0] = n[1] = (f32x16){};
      steps<AHEAD>([&](auto x) { kf[decltype(x)::value] = read_k(buf ^ 1, decltype(x)::value); });
      steps<NK>([&](auto xt) {
        constexpr int x = decltype(xt)::value;
        if constexpr (x + AHEAD < NK) kf[(x + AHEAD) % (AHEAD + 1)] = read_k(buf ^ 1, x + AHEAD);
        else if constexpr (THIS) vf[x + AHEAD - NK] = read_v(buf, x + AHEAD - NK);
        n[x / STEPS] = mma<T>(kf[x % (AHEAD + 1)], qf[x % STEPS], n[x / STEPS]);
        if constexpr (THIS) {
          share<NK, 16>(xt, [&](auto e) { weigh(decltype(e)::value); });
          keep(l[0]);
          keep(l[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    } else {
      steps<AHEAD>([&](auto x) { vf[decltype(x)::value] = read_v(buf, decltype(x)::value); });
      steps<16>([&](auto e) { weigh(decltype(e)::value); });
    }
    if constexpr (THIS) {
      steps<NP>([&](auto xt) {
        constexpr int x = decltype(xt)::value, g = x / TD;
        if constexpr (x + AHEAD < NP) vf[(x + AHEAD) % (AHEAD + 1)] = read_v(buf, x + AHEAD);
        if constexpr (x % TD == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) weights[e] = (__bf16)s[g >> 1][8 * (g & 1) + e];
        }
        acc[x % TD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[x % (AHEAD + 1)], weights, acc[x % TD], 0, 0, 0);
        if constexpr (x < NP / 2) {
          share<NP / 2, 16>(xt, [&](auto e) { weigh(16 + decltype(e)::value); });
          keep(l[0]);
          keep(l[1]);
        } else if constexpr (NEXT && !MOD) {
          share<NP / 2, 16>(std::integral_constant<int, x - NP / 2>{}, [&](auto e) { constexpr int z = 2 * decltype(e)::value; top = max_of(top, n[z >> 4][z & 15], n[z >> 4][(z & 15) + 1]); });
          keep(top);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    } else if constexpr (!MOD) {
#pragma unroll
      for (int e = 0; e < 32; ++e) top = max_of(top, n[e >> 4][e & 15]);
    }
    return top;
  };
  std::true_type yes;
  std::false_type no;
  // what the products of tile t become before the exponential, and the row's reference
  auto take_scores = [&](int t, int buf, f32x16 (&s)[2], float top, bool need) {
    const int j0 = t * KT;
    if constexpr (MOD) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) scores<SERIES>(p, s[kb], w, j0 + 32 * kb + 4 * h, cap, bias, in, out);
    }
    if (need) {
      const int hh = prism::here(h);
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const int j = 8 * g + 4 * hh;
        int4 d = make_int4(w.doc, w.doc, w.doc, w.doc);
        if (kdoc) d = *(const int4*)&kd[buf][j];
        const int dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = s[g >> 2][4 * (g & 3) + e];
          s[g >> 2][4 * (g & 3) + e] = j0 + j + e <= w.last && dd[e] == w.doc ? x : -INFINITY;
        }
      }
    }
    if (MOD || need) {
      top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 32; ++e) top = max_of(top, s[e >> 4][e & 15]);
    }
    top *= mul;
    if (__any(top > m + 8.0f)) {
      const float to = fmaxf(m, fmaxf(top, other_half(top))), f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l[0] *= f;
      l[1] *= f;
#pragma unroll
      for (int t2 = 0; t2 < TD; ++t2)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t2][e] *= f;
    }
  };
  auto landed = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
  };
  // A tile that the wave's rows do not see is masked, not skipped: one straight path through the loop keeps its registers in place.
  auto next_scores = [&](int t, const int4& docs, int buf, f32x16 (&n)[2], float top) {
    bool need;
    const bool any = tile_seen<KT>(p, lim, docs, t, need);
    take_scores(t, buf, n, top, need || !any);
  };
  int4 docs;   // of the next tile's keys
  auto step = [&](int t, int buf, f32x16 (&s)[2], f32x16 (&n)[2]) __attribute__((always_inline)) {
    const int4 after = key_docs<KT>(p, b, min(t + 2, t1 - 1));
    landed();   // keys t + 1 and values t are there; keys t and values t - 1 have been read by all waves
    if (t + 2 < t1) issue_k(t + 2, after.z, buf);
    issue_v(t + 1, docs.z, buf ^ 1);
    next_scores(t + 1, docs, buf ^ 1, n, products(yes, yes, buf, s, n));
    docs = after;
  };
  if (t0 < t1 && lim.last < 0) {   // a wave without rows only takes its share of the loads
    issue_k(t0, key_docs<KT>(p, b, t0).z, 0);
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1;
      landed();
      if (t + 1 < t1) issue_k(t + 1, key_docs<KT>(p, b, t + 1).z, buf ^ 1);
      issue_v(t, key_docs<KT>(p, b, t).z, buf);
    }
    landed();
  } else if (t0 < t1) {
    const int4 first = key_docs<KT>(p, b, t0);
    issue_k(t0, first.z, 0);
    docs = key_docs<KT>(p, b, min(t0 + 1, t1 - 1));
    landed();
    if (t0 + 1 < t1) issue_k(t0 + 1, docs.z, 1);
    issue_v(t0, first.z, 0);
    next_scores(t0, first, 0, sa, products(yes, no, 1, sb, sa));
    int t = t0;
    for (; t + 2 < t1; t += 2) {
      step(t, 0, sa, sb);
      step(t + 1, 1, sb, sa);
    }
    if (t + 1 < t1) {
      step(t, 0, sa, sb);
      landed();
      products(no, yes, 1, sb, sa);
    } else {
      landed();
      products(no, yes, 0, sa, sb);
    }
  }
  float sum = l[0] + l[1];
  sum += other_half(sum);
  const int re = tile * 128 + wave * 32 + (prism::here(lane) & 31), ie = re / p.G;   // (again, rather than kept)
  finish<T, DP>(p, acc, m, sum, split, pair, b, ie, kh * p.G + re - ie * p.G, re, h);
}

// Few rows (32 of a pair at most, as when single tokens are generated for a group of heads): the time is that of reading the keys and values once.  Every wave
// takes blocks of 32 keys of its own, with no barrier between them, through its own part of LDS (as an operand straight from memory every load of keys would touch 32 lines):
// the keys are read into registers at once, which makes room for the next block's, the values lie in two blocks.  The waves' results are joined in LDS.
// 8 tokens of 32 heads on 8 of 128, 4096 to 16384 keys, capped: 75 us and 5 for the join, 4.5 TB/s (waves wait for data 42 % of their cycles); with the kernel above 105.  One token of 8 heads on 2, 32768 keys: 13.9 and 20.2; 8 on
// 2048 keys each: 21.9 and 19.5, where its join of four waves shows.
template <int DP, bool MOD, bool SERIES>
__global__ void __launch_bounds__(NT, 2) attention_few_kernel(Attn p) {
  typedef __bf16 T;
  using L = Lds<T, DP>;
  constexpr int STEPS = L::STEPS, TB = 32 * L::RB, TD = DP / 32, LOADS = 32 * L::CPR / 64, LD = DP + 4;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // keys, and two blocks of values of each wave; at the end [wave][32][LD] floats
  __shared__ float ml[NW][32][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, r = lane & 31;
  const int id = place(blockIdx.x, gridDim.x), split = id % p.nsplit, pair = id / p.nsplit, b = pair / p.hk, kh = pair - b * p.hk;
  const int keys = keys_of(p, b);
  const Row w = row_of(p, b, kh, r, keys);
  const Limits lim = limits_of(p, w, b, kh, r, keys);
  const int blocks = (lim.last + 32) / 32, per = (blocks + p.nsplit - 1) / p.nsplit, b0 = split * per, b1 = min(blocks, b0 + per);
  Frag<T, DP> qf, kf;
  {
    const int i = r / p.G;
    load_row<T, DP>(qf, true, p.dim, h, w.last < 0 ? nullptr : (const T*)p.q + b * p.qs[0] + i * p.qs[1] + (kh * p.G + r - i * p.G) * p.qs[2]);
  }
  const T* kbase = (const T*)p.k + b * p.ks[0] + kh * p.ks[2];
  const T* vbase = (const T*)p.v + b * p.vs[0] + kh * p.vs[2];
  char* mine = smem + wave * 3 * TB;
  // keys past the end: the last one again, masked
  auto issue = [&](int block, const T* base, long long stride, char* to) {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int x = u * 64 + lane, row = x / L::CPR, c = (x % L::CPR) ^ L::swizzle(row);
      const T* from = base + (long long)min(block * 32 + row, keys - 1) * stride + c * L::EPC;
      __builtin_amdgcn_global_load_lds((gptr_t)(c * L::EPC < p.dim ? (const void*)from : (const void*)zero_page), (lptr_t)(to + u * 1024), 16, 0, 0);
    }
  };
  f32x16 acc[TD];
#pragma unroll
  for (int t = 0; t < TD; ++t) acc[t] = (f32x16){};
  float m = -3.4e38f, l = 0.0f;
  const bool cap = MOD && p.cap > 0.0f, bias = MOD && p.slopes != nullptr;
  const float mul = MOD ? 1.0f : p.scale * LOG2E, in = cap ? p.scale / p.cap : p.scale * LOG2E, out = p.cap * LOG2E;
  int buf = 0;
  if (b0 + wave < b1) {
    issue(b0 + wave, kbase, p.ks[1], mine);
    issue(b0 + wave, vbase, p.vs[1], mine + TB);
  }
  for (int block = b0 + wave; block < b1; block += NW, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
#pragma unroll
    for (int x = 0; x < STEPS; ++x) kf[x] = lds_read16(lds_address(mine) + r * L::RB + (((2 * x + h) ^ L::swizzle(r)) << 4));
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the keys are in registers, their place is free
    __builtin_amdgcn_sched_barrier(0);
    if (block + NW < b1) {
      issue(block + NW, kbase, p.ks[1], mine);
      issue(block + NW, vbase, p.vs[1], mine + TB + (buf ^ 1) * TB);
    }
    f32x16 s = {};
#pragma unroll
    for (int x = 0; x < STEPS; ++x) s = mma<T>(kf[x], qf[x], s);
    const int j0 = block * 32 + 4 * h;
    if constexpr (MOD) scores<SERIES>(p, s, w, j0, cap, bias, in, out);
    if (block * 32 + 31 > lim.first) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = j0 + 8 * (e >> 2) + (e & 3) <= w.last ? s[e] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max_of(top, s[e]);
    top *= mul;
    if (__any(top > m + 8.0f)) {
      const float to = fmaxf(m, fmaxf(top, other_half(top))), f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int t = 0; t < TD; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= f;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] * mul - m);
      l += s[e];
    }
    columns_by<T, DP>(acc, mine + TB + buf * TB, 0, s, lane);
  }
  l += other_half(l);
  __syncthreads();
  float* all = (float*)smem;
#pragma unroll
  for (int t = 0; t < TD; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[t][4 * g + e];
      *(f32x4*)&all[(wave * 32 + r) * LD + 32 * t + 8 * g + 4 * h] = v;
    }
  if (h == 0) { ml[wave][r][0] = m; ml[wave][r][1] = l; }
  __syncthreads();
  for (int x = tid; x < p.R * (DP / 4); x += NT) {
    const int row = x / (DP / 4), d = (x % (DP / 4)) * 4;
    float top = -3.4e38f, sum = 0.0f;
#pragma unroll
    for (int q = 0; q < NW; ++q) top = fmaxf(top, ml[q][row][0]);
    f32x4 v = {};
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      const float f = __builtin_amdgcn_exp2f(ml[q][row][0] - top);
      sum += ml[q][row][1] * f;
      if (ml[q][row][1] != 0.0f) v += *(const f32x4*)&all[(q * 32 + row) * LD + d] * f;
    }
    const int i = row / p.G, head = kh * p.G + row - i * p.G;
    if (p.nsplit > 1) {
      const long long at = ((long long)split * p.batch * p.hk + pair) * p.R + row;
      if (d < p.dim) *(f32x4*)(p.part + at * p.dim + d) = v;
      if (d == 0) { p.part_ml[2 * at] = top; p.part_ml[2 * at + 1] = sum; }
    } else {
      if (d < p.dim) store4<T>((T*)p.out + b * p.os[0] + i * p.os[1] + head * p.os[2] + d, v * (sum == 0.0f ? 0.0f : 1.0f / sum), true, 4);
      if (d == 0 && p.lse) p.lse[((long long)b * p.hq + head) * p.n + i] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.0f / LOG2E);
    }
  }
}

// The parts of a row's keys (64 at most) joined.  MANY: by a workgroup, whose waves take every fourth part; else (eight at most) by a wave.  Nothing is waited for before
// all parts of a wave are on their way.
template <typename T, bool MANY> __global__ void __launch_bounds__(256) attention_join_kernel(Attn p) {
  constexpr int EVERY = MANY ? NW : 1, PARTS = MANY ? 16 : 8;
  __shared__ float other[MANY ? NW : 1][128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long rows = (long long)p.batch * p.hk * p.R, row = MANY ? blockIdx.x : (long long)blockIdx.x * NW + wave;
  if (row >= rows) return;
  const int first = MANY ? wave : 0;
  float m = -3.4e38f, l = 0.0f;
  if (lane < p.nsplit) {
    m = p.part_ml[2 * (lane * rows + row)];
    l = p.part_ml[2 * (lane * rows + row) + 1];
  }
  float v[PARTS][2];
#pragma unroll
  for (int s = 0; s < PARTS; ++s)
    if (first + EVERY * s < p.nsplit)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (lane + 64 * x < p.dim) v[s][x] = p.part[((first + EVERY * s) * rows + row) * p.dim + lane + 64 * x];
  float top = m;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
  const float f = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m - top);   // 0 too where nothing was written
  float sum = l * f, o[2] = {0.0f, 0.0f};
#pragma unroll
  for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
#pragma unroll
  for (int s = 0; s < PARTS; ++s) {
    const float fs = __shfl(f, (first + EVERY * s) & 63);
    if (first + EVERY * s < p.nsplit && fs != 0.0f)
#pragma unroll
      for (int x = 0; x < 2; ++x) o[x] += v[s][x] * fs;
  }
  const int pair = (int)(row / p.R), r = (int)(row - (long long)pair * p.R), b = pair / p.hk, kh = pair - b * p.hk, i = r / p.G, head = kh * p.G + r - i * p.G;
  T* to = (T*)p.out + b * p.os[0] + i * p.os[1] + head * p.os[2];
  if constexpr (MANY) {
    other[wave][lane] = o[0];
    other[wave][lane + 64] = o[1];
    __syncthreads();
    const int d = threadIdx.x;
    if (d < p.dim) to[d] = (T)(sum == 0.0f ? 0.0f : (other[0][d] + other[1][d] + other[2][d] + other[3][d]) / sum);
    if (d != 0) return;
  } else {
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (lane + 64 * x < p.dim) to[lane + 64 * x] = (T)(sum == 0.0f ? 0.0f : o[x] / sum);
    if (lane != 0) return;
  }
  if (p.lse) p.lse[((long long)b * p.hq + head) * p.n + i] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.0f / LOG2E);
}

template <typename T, int DP> int launch(Attn& p, bool few, hipStream_t s) {
  int bytes = 4 * key_tile<T>() * Lds<T, DP>::RB;
  void (*kernel)(Attn);
  if constexpr (sizeof(T) == 4) {
    kernel = attention_kernel<T, DP>;
  } else {
    const bool mod = p.cap > 0.0f || p.slopes, series = p.cap > CAP_SERIES;
    if (few) {
      kernel = series ? attention_few_kernel<DP, true, true> : mod ? attention_few_kernel<DP, true, false> : attention_few_kernel<DP, false, false>;
      bytes = NW * 3 * 32 * Lds<T, DP>::RB;
    } else {
      kernel = series ? attention_bf16_kernel<DP, true, true> : mod ? attention_bf16_kernel<DP, true, false> : attention_bf16_kernel<DP, false, false>;
    }
  }
  const int rc = allow_dynamic_lds((const void*)kernel, bytes);
  if (rc != PRISM_OK) return rc;
  const long long rows = (long long)p.batch * p.hk * p.R;
  {
    ProfScope prof(PK_ATTENTION, s);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.batch * p.hk * p.row_tiles * p.nsplit), dim3(NT), bytes, s, p);
  }
  if (p.nsplit > 1) {
    ProfScope prof(PK_ATTENTION_JOIN, s);
    if (p.nsplit > 8) hipLaunchKernelGGL((attention_join_kernel<T, true>), dim3((unsigned)rows), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((attention_join_kernel<T, false>), dim3((unsigned)((rows + NW - 1) / NW)), dim3(256), 0, s, p);
  }
  return PRISM_OK;
}

}  // namespace

AttnPlan attention_plan(const prism_attention_desc& d, int dt, bool backward) {
  AttnPlan a = {};
  const long long pairs = (long long)d.batch * d.k_heads, R = (long long)(d.q_heads / d.k_heads) * d.q_len;
  const int kt = dt == PRISM_F32 ? 32 : 64;
  // Launches that leave CUs without work are cut along the other axis, into parts of four tiles at least: 512 workgroups, two per CU.  Under the causal mask parts are of
  // unequal length; in fp32, where products outweigh the join, twice as many even that out (2 x 2048 x 8 heads of 80: forward 222 us with 512, 153 with 1024; gradients of heads of
  // 64: 462 and 392).  Not where one workgroup fits a CU (gradients of heads of 80: 547 and 562) nor in bf16 (2 x 1111, heads of 128: 88 and 101).
  const int target = dt == PRISM_F32 && d.causal && !(backward && d.head_dim > 64) ? 1024 : 512;
  auto parts = [target](long long groups, long long tiles) {
    if (groups == 0) return 1;
    const long long want = target / groups, most = (tiles + 3) / 4;
    const long long n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
  };
  a.split = parts(pairs * ((R + 127) / 128), (d.k_len + kt - 1) / kt);
  a.few = !backward && dt == PRISM_BF16 && R <= 32 && !d.q_doc;
  if (a.few && pairs > 0) {   // parts of 256 keys (two blocks a wave) at least, twice the workgroups that run at once: sequences of unequal length.  8 tokens of 32 heads on 8 key heads
    // of 128, 4096 to 16384 keys: 512 workgroups 78 us, 1024 84, 1536 95
    const long long want = (512 + pairs - 1) / pairs, most = (d.k_len + 255) / 256;
    const long long n = want < most ? want : most;
    a.split = (int)(n < 1 ? 1 : n > 64 ? 64 : n);
  }
  // dk and dv: the rows of a key tile are many or few under the causal mask.  Up to 512 key tiles (two workgroups per CU) are cut into parts of equal length,
  // 1024 at most; 2 x 4096 x 16 heads of 128 on 4 key heads: 628 us in two parts each, 545 in 512 parts of equal length, 509 in 1024 (with their sum).
  const int key_tiles = (d.k_len + 127) / 128;
  a.parts = 1;
  a.items = key_tiles;
  if (backward && pairs * key_tiles > 0 && pairs * key_tiles <= 512) {
    long long all = 0;
    for (int k = 0; k < key_tiles; ++k) all += rows_of_key_tile(d.causal, d.prefix, d.q_len, d.k_len, (int)(R / (d.q_len ? d.q_len : 1)), k);
    long long chunk = (all * pairs + 1023) / 1024;
    for (chunk = chunk < 4 * kt ? 4 * kt : (chunk + 31) / 32 * 32;; chunk += (chunk / 16 + 31) / 32 * 32) {
      a.items = 0;
      a.parts = 1;
      for (int k = 0; k < key_tiles; ++k) {
        const int n = parts_of(rows_of_key_tile(d.causal, d.prefix, d.q_len, d.k_len, (int)(R / (d.q_len ? d.q_len : 1)), k), (int)chunk);
        a.items += n;
        if (n > a.parts) a.parts = n;
      }
      if (a.items * pairs <= 1024) break;
    }
    a.chunk = a.parts > 1 ? (int)chunk : 0;
  }
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = (at + bytes + 255) & ~(size_t)255;
    return o;
  };
  if (d.q_doc) take((size_t)d.batch * ((d.q_len + 63) / 64 + (d.k_len + 63) / 64) * sizeof(int4));
  if (backward) a.o_stat = take(((size_t)pairs * 2 * R + 64) * sizeof(float));
  size_t part = a.split > 1 ? (size_t)a.split * pairs * R * d.head_dim * sizeof(float) : 0;
  const size_t dkv = a.parts > 1 ? (size_t)2 * a.parts * pairs * d.k_len * d.head_dim * sizeof(float) : 0;
  a.o_part = take(part > dkv ? part : dkv);
  a.o_ml = take(a.split > 1 && !backward ? (size_t)a.split * pairs * R * 2 * sizeof(float) : 0);
  a.total = at;
  return a;
}

void launch_doc_ranges(const prism_attention_desc& d, int4* to, hipStream_t s) {
  const long long blocks = ((long long)(d.q_len + 63) / 64 + (d.k_len + 63) / 64) * d.batch;
  if (!d.q_doc || blocks == 0) return;
  ProfScope prof(PK_ATTENTION_DOCS, s);
  hipLaunchKernelGGL(doc_range_kernel, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, s, d.q_doc, d.k_doc, to, d.q_len, d.k_len, d.batch);
}

int launch_attention(const void* q, const void* k, const void* v, void* out, float* lse, int dt, const prism_attention_desc& d, char* ws, hipStream_t s) {
  const AttnPlan plan = attention_plan(d, dt, false);
  Attn p = attn_common(q, k, v, dt, d, ws);
  launch_doc_ranges(d, (int4*)ws, s);
  p.out = out;
  p.lse = lse;
  set_strides(p.os, d.out);
  p.nsplit = plan.split;
  p.part = (float*)(ws + plan.o_part);
  p.part_ml = (float*)(ws + plan.o_ml);
  p.direct = p.direct && rows_are_vectors(out, d.out, dt);
  // The parts were counted for the kernel that the sizes ask for; what it cannot read (rows that are no whole vectors) the other one takes in the same parts.
  const bool few = plan.few && p.direct;
  if (dt == PRISM_F32)
    return d.head_dim <= 32 ? launch<float, 32>(p, few, s) : d.head_dim <= 64 ? launch<float, 64>(p, few, s) : d.head_dim <= 96 ? launch<float, 96>(p, few, s) : launch<float, 128>(p, few, s);
  return d.head_dim <= 64 ? launch<__bf16, 64>(p, few, s) : d.head_dim <= 96 ? launch<__bf16, 96>(p, few, s) : launch<__bf16, 128>(p, few, s);
}

}  // namespace prism
