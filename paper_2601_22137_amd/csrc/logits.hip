// What is computed from rows of logits and one token of each: its log-probability, losses of it, and the logits' gradients.
//
//   logp = s z_t - lse, lse = log sum_j exp(s z_j);   dz_j = s d ([j = t] - exp(s z_j - lse)), d = the derivative of the loss by logp
//   with o = sum over j other than t of exp(s (z_j - z_t)):   logp = -log(1 + o), 1 - p_t = o / (1 + o), dz_t = s d (1 - p_t)
//   loss = sum w l,  l = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(f) - f - 1),  r = exp(logp - old), f = ref - logp;  without old l = -A logp + ...
//   dl / dlogp = -(r A where r A <= clip(r) A, else 0) + kl (1 - exp(f))
//
// A row is one workgroup's (or one wave's, to 4096 logits of bf16).  Its exponentials are taken in base 2 relative to a running maximum m, exp2(c (z - m)), c = s log2 e, every thread with its own, joined
// at the end: the difference first, so that logits of the type's lowest value (masks) neither overflow nor differ from one another.  The sum is over the others than the token, in 32 bits to its end,
// joins too: o has its errors, and so 1 - p_t and logp have them relative to themselves, however close to certain the token is.  The loss follows from logp in 64 bits: a ratio next to where it is
// cut off decides about a row's gradient.
//
// Loss and gradient in one pass hold the row in registers, up to 16384 vectors of 16 bytes, so that it is read once and written once: 8192 x 32768 bf16 172 us (1013 MB, 5.9 TB/s, vector units 73 % busy),
// 2048 x 131072 204 us (5.0 TB/s: the registers of a CU hold one such row, and nothing reads while it is computed).  Read twice, the second time from the caches: 249 and 266.  Log-probabilities
// alone, 4096 x 131072: 165 us, 6.5 TB/s.  The gradient of given derivatives, in the same way: 8192 x 32768 201 us, 4096 x 32000 fp32 181.  Two transcendental instructions a logit, four cycles each, are half of what the vector units do.
#include <cmath>

#include "layer.h"
#include "row_vector.h"

namespace prism {
namespace {

struct Logits {
  const void *z, *tokens;
  void* dz;
  float *logp, *lse, *dlogp;             // results
  const float *dlogp_given, *lse_given;  // backward
  const float *advantages, *old, *ref, *weights;
  double *losses, *mean;                 // weighted losses of the rows; one over the number of rows with a token (null: every workgroup counts them itself)
  long long rows, zs, ds;
  int vocabulary;
  float c, c_rest, scale;                // scale log2 e, rounded; fp32: rounded down and the rest, which is positive so that infinite differences keep their sign
  double low, high, kl, exact_scale;
  bool wide;
};

constexpr double LN2 = 0.69314718055994530942;

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// c (z - m): fp32 with the rest of c, whose rounding would show there (of a difference of 20: 4e-7 of the exponential).  bf16 leaves it out, an instruction in nine: its logits are rounded by 2^-8 of
// themselves, and logp and lse take 2^-24 of the mean distance from the largest, 3e-7 of 5.
template <typename T> __device__ inline float power(const Logits& p, float z, float m) {
  const float d = z - m;
  if constexpr (sizeof(T) == 4) return fmaf(d, p.c, d * p.c_rest);
  else return d * p.c;
}

// exp2(c (z - m)) of many z.  bf16 takes c z - (c m rounded) as one fused product and makes up for that rounding once, by the factor `rest`; not where c m is so large that its
// rounding is no longer small, or overflows (masks of the lowest value).  One instruction in nine of an exponential less: the vector units bound these kernels as much as memory does.
struct Reference {
  float m, cm, rest;
  bool fused;
  __device__ Reference(const Logits& p, float m, bool bf16) : m(m), cm(m * p.c) {
    fused = bf16 && fabsf(cm) < 1048576.0f;
    rest = fused ? exp2_of(-fmaf(m, p.c, -cm)) : 1.0f;
  }
};
template <typename T, bool FUSED> __device__ inline float exp_of(const Logits& p, const Reference& r, float z) {
  return exp2_of(FUSED ? fmaf(z, p.c, -r.cm) : power<T>(p, z, r.m));
}
// f(whether fused), a constant
template <typename T, typename F> __device__ inline void either(const Reference& r, F&& f) {
  if constexpr (sizeof(T) == 2) {
    if (r.fused) return f(std::true_type{});
  }
  f(std::false_type{});
}

// sum_j 2^(c z_j) = s 2^(c m); no terms: m = -inf, s = 0
struct Sum {
  float m = -INFINITY, s = 0.0f;
  __device__ float reference() const { return m == -INFINITY ? 0.0f : m; }
  template <typename T> __device__ void raise(const Logits& p, float to) {
    if (to > m) {
      s *= exp2_of(power<T>(p, m, to));
      m = to;
    }
  }
  template <typename T> __device__ void join(const Logits& p, float om, float os) {
    const float to = fmaxf(m, om), by = to == -INFINITY ? 0.0f : to;
    s = s * exp2_of(power<T>(p, m, by)) + os * exp2_of(power<T>(p, om, by));
    m = to;
  }
};

// Entry `at` of a vector, if it has one.  By words: entries of 16 bits, one by one, take twice the instructions.
template <typename T> __device__ inline void set_entry(typename Vec<T>::type& v, int at, float x) {
  typedef unsigned words __attribute__((ext_vector_type(4)));
  words w = __builtin_bit_cast(words, v);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = i == at ? __builtin_bit_cast(unsigned, x) : w[i];
  } else {
    const unsigned stays = at & 1 ? 0x0000FFFFu : 0xFFFF0000u, put = __builtin_bit_cast(unsigned short, (T)x) * 0x10001u & ~stays;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = i == at >> 1 ? (w[i] & stays) | put : w[i];
  }
  v = __builtin_bit_cast(typename Vec<T>::type, w);
}

// The sum over a row without its token t.  The row is read in pieces of K vectors a thread, all on their way before the first is used.
template <typename T, int THREADS, bool PAST> __device__ inline Sum own_sum(const Logits& p, const T* z, int t) {
  constexpr int N = Vec<T>::N, K = 4;
  using V = typename Vec<T>::type;
  Sum a;
  for (int first = 0; first < p.vocabulary; first += K * THREADS * N) {
    V v[K];
#pragma unroll
    for (int j = 0; j < K; ++j) v[j] = load_vector<T, PAST>(z + first + j * THREADS * N, (int)threadIdx.x * N, p.vocabulary - first - j * THREADS * N, -INFINITY);
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int place = t - first - j * THREADS * N;                      // the same in all threads: one piece has it
      if ((unsigned)place < (unsigned)(THREADS * N)) set_entry<T>(v[j], place - (int)threadIdx.x * N, -INFINITY);
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) top = fmaxf(top, (float)v[j][e]);
    a.raise<T>(p, top);
    const Reference r(p, a.reference(), sizeof(T) == 2);
    float part[4] = {};
    either<T>(r, [&](auto fused) {
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (first + j * THREADS * N >= p.vocabulary) break;               // (nothing of the row in this piece)
        as_loaded<T>(v[j]);
#pragma unroll
        for (int e = 0; e < N; ++e) part[e & 3] += exp_of<T, fused.value>(p, r, (float)v[j][e]);
      }
    });
    a.s += ((part[0] + part[1]) + (part[2] + part[3])) * r.rest;
  }
  return a;
}

// The sum of the workgroup, in every thread
template <typename T, int THREADS> __device__ inline Sum whole_row(const Logits& p, Sum a, float2* memory) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) a.join<T>(p, __shfl_xor(a.m, d), __shfl_xor(a.s, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) memory[threadIdx.x >> 6] = make_float2(a.m, a.s);
  __syncthreads();
  Sum b;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) b.join<T>(p, memory[w].x, memory[w].y);
  return b;
}

__device__ inline int token_of(const Logits& p, long long row) {
  const long long t = p.wide ? ((const long long*)p.tokens)[row] : (long long)((const int*)p.tokens)[row];
  return t >= 0 && t < p.vocabulary ? (int)t : -1;
}

// What is given for a row, read ahead
struct Given {
  int token;
  float weight, advantage, old, ref;     // backward: weight is the derivative by logp
};
__device__ inline Given given_for(const Logits& p, long long row) {
  Given g = {__builtin_amdgcn_readfirstlane(token_of(p, row)), 0.0f, 1.0f, 0.0f, 0.0f};
  if (p.weights) g.weight = p.weights[row];
  if (p.dlogp_given) g.weight = p.dlogp_given[row];
  if (p.advantages) g.advantage = p.advantages[row];
  if (p.old) g.old = p.old[row];
  if (p.kl != 0.0) g.ref = p.ref[row];
  return g;
}

// exp2(c (x - y)), x <= y, good to what the instruction is, 1 ulp in 32 bits, however far they are apart: with what the roundings of the difference, of the factor and of their product left over
__device__ inline float exp_of_difference(const Logits& p, float x, float y) {
  const float d = x - y, back = d - x, rest = (x - (d - back)) - (y + back), k = d * p.c;
  return k < -150.0f ? 0.0f : exp2_of(k) * fmaf(fmaf(d, p.c, -k) + fmaf(d, p.c_rest, rest * p.c), (float)LN2, 1.0f);
}

// log(1 + y), y from -2^-20, NaN for NaN: 1 + y = f 2^k, f next to 1, and log f = 2 artanh((f - 1) / (f + 1)), its series cut off where it is 4e-14 of it; f - 1 is y where k is 0, so that small ones
// keep their digits.  (The library's log and log1p are good to a unit of 64 bits, with three times the instructions and, log1p, a dozen registers more, for a sum in 32 bits.)
__device__ inline double log_of_one_and(double y) {
  double f = __builtin_amdgcn_frexp_mant(1.0 + y);
  int k = __builtin_amdgcn_frexp_exp(1.0 + y);
  if (f < 0.70710678118654752440) {
    f *= 2.0;
    --k;
  }
  double r = __builtin_amdgcn_rcp(f + 1.0);
  r = fma(fma(-(f + 1.0), r, 1.0), r, r);
  const double x = (k == 0 ? y : f - 1.0) * r, q = x * x;
  double series = 2.0 / 15;
#pragma unroll
  for (int i = 13; i > 1; i -= 2) series = fma(series, q, 2.0 / i);
  return fma((double)k, LN2, fma(series * q, x, 2.0 * x));
}

// The sum over a row's other logits beside its token's exponential e = exp(-|s (m - z)|), which is as good as that sum.  z: the logit of the token
struct Others {
  float e;
  bool above;                   // one of them is, m > z: everything relative to m then, to z otherwise
  __device__ Others(const Logits& p, const Sum& a, float z) : above(a.m > z) { e = exp_of_difference(p, above ? z : a.m, above ? a.m : z); }
  // all of them, less 1
  __device__ float rest(const Sum& a) const { return above ? (a.s - 1.0f) + e : a.s * e; }
  // 1 - p_t
  __device__ float share(const Sum& a) const { return (above ? a.s : a.s * e) * __builtin_amdgcn_rcpf(1.0f + rest(a)); }
  // logp = -max(0, s (m - z)) - this
  __device__ double log_of_all(const Sum& a) const { return log_of_one_and(rest(a)); }
};

__device__ inline float share_of_one(float z) { return z == -INFINITY ? 1.0f : z - z; }         // no others: 0, and NaN stays
__device__ inline float share_of(const Logits& p, const Sum& a, float z) { return a.s == 0.0f ? share_of_one(z) : Others(p, a, z).share(a); }

// What one thread computes of a row: its results, and the gradient at the token, s d (1 - p_t)
__device__ inline float finish_row(const Logits& p, long long row, const Given& g, int count, const Sum& a, float z) {
  if (p.dlogp_given) return g.weight * p.scale * share_of(p, a, z);
  double logp, lse;
  float share;
  if (a.s == 0.0f) {            // no others
    share = share_of_one(z);
    logp = z == -INFINITY ? -INFINITY : share;
    lse = z * p.exact_scale;
  } else {
    const Others o(p, a, z);
    share = o.share(a);
    const double l = o.log_of_all(a);
    logp = 0.0 - (o.above ? ((double)a.m - z) * p.exact_scale + l : l);
    lse = (o.above ? a.m : z) * p.exact_scale + l;
  }
  if (p.logp) p.logp[row] = (float)logp;
  if (p.lse) p.lse[row] = (float)lse;
  if (!p.losses) return 0.0f;
  const double w = p.weights ? (double)g.weight : p.mean ? *p.mean : 1.0 / count;
  double l = 0.0, d = 0.0;
  if (w != 0.0) {
    const double A = g.advantage;
    if (p.old) {
      const double r = exp(logp - g.old), low = 1.0 - p.low, high = 1.0 + p.high, held = (r < low ? low : r > high ? high : r) * A, free = r * A;
      if (free <= held || r != r || A != A) {
        l = -free;
        d = -free;
      } else {
        l = -held;
      }
    } else {
      l = -A * logp;
      d = -A;
    }
    if (p.kl != 0.0) {
      const double f = g.ref - logp, e = expm1(f);
      l += p.kl * (e - f);
      d -= p.kl * e;
    }
    l *= w;
    d *= w;
  }
  p.losses[row] = l;
  if (p.dlogp) p.dlogp[row] = (float)d;
  return (float)d * p.scale * share;
}

// The token's logit; +inf is no number here, as it is among the others (inf less inf)
template <typename T> __device__ inline float logit_of(const T* z, int t) {
  const float x = (float)z[t];
  return x < INFINITY ? x : NAN;
}
// What the exponentials of the others are multiplied by; no others: 0, and NaN as ever where the token's gradient is
__device__ inline float factor_of(const Sum& a, float token) { return a.s == 0.0f ? 0.0f * token : token / a.s; }

// Rows with a token, by the whole workgroup
template <int THREADS> __device__ inline int count_rows(const Logits& p) {
  int n = 0;
  if (p.losses && !p.weights && !p.mean)
    for (long long first = 0; first < p.rows; first += THREADS) n += __syncthreads_count(first + threadIdx.x < p.rows && token_of(p, first + threadIdx.x) >= 0);
  return n;
}

// A row without a token
__device__ inline void skip_row(const Logits& p, long long row) {
  if (p.logp) p.logp[row] = 0.0f;
  if (p.lse) p.lse[row] = 0.0f;
  if (p.dlogp) p.dlogp[row] = 0.0f;
  if (p.losses) p.losses[row] = 0.0;
}

template <typename T> __device__ inline void clear_row(const Logits& p, long long row, int threads) {
  T* dz = (T*)p.dz + row * p.ds;
  for (int at = threadIdx.x * Vec<T>::N; at < p.vocabulary; at += threads * Vec<T>::N) store_vector(dz, at, p.vocabulary, typename Vec<T>::type{});
}

// A vector of the gradient, the token's entry aside: -exp2(c (z - m)) factor; factor has the reference's rest in it
template <typename T, bool FUSED>
__device__ inline typename Vec<T>::type gradient(const Logits& p, const Reference& r, const typename Vec<T>::type& v, float factor) {
  constexpr int N = Vec<T>::N;
  float g[N];
#pragma unroll
  for (int e = 0; e < N; ++e) g[e] = exp_of<T, FUSED>(p, r, (float)v[e]) * -factor;
  return rounded<T>(g);
}

template <typename T, int THREADS, bool GRAD, bool PAST>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4))) logits_kernel(Logits p) {
  constexpr int N = Vec<T>::N;
  __shared__ float2 memory[THREADS / 64];
  __shared__ float result;
  const int count = count_rows<THREADS>(p);
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const Given g = given_for(p, row);
    const int t = g.token;
    if (t < 0) {
      if (threadIdx.x == 0) skip_row(p, row);
      if constexpr (GRAD) clear_row<T>(p, row, THREADS);
      continue;
    }
    const T* z = (const T*)p.z + row * p.zs;
    const float zt = logit_of(z, t);
    const Sum a = whole_row<T, THREADS>(p, own_sum<T, THREADS, PAST>(p, z, t), memory);
    if (threadIdx.x == 0) result = finish_row(p, row, g, count, a, zt);
    if constexpr (GRAD) {
      __syncthreads();
      const Reference r(p, a.reference(), sizeof(T) == 2);
      const float own = result, factor = factor_of(a, own) * r.rest;
      T* dz = (T*)p.dz + row * p.ds;
      either<T>(r, [&](auto fused) {
        for (int first = 0; first < p.vocabulary; first += 4 * THREADS * N) {
          typename Vec<T>::type v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = load_vector(z + first + j * THREADS * N, (int)threadIdx.x * N, p.vocabulary - first - j * THREADS * N, -INFINITY);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int width = p.vocabulary - first - j * THREADS * N, place = t - first - j * THREADS * N;
            if (width <= 0) break;
            as_loaded<T>(v[j]);
            typename Vec<T>::type o = gradient<T, fused.value>(p, r, v[j], factor);
            if ((unsigned)place < (unsigned)(THREADS * N)) set_entry<T>(o, place - (int)threadIdx.x * N, own);
            store_vector(dz + first + j * THREADS * N, (int)threadIdx.x * N, width, o);
          }
        }
      });
      __syncthreads();
    }
  }
}

// The same with the row in registers, NV vectors a thread: loss and gradient, or the gradient alone, read it once
template <typename T, int THREADS, int NV, bool PAST>
__global__ void __launch_bounds__(THREADS) logits_held_kernel(Logits p) {
  constexpr int N = Vec<T>::N;
  using V = typename Vec<T>::type;
  __shared__ float2 memory[THREADS / 64];
  __shared__ float result;
  const long long row = blockIdx.x;
  const Given g = given_for(p, row);
  const int t = g.token;
  if (t < 0) {
    if (threadIdx.x == 0) skip_row(p, row);
    clear_row<T>(p, row, THREADS);
    return;
  }
  const T* z = (const T*)p.z + row * p.zs;
  const float zt = logit_of(z, t);
  const int at = (int)threadIdx.x * N;       // in each of NV pieces of the row, whose beginnings all lanes share: one offset takes fewer registers than NV
  V v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) v[j] = load_vector<T, PAST>(z + j * THREADS * N, at, p.vocabulary - j * THREADS * N, -INFINITY);
  const int count = count_rows<THREADS>(p);         // (while the row is under way)
  float top = -INFINITY, part[4] = {};
#pragma unroll
  for (int j = 0; j < NV; ++j) {                    // the sum is over the others than the token
    const int place = t - j * THREADS * N;
    if ((unsigned)place < (unsigned)(THREADS * N)) set_entry<T>(v[j], place - at, -INFINITY);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, (float)v[j][e]);
  Sum a;
  a.m = top;
  const Reference own(p, a.reference(), sizeof(T) == 2);
  either<T>(own, [&](auto fused) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * THREADS * N >= p.vocabulary) break;          // (nothing of the row in this piece)
      as_loaded<T>(v[j]);
#pragma unroll
      for (int e = 0; e < N; ++e) part[e & 3] += exp_of<T, fused.value>(p, own, (float)v[j][e]);
    }
  });
  a.s = ((part[0] + part[1]) + (part[2] + part[3])) * own.rest;
  a = whole_row<T, THREADS>(p, a, memory);
  if (threadIdx.x == 0) result = finish_row(p, row, g, count, a, zt);
  __syncthreads();
  const Reference r(p, a.reference(), sizeof(T) == 2);
  const float token = result, factor = factor_of(a, token) * r.rest;
  T* dz = (T*)p.dz + row * p.ds;
  either<T>(r, [&](auto fused) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * THREADS * N >= p.vocabulary) break;
      as_loaded<T>(v[j]);
      const int width = p.vocabulary - j * THREADS * N, place = t - j * THREADS * N;
      V o = gradient<T, fused.value>(p, r, v[j], factor);
      if ((unsigned)place < (unsigned)(THREADS * N)) set_entry<T>(o, place - at, token);
      if constexpr (PAST) stream_vector_to(dz + j * THREADS * N, at, width, o);
      else store_vector(dz + j * THREADS * N, at, width, o);
    }
  });
}

// The gradient of rows that registers do not hold is taken from lse, up to this one as it was rounded: probabilities are off by 2^-24 |lse|, 2^-20 here and 2^-19 in bf16, whose own
// rounding is 2^-8.  A row beyond is summed once more (1000 x 131072 fp32: 312 us, 228 without).
template <typename T> constexpr float MOST_LSE = sizeof(T) == 4 ? 32.0f : 64.0f;

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(6))) logprob_backward_kernel(Logits p) {
  constexpr int N = Vec<T>::N, K = 4;
  using V = typename Vec<T>::type;
  __shared__ float2 memory[THREADS / 64];
  __shared__ float sums[THREADS / 32];
  int turn = 0;
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int t = __builtin_amdgcn_readfirstlane(token_of(p, row));
    if (t < 0) {
      clear_row<T>(p, row, THREADS);
      continue;
    }
    const T* z = (const T*)p.z + row * p.zs;
    T* dz = (T*)p.dz + row * p.ds;
    const float d = p.dlogp_given[row] * p.scale, lse = p.lse_given[row];
    const bool given = fabsf(lse) <= MOST_LSE<T>;
    float m, factor, token;
    if (given) {                         // the reference is lse / s, rounded; the factor makes up for its rounding
      const double exact = (double)lse / p.exact_scale;
      m = (float)exact;
      factor = d * exp2_of((float)((m - exact) * p.c));
    } else {                             // lse itself is rounded by too much: the sum once more
      const float zt = logit_of(z, t);   // (before the barriers, and dlogits may be the logits)
      const Sum a = whole_row<T, THREADS>(p, own_sum<T, THREADS, false>(p, z, t), memory);
      m = a.reference();
      token = d * share_of(p, a, zt);
      factor = factor_of(a, token);
    }
    const Reference r(p, m, sizeof(T) == 2);
    factor *= r.rest;
    float part[4] = {}, zt = 0.0f;       // of the others' exponentials; the token's logit, in the thread that has it
    either<T>(r, [&](auto fused) {
      for (int first = 0; first < p.vocabulary; first += K * THREADS * N) {
        V v[K];
#pragma unroll
        for (int j = 0; j < K; ++j) v[j] = load_vector(z + first + j * THREADS * N, (int)threadIdx.x * N, p.vocabulary - first - j * THREADS * N, -INFINITY);
#pragma unroll
        for (int j = 0; j < K; ++j) {
          const int width = p.vocabulary - first - j * THREADS * N, place = t - first - j * THREADS * N;
          if (width <= 0) break;
          as_loaded<T>(v[j]);
          if ((unsigned)place < (unsigned)(THREADS * N)) {
#pragma unroll
            for (int e = 0; e < N; ++e) zt = e == place - (int)threadIdx.x * N ? (float)v[j][e] : zt;
            set_entry<T>(v[j], place - (int)threadIdx.x * N, -INFINITY);
          }
          float g[N];
#pragma unroll
          for (int e = 0; e < N; ++e) {
            g[e] = exp_of<T, fused.value>(p, r, (float)v[j][e]);
            part[e & 3] += g[e];
            g[e] *= -factor;
          }
          store_vector(dz + first + j * THREADS * N, (int)threadIdx.x * N, width, rounded<T>(g));
        }
      }
    });
    // the token's by the thread that had it: d times the others' share of all, in which the rounding of lse is no more
    const float others = given ? row_sum<THREADS>((part[0] + part[1]) + (part[2] + part[3]), sums, turn++) : 0.0f;
    if (t / N % THREADS == (int)threadIdx.x) {
      if (given) {
        either<T>(r, [&](auto fused) { token = exp_of<T, fused.value>(p, r, zt); });
        token = d * (others / (others + token));
      }
      dz[t] = (T)token;
    }
  }
}

__device__ inline double block_sum(double v, double* memory) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) memory[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) v += memory[w];
  return v;
}

// One over the number of rows with a token
__global__ void __launch_bounds__(1024) count_rows_kernel(Logits p) {
  __shared__ double memory[16];
  int own = 0;
#pragma unroll 16
  for (long long row = threadIdx.x; row < p.rows; row += 1024) own += token_of(p, row) >= 0;
  const double n = block_sum(own, memory);
  if (threadIdx.x == 0) *p.mean = n > 0.0 ? 1.0 / n : 0.0;
}

__global__ void __launch_bounds__(1024) loss_sum_kernel(Logits p, float* loss) {
  __shared__ double memory[16];
  double v = 0.0, part[8] = {};
  const long long most = p.rows - p.rows % 8192;
  for (long long row = threadIdx.x; row < most; row += 8192) {          // eight reads on their way at a time
#pragma unroll
    for (int i = 0; i < 8; ++i) part[i] += p.losses[row + 1024 * i];
  }
  for (long long row = most + threadIdx.x; row < p.rows; row += 1024) v += p.losses[row];
#pragma unroll
  for (int i = 0; i < 8; ++i) v += part[i];
  v = block_sum(v, memory);
  if (threadIdx.x == 0) *loss = (float)v;
}

constexpr long long MOST_BLOCKS = 1 << 20;

Logits common(const void* z, const void* tokens, int dt, const prism_logits_desc& d) {
  Logits p = {};
  p.z = z; p.tokens = tokens;
  p.rows = d.rows; p.zs = d.logits_stride; p.ds = d.dlogits_stride; p.vocabulary = d.vocabulary; p.wide = d.wide_tokens;
  p.scale = (float)d.scale; p.exact_scale = d.scale;
  const double c = d.scale / LN2;
  p.c = (float)c;
  if (dt == PRISM_F32 && p.c >= c) p.c = std::nextafterf(p.c, 0.0f);
  p.c_rest = (float)(c - p.c);
  return p;
}

// Threads of a row that is read in pieces, whatever the number of rows, so that a row's results do not depend on what else is in the call.  Four vectors a thread are under way at a time, and fewer
// threads waste fewer of them (log-probabilities of 16384 rows of 8000 logits, bf16: 64 threads 44 us, 256 67).
int threads_of(int vocabulary) {
  const int vectors = (vocabulary + 7) / 8;
  return vectors <= 1024 ? 64 : vectors <= 4096 ? 256 : 512;
}

// Logits that do not fit the card's last cache are read past the caches where they are read once: 4096 x 131072 bf16, log-probabilities alone 165 us (177 through them)
template <typename T> bool past(const Logits& p) { return p.rows * p.vocabulary * (long long)sizeof(T) > (256ll << 20); }

template <typename T, int THREADS> void launch(const Logits& p, bool back, hipStream_t s) {
  void (*kernel)(Logits) = back ? logprob_backward_kernel<T, THREADS> : p.dz ? logits_kernel<T, THREADS, true, false> : past<T>(p) ? logits_kernel<T, THREADS, false, true> :
                                  logits_kernel<T, THREADS, false, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.rows < MOST_BLOCKS ? p.rows : MOST_BLOCKS)), dim3(THREADS), 0, s, p);
}
template <typename T> void by_threads(const Logits& p, int threads, bool back, hipStream_t s) {
  if (threads == 64) launch<T, 64>(p, back, s);
  else if (threads == 256) launch<T, 256>(p, back, s);
  else launch<T, 512>(p, back, s);
}

// The kernel that holds rows of that many vectors, or none
template <typename T, bool PAST> void (*held_kernel(int vectors, int& threads))(Logits) {
  if (vectors <= 64 * 8) return threads = 64, vectors <= 64 * 4 ? logits_held_kernel<T, 64, 4, PAST> : logits_held_kernel<T, 64, 8, PAST>;
  if (vectors <= 256 * 8) return threads = 256, vectors <= 256 * 4 ? logits_held_kernel<T, 256, 4, PAST> : logits_held_kernel<T, 256, 8, PAST>;
  if (vectors <= 512 * 5) return threads = 512, logits_held_kernel<T, 512, 5, PAST>;         // (three pieces of eight would hold nothing: 8192 x 20000 bf16 120 us, 124 in eight)
  if (vectors <= 512 * 8) return threads = 512, logits_held_kernel<T, 512, 8, PAST>;
  if (vectors <= 512 * 16) return threads = 512, logits_held_kernel<T, 512, 16, PAST>;        // two workgroups a CU: 2684 x 50001 bf16 133 us, with 1024 threads 159
  if (vectors <= 1024 * 16) return threads = 1024, logits_held_kernel<T, 1024, 16, PAST>;
  return nullptr;
}
template <typename T> bool held(const Logits& p, hipStream_t s) {
  int threads = 0;
  const int vectors = (p.vocabulary + Vec<T>::N - 1) / Vec<T>::N;
  void (*kernel)(Logits) = p.rows > MOST_BLOCKS ? nullptr : past<T>(p) ? held_kernel<T, true>(vectors, threads) : held_kernel<T, false>(vectors, threads);
  if (kernel) hipLaunchKernelGGL(kernel, dim3((unsigned)p.rows), dim3(threads), 0, s, p);
  return kernel != nullptr;
}

void by_type(const Logits& p, int dt, bool back, hipStream_t s) {
  if (p.dz && (dt == PRISM_F32 ? held<float>(p, s) : held<__bf16>(p, s))) return;
  if (dt == PRISM_F32) by_threads<float>(p, threads_of(p.vocabulary), back, s);
  else by_threads<__bf16>(p, threads_of(p.vocabulary), back, s);
}

}  // namespace

int launch_logprob(const void* z, const void* tokens, float* logp, float* lse, int dt, const prism_logits_desc& d, hipStream_t s) {
  ProfScope prof(PK_LOGPROB, s);
  Logits p = common(z, tokens, dt, d);
  p.logp = logp; p.lse = lse;
  by_type(p, dt, false, s);
  return PRISM_OK;
}

int launch_logprob_backward(const float* dlogp, const void* z, const void* tokens, const float* lse, void* dz, int dt, const prism_logits_desc& d, hipStream_t s) {
  ProfScope prof(PK_LOGPROB_BACKWARD, s);
  Logits p = common(z, tokens, dt, d);
  p.dlogp_given = dlogp; p.lse_given = lse; p.dz = dz;
  by_type(p, dt, true, s);
  return PRISM_OK;
}

size_t policy_loss_bytes(const prism_logits_desc& d) { return (size_t)(d.rows + 1) * sizeof(double); }

int launch_policy_loss(const void* z, const void* tokens, float* loss, float* logp, float* lse, float* dlogp, void* dz, int dt, const prism_logits_desc& d, char* ws,
                       hipStream_t s) {
  Logits p = common(z, tokens, dt, d);
  p.logp = logp; p.lse = lse; p.dlogp = dlogp; p.dz = dz;
  p.advantages = d.advantages; p.old = d.old_logp; p.ref = d.ref_logp; p.weights = d.weights;
  p.low = d.clip_low; p.high = d.clip_high; p.kl = d.kl;
  p.losses = (double*)ws + 1;
  // a launch of its own counts the rows if there are many: a workgroup reads as many tokens as it has logits otherwise
  if (!p.weights && (p.rows > 4096 || p.rows * 16 > p.vocabulary)) p.mean = (double*)ws;
  {
    ProfScope prof(PK_LOSS_SUM, s);
    if (p.mean) hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, p);
  }
  if (p.rows) {
    ProfScope prof(PK_POLICY_LOSS, s);
    by_type(p, dt, false, s);
  }
  ProfScope prof(PK_LOSS_SUM, s);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, s, p, loss);
  return PRISM_OK;
}

}  // namespace prism
