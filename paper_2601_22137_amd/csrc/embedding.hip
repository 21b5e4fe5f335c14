// Rows of a table by token, times a factor, and the table's gradient.
//
//   out[i] = scale table[token[i]], 0 for a token that is no row;   dtable[v] = scale sum over i with token[i] = v of dout[i], 0 for a row without a token
//
// The gradient is a sum over sorted tokens, so that the same call gives the same bits whatever the order in which workgroups run:
//   sort   a workgroup has a range of the table's rows, about a 256th; it goes through all tokens, counts those of each of its rows and those before its range, keeps its own in LDS and puts
//          them, 64 at a time, in their places.  Nothing passes between workgroups.  65536 tokens, 32768 rows: 16.7 us (every workgroup looks at every token, and the one with the commonest has the most to do); 16384
//          tokens: 9.
//   sums   the sorted tokens are cut into tiles of equal length; a wave adds up the rows of dout of a tile, 64 vectors of 16 bytes wide, eight rows under way, in 32 bits.  A run of equal
//          tokens that lies in one tile goes straight to the table; what crosses a border is kept as partial sums.  Other waves clear the rows without tokens.  Memory: 65536 x 768
//          bf16 into 32768 rows 30 us, 161 MB; 16384 x 4096 into 131072 rows 213 us, 1216 MB, most of them zeros (a fill alone runs at 6.8 TB/s).
//   join   partial sums of a run in their order, in 64 bits, long runs by eight waves together: 8 to 9 us, a chain of five dependent reads.
// The lookup: 65536 x 768 from 32768 rows 23 us (147 MB), 16384 x 4096 from 131072 rows 50 us (229 MB, rows at random); a few tokens: 3 us, and the host's call.
#include "layer.h"
#include "row_vector.h"

namespace prism {
namespace {

constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, MAX_RANGE = 512, LIST = 512, AHEAD = 8, SUM_AHEAD = 8;

// Token i as an unsigned number; what is no row of a table is 2^31 or more, or past its rows
template <typename I> __device__ inline unsigned token_at(const void* tokens, long long i) {
  const I t = ((const I*)tokens)[i];
  return sizeof(I) == 8 && (unsigned long long)t >> 32 ? 0xFFFFFFFFu : (unsigned)t;
}

// Where lane vector c of a row begins.  The last one ends with the row and may repeat entries of the one before (the same values are then stored twice), so that every
// vector is whole; WHOLE: the row has a vector's entries at least.
template <typename T, bool WHOLE> __device__ inline int column(int c, int width) { return WHOLE && c > width - Vec<T>::N ? width - Vec<T>::N : c; }
template <typename T, bool WHOLE> __device__ inline typename Vec<T>::type load_piece(const T* row, int c, int width) {
  if constexpr (WHOLE) return *(const typename Vec<T>::type*)(row + c);
  else return load_vector(row, c, width);
}
template <typename T, bool WHOLE, bool PAST> __device__ inline void store_piece(T* row, int c, int width, const typename Vec<T>::type& v) {
  if constexpr (WHOLE && PAST) __builtin_nontemporal_store(v, (typename Vec<T>::type*)(row + c));
  else if constexpr (WHOLE) *(typename Vec<T>::type*)(row + c) = v;
  else store_vector(row, c, width, v);
}

// The lookup's result goes past the caches where it fills a quarter of the last one, dout where it and the table fill half of it: 65536 tokens x 768 bf16, 32768 rows, 78 us among others (93 through them).
// The table's gradient does not: 16384 x 4096 into 131072 rows, with the lookup, 294 us past the caches, 283 through them.
template <typename T> bool fills(long long rows, int width, int megabytes) { return rows * width * (long long)sizeof(T) > (long long)megabytes << 20; }

struct Lookup {
  const void *table, *tokens;
  void* out;
  long long count, rows, ts, os;
  int width, lanes;             // lanes (a power of two up to 256) share a row
  float scale;
};

template <typename T, typename I, bool WHOLE, bool PAST> __global__ void __launch_bounds__(256) embedding_kernel(Lookup p) {
  using V = typename Vec<T>::type;
  constexpr int N = Vec<T>::N, NV = 4;
  const int lane = threadIdx.x & (p.lanes - 1), per = 256 / p.lanes;
  for (long long i = (long long)blockIdx.x * per + threadIdx.x / p.lanes; i < p.count; i += (long long)gridDim.x * per) {
    const unsigned t = token_at<I>(p.tokens, i);
    const bool there = t < p.rows;
    const T* row = (const T*)p.table + (there ? t : 0) * p.ts;
    T* to = (T*)p.out + i * p.os;
    for (int first = 0; first < p.width; first += p.lanes * N * NV) {
      V v[NV] = {};
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (first + j * p.lanes * N < p.width && there) v[j] = load_piece<T, WHOLE>(row, column<T, WHOLE>(first + (j * p.lanes + lane) * N, p.width), p.width);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (first + j * p.lanes * N >= p.width) break;
        float o[N];
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = there ? (float)v[j][e] * p.scale : 0.0f;
        store_piece<T, WHOLE, PAST>(to, column<T, WHOLE>(first + (j * p.lanes + lane) * N, p.width), p.width, rounded<T>(o));
      }
    }
  }
}

struct Sorted {
  const void* tokens;
  int* starts;                  // [rows + 1]: where a row's tokens begin
  int2* sorted;                 // (token, index), by token and then index
  int count;
  unsigned range;
  long long rows;
};

template <typename I> __global__ void __launch_bounds__(SORT_THREADS) embedding_sort_kernel(Sorted p) {
  __shared__ int places[MAX_RANGE * SORT_WAVES];        // [row of the range][wave]: counts, then where the wave's next one goes
  __shared__ int2 lists[SORT_WAVES][LIST];              // the range's tokens among a wave's: (row of the range, index), in their order
  __shared__ int sums[SORT_WAVES];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const unsigned rows = (unsigned)p.rows, first = blockIdx.x * p.range, range = rows - first < p.range ? rows - first : p.range;
  const int slots = range * SORT_WAVES;
  for (int i = threadIdx.x; i < slots; i += SORT_THREADS) places[i] = 0;
  __syncthreads();
  // a wave has a part of the tokens, in whole sixty-fours
  const int part = ((p.count + SORT_THREADS - 1) / SORT_THREADS) * 64;
  const int begin = (int)((long long)wave * part < p.count ? wave * part : p.count), end = p.count - begin < part ? p.count : begin + part;
  auto load = [&](int i0, unsigned (&t)[AHEAD]) {
    if (i0 + 64 * AHEAD <= end) {            // (the same base for all lanes: no arithmetic for addresses)
      const I* from = (const I*)p.tokens + i0;
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) t[j] = token_at<I>(from, 64 * j + lane);
      return;
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + 64 * j + lane;
      t[j] = i < end ? token_at<I>(p.tokens, i) : 0xFFFFFFFFu;
    }
  };
  int below = 0, listed = 0;                            // of the wave; listed: all of them, also those for which the list has no room
  for (int i0 = begin; i0 < end; i0 += 64 * AHEAD) {
    unsigned t[AHEAD];
    load(i0, t);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const unsigned at = t[j] - first;
      below += __popcll(__ballot(t[j] < first));
      const unsigned long long some = __ballot(at < range);
      if (!some) continue;
      if (at < range) {
        atomicAdd(&places[at * SORT_WAVES + wave], 1);
        const int place = listed + __popcll(some & ((1ull << lane) - 1));
        if (place < LIST) lists[wave][place] = make_int2(at, i0 + 64 * j + lane);
      }
      listed += __popcll(some);
    }
  }
  // all tokens before the range
  if (lane == 0) sums[wave] = below;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) base += sums[w];
  __syncthreads();
  // exclusive sums over (row, wave): a thread takes consecutive slots
  constexpr int EACH = MAX_RANGE * SORT_WAVES / SORT_THREADS;
  int mine[EACH], total = 0;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int i = threadIdx.x * EACH + j;
    mine[j] = i < slots ? places[i] : 0;
    total += mine[j];
  }
  int before = total;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int up = __shfl_up(before, d);
    if (lane >= d) before += up;
  }
  if (lane == 63) sums[wave] = before;
  __syncthreads();
  before += base - total;
  for (int w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int i = threadIdx.x * EACH + j;
    if (i < slots) {
      places[i] = before;
      if (i % SORT_WAVES == 0) p.starts[first + i / SORT_WAVES] = before;
    }
    before += mine[j];
  }
  if (threadIdx.x == SORT_THREADS - 1 && first + range == rows) p.starts[rows] = before;
  __syncthreads();
  // 64 tokens into their places: lanes of the same row find each other by its bits, the first of them takes their places together
  const int bits = range > 1 ? 32 - __clz((int)range - 1) : 0;
  auto place = [&](bool in, int at, int i) {
    unsigned long long same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((at >> b) & 1);
      same &= (at >> b) & 1 ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << lane) - 1)), leader = in ? __ffsll((long long)same) - 1 : lane;
    int to = 0;
    if (in && before == 0) to = atomicAdd(&places[at * SORT_WAVES + wave], __popcll(same));
    to = __shfl(to, leader) + before;
    if (in) p.sorted[to] = make_int2((int)first + at, i);
  };
  if (listed <= LIST) {
    for (int k = 0; k < listed; k += 64) {
      const int2 e = k + lane < listed ? lists[wave][k + lane] : make_int2(0, 0);
      place(k + lane < listed, e.x, e.y);
    }
  } else {
    for (int i0 = begin; i0 < end; i0 += 64 * AHEAD) {
      unsigned t[AHEAD];
      load(i0, t);
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const unsigned at = t[j] - first;
        if (__ballot(at < range)) place(at < range, (int)at, i0 + 64 * j + lane);
      }
    }
  }
}

struct Sums {
  const void* dout;
  void* dtable;
  const int* starts;
  const int2* sorted;
  float* part;                  // [tile][run that came in, run that goes on][chunks x 64 vectors]
  long long rows, ds, ts;
  int width, tile, chunks, tile_waves, clear;   // clear: rows that a wave looks at together to clear those without tokens
  float scale;
};

template <typename T, bool WHOLE> __device__ inline void put(const Sums& p, int token, int c, const float (&sum)[Vec<T>::N]) {
  float o[Vec<T>::N];
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) o[e] = sum[e] * p.scale;
  store_piece<T, WHOLE, false>((T*)p.dtable + token * p.ts, column<T, WHOLE>(c, p.width), p.width, rounded<T>(o));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T> __device__ inline f32x4* part_of(const Sums& p, int tile, int which, int c) {
  return (f32x4*)(p.part + ((size_t)tile * 2 + which) * (p.chunks * 64 * Vec<T>::N) + c);
}
template <typename T> __device__ inline void keep(const Sums& p, int tile, int which, int c, const float (&sum)[Vec<T>::N]) {
  f32x4* to = part_of<T>(p, tile, which, c);
#pragma unroll
  for (int e = 0; e < Vec<T>::N; e += 4) to[e / 4] = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
}

template <typename T, bool WHOLE, bool PAST> __global__ void __launch_bounds__(256) embedding_sums_kernel(Sums p) {
  using V = typename Vec<T>::type;
  constexpr int N = Vec<T>::N;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (wave >= p.tile_waves) {
    // some neighbouring rows at a time, each lane looks at one
    const long long stride = (long long)(gridDim.x * 4 - p.tile_waves) * p.clear;
    for (long long first = (long long)(wave - p.tile_waves) * p.clear; first < p.rows; first += stride) {
      const long long row = first + lane;
      const bool empty = lane < p.clear && row < p.rows && p.starts[row] == p.starts[row + 1];
      for (unsigned long long left = __ballot(empty); left; left &= left - 1) {
        T* to = (T*)p.dtable + (first + __ffsll((long long)left) - 1) * p.ts;
        for (int c = lane * N; c < p.width; c += 64 * N) store_piece<T, WHOLE, false>(to, column<T, WHOLE>(c, p.width), p.width, V{});
      }
    }
    return;
  }
  const int count = p.starts[p.rows], tile = wave / p.chunks, c = ((wave - tile * p.chunks) * 64 + lane) * N, from = column<T, WHOLE>(c, p.width);
  const long long begin = (long long)tile * p.tile;
  if (begin >= count) return;
  const long long end = count - begin < p.tile ? count : begin + p.tile;
  const int last = begin ? p.sorted[begin - 1].x : -1, next = end < count ? p.sorted[end].x : -1;     // tokens before and behind the tile
  int token = -1;
  bool inside = false;                      // the run began in this tile
  float sum[N] = {};
  for (long long b = begin; b < end; b += 64) {
    const int here = (int)(end - b < 64 ? end - b : 64);
    const int2 mine = p.sorted[b + (lane < here ? lane : here - 1)];
    if (b == begin) {
      token = __builtin_amdgcn_readfirstlane(mine.x);
      inside = token != last;
    }
    for (int j0 = 0; j0 < here; j0 += SUM_AHEAD) {
      V v[SUM_AHEAD];
#pragma unroll
      for (int j = 0; j < SUM_AHEAD; ++j) {
        const int at = __builtin_amdgcn_readlane(mine.y, j0 + j < here ? j0 + j : here - 1);
        const T* row = (const T*)p.dout + at * p.ds;
        if constexpr (WHOLE && PAST) v[j] = __builtin_nontemporal_load((const V*)(row + from));
        else v[j] = load_piece<T, WHOLE>(row, from, p.width);
      }
#pragma unroll
      for (int j = 0; j < SUM_AHEAD; ++j) {
        if (j0 + j >= here) break;
        const int t = __builtin_amdgcn_readlane(mine.x, j0 + j);
        if (t != token) {
          if (inside) put<T, WHOLE>(p, token, c, sum);
          else keep<T>(p, tile, 0, c, sum);
#pragma unroll
          for (int e = 0; e < N; ++e) sum[e] = 0.0f;
          token = t;
          inside = true;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += (float)v[j][e];
      }
    }
  }
  if (inside && next != token) put<T, WHOLE>(p, token, c, sum);
  else keep<T>(p, tile, inside ? 1 : 0, c, sum);
}

// Partial sums of the runs that cross borders between tiles.  A workgroup has BORDERS of them and 64 vectors of 16 bytes; its waves find those that are the
// first of a run, and take the runs in turn, long ones together.
constexpr int BORDERS = 16, JOIN_WAVES = 8, LONG_RUN = 24;

template <typename T> __device__ inline void add_parts(const Sums& p, int tile, int from, int to, int c, double (&sum)[Vec<T>::N]) {
#pragma unroll 4
  for (int t = from; t < to; ++t) {
    const f32x4* part = part_of<T>(p, t, t == tile ? 1 : 0, c);
    f32x4 v[Vec<T>::N / 4];
#pragma unroll
    for (int e = 0; e < Vec<T>::N / 4; ++e) v[e] = part[e];
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) sum[e] += v[e / 4][e % 4];
  }
}

template <typename T, bool WHOLE> __global__ void __launch_bounds__(64 * JOIN_WAVES) embedding_join_kernel(Sums p) {
  constexpr int N = Vec<T>::N;
  __shared__ double sums[JOIN_WAVES][64 * N];
  __shared__ int2 runs[BORDERS];                                   // (token, end of its last tile), or -1
  const int group = blockIdx.x / p.chunks, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, count = p.starts[p.rows];
  const int c = ((blockIdx.x - group * p.chunks) * 64 + lane) * N;
  if (threadIdx.x < BORDERS) {
    const int tile = group * BORDERS + threadIdx.x;
    const long long border = (long long)(tile + 1) * p.tile;
    int2 run = make_int2(-1, 0);
    if (border < count) {
      const int token = p.sorted[border].x;
      if (p.sorted[border - 1].x == token && p.starts[token] >= tile * p.tile) run = make_int2(token, (p.starts[token + 1] - 1) / p.tile + 1);
    }
    runs[threadIdx.x] = run;
  }
  __syncthreads();
  int turn = 0;
  for (int i = 0; i < BORDERS; ++i) {
    const int tile = group * BORDERS + i, token = runs[i].x, end = runs[i].y;
    if (token < 0) continue;
    double sum[N] = {};
    float whole[N];
    if (end - tile <= LONG_RUN) {
      if (turn++ % JOIN_WAVES != wave) continue;
      add_parts<T>(p, tile, tile, end, c, sum);
#pragma unroll
      for (int e = 0; e < N; ++e) whole[e] = (float)sum[e];
      put<T, WHOLE>(p, token, c, whole);
      continue;
    }
    const int share = (end - tile + JOIN_WAVES - 1) / JOIN_WAVES, from = tile + wave * share;
    add_parts<T>(p, tile, from, from + share < end ? from + share : end, c, sum);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) sums[wave][e * 64 + lane] = sum[e];
    __syncthreads();
    if (wave) continue;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      double v = 0.0;
      for (int w = 0; w < JOIN_WAVES; ++w) v += sums[w][e * 64 + lane];
      whole[e] = (float)v;
    }
    put<T, WHOLE>(p, token, c, whole);
  }
}

int range_of(long long rows) {
  const long long r = (rows + 255) / 256;
  return (int)(r < 1 ? 1 : r > MAX_RANGE ? MAX_RANGE : r);
}
// Sorted tokens of a tile: 4096 waves and more where the tokens suffice
int tile_of(const prism_embedding_desc& d, int chunks) {
  int tile = 64;
  while (tile > 4 && (d.count + tile - 1) / tile * chunks < 4096) tile /= 2;
  while ((d.count + tile - 1) / tile * chunks > (1 << 20) && tile < (1 << 30)) tile *= 2;      // launches stay far below 2^32 work-items
  return tile;
}
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

template <typename T, typename I> void lookup(const Lookup& p, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL((p.width < Vec<T>::N ? embedding_kernel<T, I, false, false> : fills<T>(p.count, p.width, 64) ? embedding_kernel<T, I, true, true> : embedding_kernel<T, I, true, false>),
                     grid, dim3(256), 0, s, p);
}
template <typename T> void lookup(const Lookup& p, bool wide, dim3 grid, hipStream_t s) {
  if (wide) lookup<T, int64_t>(p, grid, s);
  else lookup<T, int>(p, grid, s);
}
template <typename T> void add_up(const Sums& p, long long tokens, dim3 sums, dim3 joins, hipStream_t s) {
  const bool whole = p.width >= Vec<T>::N;
  const bool past = fills<T>(tokens + p.rows, p.width, 128);
  hipLaunchKernelGGL((!whole ? embedding_sums_kernel<T, false, false> : past ? embedding_sums_kernel<T, true, true> : embedding_sums_kernel<T, true, false>), sums, dim3(256), 0, s, p);
  if (joins.x) hipLaunchKernelGGL((whole ? embedding_join_kernel<T, true> : embedding_join_kernel<T, false>), joins, dim3(64 * JOIN_WAVES), 0, s, p);
}

}  // namespace

int launch_embedding(const void* table, const void* tokens, void* out, int dt, const prism_embedding_desc& d, hipStream_t s) {
  ProfScope prof(PK_EMBEDDING, s);
  Lookup p = {};
  p.table = table; p.tokens = tokens; p.out = out;
  p.count = d.count; p.rows = d.rows; p.ts = d.table_stride; p.os = d.out_stride; p.width = d.width; p.scale = d.scale;
  const int n = dt == PRISM_F32 ? 4 : 8, vectors = (d.width + n - 1) / n;
  // a lane has four vectors under way where there are tokens enough
  p.lanes = 1;
  while (p.lanes < 256 && p.lanes < vectors && (p.lanes * 4 < vectors || d.count * p.lanes < 1 << 18)) p.lanes *= 2;
  const long long need = (d.count + 256 / p.lanes - 1) / (256 / p.lanes);
  const dim3 grid((unsigned)(need < 16384 ? need : 16384));
  if (dt == PRISM_F32) lookup<float>(p, d.wide_tokens, grid, s);
  else lookup<__bf16>(p, d.wide_tokens, grid, s);
  return PRISM_OK;
}

EmbeddingPlan embedding_plan(const prism_embedding_desc& d, int dt) {
  EmbeddingPlan P = {};
  const int n = dt == PRISM_F32 ? 4 : 8;
  P.chunks = (d.width + 64 * n - 1) / (64 * n);
  P.tile = tile_of(d, P.chunks);
  P.tiles = (int)((d.count + P.tile - 1) / P.tile);
  P.o_sorted = up((size_t)(d.rows + 1) * sizeof(int));
  P.o_part = P.o_sorted + up((size_t)d.count * sizeof(int2));
  P.total = P.o_part + up((size_t)P.tiles * 2 * P.chunks * 64 * n * sizeof(float));
  return P;
}

int launch_embedding_backward(const void* dout, const void* tokens, void* dtable, int dt, const prism_embedding_desc& d, char* ws, hipStream_t s) {
  const EmbeddingPlan P = embedding_plan(d, dt);
  Sorted q = {};
  q.tokens = tokens; q.starts = (int*)ws; q.sorted = (int2*)(ws + P.o_sorted);
  q.count = (int)d.count; q.rows = d.rows; q.range = range_of(d.rows);
  {
    ProfScope prof(PK_EMBEDDING_SORT, s);
    const dim3 grid((unsigned)((d.rows + q.range - 1) / q.range));
    if (d.wide_tokens) hipLaunchKernelGGL((embedding_sort_kernel<int64_t>), grid, dim3(SORT_THREADS), 0, s, q);
    else hipLaunchKernelGGL((embedding_sort_kernel<int>), grid, dim3(SORT_THREADS), 0, s, q);
  }
  ProfScope prof(PK_EMBEDDING_BACKWARD, s);
  Sums p = {};
  p.dout = dout; p.dtable = dtable; p.starts = q.starts; p.sorted = q.sorted; p.part = (float*)(ws + P.o_part);
  p.rows = d.rows; p.ds = d.out_stride; p.ts = d.table_stride; p.width = d.width; p.scale = d.scale;
  p.tile = P.tile; p.chunks = P.chunks; p.tile_waves = P.tiles * P.chunks;
  // 2048 workgroups clear rows, if each wave has one
  p.clear = (int)(d.rows <= 8192 ? 1 : d.rows < 64 * 8192 ? (d.rows + 8191) / 8192 : 64);
  const long long clear = (d.rows + 4 * p.clear - 1) / (4 * p.clear);
  const dim3 grid((unsigned)((p.tile_waves + 3) / 4 + (clear < 2048 ? clear : 2048)));
  const dim3 joins(P.tiles > 1 ? (unsigned)((P.tiles - 1 + BORDERS - 1) / BORDERS * P.chunks) : 0);
  if (dt == PRISM_F32) add_up<float>(p, d.count, grid, joins, s);
  else add_up<__bf16>(p, d.count, grid, joins, s);
  return PRISM_OK;
}

}  // namespace prism
