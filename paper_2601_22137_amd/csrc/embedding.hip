// Rows of a table by token, times a factor, and the table's gradient.
//
//   out[i] = scale table[token[i]], 0 for a token that is no row;   dtable[v] = scale sum over i with token[i] = v of dout[i], 0 for a row without a token
//
// The gradient is a sum over sorted tokens, so that the same call gives the same bits whatever the order in which workgroups run:
//   sort   a workgroup has a range of the table's rows; it goes through all tokens twice, counting those of each of its rows and those before its range, then
//          putting each (in its order) in its place.  Nothing passes between workgroups.
//   sums   the sorted tokens are cut into tiles of equal length; a wave adds up the rows of dout of a tile, 64 vectors of 16 bytes wide, in 32 bits.  A run of
//          equal tokens that lies in one tile goes straight to the table; what crosses a border is kept as partial sums.  Other waves clear the rows without tokens.
//   join   partial sums of a run in their order, in 64 bits.
#include "layer.h"
#include "row_vector.h"

namespace prism {
namespace {

constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, MAX_RANGE = 512;

// Token i; -1: no row of the table
template <typename I> __device__ inline int token_at(const void* tokens, long long i, long long rows) {
  const I t = ((const I*)tokens)[i];
  return t >= 0 && (long long)t < rows ? (int)t : -1;
}

struct Lookup {
  const void *table, *tokens;
  void* out;
  long long count, rows, ts, os;
  int width, lanes;             // lanes (a power of two up to 256) share a row
  float scale;
};

template <typename T, typename I> __global__ void __launch_bounds__(256) embedding_kernel(Lookup p) {
  using V = typename Vec<T>::type;
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & (p.lanes - 1), per = 256 / p.lanes;
  for (long long i = (long long)blockIdx.x * per + threadIdx.x / p.lanes; i < p.count; i += (long long)gridDim.x * per) {
    const int t = token_at<I>(p.tokens, i, p.rows);
    const T* row = (const T*)p.table + (t < 0 ? 0 : t) * p.ts;
    T* to = (T*)p.out + i * p.os;
#pragma unroll 4
    for (int c = lane * N; c < p.width; c += p.lanes * N) {
      V v = {};
      if (t >= 0) {
        v = load_vector(row, c, p.width);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)((float)v[e] * p.scale);
      }
      store_vector(to, c, p.width, v);
    }
  }
}

struct Sorted {
  const void* tokens;
  int* starts;                  // [rows + 1]: where a row's tokens begin
  int2* sorted;                 // (token, index), by token and then index
  int count, range;
  long long rows;
};

template <typename I> __global__ void __launch_bounds__(SORT_THREADS) embedding_sort_kernel(Sorted p) {
  __shared__ int places[MAX_RANGE * SORT_WAVES];        // [row of the range][wave]: counts, then where the wave's next one goes
  __shared__ int sums[SORT_WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long first = (long long)blockIdx.x * p.range;
  const int range = (int)(p.rows - first < p.range ? p.rows - first : p.range), slots = range * SORT_WAVES;
  for (int i = threadIdx.x; i < slots; i += SORT_THREADS) places[i] = 0;
  __syncthreads();
  // a wave has a part of the tokens, in whole sixty-fours
  const int part = ((p.count + SORT_THREADS - 1) / SORT_THREADS) * 64;
  const int begin = (int)((long long)wave * part < p.count ? wave * part : p.count), end = p.count - begin < part ? p.count : begin + part;
  int below = 0;
#pragma unroll 8
  for (int i = begin + lane; i < end; i += 64) {
    const int t = token_at<I>(p.tokens, i, p.rows);
    if (t < 0) continue;
    const long long at = t - first;
    if (at < 0) ++below;
    else if (at < range) atomicAdd(&places[(int)at * SORT_WAVES + wave], 1);
  }
  // all tokens before the range
#pragma unroll
  for (int d = 1; d < 64; d *= 2) below += __shfl_xor(below, d);
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
  if (threadIdx.x == SORT_THREADS - 1 && first + range == p.rows) p.starts[p.rows] = before;
  __syncthreads();
#pragma unroll 4
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int i = i0 + lane, t = i < end ? token_at<I>(p.tokens, i, p.rows) : -1;
    const long long at = t - first;
    const bool in = t >= 0 && at >= 0 && at < range;
    unsigned long long left = __ballot(in);
    while (left) {              // one turn for each row that a token of these 64 names
      const int leader = __ffsll((long long)left) - 1, row = __shfl((int)at, leader);
      const unsigned long long same = __ballot(in && (int)at == row);
      int place = 0;
      if (lane == leader) place = atomicAdd(&places[row * SORT_WAVES + wave], __popcll(same));
      place = __shfl(place, leader);
      if ((same >> lane) & 1) p.sorted[place + __popcll(same & ((1ull << lane) - 1))] = make_int2(t, i);
      left &= ~same;
    }
  }
}

struct Sums {
  const void* dout;
  void* dtable;
  const int* starts;
  const int2* sorted;
  float* part;                  // [tile][run that came in, run that goes on][width]
  long long rows, ds, ts;
  int width, tile, tiles, chunks, tile_waves;
  float scale;
};

template <typename T> __device__ inline void put(const Sums& p, int token, int c, const float (&sum)[Vec<T>::N]) {
  typename Vec<T>::type o;
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e) o[e] = (T)(sum[e] * p.scale);
  store_vector((T*)p.dtable + token * p.ts, c, p.width, o);
}

template <typename T> __global__ void __launch_bounds__(256) embedding_sums_kernel(Sums p) {
  using V = typename Vec<T>::type;
  constexpr int N = Vec<T>::N, AHEAD = 8;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63, count = p.starts[p.rows];
  if (wave >= p.tile_waves) {
    const int others = gridDim.x * 4 - p.tile_waves;
    for (long long row = wave - p.tile_waves; row < p.rows; row += others) {
      if (p.starts[row] != p.starts[row + 1]) continue;
      for (int c = lane * N; c < p.width; c += 64 * N) store_vector((T*)p.dtable + row * p.ts, c, p.width, V{});
    }
    return;
  }
  const int tile = wave / p.chunks, c = ((wave - tile * p.chunks) * 64 + lane) * N, begin = tile * p.tile;
  if (begin >= count) return;
  const int end = count - begin < p.tile ? count : begin + p.tile;
  int token = p.sorted[begin].x;
  bool inside = begin == 0 || p.sorted[begin - 1].x != token;      // the run began in this tile
  float sum[N] = {};
  for (int i0 = begin; i0 < end; i0 += AHEAD) {
    V v[AHEAD];
    int2 at[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      at[j] = p.sorted[i0 + j < end ? i0 + j : end - 1];
      v[j] = load_vector((const T*)p.dout + at[j].y * p.ds, c, i0 + j < end ? p.width : 0);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j >= end) break;
      if (at[j].x != token) {
        if (inside) put<T>(p, token, c, sum);
        else {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (c + e < p.width) p.part[(size_t)tile * 2 * p.width + c + e] = sum[e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.0f;
        token = at[j].x;
        inside = true;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += (float)v[j][e];
    }
  }
  const bool goes_on = end < count && p.sorted[end].x == token;
  if (inside && !goes_on) {
    put<T>(p, token, c, sum);
    return;
  }
  float* part = p.part + ((size_t)tile * 2 + (inside ? 1 : 0)) * p.width;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (c + e < p.width) part[c + e] = sum[e];
}

// A workgroup for each border between tiles and 64 vectors: the first border of a run adds it up, each of its waves a share of the tiles
template <typename T> __global__ void __launch_bounds__(512) embedding_join_kernel(Sums p) {
  constexpr int N = Vec<T>::N;
  const int tile = blockIdx.x / p.chunks, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, border = (tile + 1) * p.tile, count = p.starts[p.rows];
  if (border >= count) return;
  const int token = p.sorted[border].x;
  if (p.sorted[border - 1].x != token) return;
  const int start = p.starts[token], stop = p.starts[token + 1];
  if (start < tile * p.tile) return;                               // an earlier border's
  const int c = ((blockIdx.x - tile * p.chunks) * 64 + lane) * N, last = (stop - 1) / p.tile, all = last - tile + 1, share = (all + 7) / 8;
  const int from = tile + wave * share, to = from + share <= last + 1 ? from + share : last + 1;
  double sum[N] = {};
#pragma unroll 4
  for (int t = from; t < to; ++t) {
    const float* part = p.part + ((size_t)t * 2 + (t == tile ? 1 : 0)) * p.width;
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += c + e < p.width ? part[c + e] : 0.0f;
  }
  __shared__ double sums[8][64 * N];
#pragma unroll
  for (int e = 0; e < N; ++e) sums[wave][e * 64 + lane] = sum[e];
  __syncthreads();
  if (wave) return;
  float whole[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    double v = 0.0;
    for (int w = 0; w < 8; ++w) v += sums[w][e * 64 + lane];
    whole[e] = (float)v;
  }
  put<T>(p, token, c, whole);
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

}  // namespace

int launch_embedding(const void* table, const void* tokens, void* out, int dt, const prism_embedding_desc& d, hipStream_t s) {
  ProfScope prof(PK_EMBEDDING, s);
  Lookup p = {};
  p.table = table; p.tokens = tokens; p.out = out;
  p.count = d.count; p.rows = d.rows; p.ts = d.table_stride; p.os = d.out_stride; p.width = d.width; p.scale = d.scale;
  const int n = dt == PRISM_F32 ? 4 : 8, vectors = (d.width + n - 1) / n;
  p.lanes = 256;
  while (p.lanes > 1 && (p.lanes > vectors || (vectors + p.lanes - 1) / p.lanes * p.lanes > vectors + vectors / 8)) p.lanes /= 2;
  const long long need = (d.count + 256 / p.lanes - 1) / (256 / p.lanes);
  const dim3 grid((unsigned)(need < 16384 ? need : 16384));
  if (dt == PRISM_F32) {
    if (d.wide_tokens) hipLaunchKernelGGL((embedding_kernel<float, int64_t>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((embedding_kernel<float, int>), grid, dim3(256), 0, s, p);
  } else {
    if (d.wide_tokens) hipLaunchKernelGGL((embedding_kernel<__bf16, int64_t>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((embedding_kernel<__bf16, int>), grid, dim3(256), 0, s, p);
  }
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
  P.total = P.o_part + up((size_t)P.tiles * 2 * d.width * sizeof(float));
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
  p.tile = P.tile; p.tiles = P.tiles; p.chunks = P.chunks; p.tile_waves = P.tiles * P.chunks;
  // a wave clears rows until 2048 workgroups are at work
  const long long clear = (d.rows + 3) / 4;
  const dim3 grid((unsigned)((p.tile_waves + 3) / 4 + (clear < 2048 ? clear : 2048)));
  if (dt == PRISM_F32) hipLaunchKernelGGL((embedding_sums_kernel<float>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((embedding_sums_kernel<__bf16>), grid, dim3(256), 0, s, p);
  if (P.tiles > 1) {
    const dim3 joins((unsigned)((P.tiles - 1) * P.chunks));
    if (dt == PRISM_F32) hipLaunchKernelGGL((embedding_join_kernel<float>), joins, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((embedding_join_kernel<__bf16>), joins, dim3(512), 0, s, p);
  }
  return PRISM_OK;
}

}  // namespace prism
