// Embedding lookup with scaling, and its gradient by sorted ids.
#include "op_common.h"

#include <algorithm>

using namespace xrl;

namespace {

// ---- lookup: out[t, :] = scale * table[id_t, :]
struct EmbedArgs {
  const void *table;
  const int32_t *ids;
  void *out;
  int64_t table_stride, out_stride, n;
  int vocab, dim, lanes;        // lanes: threads that share a row, a power of two up to 256
  float scale;
};

// Bound by memory: the distinct rows read, the results written.
template <typename TT, typename TO, int VEC, int ROWS, bool STREAM>
__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs a) {
  const int lane = threadIdx.x & (a.lanes - 1), per = 256 / a.lanes;
  for (int64_t t0 = ((int64_t)blockIdx.x * per + threadIdx.x / a.lanes) * ROWS; t0 < a.n; t0 += (int64_t)gridDim.x * per * ROWS) {
    const int rows = (int)(a.n - t0 < ROWS ? a.n - t0 : ROWS);
    int id[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      id[r] = r < rows ? a.ids[t0 + r] : -1;
      if ((unsigned)id[r] >= (unsigned)a.vocab) id[r] = -1;
    }
    for (int c = lane * VEC; c < a.dim; c += a.lanes * VEC) {
      if (c + VEC <= a.dim) {
        Piece<TT, VEC> x[ROWS];
        if (a.vocab > 0)
#pragma unroll
          for (int r = 0; r < ROWS; ++r) x[r] = load_piece<TT, VEC>((const TT *)a.table + (int64_t)(id[r] >= 0 ? id[r] : 0) * a.table_stride + c);
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          if (r < rows) {
            float v[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = id[r] >= 0 ? a.scale * (float)x[r].v[j] : 0.f;
            store_piece<TO, VEC, STREAM>((TO *)a.out + (t0 + r) * a.out_stride + c, v);
          }
      } else {
        for (int r = 0; r < rows; ++r)
          for (int j = c; j < a.dim; ++j)
            ((TO *)a.out)[(t0 + r) * a.out_stride + j] =
                (TO)(id[r] >= 0 ? a.scale * (float)((const TT *)a.table)[(int64_t)id[r] * a.table_stride + j] : 0.f);
      }
    }
  }
}

// A thread takes 16 bytes of the narrower of the two types. Results that are streamed past the caches are taken two rows a thread, whose ids and
// pieces are then on their way together. us, four sets of inputs in turn, cached one row / cached two / streamed one / streamed two: 65536 x 768 from
// fp32 to bf16 49 / 45 / 38 / 33, 65536 x 1024 in bf16 52 / 46 / 33 / 29, 131072 x 512 in fp32 88 / 90 / 86 / 76.
template <typename TT, typename TO>
int launch_embed(const xrl_ctx *c, EmbedArgs &a) {
  constexpr int VEC = sizeof(TT) + sizeof(TO) == 8 ? 4 : 8;
  const int pieces = (a.dim + VEC - 1) / VEC;
  a.lanes = 1;
  while (a.lanes < pieces && a.lanes < 256) a.lanes *= 2;
  const bool stream = streams(a.n * a.dim * (int64_t)sizeof(TO));
  const int64_t per = 256 / a.lanes * (stream ? 2 : 1);
  const dim3 grid((unsigned)std::min<int64_t>((a.n + per - 1) / per, kMaxBlocks));
  if (stream) embed_kernel<TT, TO, VEC, 2, true><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  else embed_kernel<TT, TO, VEC, 1, false><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

// ---- gradient
// The columns of a thread: N from `at` on, of which the first `skip` are another thread's too and not stored. (The last thread of a row reads back into its
// neighbour's columns, a thread behind the row all of them, so that every thread's loads are the same: one that is made in a branch of its own is
// waited for at that branch's end. dim >= N.)
template <int N>
struct Columns {
  int at, skip;
  __device__ Columns(int c, int dim) : at(c + N <= dim ? c : dim - N), skip(c - at) {}
};

// Few ids: a block per place t and slab of columns. It ends at once if the id stands before t; else it adds up all places of the id, wave w those of the
// w-th eighth of the places from t on, and the eight sums in order. One launch and no workspace; the work grows with the square of the ids. us a call, this /
// ranked and summed: 2048 long-tailed ids, 128 columns in fp32 6 / 15, 1024 in bf16 17 / 20, 2048 in fp32 40 / 18 (1024 of these 19 / 15, 768 14 / 14, 512
// 10 / 14); 2048 times one id, 128 columns 21 / 15, 1024 39 / 17.
constexpr int kFewIds = 768, kFewSlabIds = 2048, kFewWaves = 8;   // however many slabs, and of one or two

struct FewArgs {
  const int32_t *ids;
  const void *dout;
  float *dtable;
  int64_t dout_stride, dtable_stride;
  int n, vocab, dim;
  float scale;
};

template <typename T, int VEC>
__global__ __launch_bounds__(kFewWaves * 64) void embed_few_kernel(const FewArgs a) {
  touch_args(a);
  const int t = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int id = a.ids[t];
  if ((unsigned)id >= (unsigned)a.vocab) return;
  int before = 0;
  for (int i = threadIdx.x; i < t; i += kFewWaves * 64) before |= a.ids[i] == id;
  if (__syncthreads_or(before)) return;
  const Columns<VEC> c(((int)blockIdx.y * 64 + lane) * VEC, a.dim);
  const int chunks = (a.n - t + 63) / 64, per = (chunks + kFewWaves - 1) / kFewWaves;
  const int i0 = t + w * per * 64, i1 = i0 + per * 64 < a.n ? i0 + per * 64 : a.n;
  float acc[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
  for (int i = i0; i < i1; i += 64) {
    unsigned long long here = __ballot(i + lane < i1 && a.ids[i + lane < i1 ? i + lane : i] == id);
    while (here) {
      constexpr int BATCH = 8;
      Piece<T, VEC> v[BATCH];
      int got = 0;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (!here) break;
        v[k] = load_piece<T, VEC>((const T *)a.dout + (int64_t)(i + __ffsll(here) - 1) * a.dout_stride + c.at);
        here &= here - 1;
        got = k + 1;
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
        if (k < got)
#pragma unroll
          for (int j = 0; j < VEC; ++j) acc[j] += (float)v[k].v[j];
    }
  }
  __shared__ float part[kFewWaves - 1][64][VEC + 1];
  if (w)
#pragma unroll
    for (int j = 0; j < VEC; ++j) part[w - 1][lane][j] = acc[j];
  __syncthreads();
  if (w) return;
  float *p = a.dtable + (int64_t)id * a.dtable_stride + c.at;
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
#pragma unroll
    for (int k = 0; k < kFewWaves - 1; ++k) acc[j] += part[k][lane][j];
    if (j >= c.skip) p[j] += a.scale * acc[j];
  }
}

// A small table: no sort. A block takes consecutive places and 64 C columns; each of its four waves adds its quarter of the rows, one after another, into a
// table of its own in LDS, a lane C columns (so every sum has one order), and the four tables in order are the block's. A second launch adds up the
// blocks' in order. Ids outside the vocabulary go to a row behind the table. Four rows are added at once, or each would wait for the one before, 130
// clocks through the LDS; of equal ids among them one takes the other's sum in registers (16.7 us where waiting for those alone takes 18.1; the LDS's own atomic
// additions of floats, 12 clocks a lane, take 90). Two columns a lane up to 24 ids; the
// more ids the fewer waves the LDS has room for: up to 64 ids and 512 columns one column a lane, beyond the sort. us a call, this / sorted: 77013 x 128 in
// fp32, 8 ids 14 / 31, 40 17 / 26, 64 20 / 26, 100 26 / 23; 77013 x 1024 in bf16, 8 ids 38 / 54, 24 43 / 49, 40 68 / 47, 100 115 / 47.
constexpr int kBinIds = 64, kBinWaves = 4, kBinWideIds = 24, kBinDim = 512;

struct BinArgs {
  const int32_t *ids;
  const void *dout;
  float *dtable, *partial;      // partial [blocks][vocab][dim]
  unsigned *seen;               // [blocks][kBinIds / 32] bits of the ids that a block met
  int64_t dout_stride, dtable_stride, n;
  int vocab, dim, per, blocks;  // per: places of a wave, a multiple of 64
  float scale;
};

template <typename T, int C>
__global__ __launch_bounds__(kBinWaves * 64) void embed_bins_kernel(const BinArgs a) {
  touch_args(a);
  constexpr int AHEAD = 16;
  extern __shared__ __align__(16) float bins[];
  __shared__ unsigned seen[kBinIds / 32];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), table = (a.vocab + 1) * 64 * C;
  for (int i = threadIdx.x; i < kBinWaves * table / 4; i += kBinWaves * 64) ((f32x4 *)bins)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (threadIdx.x < kBinIds / 32) seen[threadIdx.x] = 0;
  __syncthreads();
  const Columns<C> c((int)blockIdx.y * 64 * C + lane * C, a.dim);
  float *mine = bins + w * table + lane;
  const int64_t r0 = ((int64_t)blockIdx.x * kBinWaves + w) * a.per;
  for (int64_t r = r0; r < r0 + a.per && r < a.n; r += 64) {
    int id = r + lane < a.n ? a.ids[r + lane] : -1;
    if ((unsigned)id >= (unsigned)a.vocab) id = a.vocab;
    else atomicOr(&seen[id >> 5], 1u << (id & 31));
    Piece<T, C> v[2][AHEAD];
    auto request = [&](int h, int q) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int64_t row = r + q + u < a.n ? r + q + u : a.n - 1;      // (behind the end the id is no row's)
        v[h][u] = load_piece<T, C>((const T *)a.dout + row * a.dout_stride + c.at);
      }
    };
    request(0, 0);
#pragma unroll
    for (int q = 0; q < 64; q += AHEAD) {
      if (r + q >= a.n) break;
      const int h = q / AHEAD & 1;
      if (q + AHEAD < 64) request(h ^ 1, q + AHEAD);
#pragma unroll
      for (int u = 0; u < AHEAD; u += 4) {
        int to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) to[k] = __builtin_amdgcn_readlane(id, q + u + k) * 64 * C;
        float x[4][C];                                      // four rows of the table at once
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < C; ++j) x[k][j] = mine[to[k] + j * 64];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < C; ++j) {
            float old = x[k][j];                            // of an id that came before among the four: the sum so far
#pragma unroll
            for (int l = 0; l < k; ++l) old = to[l] == to[k] ? x[l][j] : old;
            x[k][j] = old + (float)v[h][u + k].v[j];
          }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < C; ++j) mine[to[k] + j * 64] = x[k][j];
      }
    }
  }
  __syncthreads();
  for (int v = w; v < a.vocab; v += kBinWaves) {
    const float *from = bins + v * 64 * C + lane;
    float *to = a.partial + ((int64_t)blockIdx.x * a.vocab + v) * a.dim + c.at;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float sum = from[j * 64];
#pragma unroll
      for (int k = 1; k < kBinWaves; ++k) sum += from[k * table + j * 64];
      if (j >= c.skip) to[j] = sum;
    }
  }
  if (blockIdx.y == 0 && threadIdx.x < kBinIds / 32) a.seen[blockIdx.x * (kBinIds / 32) + threadIdx.x] = seen[threadIdx.x];
}

// A block per id and 64 columns: sixteen waves a part of the blocks' sums each, and their sums in order.
__global__ __launch_bounds__(1024) void embed_bins_join_kernel(const BinArgs a) {
  touch_args(a);
  __shared__ float part[15][64];
  const int id = blockIdx.x, lane = threadIdx.x & 63, g = threadIdx.x >> 6, c = (int)blockIdx.y * 64 + lane;
  bool met = false;
  for (int b = threadIdx.x; b < a.blocks; b += 1024) met = met || (a.seen[b * (kBinIds / 32) + (id >> 5)] >> (id & 31) & 1);
  if (!__syncthreads_or(met)) return;
  const int per = (a.blocks + 15) / 16, b0 = g * per, b1 = b0 + per < a.blocks ? b0 + per : a.blocks;
  float sum = 0.f;
  if (c < a.dim)
    for (int b = b0; b < b1; b += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = b + u < b1 ? a.partial[((int64_t)(b + u) * a.vocab + id) * a.dim + c] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += x[u];
    }
  if (g) part[g - 1][lane] = sum;
  __syncthreads();
  if (g || c >= a.dim) return;
  for (int k = 0; k < 15; ++k) sum += part[k][lane];
  a.dtable[(int64_t)id * a.dtable_stride + c] += a.scale * sum;
}

// More ids: sorted pairs (id, t) by a stable radix sort of up to kDigitBits bits a pass. Ids outside the vocabulary sort behind all others, as
// `vocab`. A pass is two launches: one counts each block's digits, one moves the pairs.
constexpr int kDigitBits = 10, kSortBlocks = 64, kSortThreads = 512, kSortWaves = kSortThreads / 64;

struct SortArgs {
  const int32_t *ids;           // first pass: the items are (ids[t], t)
  const uint2 *in;              // later passes
  uint2 *out;
  int32_t *hist;                // [blocks][1 << bits]
  int32_t *clear;               // zeroed by the counting launch
  int64_t n;
  int vocab, shift, bits, per_wave;   // per_wave: consecutive items of a wave, a multiple of 64
};

__device__ __forceinline__ uint2 sort_item(const SortArgs &a, int id, int64_t i) {
  return make_uint2((unsigned)id < (unsigned)a.vocab ? (unsigned)id : (unsigned)a.vocab, (unsigned)i);
}
// Items i, i + step, .. (kAhead of them; the first one for those from `end` on): all are on their way together.
constexpr int kAhead = 4;
struct Items {
  uint2 x[kAhead];
};
__device__ __forceinline__ Items sort_items(const SortArgs &a, int64_t i, int step, int64_t end) {
  Items v;
  int64_t at[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) at[k] = i + k * step < end ? i + k * step : 0;
  if (a.ids) {
    int id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = a.ids[at[k]];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v.x[k] = sort_item(a, id[k], at[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v.x[k] = a.in[at[k]];
  }
  return v;
}

__global__ __launch_bounds__(kSortThreads) void embed_sort_count_kernel(const SortArgs a) {
  touch_args(a);
  __shared__ int cnt[1 << kDigitBits];
  const int digits = 1 << a.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) cnt[d] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * kSortWaves * a.per_wave;
  const int64_t i1 = i0 + (int64_t)kSortWaves * a.per_wave < a.n ? i0 + (int64_t)kSortWaves * a.per_wave : a.n;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kAhead * kSortThreads) {
    const Items v = sort_items(a, i, kSortThreads, i1);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * kSortThreads < i1) atomicAdd(&cnt[(v.x[k].x >> a.shift) & (digits - 1)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) a.hist[(size_t)blockIdx.x * digits + d] = cnt[d];
}

__global__ __launch_bounds__(kSortThreads) void embed_sort_scatter_kernel(const SortArgs a) {
  touch_args(a);
  __shared__ int off[kSortWaves][1 << kDigitBits];
  __shared__ int total[1 << kDigitBits], before[1 << kDigitBits], wave_sum[kSortWaves];
  const int digits = 1 << a.bits, t = threadIdx.x, lane = t & 63, w = t >> 6;
  for (int k = 0; k < kSortWaves; ++k)
    for (int d = t; d < digits; d += kSortThreads) off[k][d] = 0;
  for (int d = t; d < digits; d += kSortThreads) total[d] = before[d] = 0;
  __syncthreads();
  const int64_t w0 = ((int64_t)blockIdx.x * kSortWaves + w) * a.per_wave;
  const int64_t w1 = w0 + a.per_wave < a.n ? w0 + a.per_wave : a.n;
  const Items first = sort_items(a, w0 + lane, 64, w1);
  for (int64_t i0 = w0; i0 < w1; i0 += kAhead * 64) {
    const Items v = i0 == w0 ? first : sort_items(a, i0 + lane, 64, w1);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k * 64 + lane < w1) atomicAdd(&off[w][(v.x[k].x >> a.shift) & (digits - 1)], 1);
  }
  // of each digit: the items of all blocks, and those of the blocks before; digits x blocks dealt to the threads, eight requests at a time
  {
    const int d = t & (digits - 1), slices = digits < kSortThreads ? kSortThreads / digits : 1;
    for (int dd = d; dd < digits; dd += kSortThreads) {
      int sum = 0, mine = 0;
      for (int b = digits < kSortThreads ? t / digits : 0; b < (int)gridDim.x; b += 8 * slices) {
        int h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) h[k] = b + k * slices < (int)gridDim.x ? a.hist[(size_t)(b + k * slices) * digits + dd] : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sum += h[k];
          mine += b + k * slices < (int)blockIdx.x ? h[k] : 0;
        }
      }
      atomicAdd(&total[dd], sum);
      atomicAdd(&before[dd], mine);
    }
  }
  __syncthreads();
  // exclusive sums over the digits: thread t takes digits [t * per, ...)
  const int per = (digits + kSortThreads - 1) / kSortThreads;
  int own = 0;
  for (int k = 0; k < per; ++k) own += t * per + k < digits ? total[t * per + k] : 0;
  int inc = own;
  for (int s = 1; s < 64; s *= 2) {
    const int y = __shfl_up(inc, s);
    if (lane >= s) inc += y;
  }
  if (lane == 63) wave_sum[w] = inc;
  __syncthreads();
  int base = inc - own;
  for (int k = 0; k < w; ++k) base += wave_sum[k];
  for (int k = 0; k < per; ++k) {
    const int d = t * per + k;
    if (d < digits) {
      int at = base + before[d];
      base += total[d];
      for (int q = 0; q < kSortWaves; ++q) {             // digit d's first place for each wave
        const int x = off[q][d];
        off[q][d] = at;
        at += x;
      }
    }
  }
  __syncthreads();
  int *mine = off[w];
  for (int64_t i0 = w0; i0 < w1; i0 += kAhead * 64) {
    const Items v = i0 == w0 ? first : sort_items(a, i0 + lane, 64, w1);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + k * 64 >= w1) break;
      const bool in = i0 + k * 64 + lane < w1;
      const int d = (int)((v.x[k].x >> a.shift) & (unsigned)(digits - 1));
      unsigned long long same = __ballot(in);
      for (int b = 0; b < a.bits; ++b) {
        const unsigned long long m = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? m : ~m;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const int place = mine[d] + rank;
      __builtin_amdgcn_wave_barrier();
      if (in && rank == 0) mine[d] = place + __popcll(same);
      __threadfence_block();
      __builtin_amdgcn_wave_barrier();
      if (in) a.out[place] = v.x[k];
    }
  }
}

// Up to kRankIds ids: the same pairs in one launch, each place from the count of the pairs before it. A block ranks 32 of them against all ids, which it has in
// LDS; lane l of a half wave has place t0 + l % 32, and the 32 half waves share out the ids, four at a time. Two instructions an id and place, n^2 of them,
// against the latency of two launches for each of the sort's passes. us a call, ranked / sorted: two passes, 128 columns in fp32, 3000 ids 16 / 29, 8192 21 / 31,
// 12288 30 / 32, 1024 in bf16, 8192 28 / 38, 12288 40 / 42; one pass (vocab < 1024), 512 in fp32, 8192 24 / 26, 12288 36 / 30.
constexpr int kRankIds = 12288, kRankIdsOnePass = 8192, kRankPlaces = 32;

__global__ __launch_bounds__(1024) void embed_rank_kernel(const SortArgs a) {
  touch_args(a);
  __shared__ __align__(16) int key[kRankIds];
  __shared__ int rank[kRankPlaces];
  const int n = (int)a.n, t0 = blockIdx.x * kRankPlaces, own = threadIdx.x & (kRankPlaces - 1), slot = threadIdx.x / kRankPlaces;
  const int padded = (n + kRankPlaces - 1) / kRankPlaces * kRankPlaces;
  for (int i0 = threadIdx.x; i0 < padded; i0 += kAhead * 1024) {
    const Items v = sort_items(a, i0, 1024, n);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * 1024;
      if (i < padded) key[i] = i < n ? (int)v.x[k].x : 0x7fffffff;
    }
  }
  if (threadIdx.x < kRankPlaces) rank[threadIdx.x] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
  __syncthreads();
  const int mine = key[t0 + own];
  int before = 0;
  auto count = [&](int from, int to, int bound) {          // chunks of four ids
#pragma unroll 4
    for (int k = from + slot; k < to; k += 32) {
      const int4 x = *(const int4 *)&key[4 * k];
      before += (x.x < bound) + (x.y < bound) + (x.z < bound) + (x.w < bound);
    }
  };
  count(0, t0 / 4, mine < 0x7fffffff ? mine + 1 : mine);   // equal ids that stand before count, those behind do not
  count(t0 / 4 + kRankPlaces / 4, padded / 4, mine);
  const int other = key[t0 + slot];                        // of the block's own places each half wave takes one
  before += other < mine || (other == mine && slot < own);
  atomicAdd(&rank[own], before);
  __syncthreads();
  if (threadIdx.x < kRankPlaces && t0 + (int)threadIdx.x < n) a.out[rank[threadIdx.x]] = make_uint2((unsigned)mine, (unsigned)(t0 + threadIdx.x));
}

// Sums over runs of equal ids. A group of `lanes` threads takes a window of consecutive sorted pairs, in their order; a batch's rows, and the rows of the
// table that its runs are added to, are requested together. A run inside the window is added to its row of the table. The piece of a run that began
// before goes to carry[window][0], that of one that goes on behind it to carry[window][1]; a window that such a run begins in is listed, and
// embed_join_kernel adds up the run's pieces.
// Groups that are whole waves keep their pairs in scalar registers; there a window is of 32 pairs from eight waves a compute unit on, else of 16. us a call,
// 32 / 16: 65536 long-tailed ids of 1024 columns in bf16 85 / 95, 77013 of 512 in fp32 75 / 80; of 1024 in bf16 8192 36 / 28, 16384 50 / 46.
// Bound by memory from some 30000 ids of 1024 columns on (the 65536: 58 us of this kernel for the gradient and two passes over the rows it meets,
// 263 MB), below by latency. All loads of a batch are on their way together: none stands in a branch that also takes its value apart, which would be waited
// for there (62 us, and 13 more at 8192 ids). Batches of eight rows but for windows of 16 in bf16, whose registers they would double: us, four / eight, the
// 65536 88 / 85, 12288 of 128 columns in fp32 31 / 30, 12288 of 1024 in bf16 39 / 41.
constexpr int kJoinWaves = 8;

struct SumArgs {
  const uint2 *items;
  const void *dout;
  float *dtable, *carry;        // carry [windows][2][dim]
  int32_t *listed;              // how many windows are listed,
  int2 *list;                   // and which, with the run's id (in any order)
  int64_t dout_stride, dtable_stride, n;
  int vocab, dim, lanes, window;
  float scale;
};

template <typename T, int VEC, bool WHOLE, int kWindow, bool STREAM>
__global__ __launch_bounds__(256) void embed_sum_kernel(const SumArgs a) {
  touch_args(a);
  constexpr int BATCH = kWindow == 32 || sizeof(T) == 4 ? 8 : 4;
  const int lane = threadIdx.x & (a.lanes - 1);
  int in_block = threadIdx.x / a.lanes;
  if (WHOLE) in_block = __builtin_amdgcn_readfirstlane(in_block);   // whole waves: their pairs are in scalar registers
  const int64_t w = (int64_t)blockIdx.x * (256 / a.lanes) + in_block;
  const int64_t i0 = w * kWindow;
  if (i0 >= a.n) return;
  const unsigned vocab = (unsigned)a.vocab;
  // The window's pairs, and the ids around it (in front of the first pair and behind the last: no row's).
  unsigned id[kWindow + 2];
  int at[kWindow];
  auto pair = [&](int i) {
    const int64_t k = i0 + i - 1;
    const bool in = k >= 0 && k < a.n;
    uint2 x = a.items[in ? k : i0];
    if (!in) x.x = k < 0 ? ~0u : vocab;
    return x;
  };
  if constexpr (WHOLE) {                                 // one a lane
    const uint2 x = pair((int)(threadIdx.x & 63) < kWindow + 2 ? (int)(threadIdx.x & 63) : 0);
#pragma unroll
    for (int i = 0; i < kWindow + 2; ++i) {
      id[i] = __builtin_amdgcn_readlane((int)x.x, i);
      if (i >= 1 && i <= kWindow) at[i - 1] = __builtin_amdgcn_readlane((int)x.y, i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWindow + 2; ++i) {
      const uint2 x = pair(i);
      id[i] = x.x;
      if (i >= 1 && i <= kWindow) at[i - 1] = (int)x.y;
    }
  }
  const Columns<VEC> c(((int)blockIdx.y * a.lanes + lane) * VEC, a.dim);
  if (c.skip >= VEC || id[1] >= vocab) return;           // (ids that are no row's stand at the end)
  float acc[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
  bool head = id[0] == id[1];                            // the run at hand began before the window
#pragma unroll
  for (int b0 = 0; b0 < kWindow; b0 += BATCH) {
    Piece<T, VEC> v[BATCH];
    Piece<float, VEC> old[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b0 + k;
      v[k] = load_piece<T, VEC, STREAM>((const T *)a.dout + (int64_t)at[i] * a.dout_stride + c.at);
      if (id[i + 2] != id[i + 1] && id[i + 1] < vocab) old[k] = load_piece<float, VEC>(a.dtable + (int64_t)id[i + 1] * a.dtable_stride + c.at);
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = b0 + k;
      if (id[i + 1] >= vocab) continue;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += (float)v[k].v[j];
      const bool goes_on = id[i + 2] == id[i + 1];
      if (goes_on && i < kWindow - 1) continue;
      if (head || goes_on) {
        store_piece<float, VEC>(a.carry + ((size_t)w * 2 + (head ? 0 : 1)) * a.dim + c.at, acc);   // (what two threads store is the same)
        if (!head && lane == 0 && blockIdx.y == 0) a.list[atomicAdd(a.listed, 1)] = make_int2((int)w, (int)id[i + 1]);
      } else {
        float *p = a.dtable + (int64_t)id[i + 1] * a.dtable_stride + c.at, s[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[j] = old[k].v[j] + a.scale * acc[j];
        if (c.skip == 0) store_piece<float, VEC, STREAM>(p, s);
        else
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (j >= c.skip) p[j] = s[j];
      }
      head = false;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
    }
  }
}

// The run that the listed window w begins: its id, and its pieces, one in each window from w on that it reaches.
struct Run {
  int64_t w, pieces;
  unsigned id;
};
__device__ __forceinline__ Run run_of(const SumArgs &a, int listed, int lane) {
  Run r;
  const int2 x = a.list[listed];
  r.w = x.x;
  r.id = (unsigned)x.y;
  // windows behind w that begin with the id: 64 probes at once, each level 64 times as fine
  const int64_t windows = (a.n + a.window - 1) / a.window;
  auto follow = [&](int64_t from, int64_t s) {
    const int64_t k = from + (lane + 1) * s;
    return s * __popcll(__ballot(k < windows && a.items[k < windows ? k * a.window : 0].x == r.id));
  };
  int64_t more = follow(r.w, 1);
  if (more == 64) {                                       // (few are that long)
    more = 0;
    for (int64_t s = (int64_t)1 << 18; s; s >>= 6)
      if (s == 1 || s < windows) more += follow(r.w + more, s);
  }
  r.pieces = more + 1;
  return r;
}
// Pieces [p0, p1) of a run added up in their order, eight requests at a time.
template <int N>
__device__ __forceinline__ void add_pieces(const SumArgs &a, const Run &r, int64_t p0, int64_t p1, const Columns<N> &c, float *sum) {
#pragma unroll
  for (int j = 0; j < N; ++j) sum[j] = 0.f;
  const float *src = a.carry + (size_t)r.w * 2 * a.dim + c.at;
  for (int64_t k = p0; k < p1; k += 8) {
    Piece<float, N> x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (k + u < p1) x[u] = load_piece<float, N>(src + ((size_t)(k + u) * 2 + (k + u == 0)) * a.dim);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (k + u < p1)
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += x[u].v[j];
  }
}
template <int N>
__device__ __forceinline__ void add_run(const SumArgs &a, const Run &r, const Columns<N> &c, const Piece<float, N> &old, const float *sum) {
  float *p = a.dtable + (int64_t)r.id * a.dtable_stride + c.at;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j >= c.skip) p[j] = old.v[j] + a.scale * sum[j];
}

// The runs that go over windows, 64 N columns a block: each wave takes a listed window and adds up the run's pieces if they are few; the runs of many
// pieces are then taken by all waves of the block, a part of the pieces each, and their sums in order. A block for every run leaves most of its waves
// idle, a wave for every run is long at an id that fills the batch: us of this kernel at 65536 long-tailed ids of 1024 columns, and of the whole
// call at 131072 times the same id of 128 columns: sixteen waves a run 49 and 113, four 17 and 263, this 19 and 197; since
// the row of the table is asked for together with the pieces and the nearest 64 windows are looked at first, 14 and 150 (of which this kernel is 112: one
// compute unit takes in 4 MB).
constexpr int kFewPieces = 32;
template <int N>
__global__ __launch_bounds__(kJoinWaves * 64) void embed_join_kernel(const SumArgs a) {
  touch_args(a);
  __shared__ float part[kJoinWaves - 1][64 * N];
  __shared__ int many[kJoinWaves];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, listed = *a.listed;
  const Columns<N> c(((int)blockIdx.y * 64 + lane) * N, a.dim);
  for (int q0 = blockIdx.x; q0 < listed; q0 += gridDim.x * kJoinWaves) {   // neighbours in the list go to different blocks
    bool left = false;
    const int q = q0 + g * (int)gridDim.x;
    if (q < listed) {
      const Run r = run_of(a, q, lane);
      left = r.pieces > kFewPieces;
      if (!left) {
        const Piece<float, N> old = load_piece<float, N>(a.dtable + (int64_t)r.id * a.dtable_stride + c.at);
        float sum[N];
        add_pieces<N>(a, r, 0, r.pieces, c, sum);
        add_run<N>(a, r, c, old, sum);
      }
    }
    if (!__syncthreads_or(left)) continue;
    if (lane == 0) many[g] = left;
    __syncthreads();
    for (int k = 0; k < kJoinWaves; ++k) {
      if (!many[k]) continue;
      const Run r = run_of(a, q0 + k * (int)gridDim.x, lane);
      const int64_t per = (r.pieces + kJoinWaves - 1) / kJoinWaves, p0 = g * per, p1 = p0 + per < r.pieces ? p0 + per : r.pieces;
      const Piece<float, N> old = load_piece<float, N>(a.dtable + (int64_t)r.id * a.dtable_stride + c.at);
      float sum[N];
      add_pieces<N>(a, r, p0, p1, c, sum);
      if (g)
#pragma unroll
        for (int j = 0; j < N; ++j) part[g - 1][lane * N + j] = sum[j];
      __syncthreads();
      if (g == 0) {
        for (int u = 0; u < kJoinWaves - 1; ++u)
#pragma unroll
          for (int j = 0; j < N; ++j) sum[j] += part[u][lane * N + j];
        add_run<N>(a, r, c, old, sum);
      }
      __syncthreads();
    }
  }
}

template <typename T, int C>
int launch_embed_bins(xrl_ctx *c, BinArgs &a, const char *who) {
  const int n_cu = op_compute_units(c), slabs = (a.dim + 64 * C - 1) / (64 * C), lds = kBinWaves * (a.vocab + 1) * 64 * C * 4;
  static const hipError_t allowed =
      hipFuncSetAttribute((const void *)embed_bins_kernel<T, C>, hipFuncAttributeMaxDynamicSharedMemorySize, kBinWaves * ((C == 2 ? kBinWideIds : kBinIds) + 1) * 64 * C * 4);
  if (allowed != hipSuccess) return fail(XRL_ERR_HIP, "%s: %d bytes of LDS: %s", who, lds, hipGetErrorString(allowed));
  // as many blocks as the LDS lets run at once, of 64 places a wave at least: what they write is then at most half of what they read
  const int64_t at_once = std::max<int64_t>(1, (int64_t)n_cu * std::min(8, 163840 / (lds + 64)) / slabs);
  a.per = (int)(std::max<int64_t>(64, (a.n + kBinWaves * at_once - 1) / (kBinWaves * at_once)) + 63) / 64 * 64;
  a.blocks = (int)((a.n + (int64_t)kBinWaves * a.per - 1) / ((int64_t)kBinWaves * a.per));
  const size_t o_p = op_align((size_t)a.blocks * (kBinIds / 32) * 4);
  char *ws = nullptr;
  if (int rc = op_workspace(c, o_p + (size_t)a.blocks * a.vocab * a.dim * 4, &ws, who)) return rc;
  a.seen = (unsigned *)ws;
  a.partial = (float *)(ws + o_p);
  embed_bins_kernel<T, C><<<dim3((unsigned)a.blocks, (unsigned)slabs), dim3(kBinWaves * 64), lds, op_stream(c)>>>(a);
  embed_bins_join_kernel<<<dim3((unsigned)a.vocab, (unsigned)((a.dim + 63) / 64)), dim3(1024), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

template <typename T, int VEC>
int launch_embed_few(const xrl_ctx *c, const FewArgs &a) {
  embed_few_kernel<T, VEC><<<dim3((unsigned)a.n, (unsigned)((a.dim + 64 * VEC - 1) / (64 * VEC))), dim3(kFewWaves * 64), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

// Threads that share a row of the gradient, and pairs of a window.
void sum_shape(const xrl_ctx *c, int elem, int dim, int64_t n, int *lanes, int *window) {
  const int vec = dim >= 16 / elem ? 16 / elem : 1, pieces = (dim + vec - 1) / vec;
  *lanes = 1;
  while (*lanes < pieces && *lanes < 256) *lanes *= 2;
  *window = *lanes >= 64 && n / 32 * (*lanes / 64) >= 8 * op_compute_units(c) ? 32 : 16;
}

template <typename T, int VEC, bool STREAM>
void launch_sum_kernel(const xrl_ctx *c, const SumArgs &a, dim3 grid) {
  if (a.window == 32) embed_sum_kernel<T, VEC, true, 32, STREAM><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  else if (a.lanes >= 64) embed_sum_kernel<T, VEC, true, 16, STREAM><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  else embed_sum_kernel<T, VEC, false, 16, STREAM><<<grid, dim3(256), 0, op_stream(c)>>>(a);
}
template <typename T>
int launch_embed_sums(const xrl_ctx *c, SumArgs &a) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const int64_t windows = (a.n + a.window - 1) / a.window, per = 256 / a.lanes;
  const int vec = a.dim >= VEC ? VEC : 1, pieces = (a.dim + vec - 1) / vec;
  const dim3 grid((unsigned)((windows + per - 1) / per), (unsigned)((pieces + a.lanes - 1) / a.lanes));
  // A gradient of more than 64 MB is read, and the table's rows are stored, past the caches: 65536 x 1024 in bf16 107 / 85 us a call; but 77013 x 128 in
  // fp32, 39 MB that the last-level cache may still have, 53 / 55.
  const bool stream = a.n * a.dim * (int64_t)sizeof(T) > (int64_t)64 << 20;
  if (vec == 1) embed_sum_kernel<T, 1, false, 16, false><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  else if (stream) launch_sum_kernel<T, VEC, true>(c, a, grid);
  else launch_sum_kernel<T, VEC, false>(c, a, grid);
  const dim3 join((unsigned)std::min<int64_t>(windows, 2 * op_compute_units(c)), (unsigned)((a.dim + 255) / 256));
  if (a.dim >= 4) embed_join_kernel<4><<<join, dim3(kJoinWaves * 64), 0, op_stream(c)>>>(a);
  else embed_join_kernel<1><<<join, dim3(kJoinWaves * 64), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

}  // namespace

extern "C" {

int xrl_embedding(xrl_ctx *c, const void *d_table, int32_t table_type, int64_t table_stride, int64_t vocab, int64_t dim,
                  const int32_t *d_ids, int64_t n, float scale, void *d_out, int32_t out_type, int64_t out_stride) {
  if (!c) return fail(XRL_ERR_NULL, "xrl_embedding: ctx is NULL");
  if (!op_type_ok(table_type) || !op_type_ok(out_type)) return fail(XRL_ERR_UNSUPPORTED, "xrl_embedding: types %d and %d", table_type, out_type);
  if (n < 0 || vocab < 0 || dim < 0 || table_stride < dim || out_stride < dim)
    return fail(XRL_ERR_SHAPE, "xrl_embedding: n = %lld, vocab = %lld, dim = %lld, strides %lld and %lld", (long long)n, (long long)vocab,
                (long long)dim, (long long)table_stride, (long long)out_stride);
  if (vocab > INT32_MAX || dim > (1 << 24)) return fail(XRL_ERR_UNSUPPORTED, "xrl_embedding: vocab = %lld, dim = %lld", (long long)vocab, (long long)dim);
  if (n == 0 || dim == 0) return XRL_OK;
  if (!d_ids || !d_out || (vocab > 0 && !d_table)) return fail(XRL_ERR_NULL, "xrl_embedding: NULL device pointer");
  const int te = table_type == XRL_PREC_BF16 ? 2 : 4, oe = out_type == XRL_PREC_BF16 ? 2 : 4;
  if ((uintptr_t)d_table % te || (uintptr_t)d_out % oe || (uintptr_t)d_ids % 4)
    return fail(XRL_ERR_SHAPE, "xrl_embedding: a pointer that is no multiple of its elements' size");
  EmbedArgs a = {d_table, d_ids, d_out, table_stride, out_stride, n, (int)vocab, (int)dim, 0, scale};
  if (table_type == XRL_PREC_FP32)
    return out_type == XRL_PREC_FP32 ? launch_embed<float, float>(c, a) : launch_embed<float, bf16_t>(c, a);
  return out_type == XRL_PREC_FP32 ? launch_embed<bf16_t, float>(c, a) : launch_embed<bf16_t, bf16_t>(c, a);
}

int xrl_embedding_backward(xrl_ctx *c, const void *d_dout, int32_t dout_type, int64_t dout_stride, const int32_t *d_ids,
                           int64_t n, int64_t vocab, int64_t dim, float scale, float *d_dtable, int64_t dtable_stride) {
  const char *who = "xrl_embedding_backward";
  if (!c) return fail(XRL_ERR_NULL, "%s: ctx is NULL", who);
  if (!op_type_ok(dout_type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, dout_type);
  if (n < 0 || vocab < 0 || dim < 0 || (dout_stride < dim && dout_stride != 0) || dtable_stride < dim)   // (0: one row for all, as a broadcast's gradient has)
    return fail(XRL_ERR_SHAPE, "%s: n = %lld, vocab = %lld, dim = %lld, strides %lld and %lld", who, (long long)n, (long long)vocab,
                (long long)dim, (long long)dout_stride, (long long)dtable_stride);
  if (n >= 1 << 27 || vocab >= 1 << 30 || dim > (1 << 20))
    return fail(XRL_ERR_UNSUPPORTED, "%s: n = %lld, vocab = %lld, dim = %lld", who, (long long)n, (long long)vocab, (long long)dim);
  if (n == 0 || dim == 0 || vocab == 0) return XRL_OK;
  if (!d_ids || !d_dout || !d_dtable) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if ((uintptr_t)d_dout % (dout_type == XRL_PREC_BF16 ? 2 : 4) || (uintptr_t)d_dtable % 4 || (uintptr_t)d_ids % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  const int64_t slabs = (dim * (dout_type == XRL_PREC_BF16 ? 2 : 4) + 1023) / 1024;
  if (n <= (slabs <= 2 ? kFewSlabIds : kFewIds)) {
    const FewArgs a = {d_ids, d_dout, d_dtable, dout_stride, dtable_stride, (int)n, (int)vocab, (int)dim, scale};
    if (dout_type == XRL_PREC_BF16) return dim >= 8 ? launch_embed_few<bf16_t, 8>(c, a) : launch_embed_few<bf16_t, 1>(c, a);
    return dim >= 4 ? launch_embed_few<float, 4>(c, a) : launch_embed_few<float, 1>(c, a);
  }
  if (vocab <= kBinWideIds || (vocab <= kBinIds && dim <= kBinDim)) {
    BinArgs a = {d_ids, d_dout, d_dtable, nullptr, nullptr, dout_stride, dtable_stride, n, (int)vocab, (int)dim, 0, 0, scale};
    if (vocab <= kBinWideIds && dim > 1) return dout_type == XRL_PREC_BF16 ? launch_embed_bins<bf16_t, 2>(c, a, who) : launch_embed_bins<float, 2>(c, a, who);
    return dout_type == XRL_PREC_BF16 ? launch_embed_bins<bf16_t, 1>(c, a, who) : launch_embed_bins<float, 1>(c, a, who);
  }
  int bits = 1;
  while ((vocab >> bits) > 0) ++bits;                   // of the largest key, `vocab`
  const int passes = (bits + kDigitBits - 1) / kDigitBits, per_pass = (bits + passes - 1) / passes;
  SortArgs s = {};
  s.n = n; s.vocab = (int)vocab; s.bits = per_pass;
  const int64_t per_wave = std::max<int64_t>(256, (n + (int64_t)kSortBlocks * kSortWaves - 1) / ((int64_t)kSortBlocks * kSortWaves));
  s.per_wave = (int)((per_wave + 63) / 64 * 64);
  const int blocks = (int)((n + (int64_t)s.per_wave * kSortWaves - 1) / ((int64_t)s.per_wave * kSortWaves));
  int lanes, window;
  sum_shape(c, dout_type == XRL_PREC_BF16 ? 2 : 4, (int)dim, n, &lanes, &window);
  const int64_t windows = (n + window - 1) / window;
  const int64_t hist = (int64_t)blocks << per_pass;      // counters of one pass
  const size_t o_b = op_align((size_t)n * 8), o_h = 2 * o_b, o_l = o_h + op_align((size_t)(hist + 1) * 4),
               o_c = o_l + op_align((size_t)windows * 8);
  char *ws = nullptr;
  if (int rc = op_workspace(c, o_c + (size_t)windows * 2 * dim * 4, &ws, who)) return rc;
  uint2 *x = (uint2 *)ws, *y = (uint2 *)(ws + o_b);
  const bool ranked = n <= (passes > 1 ? kRankIds : kRankIdsOnePass);
  s.hist = (int32_t *)(ws + o_h);
  s.clear = s.hist + hist;                               // the list's length
  if (ranked) {
    s.ids = d_ids;
    s.out = x;
    embed_rank_kernel<<<dim3((unsigned)((n + kRankPlaces - 1) / kRankPlaces)), dim3(1024), 0, op_stream(c)>>>(s);
  }
  for (int p = 0; p < passes && !ranked; ++p) {
    s.ids = p == 0 ? d_ids : nullptr;
    s.in = x; s.out = y; s.shift = p * per_pass;
    embed_sort_count_kernel<<<dim3(blocks), dim3(kSortThreads), 0, op_stream(c)>>>(s);
    embed_sort_scatter_kernel<<<dim3(blocks), dim3(kSortThreads), 0, op_stream(c)>>>(s);
    std::swap(x, y);
  }
  OP_TRY(hipGetLastError());
  SumArgs a = {x, d_dout, d_dtable, (float *)(ws + o_c), s.clear, (int2 *)(ws + o_l), dout_stride, dtable_stride, n,
               (int)vocab, (int)dim, lanes, window, scale};
  return dout_type == XRL_PREC_BF16 ? launch_embed_sums<bf16_t>(c, a) : launch_embed_sums<float>(c, a);
}

}  // extern "C"
