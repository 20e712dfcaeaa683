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

template <typename TT, typename TO, int VEC>
__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs a) {
  const int lane = threadIdx.x & (a.lanes - 1);
  const int per = 256 / a.lanes;
  for (int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / a.lanes; t < a.n; t += (int64_t)gridDim.x * per) {
    const int id = a.ids[t];
    const bool in = (unsigned)id < (unsigned)a.vocab;
    const TT *row = (const TT *)a.table + (in ? (int64_t)id * a.table_stride : 0);
    TO *out = (TO *)a.out + t * a.out_stride;
    for (int c = lane * VEC; c < a.dim; c += a.lanes * VEC) {
      if (c + VEC <= a.dim) {
        float v[VEC];
        if (in) {
          const Piece<TT, VEC> x = load_piece<TT, VEC>(row + c);
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] = a.scale * (float)x.v[j];
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] = 0.f;
        }
        store_piece<TO, VEC>(out + c, v);
      } else {
        for (int j = c; j < a.dim; ++j) out[j] = (TO)(in ? a.scale * (float)row[j] : 0.f);
      }
    }
  }
}

template <typename TT, typename TO>
int launch_embed(const xrl_ctx *c, EmbedArgs &a) {
  constexpr int VEC = 8;
  const int pieces = (a.dim + VEC - 1) / VEC;
  a.lanes = 1;
  while (a.lanes < pieces && a.lanes < 256) a.lanes *= 2;
  const int64_t per = 256 / a.lanes, blocks = std::min<int64_t>((a.n + per - 1) / per, kMaxBlocks);
  embed_kernel<TT, TO, VEC><<<dim3((unsigned)blocks), dim3(256), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

// ---- gradient
// Sorted pairs (id, t): a stable radix sort by up to kDigitBits bits a pass. Ids outside the vocabulary sort behind all others, as `vocab`.
constexpr int kDigitBits = 10, kSortBlocks = 64, kSortThreads = 512, kSortWaves = kSortThreads / 64;

struct SortArgs {
  const int32_t *ids;           // first pass: the items are (ids[t], t)
  const uint2 *in;              // later passes
  uint2 *out;
  int32_t *hist;                // [blocks][1 << bits]
  int64_t n;
  int vocab, shift, bits, per_wave;   // per_wave: consecutive items of a wave, a multiple of 64
};

__device__ __forceinline__ uint2 sort_item(const SortArgs &a, int64_t i) {
  if (!a.ids) return a.in[i];
  const int id = a.ids[i];
  return make_uint2((unsigned)id < (unsigned)a.vocab ? (unsigned)id : (unsigned)a.vocab, (unsigned)i);
}

__global__ __launch_bounds__(kSortThreads) void embed_sort_count_kernel(const SortArgs a) {
  __shared__ int cnt[1 << kDigitBits];
  const int digits = 1 << a.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) cnt[d] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * kSortWaves * a.per_wave;
  const int64_t i1 = i0 + (int64_t)kSortWaves * a.per_wave < a.n ? i0 + (int64_t)kSortWaves * a.per_wave : a.n;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads) atomicAdd(&cnt[(sort_item(a, i).x >> a.shift) & (digits - 1)], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) a.hist[(size_t)blockIdx.x * digits + d] = cnt[d];
}

__global__ __launch_bounds__(kSortThreads) void embed_sort_scatter_kernel(const SortArgs a) {
  __shared__ int off[kSortWaves][1 << kDigitBits];
  __shared__ int total[1 << kDigitBits], wave_sum[kSortWaves];
  const int digits = 1 << a.bits, t = threadIdx.x, lane = t & 63, w = t >> 6;
  for (int k = 0; k < kSortWaves; ++k)
    for (int d = t; d < digits; d += kSortThreads) off[k][d] = 0;
  __syncthreads();
  const int64_t w0 = ((int64_t)blockIdx.x * kSortWaves + w) * a.per_wave;
  for (int k = lane; k < a.per_wave; k += 64)
    if (w0 + k < a.n) atomicAdd(&off[w][(sort_item(a, w0 + k).x >> a.shift) & (digits - 1)], 1);
  // of each digit: the items of all blocks, and those of the blocks before
  int before[(1 << kDigitBits) / kSortThreads];
#pragma unroll
  for (int q = 0; q < (1 << kDigitBits) / kSortThreads; ++q) {
    const int d = t + q * kSortThreads;
    int sum = 0, mine = 0;
    if (d < digits)
      for (int b = 0; b < (int)gridDim.x; ++b) {
        const int h = a.hist[(size_t)b * digits + d];
        mine += b < (int)blockIdx.x ? h : 0;
        sum += h;
      }
    before[q] = mine;
    if (d < digits) total[d] = sum;
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
  for (int k = 0; k < per; ++k)
    if (t * per + k < digits) {
      const int x = total[t * per + k];
      total[t * per + k] = base;
      base += x;
    }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < (1 << kDigitBits) / kSortThreads; ++q) {
    const int d = t + q * kSortThreads;
    if (d < digits) {
      int at = total[d] + before[q];
      for (int k = 0; k < kSortWaves; ++k) {       // digit d's first place for each wave
        const int x = off[k][d];
        off[k][d] = at;
        at += x;
      }
    }
  }
  __syncthreads();
  volatile int *mine = off[w];
  for (int k = 0; k < a.per_wave; k += 64) {
    const int64_t i = w0 + k + lane;
    const bool in = i < a.n;
    const uint2 x = in ? sort_item(a, i) : make_uint2(0, 0);
    const int d = (int)((x.x >> a.shift) & (unsigned)(digits - 1));
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
    if (in) a.out[place] = x;
  }
}

// Sums over runs of equal ids. A group of `lanes` threads takes kWindow consecutive sorted pairs, in their order. A run inside the window is
// added to its row of the table; the piece of a run that began before goes to carry[window][0], that of one that goes on behind it to
// carry[window][1], and embed_join_kernel adds up the pieces of each such run.
constexpr int kWindow = 32;

struct SumArgs {
  const uint2 *items;
  const void *dout;
  float *dtable, *carry;        // carry [windows][2][dim]
  int64_t dout_stride, dtable_stride, n;
  int vocab, dim, lanes;
  float scale;
};

template <typename T, int VEC, int BATCH>
__global__ __launch_bounds__(256) void embed_sum_kernel(const SumArgs a) {
  const int lane = threadIdx.x & (a.lanes - 1);
  const int64_t w = (int64_t)blockIdx.x * (256 / a.lanes) + threadIdx.x / a.lanes;
  const int64_t i0 = w * kWindow;
  if (i0 >= a.n) return;
  const int c = ((int)blockIdx.y * a.lanes + lane) * VEC;
  if (c >= a.dim) return;
  const int nv = a.dim - c < VEC ? a.dim - c : VEC;     // columns of this thread
  const int len = (int)(a.n - i0 < kWindow ? a.n - i0 : kWindow);
  const uint2 *it = a.items + i0;
  const unsigned before = i0 > 0 ? it[-1].x : ~0u, behind = i0 + len < a.n ? it[len].x : ~0u;
  float acc[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
  bool first = true;                                     // in the window's first run
  for (int b0 = 0; b0 < len; b0 += BATCH) {
    uint2 x[BATCH];
    Piece<T, VEC> v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) x[i] = b0 + i < len ? it[b0 + i] : make_uint2((unsigned)a.vocab, 0);
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (x[i].x < (unsigned)a.vocab) {
        const T *p = (const T *)a.dout + (int64_t)x[i].y * a.dout_stride + c;
        if (nv == VEC) v[i] = load_piece<T, VEC>(p);
        else
          for (int j = 0; j < VEC; ++j) v[i].v[j] = j < nv ? p[j] : (T)0.f;
      }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (x[i].x >= (unsigned)a.vocab) continue;         // behind the end, or no row's id
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += (float)v[i].v[j];
      const bool last = b0 + i == len - 1;
      const unsigned next = last ? behind : it[b0 + i + 1].x;
      if (next == x[i].x && !last) continue;
      const bool head = first && before == x[i].x, goes_on = next == x[i].x;
      float *p = head || goes_on ? a.carry + ((size_t)w * 2 + (head ? 0 : 1)) * a.dim + c
                                 : a.dtable + (int64_t)x[i].x * a.dtable_stride + c;
      if (head || goes_on) {
        for (int j = 0; j < nv; ++j) p[j] = acc[j];
      } else {
        for (int j = 0; j < nv; ++j) p[j] += a.scale * acc[j];
      }
      first = false;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
    }
  }
}

// A block per window: if its last run begins in it and goes on, the run's pieces in sixteen parts, and the parts in order.
__global__ __launch_bounds__(1024) void embed_join_kernel(const SumArgs a) {
  const int64_t w = blockIdx.x, i1 = (w + 1) * kWindow;
  if (i1 >= a.n) return;
  const unsigned id = a.items[i1 - 1].x;
  if (id >= (unsigned)a.vocab || a.items[i1].x != id) return;
  if (a.items[i1 - kWindow].x == id && w > 0 && a.items[i1 - kWindow - 1].x == id) return;   // began before
  // the first pair behind the run
  int64_t lo = i1, hi = a.n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (a.items[mid].x <= id) lo = mid + 1; else hi = mid;
  }
  const int64_t w_end = (lo + kWindow - 1) / kWindow;   // windows w + 1 .. w_end - 1 hold its other pieces
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int c = (int)blockIdx.y * 64 + lane;
  const int64_t n = w_end - w, per = (n + 15) / 16, p0 = g * per, p1 = p0 + per < n ? p0 + per : n;
  float sum = 0.f;
  if (c < a.dim)
    for (int64_t k = p0; k < p1; ++k) sum += a.carry[((size_t)(w + k) * 2 + (k == 0 ? 1 : 0)) * a.dim + c];
  part[g][lane] = sum;
  __syncthreads();
  if (g || c >= a.dim) return;
  for (int k = 1; k < 16; ++k) sum += part[k][lane];
  float *p = a.dtable + (int64_t)id * a.dtable_stride + c;
  *p += a.scale * sum;
}

template <typename T>
int launch_embed_sums(const xrl_ctx *c, SumArgs &a) {
  constexpr int VEC = sizeof(T) == 2 ? 8 : 4;
  const int pieces = (a.dim + VEC - 1) / VEC;
  a.lanes = 1;
  while (a.lanes < pieces && a.lanes < 256) a.lanes *= 2;
  const int64_t windows = (a.n + kWindow - 1) / kWindow, per = 256 / a.lanes;
  embed_sum_kernel<T, VEC, 4><<<dim3((unsigned)((windows + per - 1) / per), (unsigned)((pieces + a.lanes - 1) / a.lanes)), dim3(256), 0,
                                op_stream(c)>>>(a);
  embed_join_kernel<<<dim3((unsigned)windows, (unsigned)((a.dim + 63) / 64)), dim3(1024), 0, op_stream(c)>>>(a);
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
  if (n < 0 || vocab < 0 || dim < 0 || dout_stride < dim || dtable_stride < dim)
    return fail(XRL_ERR_SHAPE, "%s: n = %lld, vocab = %lld, dim = %lld, strides %lld and %lld", who, (long long)n, (long long)vocab,
                (long long)dim, (long long)dout_stride, (long long)dtable_stride);
  if (n >= 1 << 27 || vocab >= 1 << 30 || dim > (1 << 20))
    return fail(XRL_ERR_UNSUPPORTED, "%s: n = %lld, vocab = %lld, dim = %lld", who, (long long)n, (long long)vocab, (long long)dim);
  if (n == 0 || dim == 0 || vocab == 0) return XRL_OK;
  if (!d_ids || !d_dout || !d_dtable) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if ((uintptr_t)d_dout % (dout_type == XRL_PREC_BF16 ? 2 : 4) || (uintptr_t)d_dtable % 4 || (uintptr_t)d_ids % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  int bits = 1;
  while ((vocab >> bits) > 0) ++bits;                   // of the largest key, `vocab`
  const int passes = (bits + kDigitBits - 1) / kDigitBits, per_pass = (bits + passes - 1) / passes;
  SortArgs s = {};
  s.n = n; s.vocab = (int)vocab; s.bits = per_pass;
  const int64_t per_wave = std::max<int64_t>(256, (n + (int64_t)kSortBlocks * kSortWaves - 1) / ((int64_t)kSortBlocks * kSortWaves));
  s.per_wave = (int)((per_wave + 63) / 64 * 64);
  const int blocks = (int)((n + (int64_t)s.per_wave * kSortWaves - 1) / ((int64_t)s.per_wave * kSortWaves));
  const int64_t windows = (n + kWindow - 1) / kWindow;
  const size_t o_b = op_align((size_t)n * 8), o_h = 2 * o_b, o_c = o_h + op_align((size_t)blocks * ((size_t)4 << per_pass));
  char *ws = nullptr;
  if (int rc = op_workspace(c, o_c + (size_t)windows * 2 * dim * 4, &ws, who)) return rc;
  uint2 *x = (uint2 *)ws, *y = (uint2 *)(ws + o_b);
  s.hist = (int32_t *)(ws + o_h);
  for (int p = 0; p < passes; ++p) {
    s.ids = p == 0 ? d_ids : nullptr;
    s.in = x; s.out = y; s.shift = p * per_pass;
    embed_sort_count_kernel<<<dim3(blocks), dim3(kSortThreads), 0, op_stream(c)>>>(s);
    embed_sort_scatter_kernel<<<dim3(blocks), dim3(kSortThreads), 0, op_stream(c)>>>(s);
    std::swap(x, y);
  }
  OP_TRY(hipGetLastError());
  SumArgs a = {x, d_dout, d_dtable, (float *)(ws + o_c), dout_stride, dtable_stride, n, (int)vocab, (int)dim, 0, scale};
  return dout_type == XRL_PREC_BF16 ? launch_embed_sums<bf16_t>(c, a) : launch_embed_sums<float>(c, a);
}

}  // extern "C"
