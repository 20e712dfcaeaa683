// What the kernels of attention over packed sequences share: arguments, the places of blocks, checks and launches.
#pragma once
#include "attn_tile.hip.h"

#include <algorithm>
#include <cmath>

using namespace xrl;

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.0e38f;                 // a maximum that no score has reached yet

struct Heads {
  void *p;
  int64_t stride, head_stride;
};

struct AttnArgs {
  const int32_t *q_ptr, *k_ptr;
  int64_t seqs, n_q, n_k, blocks, block0;           // block0: first block of this launch
  int q_heads, kv_heads, causal;
  int dim, dim_in;                                  // of a head; of what is read, whole pieces of 16 bytes
  bool quads;                                       // four columns of a result may be stored together
  float scale;
  Heads q, k, v, out, dout, dq, dk, dv;
  float *lse;                                       // [n_q, q_heads]
  float *stat_lse, *stat_delta;                     // [q_heads, n_q]: lse log2(e) and do . o
};

// Tiles in LDS at a time: the next one's loads run while one is worked on. A wave by itself, for short sequences, has one: it seldom has a second tile, and twice as many such waves
// fit on a compute unit.
template <int WAVES>
constexpr int kBuffers = WAVES == 1 ? 1 : 2;

template <typename T>
__device__ __forceinline__ T *head_at(const Heads &x, int64_t row, int head) { return (T *)x.p + row * x.stride + head * x.head_stride; }

// Block -> tile of rows and head. Blocks are dealt to the eight XCDs in turn: the heads of one row tile follow each other, those that share keys at a distance of kv_heads,
// so that with eight of these (or a multiple) an XCD's L2 holds the keys of its own heads alone. Under a causal mask a sequence's last queries and its first keys have the
// most work, in proportion to their tile's number from the other end: of up to 64 sequences the tiles with the most work come first, whichever sequence they are of (of more, each
// sequence's own). us, forward and backward of 16 sequences of 330 to 3300 rows, 16 heads of 64: 563 sequence by sequence, 419 in this order.
struct Place {
  int64_t seq;
  int head, tile;
};
__device__ __forceinline__ int head_of(const AttnArgs &a, int heads, int h) {
  const int group = heads / a.kv_heads;
  return h % a.kv_heads * group + h / a.kv_heads;
}
__device__ __forceinline__ bool place_of(const AttnArgs &a, const int32_t *ptr, int64_t n, int heads, int bm, bool last_first, int lane, Place &o) {
  const int64_t b = a.block0 + blockIdx.x;
  o.head = head_of(a, heads, (int)(b % heads));
  if (a.seqs <= 64) {
    const Span mine = lane < a.seqs ? span_of(ptr, lane, n) : Span{0, 0};
    const int tiles = (mine.len + bm - 1) / bm;
    int64_t u = b / heads;
    // level: how many tiles from its own end on; between two sequences' numbers of tiles as many sequences have one at every level
    int level = -wave_min(-tiles);
    while (level > 0) {
      const unsigned long long have = __ballot(tiles >= level);
      const int count = __popcll(have), next = -wave_min(tiles < level ? -tiles : 0);
      const int64_t here = (int64_t)count * (level - next);
      if (u < here) {
        level -= (int)(u / count);
        const int k = (int)(u % count);              // the k-th of them
        const int before = __popcll(have & ((1ull << lane) - 1));
        const int seq = __ffsll(__ballot((have >> lane & 1) && before == k)) - 1;
        o.seq = seq;
        o.tile = last_first ? level - 1 : __shfl(tiles, seq) - level;
        return true;
      }
      u -= here;
      level = next;
    }
    return false;
  }
  const int64_t u = last_first ? a.blocks / heads - 1 - b / heads : b / heads;
  o.seq = sequence_of(ptr, a.seqs, n, bm, u, lane);
  if (o.seq < 0) return false;
  const int64_t t = u - (end_at(ptr, o.seq, n) / bm + o.seq);
  o.tile = t < (1 << 30) ? (int)t : 1 << 30;
  return true;
}

// Short sequences: a tile is 32 rows that follow each other in the packed tensor, of whatever sequences, a row a lane, and goes over the rows of the other side that any of
// them meets. A sequence by itself would leave most of a tile empty. (Where in a tile its keys lie then depends on its place among the others, and so do the last bits of its sums.)
// us, forward and backward of 1024 sequences of 1 to 24 rows with 4 heads of 32 in fp32: 60 by a tile a sequence, 35 by mixed ones.
//
// Taken where sequences have at most 128 rows on average on both sides. 16384 rows in sequences of one length, mixed tiles and (>) tiles of 128 rows of one sequence, forward + backward in
// us: 4 heads of 32 in fp32 16 + 44 > 22 + 72 at 96 rows, 20 + 56 > 29 + 111 at 128, 22 + 66 > 29 + 92 at 192, 29 + 88 > 25 + 79 at 256; 32 heads of 128 in bf16 118 + 304 > 137 + 318, 125 + 358 >
// 126 + 395, 137 + 378 > 143 + 356, 148 + 445 > 131 + 357.
// The rule goes by the mean alone: 8192 rows between 200 sequences of 20, 16 heads of 64 in bf16, are 60 on average and take 321 us forward and 1599 backward in mixed tiles, where the long one by
// itself takes 171 and 827 and the short ones 10 and 31.
inline bool mixes(const AttnArgs &a) { return a.n_q <= 128 * a.seqs && a.n_k <= 128 * a.seqs; }
// Few rows over many of the other side: a wave a tile of 32 of one sequence's rows.
// us, attention of 8192 queries over 600 keys a sequence, by such waves and by blocks of four: 16 heads of 64 in bf16, 8 queries a sequence 243 and 415, 64: 51 and 61, 128: 48 and 39.
inline bool few_rows(const AttnArgs &a, int64_t n) { return n <= 64 * a.seqs; }

// What the lane's row meets: rows [lo, hi) of the other tensor (keys that a query sees; queries that see a key); and over the wave the first and the last of these, and what all
// rows meet.
struct Meets {
  bool there;                                       // the row is one of a sequence
  int lo, hi, first, last, all_lo, all_hi;
};
// The row's own tensor has the ends `ptr` and n rows, the other one `other` and m; `keys`: the row is a key.
__device__ __forceinline__ Meets meets_of(const AttnArgs &a, const int32_t *ptr, int64_t n, const int32_t *other, int64_t m, bool keys, int64_t tile, int lane) {
  const int64_t row0 = 32 * tile, row = row0 + (lane & 31);
  int64_t s0 = last_begun(ptr, a.seqs, n, row0, lane), s = -1;
  if (s0 < 0) s0 = 0;
  // so many of the sequences behind it have begun at the lane's row or in front of it, 64 of them at a time
  for (bool more = true; __ballot(more); s0 += 64) {
    const int64_t end = s0 + 1 + lane < a.seqs ? end_at(ptr, s0 + 1 + lane, n) : INT64_MAX;
    const int e = end <= INT32_MAX ? (int)end : INT32_MAX;
    int count = 0;                                  // (the ends do not fall: by halves)
#pragma unroll
    for (int step = 32; step > 0; step /= 2) count += __shfl(e, count + step - 1) <= row ? step : 0;
    count += __shfl(e, count) <= row ? 1 : 0;
    if (more && count < 64) s = s0 + count;
    more = more && count == 64;
  }
  Meets o;
  const Span mine = span_of(ptr, s, n), that = span_of(other, s, m);
  const int at = (int)(row - mine.begin);
  o.there = row >= mine.begin && at < mine.len;
  int lo = 0, hi = that.len;
  if (a.causal && keys) {                           // from the first row that sees the key on
    const int i = at - (mine.len - that.len);
    lo = i < 0 ? 0 : i < hi ? i : hi;
  } else if (a.causal) {
    const int e = at + 1 + that.len - mine.len;
    hi = e < 0 ? 0 : e < hi ? e : hi;
  }
  const bool some = o.there && lo < hi;
  o.lo = some ? (int)that.begin + lo : 0;
  o.hi = some ? (int)that.begin + hi : 0;
  o.first = wave_min(some ? o.lo : INT32_MAX);
  o.last = -wave_min(-o.hi);
  o.all_lo = -wave_min(o.there ? some ? -o.lo : -INT32_MAX : 0);
  o.all_hi = wave_min(o.there ? o.hi : INT32_MAX);
  if (o.first > o.last) o.first = o.last;
  return o;
}

// A lane's row of queries, and the keys that its block goes over: `keys` of them from row key0 of their tensor on, of which the row sees [from, mine); all rows of the wave see
// [all_from, all_see), and any of them keys below any_sees.
struct Queries {
  int head;
  int64_t row, key0;
  bool there;
  int keys, from, mine, all_from, all_see, any_sees;
};
template <int WAVES, bool MIXED>
__device__ __forceinline__ bool queries_of(const AttnArgs &a, int wave, int lane, Queries &o) {
  constexpr int BM = 32 * WAVES;
  if constexpr (MIXED) {
    static_assert(WAVES == 1);
    const int64_t b = a.block0 + blockIdx.x;
    const Meets x = meets_of(a, a.q_ptr, a.n_q, a.k_ptr, a.n_k, false, b / a.q_heads, lane);
    o.head = head_of(a, a.q_heads, (int)(b % a.q_heads));
    o.there = x.there;
    o.row = x.there ? 32 * (b / a.q_heads) + (lane & 31) : 0;
    o.key0 = x.first;
    o.keys = o.any_sees = __builtin_amdgcn_readfirstlane(x.last - x.first);
    o.from = x.lo - x.first;
    o.mine = x.hi - x.first;
    o.all_from = x.all_lo - x.first;
    o.all_see = x.all_hi - x.first;
    return true;
  } else {
    Place at;
    if (!place_of(a, a.q_ptr, a.n_q, a.q_heads, BM, true, lane, at)) return false;
    const Span qs = span_of(a.q_ptr, at.seq, a.n_q), ks = span_of(a.k_ptr, at.seq, a.n_k);
    const int i0 = __builtin_amdgcn_readfirstlane(at.tile < (qs.len + BM - 1) / BM ? at.tile * BM : -1);
    if (i0 < 0) return false;
    const int len_k = __builtin_amdgcn_readfirstlane(ks.len), off = __builtin_amdgcn_readfirstlane(ks.len - qs.len);
    auto keys_of = [&](int i) { const int e = a.causal ? i + 1 + off : len_k; return e < 0 ? 0 : e < len_k ? e : len_k; };
    const int last = (i0 + BM < qs.len ? i0 + BM : qs.len) - 1, w0 = i0 + 32 * wave, w1 = w0 + 31 < last ? w0 + 31 : last, i = w0 + (lane & 31);
    o.head = at.head;
    o.there = i < qs.len;
    o.row = qs.begin + (o.there ? i : 0);
    o.key0 = ks.begin;
    o.keys = __builtin_amdgcn_readfirstlane(keys_of(last));
    o.from = o.all_from = 0;
    o.mine = keys_of(i);
    o.all_see = __builtin_amdgcn_readfirstlane(w0 <= last ? keys_of(w0) : 0);
    o.any_sees = __builtin_amdgcn_readfirstlane(w0 <= last ? keys_of(w1) : 0);
    return true;
  }
}

// Rows [n, heads, dim] that are written must lie apart; rows that are read may not (broadcast inputs).
inline bool lies_apart(const xrl_heads &x, int64_t n, int heads, int dim) {
  const int64_t s = n > 1 ? x.stride : INT64_MAX, h = heads > 1 ? x.head_stride : INT64_MAX;
  const int64_t inner = std::min(s, h), count = s < h ? n : heads, outer = std::max(s, h);
  if (inner != INT64_MAX && inner < dim) return false;
  return outer == INT64_MAX || outer - dim >= (count - 1) * inner;
}

// Checks a tensor of n rows. `quads` (of what is written): whether four columns of every row may be stored together.
inline int check_heads(const xrl_heads *x, int64_t n, int heads, int dim, int es, const char *name, const char *who, Heads &o, bool *quads = nullptr) {
  if (!x || (n > 0 && !x->d_data)) return fail(XRL_ERR_NULL, "%s: %s is NULL", who, name);
  if ((uintptr_t)x->d_data % es) return fail(XRL_ERR_SHAPE, "%s: %s: a pointer that is no multiple of its elements' size", who, name);
  if (x->stride < 0 || x->head_stride < 0 || (quads && !lies_apart(*x, n, heads, dim)))
    return fail(XRL_ERR_SHAPE, "%s: %s: strides %lld and %lld", who, name, (long long)x->stride, (long long)x->head_stride);
  if (n > 1 && x->stride > (1 << 23)) return fail(XRL_ERR_UNSUPPORTED, "%s: %s: stride %lld (at most 2^23)", who, name, (long long)x->stride);
  o = {x->d_data, n > 1 ? x->stride : 0, heads > 1 ? x->head_stride : 0};
  if (quads) *quads = *quads && dim % 4 == 0 && (uintptr_t)x->d_data % (4 * es) == 0 && o.stride % 4 == 0 && o.head_stride % 4 == 0;
  return XRL_OK;
}

inline int check_attention(const xrl_ctx *c, const xrl_attention_desc *d, const char *who, AttnArgs &a) {
  if (!c || !d) return fail(XRL_ERR_NULL, "%s: ctx or desc is NULL", who);
  if (!op_type_ok(d->type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, d->type);
  if (d->n_seqs < 0 || d->n_q < 0 || d->n_k < 0 || d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads || d->dim < 1)
    return fail(XRL_ERR_SHAPE, "%s: %lld sequences, %lld and %lld rows, %d and %d heads of %d", who, (long long)d->n_seqs, (long long)d->n_q, (long long)d->n_k,
                d->q_heads, d->kv_heads, d->dim);
  if (d->dim > 128 || d->q_heads > 65536 || d->n_q > INT32_MAX - 65536 || d->n_k > INT32_MAX - 65536 || d->n_seqs > INT32_MAX)
    return fail(XRL_ERR_UNSUPPORTED, "%s: heads of %d (at most 128), %d heads, %lld and %lld rows", who, d->dim, d->q_heads, (long long)d->n_q, (long long)d->n_k);
  if (!(d->scale > 0.f) || !std::isfinite(d->scale * kLog2e)) return fail(XRL_ERR_VALUE, "%s: scale %g", who, (double)d->scale);
  if (d->n_seqs > 0 && (!d->d_q_ptr || !d->d_k_ptr)) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d->d_q_ptr | (uintptr_t)d->d_k_ptr) % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a = AttnArgs{};
  a.q_ptr = d->d_q_ptr; a.k_ptr = d->d_k_ptr;
  a.seqs = d->n_seqs; a.n_q = d->n_q; a.n_k = d->n_k;
  a.q_heads = d->q_heads; a.kv_heads = d->kv_heads; a.dim = d->dim; a.causal = d->causal;
  a.scale = d->scale;
  a.dim_in = d->dim;
  a.quads = true;
  return XRL_OK;
}

// What is read has to lie in rows at multiples of 16 bytes, of whole pieces of 16 bytes: a tensor that does not is copied into the workspace first, in rows of
// dim_in columns with zeros behind dim. (Reading odd rows element by element in the attention itself took registers that every call would have paid for.)
struct Repack {
  const void *from;
  void *to;
  int64_t stride, head_stride, n;                   // of `from`; rows
  int heads, dim, dim_in;
};
template <typename T>
__global__ __launch_bounds__(256) void repack_kernel(const Repack r) {
  constexpr int V = 16 / (int)sizeof(T);
  const int pieces = r.dim_in / V;
  const int64_t total = r.n * r.heads * pieces;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t row = e / (r.heads * pieces);
    const int rest = (int)(e % (r.heads * pieces)), head = rest / pieces, d0 = rest % pieces * V;
    const T *p = (const T *)r.from + row * r.stride + head * r.head_stride;
    Piece<T, V> x;
#pragma unroll
    for (int j = 0; j < V; ++j) x.v[j] = d0 + j < r.dim ? p[d0 + j] : (T)0.f;
    __builtin_memcpy(__builtin_assume_aligned((T *)r.to + e * V, 16), &x, 16);
  }
}
// The tensors of a call that are read: those that have to be copied get their place behind `bytes` of the workspace.
struct Inputs {
  struct { Heads *h; int64_t n; int heads; size_t at; } list[5];
  int count = 0;
  size_t bytes = 0;
  int es, dim, dim_in;
  Inputs(int type, int dim_) : es(type == XRL_PREC_BF16 ? 2 : 4), dim(dim_), dim_in((dim_ * es + 15) / 16 * 16 / es) {}
  void add(Heads &h, int64_t n, int heads) {
    const bool aligned = dim == dim_in && (uintptr_t)h.p % 16 == 0 && h.stride * es % 16 == 0 && h.head_stride * es % 16 == 0;
    if (aligned || n == 0) return;
    list[count++] = {&h, n, heads, bytes};
    bytes += op_align((size_t)n * heads * dim_in * es);
  }
  void copy(const xrl_ctx *c, char *ws) {
    for (int i = 0; i < count; ++i) {
      Heads &h = *list[i].h;
      const Repack r = {h.p, ws + list[i].at, h.stride, h.head_stride, list[i].n, list[i].heads, dim, dim_in};
      const int64_t blocks = std::min<int64_t>((r.n * r.heads * (dim_in * es / 16) + 255) / 256, 16384);
      if (es == 2) repack_kernel<bf16_t><<<dim3((unsigned)blocks), dim3(256), 0, op_stream(c)>>>(r);
      else repack_kernel<float><<<dim3((unsigned)blocks), dim3(256), 0, op_stream(c)>>>(r);
      h = {r.to, (int64_t)r.heads * dim_in, dim_in};
    }
  }
};

// Launches `kernel` over the tiles of 32 rows of n that follow each other, for each of `heads` heads.
template <typename K>
void launch_mixed(const xrl_ctx *c, AttnArgs &a, K kernel, int64_t n, int heads) {
  a.blocks = (n + 31) / 32 * heads;
  for (a.block0 = 0; a.block0 < a.blocks; a.block0 += kMaxBlocks)
    kernel<<<dim3((unsigned)std::min(a.blocks - a.block0, kMaxBlocks)), dim3(64), 0, op_stream(c)>>>(a);
}
// Launches `kernel` over all tiles of bm rows of n, in seqs sequences, for each of `heads` heads.
template <typename K>
void launch_tiles(const xrl_ctx *c, AttnArgs &a, K kernel, int64_t n, int heads, int bm, int threads) {
  a.blocks = (n / bm + a.seqs) * heads;
  for (a.block0 = 0; a.block0 < a.blocks; a.block0 += kMaxBlocks)
    kernel<<<dim3((unsigned)std::min(a.blocks - a.block0, kMaxBlocks)), dim3(threads), 0, op_stream(c)>>>(a);
}

}  // namespace
