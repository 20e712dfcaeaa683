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
__device__ __forceinline__ bool place_of(const AttnArgs &a, const int32_t *ptr, int64_t n, int heads, int bm, bool last_first, int lane, Place &o) {
  const int64_t b = a.block0 + blockIdx.x;
  const int h = (int)(b % heads);
  const int group = heads / a.kv_heads;
  o.head = h % a.kv_heads * group + h / a.kv_heads;
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

// Bits of a wave's tile that count: keys [j0, j0 + 32) against row i, which sees those below `end`.
__device__ __forceinline__ bool sees(int j, int end) { return j < end; }

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

// Launches `kernel` over all tiles of bm rows of n, in seqs sequences, for each of `heads` heads.
template <typename K>
void launch_tiles(const xrl_ctx *c, AttnArgs &a, K kernel, int64_t n, int heads, int bm, int threads) {
  a.blocks = (n / bm + a.seqs) * heads;
  for (a.block0 = 0; a.block0 < a.blocks; a.block0 += kMaxBlocks)
    kernel<<<dim3((unsigned)std::min(a.blocks - a.block0, kMaxBlocks)), dim3(threads), 0, op_stream(c)>>>(a);
}

}  // namespace
