// A paged cache of keys and values: writing the new tokens' rows, and their attention over all tokens of their sequences.
//
// The formulas are attention's (op_attention.hip), with key j of sequence s at cache row [table[s][j / page]][j % page]. The queries of the heads that share keys lie side by side: column
// (token, head of the group) is a lane of the accumulator tile, so that one pass over a sequence's keys serves all of them.
//
// Bound by memory for single tokens (every row of the cache is read once) and by the matrix cores for long chunks. The work is one line of tiles of KT keys: unit by unit, a unit being
// 32 WAVES columns of one sequence and one head of keys, and every block takes an equal piece of the line, whatever the lengths. Only a unit that a piece's end cuts is
// joined by a second launch from the parts, in order. Where no unit can have more than four tiles every block takes a whole one and nothing is joined.
//
// 32 sequences of 262144 tokens in all, one new token each, 32 heads on 8 of 128 in bf16 (1.07 GB): 228 us, 4.7 TB/s of the 5.18 that a large copy reaches. 509 new tokens of each of four sequences over
// 32768: 393 us, 673 TFLOP/s, of which 22 join parts. In bf16 the exponentials are rounded to it as factors of the values, as in op_attention.hip. A key's place is looked up once a tile and wave, by one
// lane, a tile ahead: page sizes of any kind end inside tiles.
#include "attn_tile.hip.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>
#include <utility>

using namespace xrl;

namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLowest = -3.0e38f;                 // a maximum that no score has reached yet

struct Rows {
  void *p;
  int64_t stride, head_stride;
};
struct Pages {
  void *p;
  int64_t page_stride, stride, head_stride;
};

// A unit that goes on in the next pieces of the line: its place, and how many of them have parts of it.
struct Split {
  int64_t seq;
  int block, kv, follow;        // block of columns; follow 0: none
};

struct CacheArgs {
  const int32_t *q_ptr, *lengths, *table;
  int64_t seqs, n_q, table_stride, n_pages, blocks, block0;   // blocks in all, the first of this launch
  int table_cols, page, q_heads, kv_heads, group, dim;
  bool quads;
  float scale;
  Rows q, out, k, v;            // k, v: the new rows
  Pages kc, vc;
  float *part, *part_sums;      // of two units a block: [2 blocks][columns][DP], and maximum and sum [2 blocks][columns][2]
  Split *splits;
};

// What a sequence has: rows of new tokens, keys, blocks of columns, tiles of a unit.
struct Seq {
  int64_t begin;
  int rows, length, keys, blocks, tiles;
};
template <int BM, int KT>
__device__ __forceinline__ Seq seq_of(const CacheArgs &a, int64_t s) {
  const Span r = span_of(a.q_ptr, s, a.n_q);
  const int64_t room = (int64_t)a.table_cols * a.page;
  const int length = a.lengths[s];
  Seq o;
  o.begin = r.begin;
  o.rows = r.len;
  o.length = length < 0 ? 0 : length;
  o.keys = o.length < room ? o.length : (int)room;
  o.blocks = (int)(((int64_t)r.len * a.group + BM - 1) / BM);
  o.tiles = o.keys > 0 ? (o.keys - 1) / KT + 1 : 1;
  return o;
}
__device__ __forceinline__ int64_t sum_scan(int64_t x, int lane) {   // over the lanes up to this one
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int64_t y = __shfl_up(x, i);
    x += lane >= i ? y : 0;
  }
  return x;
}

// Key j of a sequence: page and slot, or page -1 where there is none.
struct Slot {
  int page, slot;
};
__device__ __forceinline__ Slot slot_of(const CacheArgs &a, int64_t seq, int j) {
  const unsigned n = (unsigned)j / (unsigned)a.page;
  if (j < 0 || n >= (unsigned)a.table_cols) return {-1, 0};
  const int id = a.table[seq * a.table_stride + n];
  return {id >= 0 && id < a.n_pages ? id : -1, (int)((unsigned)j - n * (unsigned)a.page)};
}
template <typename T>
__device__ __forceinline__ T *page_row(const Pages &c, int page, int slot, int head) {
  return (T *)c.p + (int64_t)page * c.page_stride + (int64_t)slot * c.stride + (int64_t)head * c.head_stride;
}

// A wave a row of new tokens: its keys and values of all heads to their places. Rows of no sequence and places that are not there are left out.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArgs a) {
  touch_args(a);
  const int lane = threadIdx.x & 63;
  const int64_t row = a.block0 * 4 + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.n_q) return;
  const int64_t s = sequence_of_row(a.q_ptr, a.seqs, a.n_q, row, lane);
  if (s < 0) return;
  const Span r = span_of(a.q_ptr, s, a.n_q);
  const int64_t j = (int64_t)a.lengths[s] - r.len + (row - r.begin);
  if (j < 0 || j >= (int64_t)a.table_cols * a.page) return;
  const Slot at = slot_of(a, s, (int)j);
  if (at.page < 0) return;
  constexpr int V = WHOLE ? 16 / (int)sizeof(T) : 1;
  const int pieces = a.dim / V, n = a.kv_heads * pieces;
  for (int i = lane; i < 2 * n; i += 64) {
    const bool is_v = i >= n;
    const int e = is_v ? i - n : i, head = e / pieces, d = e % pieces * V;
    const Rows &from = is_v ? a.v : a.k;
    const T *p = (const T *)from.p + row * from.stride + head * from.head_stride + d;
    T *to = page_row<T>(is_v ? a.vc : a.kc, at.page, at.slot, head) + d;
    if constexpr (WHOLE) __builtin_memcpy(__builtin_assume_aligned(to, 16), __builtin_assume_aligned(p, 16), 16);
    else *to = *p;
  }
}

// Where a tile's keys and values lie: elements from the heads' own base on. A wave's table, written by one lane a key and read by the lanes that fetch the rows.
struct Places {
  int64_t k, v;
};

// KT rows of both caches into two tiles, zeros behind dim (0 times an infinity would make a score no number). WHOLE: in pieces of 16 bytes past the registers, there behind
// wait_direct_loads() and a barrier; else element by element.
__device__ const u32x4 kZeroPiece = {0, 0, 0, 0};
template <typename T, int DP, int KT, int WAVES, bool WHOLE>
__device__ __forceinline__ void stage_pages(const T *k, const T *v, unsigned places, int dim, unsigned kt, unsigned vt, int wave, int lane) {
  using L = Tile<T, DP>;
  constexpr int N = KT * L::RB / 1024, EACH = (N + WAVES - 1) / WAVES;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int n = wave + i * WAVES;
    if (N % WAVES && n >= N) break;
    const int e = n * 64 + lane, row = e / L::CPR, piece = (e % L::CPR) ^ L::swizzle(row);
    typedef int64_t i64x2 __attribute__((ext_vector_type(2)));
    const i64x2 at = *lds_at<const i64x2>(places + row * 16);
    if constexpr (WHOLE) {
      const int d = piece * L::V;
      const T *zeros = (const T *)&kZeroPiece;
      lds_direct_load16(d < dim ? k + at[0] + d : zeros, __builtin_amdgcn_readfirstlane(kt + n * 1024));
      lds_direct_load16(d < dim ? v + at[1] + d : zeros, __builtin_amdgcn_readfirstlane(vt + n * 1024));
    } else {
      typename L::vec x, y;
#pragma unroll
      for (int j = 0; j < L::V; ++j) {
        const int d = piece * L::V + j;
        x[j] = d < dim ? k[at[0] + d] : (T)0.f;
        y[j] = d < dim ? v[at[1] + d] : (T)0.f;
      }
      *lds_at<typename L::vec>(kt + (unsigned)(e * 16)) = x;
      *lds_at<typename L::vec>(vt + (unsigned)(e * 16)) = y;
    }
  }
}

// load_row, also from odd places.
template <typename T, int DP, bool WHOLE>
__device__ __forceinline__ void load_query(Vec<T> *x, const T *p, bool there, int dim, int g) {
  if constexpr (WHOLE) {
    load_row<T, DP>(x, p, there, dim, g);
  } else {
    constexpr int V = Operand<T>::V;
#pragma unroll
    for (int c = 0; c < Tile<T, DP>::SLABS; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int d = V * (2 * c + g) + j;
        x[c][j] = there && d < dim ? p[d] : (T)0.f;
      }
  }
}

// A lane's column: a new token and a head.
struct Column {
  bool there;
  int token, head;
};

template <typename T, int DP, int WAVES, int KT, bool WHOLE>
struct CacheWalk {
  using L = Tile<T, DP>;
  static constexpr int BM = 32 * WAVES, BYTES = KT * L::RB;
  const CacheArgs &a;
  unsigned base, places;        // tiles; the wave's table of places, KT of them
  int lane, wave;

  // Tiles [t0, t1) of the unit (s, block of columns, head of keys); slot: where a part of it goes, -1: all of it is here.
  __device__ __forceinline__ void unit(int64_t s, Seq seq, int block, int kv, int t0, int t1, int64_t slot) const {
    using vec = typename L::vec;
    seq.rows = __builtin_amdgcn_readfirstlane(seq.rows);
    seq.length = __builtin_amdgcn_readfirstlane(seq.length);
    seq.keys = __builtin_amdgcn_readfirstlane(seq.keys);
    block = __builtin_amdgcn_readfirstlane(block);
    kv = __builtin_amdgcn_readfirstlane(kv);
    t0 = __builtin_amdgcn_readfirstlane(t0);
    t1 = __builtin_amdgcn_readfirstlane(t1);
    const int g = lane >> 5;
    auto column = [&](int l) {                        // of lane l
      const int col = block * BM + 32 * wave + (l & 31), token = col / a.group;
      return Column{token < seq.rows, token < seq.rows ? token : 0, kv * a.group + col % a.group};
    };
    const Column mine_at = column(lane);
    // keys that a token sees
    auto keys_of = [&](int i) { const int e = seq.length - seq.rows + i + 1; return e < 0 ? 0 : e < seq.keys ? e : seq.keys; };
    const int columns = seq.rows * a.group, w0 = block * BM + 32 * wave, last = columns - 1 < w0 + 31 ? columns - 1 : w0 + 31;
    const int all_see = w0 < columns ? keys_of(w0 / a.group) : 0, any_sees = w0 < columns ? keys_of(last / a.group) : 0, mine = mine_at.there ? keys_of(mine_at.token) : 0;
    const int end = columns - 1 < block * BM + BM - 1 ? columns - 1 : block * BM + BM - 1, keys = keys_of(end / a.group);
    const int stop = t1 < (keys + KT - 1) / KT ? t1 : (keys + KT - 1) / KT;
    vec q[L::SLABS];
    load_query<T, DP, WHOLE>(q, (const T *)a.q.p + (seq.begin + mine_at.token) * a.q.stride + mine_at.head * a.q.head_stride, mine_at.there, a.dim, g);
    const float c = a.scale * kLog2e;
    const T *kb = (const T *)a.kc.p + kv * a.kc.head_stride, *vb = (const T *)a.vc.p + kv * a.vc.head_stride;
    // Keys that are not there stand for the sequence's first one, or for the cache's first row: their scores do not count.
    Slot first = slot_of(a, s, 0);
    if (first.page < 0) first = {0, 0};
    auto look_up = [&](int t) {                       // (a load that the next step waits for)
      const int j = t * KT + lane % KT;
      return j < keys ? slot_of(a, s, j) : Slot{-1, 0};
    };
    auto write_places = [&](Slot at) {                // which of the tile's keys are there
      const unsigned long long valid = __ballot(at.page >= 0);
      if (at.page < 0) at = first;
      wave_lds_fence();
      if (lane < KT) {
        typedef int64_t i64x2 __attribute__((ext_vector_type(2)));
        *lds_at<i64x2>(places + lane * 16) =
            i64x2{(int64_t)at.page * a.kc.page_stride + (int64_t)at.slot * a.kc.stride, (int64_t)at.page * a.vc.page_stride + (int64_t)at.slot * a.vc.stride};
      }
      wave_lds_fence();
      return valid;
    };
    auto pass = [&](auto safe, auto &o, int db0) {
      constexpr bool SAFE = decltype(safe)::value;
      float mc = kLowest, l = 0.f;
      for (auto &x : o) x = zero_acc();
      unsigned long long valid = 0;
      Slot next = {-1, 0};
      if (t0 < stop) {
        valid = write_places(look_up(t0));
        stage_pages<T, DP, KT, WAVES, WHOLE>(kb, vb, places, a.dim, base, base + 2 * BYTES, wave, lane);
        next = look_up(t0 + 1);
      }
      for (int t = t0; t < stop; ++t) {
        const unsigned b = (unsigned)((t - t0) & 1) * BYTES, kt = base + b, vt = kt + 2 * BYTES;
        wait_direct_loads();
        __syncthreads();
        const unsigned long long now = valid;
        if (t + 1 < stop) {
          valid = write_places(next);
          stage_pages<T, DP, KT, WAVES, WHOLE>(kb, vb, places, a.dim, base + (BYTES - b), base + (BYTES - b) + 2 * BYTES, wave, lane);
          next = look_up(t + 2);
        }
        const int j0 = t * KT;
        if (j0 >= any_sees) continue;
        const bool whole = j0 + KT <= all_see && now == ~0ull;
        // the keys that the lane's column sees, a bit each
        const int left = mine - j0;
        const unsigned long long below = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull, seen = (now & below) >> (4 * g);
        add_tile<T, DP, KT, SAFE>(kt, vt, q, c, whole, [&](int n) { return (seen >> n & 1) != 0; }, o, mc, l, lane, db0);
      }
      __syncthreads();                                // (the next tiles go where the last ones are read)
      l = half_sum(l);
      int now = lane;
      asm volatile("" : "+v"(now));                   // (computed anew: kept over the loop it is spilled)
      const Column c_at = column(now);
      if (slot < 0) {
        store_row<T>((T *)a.out.p + (seq.begin + c_at.token) * a.out.stride + c_at.head * a.out.head_stride, c_at.there, a.dim, a.quads, o, l == 0.f ? 0.f : 1.f / l, now >> 5, db0);
      } else {
        const int64_t at = slot * BM + 32 * wave + (now & 31);
        store_row<float>(a.part + at * DP, c_at.there, DP, true, o, 1.f, now >> 5, db0);
        if (c_at.there && now < 32) {
          a.part_sums[2 * at] = mc;
          a.part_sums[2 * at + 1] = l;
        }
      }
    };
    f32x16 o[L::BLOCKS];
    pass(std::false_type(), o, 0);
    bool fine = true;
#pragma unroll
    for (int db = 0; db < L::BLOCKS; ++db) fine = fine && all_finite(o[db]);
    if (WAVES == 1 ? __ballot(!fine) == 0 : !__syncthreads_or(!fine)) return;
#pragma unroll 1
    for (int db = 0; db < L::BLOCKS; ++db) {
      f32x16 one[1];
      pass(std::true_type(), one, db);
    }
  }
};

// A piece of the line each, all of it by a fixed number of blocks.
template <typename T, int DP, int WAVES, int KT, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64, DP * sizeof(T) > 256 || (WAVES == 1 && DP * sizeof(T) == 256) ? 1 : 2) void cache_attention_kernel(const CacheArgs a) {
  using W = CacheWalk<T, DP, WAVES, KT, WHOLE>;
  __shared__ __attribute__((aligned(16))) char lds[4 * W::BYTES + WAVES * KT * 16];
  touch_args(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const W walk = {a, lds_address(lds), lds_address(lds) + 4 * W::BYTES + wave * KT * 16, lane, wave};
  auto weight = [&](int64_t s) {
    if (s >= a.seqs) return (int64_t)0;
    const Seq q = seq_of<W::BM, KT>(a, s);
    return (int64_t)q.blocks * a.kv_heads * q.tiles;
  };
  auto uniform64 = [](int64_t x) {
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((uint64_t)x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
  };
  int64_t total = 0;
  for (int64_t s = lane; s < a.seqs; s += 64) total += weight(s);
  total = uniform64(__shfl(sum_scan(total, lane), 63));
  const int64_t piece = (total + a.blocks - 1) / a.blocks, x0 = piece * blockIdx.x, x1 = x0 + piece < total ? x0 + piece : total;
  if (threadIdx.x == 0) a.splits[blockIdx.x] = {0, 0, 0, 0};
  if (x0 < x1) {
    // the sequence of the piece's first tile
    int64_t s = 0, start = 0;
    for (int64_t s0 = 0; s0 < a.seqs; s0 += 64) {
      const int64_t scan = sum_scan(weight(s0 + lane), lane), all = uniform64(__shfl(scan, 63));
      if (start + all <= x0) {
        start += all;
        continue;
      }
      const int n = __ffsll(__ballot(start + scan > x0)) - 1;
      s = s0 + n;
      start += n > 0 ? uniform64(__shfl(scan, n > 0 ? n - 1 : 0)) : 0;
      break;
    }
    for (int64_t x = x0; x < x1 && s < a.seqs; ++s) {
      Seq q = seq_of<W::BM, KT>(a, s);
      q.begin = uniform64(q.begin);
      q.blocks = __builtin_amdgcn_readfirstlane(q.blocks);
      q.tiles = __builtin_amdgcn_readfirstlane(q.tiles);
      const int64_t stop = start + (int64_t)q.blocks * a.kv_heads * q.tiles;
      while (x < x1 && x < stop) {
        const int64_t n = (x - start) / q.tiles;
        const int t0 = (int)((x - start) % q.tiles), t1 = (int)(q.tiles - t0 < x1 - x ? q.tiles : t0 + (x1 - x));
        // (units of one block of columns follow each other by heads of keys)
        const int block = (int)(n / a.kv_heads), kv = (int)(n % a.kv_heads);
        const bool cut = t0 > 0 || t1 < q.tiles;
        if (t0 == 0 && cut && threadIdx.x == 0) a.splits[blockIdx.x] = {s, block, kv, (int)((q.tiles - t1 + piece - 1) / piece)};
        walk.unit(s, q, block, kv, t0, t1, cut ? 2 * (int64_t)blockIdx.x + (t0 > 0 ? 0 : 1) : -1);
        x += t1 - t0;
      }
      start = stop;
    }
  }
}

// Where units are short: a whole one a block.
template <typename T, int DP, int WAVES, int KT, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64, DP * sizeof(T) > 256 || (WAVES == 1 && DP * sizeof(T) == 256) ? 1 : 2) void cache_attention_short_kernel(const CacheArgs a) {
  using W = CacheWalk<T, DP, WAVES, KT, WHOLE>;
  __shared__ __attribute__((aligned(16))) char lds[4 * W::BYTES + WAVES * KT * 16];
  touch_args(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const W walk = {a, lds_address(lds), lds_address(lds) + 4 * W::BYTES + wave * KT * 16, lane, wave};
  const int64_t b = a.block0 + blockIdx.x, u = b / a.kv_heads;
  // (numbers of a sequence's blocks of columns: from ptr group / BM + sequences on, as in the packed kernels)
  int64_t lo = 0, hi = a.seqs;
  auto first = [&](int64_t s) { return end_at(a.q_ptr, s, a.n_q) * a.group / W::BM + s; };
  do {
    const int64_t step = (hi - lo + 63) / 64, p = lo + lane * step;
    const unsigned long long before = __ballot(p < hi && first(p < hi ? p : lo) <= u);
    const int c = ~before ? __builtin_ctzll(~before) : 64;
    if (c == 0) return;
    lo += (c - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  } while (hi - lo > 1);
  const Seq q = seq_of<W::BM, KT>(a, lo);
  const int64_t block = u - first(lo);
  if (block >= q.blocks) return;
  walk.unit(lo, q, (int)block, (int)(b % a.kv_heads), 0, q.tiles, -1);
}

// The units that end behind the piece they begin in: a column's parts, in order; 32 columns a block.
template <typename T, int DP, int BM>
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheArgs a) {
  const int64_t b = blockIdx.x;
  const Split s = a.splits[b];
  if (s.follow == 0) return;
  const Span r = span_of(a.q_ptr, s.seq, a.n_q);
  const int columns = r.len * a.group - s.block * BM < BM ? r.len * a.group - s.block * BM : BM;
  // part 0: the second place of b, then the first places of the blocks behind it
  auto at = [&](int i) { return (i == 0 ? 2 * b + 1 : 2 * (b + i)) * BM; };
  for (int e = threadIdx.x; e < 32 * (DP / 4); e += 256) {
    const int col = blockIdx.y * 32 + e / (DP / 4), d = e % (DP / 4) * 4;
    if (col >= columns || d >= a.dim) continue;
    // (eight parts' loads together: each by itself is a round trip to memory)
    float m = kLowest, l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 <= s.follow; i0 += 8) {
      float pm[8], pl[8];
      f32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t p = at(i0 + i <= s.follow ? i0 + i : s.follow) + col;
        pm[i] = a.part_sums[2 * p];
        pl[i] = a.part_sums[2 * p + 1];
        x[i] = *(const f32x4 *)(a.part + p * DP + d);
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, pm[i]);
      const float old = __builtin_amdgcn_exp2f(m - top);
      m = top;
      l *= old;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] *= old;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i0 + i > s.follow) continue;
        const float f = __builtin_amdgcn_exp2f(pm[i] - m);
        l = fmaf(f, pl[i], l);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = fmaf(f, x[i][k], v[k]);
      }
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const int token = (s.block * BM + col) / a.group, head = s.kv * a.group + (s.block * BM + col) % a.group;
    T *out = (T *)a.out.p + (r.begin + token) * a.out.stride + head * a.out.head_stride + d;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= f;
    if (a.quads) {
      store4<T>(out, v);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (d + k < a.dim) out[k] = (T)v[k];
    }
  }
}

int check_cache(const xrl_ctx *c, const xrl_cache_desc *d, const char *who, CacheArgs &a) {
  if (!c || !d) return fail(XRL_ERR_NULL, "%s: ctx or desc is NULL", who);
  if (!op_type_ok(d->type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, d->type);
  if (d->n_seqs < 0 || d->n_q < 0 || d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads || d->dim < 1 || d->page < 1 || d->n_pages < 0 ||
      d->table_cols < 0 || d->table_stride < d->table_cols)
    return fail(XRL_ERR_SHAPE, "%s: %lld sequences, %lld rows, %d and %d heads of %d, %lld pages of %d, a table of %d columns, %lld apart", who, (long long)d->n_seqs,
                (long long)d->n_q, d->q_heads, d->kv_heads, d->dim, (long long)d->n_pages, d->page, d->table_cols, (long long)d->table_stride);
  if (d->dim > 128 || d->q_heads > 65536 || d->n_q > INT32_MAX - 65536 || d->n_seqs > INT32_MAX || d->n_pages > INT32_MAX ||
      (int64_t)d->table_cols * d->page > INT32_MAX - 65536 || d->n_q * (d->q_heads / d->kv_heads) > INT32_MAX - 65536)
    return fail(XRL_ERR_UNSUPPORTED, "%s: heads of %d (at most 128), %d heads, %lld rows, %d pages of %d a sequence", who, d->dim, d->q_heads, (long long)d->n_q,
                d->table_cols, d->page);
  if (d->n_seqs > 0 && (!d->d_q_ptr || !d->d_lengths || (d->table_cols > 0 && !d->d_table))) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d->d_q_ptr | (uintptr_t)d->d_lengths | (uintptr_t)d->d_table) % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a = CacheArgs{};
  a.q_ptr = d->d_q_ptr; a.lengths = d->d_lengths; a.table = d->d_table;
  a.seqs = d->n_seqs; a.n_q = d->n_q; a.table_stride = d->table_stride; a.n_pages = d->n_pages; a.table_cols = d->table_cols; a.page = d->page;
  a.q_heads = d->q_heads; a.kv_heads = d->kv_heads; a.group = d->q_heads / d->kv_heads; a.dim = d->dim;
  return XRL_OK;
}

// Extents and strides of a tensor that is written: no two elements at one place.
bool places_apart(std::initializer_list<std::pair<int64_t, int64_t>> extents, int64_t dim) {
  std::pair<int64_t, int64_t> e[3];
  int n = 0;
  for (auto &x : extents)
    if (x.first > 1) e[n++] = {x.second, x.first};
  std::sort(e, e + n);
  int64_t reach = dim;
  for (int i = 0; i < n; ++i) {
    if (e[i].first < reach) return false;
    reach += (e[i].second - 1) * e[i].first;
  }
  return true;
}

int check_rows(const xrl_heads *x, int64_t n, int heads, int dim, int es, bool written, const char *name, const char *who, Rows &o, bool &aligned) {
  if (!x || (n > 0 && !x->d_data)) return fail(XRL_ERR_NULL, "%s: %s is NULL", who, name);
  if ((uintptr_t)x->d_data % es) return fail(XRL_ERR_SHAPE, "%s: %s: a pointer that is no multiple of its elements' size", who, name);
  if (x->stride < 0 || x->head_stride < 0 || (written && !places_apart({{n, x->stride}, {heads, x->head_stride}}, dim)))
    return fail(XRL_ERR_SHAPE, "%s: %s: strides %lld and %lld", who, name, (long long)x->stride, (long long)x->head_stride);
  o = {x->d_data, n > 1 ? x->stride : 0, heads > 1 ? x->head_stride : 0};
  aligned = aligned && (uintptr_t)x->d_data % 16 == 0 && o.stride * es % 16 == 0 && o.head_stride * es % 16 == 0;
  return XRL_OK;
}
int check_pages(const xrl_pages *x, const CacheArgs &a, int es, bool written, const char *name, const char *who, Pages &o, bool &aligned) {
  if (!x || (a.n_pages > 0 && !x->d_data)) return fail(XRL_ERR_NULL, "%s: %s is NULL", who, name);
  if ((uintptr_t)x->d_data % es) return fail(XRL_ERR_SHAPE, "%s: %s: a pointer that is no multiple of its elements' size", who, name);
  if (x->page_stride < 0 || x->stride < 0 || x->head_stride < 0 ||
      (written && !places_apart({{a.n_pages, x->page_stride}, {a.page, x->stride}, {a.kv_heads, x->head_stride}}, a.dim)))
    return fail(XRL_ERR_SHAPE, "%s: %s: strides %lld, %lld and %lld", who, name, (long long)x->page_stride, (long long)x->stride, (long long)x->head_stride);
  o = {x->d_data, a.n_pages > 1 ? x->page_stride : 0, a.page > 1 ? x->stride : 0, a.kv_heads > 1 ? x->head_stride : 0};
  aligned = aligned && (uintptr_t)x->d_data % 16 == 0 && o.page_stride * es % 16 == 0 && o.stride * es % 16 == 0 && o.head_stride * es % 16 == 0;
  return XRL_OK;
}

template <typename T, int DP, int WAVES, bool WHOLE>
int launch(xrl_ctx *c, CacheArgs &a, const char *who) {
  constexpr int KT = WAVES == 1 || sizeof(T) == 4 ? 32 : 64, BM = 32 * WAVES, LDS = 4 * KT * DP * (int)sizeof(T) + WAVES * KT * 16 + 256;
  const int64_t most = ((int64_t)a.table_cols * a.page + KT - 1) / KT;
  // (us, one new token each in fp32, 4 heads of 32, whole units and pieces: 64 sequences of up to 64 keys 13.5 and 15.6, 192 16.0 and 16.7, 256 20.4 and 15.7; 512 of 64 15.8 and 22.4, of 128
  // 26 and 30, of 512 75 and 67)
  if (most <= 4) {
    a.blocks = (a.n_q * a.group / BM + a.seqs) * a.kv_heads;
    for (a.block0 = 0; a.block0 < a.blocks; a.block0 += kMaxBlocks)
      cache_attention_short_kernel<T, DP, WAVES, KT, WHOLE><<<dim3((unsigned)std::min(a.blocks - a.block0, kMaxBlocks)), dim3(WAVES * 64), 0, op_stream(c)>>>(a);
    OP_TRY(hipGetLastError());
    return XRL_OK;
  }
  // as many blocks as run at once: by the LDS, and two waves a SIMD
  a.blocks = (int64_t)op_compute_units(c) * std::min(160 * 1024 / LDS, 8 / WAVES);
  const size_t part = op_align((size_t)a.blocks * 2 * BM * DP * 4), sums = op_align((size_t)a.blocks * 2 * BM * 8);
  char *ws = nullptr;
  if (int rc = op_workspace(c, part + sums + (size_t)a.blocks * sizeof(Split), &ws, who)) return rc;
  a.part = (float *)ws;
  a.part_sums = (float *)(ws + part);
  a.splits = (Split *)(ws + part + sums);
  cache_attention_kernel<T, DP, WAVES, KT, WHOLE><<<dim3((unsigned)a.blocks), dim3(WAVES * 64), 0, op_stream(c)>>>(a);
  cache_join_kernel<T, DP, BM><<<dim3((unsigned)a.blocks, WAVES), dim3(256), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}
template <typename T, int DP>
int launch_waves(xrl_ctx *c, CacheArgs &a, bool whole, const char *who) {
  if (!whole) return launch<T, DP, 1, false>(c, a, who);
  // Blocks of 128 columns, whose four waves share the keys' tiles, where the sequences have half as many on average, else a wave by itself. us, 32768 cached tokens of 4 sequences, 8 heads of keys
  // of 128 in bf16, a wave and four: 64 columns 70 and 54, 96 86 and 62, 192 140 and 85, 2036 1020 and 422; of 512 sequences with 4 columns and 500 keys of 64 60 and 96.
  return a.n_q * a.group >= 64 * a.seqs ? launch<T, DP, 4, true>(c, a, who) : launch<T, DP, 1, true>(c, a, who);
}
template <typename T>
int launch_dim(xrl_ctx *c, CacheArgs &a, bool whole, const char *who) {
  return a.dim <= 32 ? launch_waves<T, 32>(c, a, whole, who) : a.dim <= 64 ? launch_waves<T, 64>(c, a, whole, who) : launch_waves<T, 128>(c, a, whole, who);
}

}  // namespace

extern "C" {

int xrl_cache_write(xrl_ctx *c, const xrl_cache_desc *d, const xrl_heads *k, const xrl_heads *v, const xrl_pages *k_cache, const xrl_pages *v_cache) {
  const char *who = "xrl_cache_write";
  CacheArgs a;
  if (int rc = check_cache(c, d, who, a)) return rc;
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4;
  bool whole = d->dim * es % 16 == 0;
  if (int rc = check_rows(k, a.n_q, a.kv_heads, a.dim, es, false, "k", who, a.k, whole)) return rc;
  if (int rc = check_rows(v, a.n_q, a.kv_heads, a.dim, es, false, "v", who, a.v, whole)) return rc;
  if (int rc = check_pages(k_cache, a, es, true, "k_cache", who, a.kc, whole)) return rc;
  if (int rc = check_pages(v_cache, a, es, true, "v_cache", who, a.vc, whole)) return rc;
  if (a.n_q == 0 || a.seqs == 0 || a.n_pages == 0 || a.table_cols == 0) return XRL_OK;
  const int64_t blocks = (a.n_q + 3) / 4;
  for (a.block0 = 0; a.block0 < blocks; a.block0 += kMaxBlocks) {
    const dim3 grid((unsigned)std::min(blocks - a.block0, kMaxBlocks));
    if (es == 2) whole ? cache_write_kernel<bf16_t, true><<<grid, dim3(256), 0, op_stream(c)>>>(a) : cache_write_kernel<bf16_t, false><<<grid, dim3(256), 0, op_stream(c)>>>(a);
    else whole ? cache_write_kernel<float, true><<<grid, dim3(256), 0, op_stream(c)>>>(a) : cache_write_kernel<float, false><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  }
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

int xrl_cache_attention(xrl_ctx *c, const xrl_cache_desc *d, float scale, const xrl_heads *q, const xrl_pages *k_cache, const xrl_pages *v_cache, const xrl_heads *out) {
  const char *who = "xrl_cache_attention";
  CacheArgs a;
  if (int rc = check_cache(c, d, who, a)) return rc;
  if (!(scale > 0.f) || !std::isfinite(scale * kLog2e)) return fail(XRL_ERR_VALUE, "%s: scale %g", who, (double)scale);
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4, v = 16 / es;
  bool whole = d->dim % v == 0, quads = true;
  if (int rc = check_rows(q, a.n_q, a.q_heads, a.dim, es, false, "q", who, a.q, whole)) return rc;
  if (int rc = check_rows(out, a.n_q, a.q_heads, a.dim, es, true, "out", who, a.out, quads)) return rc;
  if (int rc = check_pages(k_cache, a, es, false, "k_cache", who, a.kc, whole)) return rc;
  if (int rc = check_pages(v_cache, a, es, false, "v_cache", who, a.vc, whole)) return rc;
  if (a.n_q == 0 || a.seqs == 0) return XRL_OK;
  a.scale = scale;
  a.quads = quads && a.dim % 4 == 0;
  if (a.n_pages == 0) a.table_cols = 0;               // no key is there
  return es == 2 ? launch_dim<bf16_t>(c, a, whole, who) : launch_dim<float>(c, a, whole, who);
}

}  // extern "C"
