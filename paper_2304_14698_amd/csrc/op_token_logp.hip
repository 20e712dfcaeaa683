// Log-probabilities of given entries of rows of logits, with entropy and the best entries, and their gradient.
#include "op_common.h"

#include <algorithm>
#include <cmath>

using namespace xrl;

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.402823466e38f;        // also a maximum that no entry has reached yet: -inf - kLowest is -inf, not NaN
constexpr int kMaxTop = 64;                        // one alternative a lane

struct LogpArgs {
  const void *logits;
  const int32_t *row_ptr;
  const uint8_t *mask;
  const int32_t *ids;
  int64_t row0, n_rows, n_cols, stride, mask_stride;   // row0: first row of this launch
  float inv_t;
  int top_k, parts;
  float *logp, *entropy, *stats, *top_logp;
  int32_t *top_ids;
  // rows in several parts: of each part the maximum, the two sums and its best entries
  float *part_sums;             // [rows][parts][3]
  float *part_top;              // [rows][parts][top_k]
  int32_t *part_ids;
  // gradient
  const float *dlogp, *dentropy;
  void *dlogits;
  int64_t dstride;
  int row_blocks, clear_blocks; // of this launch (times gridDim.x)
};

template <typename T>
struct Row {
  const T *x;
  const uint8_t *mask;
  int64_t begin;                // ragged: of the flat arrays
  int len;
};

// Row r. What a row's ends say outside the array counts as not there.
template <typename T>
__device__ __forceinline__ Row<T> row_of(const LogpArgs &a, int64_t r) {
  Row<T> o;
  if (a.row_ptr) {
    int64_t b = a.row_ptr[r], e = a.row_ptr[r + 1];
    b = b < 0 ? 0 : b;
    e = e > a.n_cols ? a.n_cols : e;
    o.begin = b;
    o.len = e > b ? (int)(e - b) : 0;
    if (o.len == 0) o.begin = 0;
    o.x = (const T *)a.logits + o.begin;
    o.mask = a.mask ? a.mask + o.begin : nullptr;
  } else {
    o.begin = r * a.stride;
    o.len = (int)a.n_cols;
    o.x = (const T *)a.logits + o.begin;
    o.mask = a.mask ? a.mask + r * a.mask_stride : nullptr;
  }
  return o;
}

// Running sums of the entries seen so far, m their largest logit: S = sum 2^t and W = sum 2^t t, t = (x - m) c with c = log2(e) / temperature.
// A t of -inf counts as -200: 2^-200 is 0 in fp32, and 0 times it is 0.
struct Sums {
  float m, s, w;
};
__device__ __forceinline__ void add_sums(Sums &a, const Sums &b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float ta = (a.m - m) * c, tb = (b.m - m) * c;
  const float ea = __builtin_amdgcn_exp2f(ta), eb = __builtin_amdgcn_exp2f(tb);
  a.w = ea * (a.w + a.s * fmaxf(ta, -200.f)) + eb * (b.w + b.s * fmaxf(tb, -200.f));
  a.s = ea * a.s + eb * b.s;
  a.m = m;
}

// The best entries of a wave, lane i the i-th: by falling logit, then by rising index. An entry that is not there: kNone.
constexpr int kNone = 0x7fffffff;
struct Best {
  float x;
  int id;
};
__device__ __forceinline__ bool better(float xa, int ia, float xb, int ib) { return xa > xb || (xa == xb && ia < ib); }
// One entry that all lanes hold the same goes into the list of k.
__device__ __forceinline__ void insert_best(Best &b, float x, int id, int lane) {
  const bool before = better(b.x, b.id, x, id);
  const int at = __popcll(__ballot(before));
  const float px = __int_as_float(lane_move<kWaveShr1, 0xf>(0, __float_as_int(b.x)));
  const int pi = lane_move<kWaveShr1, 0xf>(0, b.id);
  if (lane == at) { b.x = x; b.id = id; }
  if (lane > at) { b.x = px; b.id = pi; }
}

// The sums of all lanes of a wave, in all lanes.
__device__ __forceinline__ Sums wave_sums(const Sums &u, float c) {
  const float m = wave_max(u.m), t = (u.m - m) * c, e = __builtin_amdgcn_exp2f(t);
  return {m, wave_sum(e * u.s), wave_sum(e * (u.w + u.s * fmaxf(t, -200.f)))};
}

// The row's given entry: whether there is one, and its logit, -inf if it may not be chosen.
struct Given {
  bool none;
  float x;
};
__device__ __forceinline__ int given_id(const LogpArgs &a, int64_t r) { return (a.ids ? a.ids : (const int32_t *)a.entropy)[r]; }   // (not looked at without ids)
template <typename T>
__device__ __forceinline__ Given given_entry(const LogpArgs &a, int id, const Row<T> &row) {
  id = a.ids ? id : -1;
  T x = (T)0.f;
  uint8_t ok = 1;
  const bool in = id >= 0 && id < row.len;
  if (row.len > 0) {
    x = row.x[in ? id : 0];
    if (row.mask) ok = row.mask[in ? id : 0];
  }
  return {id < 0, in && ok ? (float)x : -INFINITY};
}

// The row's results from its sums (the same in all lanes), its given logit (lane 0) and its best entries.
__device__ __forceinline__ void finish(const LogpArgs &a, int64_t r, const Given &given, const Sums &u, const Best &best, int lane) {
  const bool any = !(u.s == 0.f);                         // (NaN: yes)
  const float ln_s = logf(u.s);
  if (lane == 0) {
    a.entropy[r] = any ? ln_s - kLn2 * (u.w / u.s) : 0.f;
    if (a.stats) {
      a.stats[2 * r] = any ? u.m : -INFINITY;
      a.stats[2 * r + 1] = any ? ln_s : -INFINITY;
    }
    if (a.logp) {
      const float v = (given.x - u.m) * a.inv_t - ln_s;
      a.logp[r] = given.none ? 0.f : any && given.x != -INFINITY ? (v < kLowest ? kLowest : v) : -INFINITY;
    }
  }
  if (lane < a.top_k) {
    const bool there = best.id != kNone;
    a.top_ids[r * a.top_k + lane] = there ? best.id : -1;
    a.top_logp[r * a.top_k + lane] = !any || (!there && u.s == u.s) ? -INFINITY : (best.x - u.m) * a.inv_t - ln_s;
  }
}

// k rounds: the best of the heads of `lists` lists of k entries each, which lie in memory one after another.
template <typename GetX, typename GetId>
__device__ __forceinline__ Best merge_best(int lists, int k, int lane, GetX get_x, GetId get_id) {
  Best out = {-INFINITY, kNone};
  int head = 0;
  float x = lane < lists ? get_x(lane, 0) : -INFINITY;
  int id = lane < lists ? get_id(lane, 0) : kNone;
  for (int n = 0; n < k; ++n) {
    const float bx = wave_max(x);
    const unsigned long long tied = __ballot(x == bx);
    int bi = __builtin_amdgcn_readlane(id, __ffsll(tied) - 1);
    if (tied & (tied - 1)) bi = wave_min(x == bx ? id : kNone);
    if (lane == n) { out.x = bx; out.id = bi; }
    if (bi == kNone) break;
    if (id == bi) {
      ++head;
      x = head < k ? get_x(lane, head) : -INFINITY;
      id = head < k ? get_id(lane, head) : kNone;
    }
  }
  return out;
}

// bf16 pieces of 16 bytes that lie 2 bytes behind a multiple of 4 take longer than all others, and every second row of an odd length has nothing else: us,
// 4096 rows of 32003 61.5, of 32002 55. Such a row's pieces are read from the element before on, five words, and shifted (then 55.4), which leaves every sum
// its order wherever the row lies; where each entry stands by itself, in the gradient, a row's pieces begin at the element before its first.
template <typename T>
__device__ __forceinline__ int lead_of(const T *p, int len) { return sizeof(T) == 2 && len > 0 ? (int)((uintptr_t)p >> 1 & 1) : 0; }

// VEC elements from such a p. (What is read beside them lies in the same words as the first and the last.)
template <typename T, int VEC>
__device__ __forceinline__ Piece<T, VEC> load_odd_piece(const T *p) {
  Piece<T, VEC> x;
  if constexpr (sizeof(T) == 2) {
    unsigned u[VEC / 2 + 1], s[VEC / 2];
    __builtin_memcpy(u, __builtin_assume_aligned(p - 1, 4), VEC * 2);
    __builtin_memcpy(u + VEC / 2, __builtin_assume_aligned(p - 1 + VEC, 4), 4);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) s[i] = __builtin_amdgcn_alignbit(u[i + 1], u[i], 16);
    __builtin_memcpy(&x, s, sizeof(x));
  } else {
    x = load_piece<T, VEC>(p);
  }
  return x;
}

// Columns col .. col + VEC - 1 of the row as fp32, -inf where nothing may be chosen and from c1 on.
template <typename T, int VEC>
__device__ __forceinline__ void fetch(const Row<T> &row, bool odd, int col, int c1, float *x) {
  if (col + VEC <= c1) {
    const Piece<T, VEC> p = odd ? load_odd_piece<T, VEC>(row.x + col) : load_piece<T, VEC>(row.x + col);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = (float)p.v[j];
    if (row.mask) {
      const Piece<uint8_t, VEC> m = load_piece<uint8_t, VEC>(row.mask + col);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = m.v[j] ? x[j] : -INFINITY;
    }
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = col + j < c1 && (!row.mask || row.mask[col + j]) ? (float)row.x[col + j] : -INFINITY;
  }
}

// The entries of x over the wave's k-th best: the largest first, so at most k of them whatever their order, the lowest column first among equals (by
// piece, then lane, then place). mx: the pieces' maxima. Entries that are taken are overwritten. One that equals the k-th best has a higher column than it.
template <int VEC, int PIECES>
__device__ __forceinline__ void take_best(float (*x)[VEC], float *mx, int n_pieces, int col, int step, int lane, int top_k, Best &best, float &bar) {
  for (int n = 0; n < top_k; ++n) {
    float v = mx[0];
#pragma unroll
    for (int p = 1; p < PIECES; ++p) v = fmaxf(v, mx[p]);
    const float top = wave_max(v);
    if (!(top > bar)) return;
    bool done = false;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (done || p >= n_pieces) continue;
      const unsigned long long have = __ballot(mx[p] == top);
      if (!have) continue;
      done = true;
      const int from = __ffsll(have) - 1;
      int at = VEC - 1;
#pragma unroll
      for (int j = VEC - 2; j >= 0; --j) at = x[p][j] == top ? j : at;
      insert_best(best, top, __builtin_amdgcn_readlane(col + p * step + at, from), lane);
      bar = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(best.x), top_k - 1));
      const int gone = lane == from ? at : -1;
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        x[p][j] = j == gone ? -INFINITY : x[p][j];
        m = fmaxf(m, x[p][j]);
      }
      mx[p] = m;
    }
    if (!done) return;
  }
}

// A team of WAVES waves takes one part of one row, 32 entries a lane at a time: their maximum first, then the two sums against the largest so
// far, then the best of them. One pass: what is read stays in registers for all three.
// Bound by memory for many long rows: 4096 x 32003 in bf16 54 us, 262 MB at 4.9 TB/s; 4096 x 32000 52; 8192 x 16001 in fp32 91, 5.8 TB/s. Bound by latency for
// few: 8 x 128256 in bf16 with the best eight 12.5 us in two launches, 8 of them without the best; 32 x 65 7. With the best entries 1000 x 8191 in fp32 under
// a mask 16, 2.5 TB/s: a round of the selection takes 0.4 us, and all else of the wave waits for it.
// Four pieces of a lane are requested together where they lie inside the row for the whole wave; each by itself was 1 to 6 % slower in long rows, 20000 x 1024
// in fp32 39 us with the best four for 31. More of them, or a step ahead, take 97 to 140 registers in place of 64, and the waves that hide it: 50 -> 60 and
// 70 us. The bounds keep eight waves a SIMD without the best entries (65536 x 200 in bf16 31.4 us with seven, 29.8) and five with them.
template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(256, TOP ? 5 : 8) void token_logp_kernel(const LogpArgs a) {
  touch_args(a);
  constexpr int VEC = 16 / (int)sizeof(T), PIECES = 32 / VEC, TEAM = WAVES * 64, TEAMS = 256 / TEAM, STEP = TEAM * VEC, GROUP = 4;
  const int t = threadIdx.x % TEAM, lane = threadIdx.x & 63, wave = t >> 6;
  const int64_t job = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
  const int64_t r = a.row0 + job / a.parts;
  const int part = (int)(job % a.parts);
  if (r >= a.n_rows) return;                              // (a whole wave, and with WAVES > 1 the whole block)
  const Row<T> row = row_of<T>(a, r);
  const bool odd = __builtin_amdgcn_readfirstlane(lead_of(row.x, row.len)) != 0;
  const float c = a.inv_t * kLog2e;
  // part `part`: columns [c0, c1), whole steps of the team
  const int steps = (row.len + STEP - 1) / STEP, per = (steps + a.parts - 1) / a.parts;
  const int64_t b0 = (int64_t)part * per * STEP, b1 = b0 + (int64_t)per * STEP;
  const int c0 = (int)(b0 < row.len ? b0 : row.len), c1 = (int)(b1 < row.len ? b1 : row.len);
  const int id = given_id(a, r);                          // (needed at the end)
  Sums u = {kLowest, 0.f, 0.f};
  Best best = {-INFINITY, kNone};
  float bar = -INFINITY;
  for (int w = c0 + wave * 64 * VEC; w < c1; w += PIECES * STEP) {   // w: the wave's first column
    const int col = w + lane * VEC, left = (c1 - w + STEP - 1) / STEP, n_pieces = left < PIECES ? left : PIECES;
    float x[PIECES][VEC], mx[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; p += GROUP) {
      if (w + (p + GROUP - 1) * STEP + 64 * VEC <= c1) {      // all of the group inside, for all lanes
        Piece<T, VEC> v[GROUP];
        if (odd)
#pragma unroll
          for (int k = 0; k < GROUP; ++k) v[k] = load_odd_piece<T, VEC>(row.x + col + (p + k) * STEP);
        else
#pragma unroll
          for (int k = 0; k < GROUP; ++k) v[k] = load_piece<T, VEC>(row.x + col + (p + k) * STEP);
#pragma unroll
        for (int k = 0; k < GROUP; ++k)
#pragma unroll
          for (int j = 0; j < VEC; ++j) x[p + k][j] = (float)v[k].v[j];
        if (row.mask) {
          Piece<uint8_t, VEC> m[GROUP];
#pragma unroll
          for (int k = 0; k < GROUP; ++k) m[k] = load_piece<uint8_t, VEC>(row.mask + col + (p + k) * STEP);
#pragma unroll
          for (int k = 0; k < GROUP; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[p + k][j] = m[k].v[j] ? x[p + k][j] : -INFINITY;
        }
      } else {
#pragma unroll
        for (int k = 0; k < GROUP; ++k)
          if (p + k < n_pieces) fetch<T, VEC>(row, odd, col + (p + k) * STEP, c1, x[p + k]);
      }
    }
    float m = u.m;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      mx[p] = -INFINITY;
      if (p < n_pieces) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) mx[p] = fmaxf(mx[p], x[p][j]);
        m = fmaxf(m, mx[p]);
      }
    }
    const float t0 = (u.m - m) * c, e0 = __builtin_amdgcn_exp2f(t0);
    u.w = e0 * (u.w + u.s * fmaxf(t0, -200.f));
    u.s *= e0;
    u.m = m;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (p < n_pieces) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float q = (x[p][j] - m) * c, e = __builtin_amdgcn_exp2f(q);
          u.s += e;
          u.w += e * fmaxf(q, -200.f);
        }
      }
    }
    if (TOP) take_best<VEC, PIECES>(x, mx, n_pieces, col, STEP, lane, a.top_k, best, bar);
  }
  u = wave_sums(u, c);
  if constexpr (WAVES > 1) {
    __shared__ float sums[WAVES][3], bx[WAVES][kMaxTop];
    __shared__ int bi[WAVES][kMaxTop];
    if (lane == 0) { sums[wave][0] = u.m; sums[wave][1] = u.s; sums[wave][2] = u.w; }
    bx[wave][lane] = best.x;
    bi[wave][lane] = best.id;
    __syncthreads();
    if (wave) return;
    for (int k = 1; k < WAVES; ++k) add_sums(u, {sums[k][0], sums[k][1], sums[k][2]}, c);
    if (TOP)
      best = merge_best(WAVES, a.top_k, lane, [&](int l, int i) { return bx[l][i]; }, [&](int l, int i) { return bi[l][i]; });
  }
  if (a.parts == 1) {
    finish(a, r, given_entry<T>(a, id, row), u, best, lane);
    return;
  }
  if (lane == 0) {
    float *p = a.part_sums + job * 3;
    p[0] = u.m; p[1] = u.s; p[2] = u.w;
  }
  if (TOP && lane < a.top_k) {
    a.part_top[job * a.top_k + lane] = best.x;
    a.part_ids[job * a.top_k + lane] = best.id;
  }
}

// A wave per row: its parts (at most 64), in order. Latency: 4 to 5 us, of which a launch is 2.7. (The lists in LDS first: 0.5 us more.)
template <typename T>
__global__ __launch_bounds__(64) void token_logp_join_kernel(const LogpArgs a) {
  const int64_t r = blockIdx.x;
  const int lane = threadIdx.x;
  touch_args(a);
  const Row<T> row = row_of<T>(a, r);
  const int id = given_id(a, r);
  const int64_t job = r * a.parts + lane;
  const bool in = lane < a.parts;
  const float *p = a.part_sums + (in ? job : 0) * 3;
  Sums u = {in ? p[0] : kLowest, in ? p[1] : 0.f, in ? p[2] : 0.f};
  u = wave_sums(u, a.inv_t * kLog2e);
  Best best = {-INFINITY, kNone};
  if (a.top_k)
    best = merge_best(a.parts, a.top_k, lane, [&](int l, int i) { return a.part_top[(r * a.parts + l) * a.top_k + i]; },
                      [&](int l, int i) { return a.part_ids[(r * a.parts + l) * a.top_k + i]; });
  finish(a, r, given_entry<T>(a, id, row), u, best, lane);
}

// dlogits_j = (1 / temperature) (g [j = id] - p_j (g + h (ln p_j + H))): with q = log2 p_j, p_j (A + B q)
// Each entry by itself; a row has a wave, or blocks of two pieces a thread or four. Bound by memory: 2048 x 50021 in bf16 78 us for 205 MB read and written, 5.3 TB/s; results of more than the L2s hold are stored past the caches.
template <typename T, bool STREAM, int TEAM>
__device__ __forceinline__ void backward_row(const LogpArgs &a, int64_t r, int t) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const Row<T> row = row_of<T>(a, r);
  // what the row has, all requested together: what is not given is read from the entropy and not looked at
  const int id0 = (a.ids ? a.ids : (const int32_t *)a.entropy)[r];
  const float logp = (a.ids ? a.logp : a.entropy)[r], g0 = (a.ids ? a.dlogp : a.entropy)[r], h0 = (a.dentropy ? a.dentropy : a.entropy)[r];
  const float m = a.stats[2 * r], ln_s = a.stats[2 * r + 1], H = a.entropy[r];
  const float c = a.inv_t * kLog2e, log2_s = ln_s * kLog2e;
  const bool any = !(m == -INFINITY);
  // whether the given entry may be chosen: from its log-probability, as in place another block may have written over its logit
  const int id = a.ids && id0 >= 0 && !(logp == -INFINITY) ? id0 : -1;
  const float g = id >= 0 ? g0 : 0.f, h = a.dentropy ? h0 : 0.f;
  const float A = -a.inv_t * (g + h * H), B = -a.inv_t * h * kLn2;
  T *out = (T *)a.dlogits + (a.row_ptr ? row.begin : r * a.dstride);
  for (int64_t col = ((int64_t)blockIdx.x * TEAM + t) * VEC - lead_of(out, row.len); col < row.len; col += (int64_t)gridDim.x * TEAM * VEC) {
    const bool whole = col >= 0 && col + VEC <= row.len;
    float x[VEC], d[VEC];
    bool ok[VEC];
    if (whole) {
      const Piece<T, VEC> p = load_piece<T, VEC>(row.x + col);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = (float)p.v[j];
      if (row.mask) {
        const Piece<uint8_t, VEC> k = load_piece<uint8_t, VEC>(row.mask + col);
#pragma unroll
        for (int j = 0; j < VEC; ++j) ok[j] = k.v[j] != 0;
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) ok[j] = true;
      }
    } else {
      T v[VEC];
      uint8_t k[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int64_t at = col + j < 0 ? 0 : col + j < row.len ? col + j : row.len - 1;
        v[j] = row.x[at];
        k[j] = row.mask ? row.mask[at] : 1;
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        ok[j] = k[j] != 0;
        x[j] = (float)v[j];
      }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float q = (x[j] - m) * c - log2_s;
      float v = __builtin_amdgcn_exp2f(q) * (A + B * fmaxf(q, -200.f));
      if (col + j == id) v += a.inv_t * g;
      d[j] = ok[j] && any && !(x[j] == -INFINITY) ? v : 0.f;
    }
    if (whole) store_piece<T, VEC, STREAM>(out + col, d);
    else
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (col + j >= 0 && col + j < row.len) out[col + j] = (T)d[j];
  }
}

// Entries of the flat array that no row covers belong to no sum: 0. As a row begins where the one before ends they lie in front of the first end and behind the
// last. Where another end lies outside these two (ends that fall), 64 entries at a time are held against all rows. Blocks of their own: with a share for every
// row's wave 20000 x 65 in bf16 took 12.5 us, 11.7 without.
template <typename T>
__device__ __forceinline__ void clear_uncovered(const LogpArgs &a, int64_t block, int64_t blocks) {
  const int64_t first_end = a.row_ptr[0], last_end = a.row_ptr[a.n_rows];
  auto inside = [&](int64_t x) { return x < 0 ? 0 : x < a.n_cols ? x : a.n_cols; };
  const int64_t front = inside(first_end), n = front + a.n_cols - inside(last_end), behind = inside(last_end) - front;
  if (block * 256 >= n) return;
  const int lane = threadIdx.x & 63;
  bool falls = false;
  for (int64_t i = lane; i <= a.n_rows; i += 8 * 64) {
    int32_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = a.row_ptr[i + k * 64 < a.n_rows ? i + k * 64 : a.n_rows];
#pragma unroll
    for (int k = 0; k < 8; ++k) falls = falls | (x[k] < first_end) | (x[k] > last_end);
  }
  falls = __ballot(falls) != 0;
  for (int64_t i0 = block * 256 + (threadIdx.x - lane); i0 < n; i0 += blocks * 256) {
    const int64_t i = i0 + lane, at = i < front ? i : i + behind;
    bool covered = false;
    if (falls)
      for (int64_t r0 = 0; r0 < a.n_rows; r0 += 64) {
        const int64_t r = r0 + lane < a.n_rows ? r0 + lane : a.n_rows - 1;
        const int b = a.row_ptr[r], e = a.row_ptr[r + 1];
        for (int k = 0; k < 64; ++k) covered = covered | (__builtin_amdgcn_readlane(b, k) <= at && at < __builtin_amdgcn_readlane(e, k));
      }
    if (i < n && !covered) ((T *)a.dlogits)[at] = (T)0.f;
  }
}

template <typename T, bool STREAM, int WAVES>
__global__ __launch_bounds__(256) void token_logp_backward_kernel(const LogpArgs a) {
  touch_args(a);
  const int64_t block = blockIdx.y + (int64_t)blockIdx.z * 32768;
  if (block >= a.row_blocks) {
    if (block < a.row_blocks + a.clear_blocks) clear_uncovered<T>(a, (block - a.row_blocks) * gridDim.x + blockIdx.x, (int64_t)a.clear_blocks * gridDim.x);
    return;
  }
  const int64_t r = a.row0 + block * (4 / WAVES) + __builtin_amdgcn_readfirstlane(threadIdx.x / (WAVES * 64));
  if (r < a.n_rows) backward_row<T, STREAM, WAVES * 64>(a, r, threadIdx.x % (WAVES * 64));
}

int check_logits(const xrl_ctx *c, const xrl_logits_desc *l, const char *who, LogpArgs &a) {
  if (!c || !l) return fail(XRL_ERR_NULL, "%s: ctx or logits is NULL", who);
  if (!op_type_ok(l->type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, l->type);
  if (!(l->temperature > 0.f) || !std::isfinite(l->temperature)) return fail(XRL_ERR_VALUE, "%s: temperature %g", who, (double)l->temperature);
  if (!std::isfinite(1.f / l->temperature * kLog2e)) return fail(XRL_ERR_VALUE, "%s: temperature %g", who, (double)l->temperature);
  if (l->n_rows < 0 || l->n_cols < 0 || (!l->d_row_ptr && (l->stride < l->n_cols || (l->d_mask && l->mask_stride != 0 && l->mask_stride < l->n_cols))))
    return fail(XRL_ERR_SHAPE, "%s: %lld rows of %lld columns, strides %lld and %lld", who, (long long)l->n_rows, (long long)l->n_cols,
                (long long)l->stride, (long long)l->mask_stride);
  if (l->n_cols > INT32_MAX - 65536 || l->n_rows > INT32_MAX)
    return fail(XRL_ERR_UNSUPPORTED, "%s: %lld rows of %lld columns", who, (long long)l->n_rows, (long long)l->n_cols);
  if (l->n_rows > 0 && l->n_cols > 0 && !l->d_logits) return fail(XRL_ERR_NULL, "%s: d_logits is NULL", who);
  if ((uintptr_t)l->d_logits % (l->type == XRL_PREC_BF16 ? 2 : 4) || (uintptr_t)l->d_row_ptr % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a = LogpArgs{};
  a.logits = l->d_logits; a.row_ptr = l->d_row_ptr; a.mask = l->d_mask;
  a.n_rows = l->n_rows; a.n_cols = l->n_cols; a.stride = l->stride; a.mask_stride = l->mask_stride;
  a.inv_t = 1.f / l->temperature;
  return XRL_OK;
}

template <typename T, bool TOP>
void launch_logp(const xrl_ctx *c, LogpArgs &a, bool wave_rows) {
  for (a.row0 = 0; a.row0 < a.n_rows; a.row0 += kMaxBlocks) {
    const int64_t jobs = std::min(a.n_rows - a.row0, kMaxBlocks) * a.parts;    // (parts > 1: of a few rows)
    if (wave_rows)
      token_logp_kernel<T, 1, TOP><<<dim3((unsigned)((jobs + 3) / 4)), dim3(256), 0, op_stream(c)>>>(a);
    else
      token_logp_kernel<T, 4, TOP><<<dim3((unsigned)jobs), dim3(256), 0, op_stream(c)>>>(a);
  }
  if (a.parts > 1) token_logp_join_kernel<T><<<dim3((unsigned)a.n_rows), dim3(64), 0, op_stream(c)>>>(a);
}

template <typename T>
void launch_backward(const xrl_ctx *c, const LogpArgs &a, dim3 grid, bool stream, bool wave_rows) {
  if (wave_rows) stream ? token_logp_backward_kernel<T, true, 1><<<grid, dim3(256), 0, op_stream(c)>>>(a) : token_logp_backward_kernel<T, false, 1><<<grid, dim3(256), 0, op_stream(c)>>>(a);
  else stream ? token_logp_backward_kernel<T, true, 4><<<grid, dim3(256), 0, op_stream(c)>>>(a) : token_logp_backward_kernel<T, false, 4><<<grid, dim3(256), 0, op_stream(c)>>>(a);
}

}  // namespace

extern "C" {

int xrl_token_logp(xrl_ctx *c, const xrl_logits_desc *logits, const int32_t *d_ids, int32_t top_k, float *d_logp,
                   float *d_entropy, float *d_stats, int32_t *d_top_ids, float *d_top_logp) {
  const char *who = "xrl_token_logp";
  LogpArgs a;
  if (int rc = check_logits(c, logits, who, a)) return rc;
  if (top_k < 0 || top_k > kMaxTop) return fail(XRL_ERR_UNSUPPORTED, "%s: top_k = %d (at most %d)", who, top_k, kMaxTop);
  if (a.n_rows == 0) return XRL_OK;
  if ((d_ids && !d_logp) || !d_entropy || (top_k > 0 && (!d_top_ids || !d_top_logp))) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d_ids | (uintptr_t)d_logp | (uintptr_t)d_entropy | (uintptr_t)d_stats | (uintptr_t)d_top_ids | (uintptr_t)d_top_logp) % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a.ids = d_ids; a.top_k = top_k; a.logp = d_logp; a.entropy = d_entropy; a.stats = d_stats; a.top_ids = d_top_ids; a.top_logp = d_top_logp;
  // A wave a row where that is one step of 2048 columns (on average, where they are ragged), or up to four where there are rows for six waves a compute unit (two
  // in fp32 without the best entries); else a block a row. us, block / wave: 10000 x 2000 in bf16 18.8 / 14.3, in fp32 20.5 / 17.5; 500 x 4000 in fp32 with the best
  // four 8.1 / 10.8, 2000 16.4 / 13.4; 1000 x 8000 in bf16 with the best eight 16 / 22, 4000 44 / 33; 8000 x 8000 31.5 / 29.8, in fp32 48.6 / 51.3.
  // Few rows of more columns than a block's step of 8192, without the best entries than five of these, are cut into parts, at most 64, which a second launch joins:
  // of 2048 columns and a wave each where such parts do not fill the chip by themselves, else of a block each. us, uncut / cut: best eight of 8 x 8000 in fp32
  // 10.5 / 12.4, of 16000 15.2 / 12.3, of 8 x 128256 in bf16 39 / 12.5 (parts of a block 14.7); without them 64 x 30000 in fp32 7.3 / 9.2, 64 x 50021 in bf16 10.2 / 8.4,
  // 16 x 128256 in fp32 20 / 8.6.
  const int64_t cols = a.row_ptr ? a.n_cols / a.n_rows : a.n_cols, n_cu = op_compute_units(c), fine = (cols + 2047) / 2048;
  const bool bf16 = logits->type == XRL_PREC_BF16;
  bool wave_rows = cols <= 2048 || (a.n_rows > 6 * n_cu && cols <= (top_k || bf16 ? 8192 : 4096));
  a.parts = 1;
  if (cols > (top_k ? 8192 : 40960)) {
    wave_rows = fine <= 64 && fine * a.n_rows <= 8 * n_cu;
    a.parts = wave_rows ? (int)fine : (int)std::max<int64_t>(1, std::min<int64_t>({4 * n_cu / a.n_rows, cols / 2048, 64}));
  }
  if (a.parts > 1) {
    const size_t jobs = (size_t)a.n_rows * a.parts, o_t = op_align(jobs * 12), o_i = o_t + op_align(jobs * top_k * 4);
    char *ws = nullptr;
    if (int rc = op_workspace(c, o_i + jobs * top_k * 4, &ws, who)) return rc;
    a.part_sums = (float *)ws; a.part_top = (float *)(ws + o_t); a.part_ids = (int32_t *)(ws + o_i);
  }
  if (bf16) top_k ? launch_logp<bf16_t, true>(c, a, wave_rows) : launch_logp<bf16_t, false>(c, a, wave_rows);
  else top_k ? launch_logp<float, true>(c, a, wave_rows) : launch_logp<float, false>(c, a, wave_rows);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

int xrl_token_logp_backward(xrl_ctx *c, const xrl_logits_desc *logits, const int32_t *d_ids, const float *d_logp,
                            const float *d_entropy, const float *d_stats, const float *d_dlogp, const float *d_dentropy,
                            void *d_dlogits, int64_t dlogits_stride) {
  const char *who = "xrl_token_logp_backward";
  LogpArgs a;
  if (int rc = check_logits(c, logits, who, a)) return rc;
  if ((a.n_rows == 0 && !a.row_ptr) || a.n_cols == 0) return XRL_OK;
  if (!d_dlogits || (a.n_rows > 0 && (!d_entropy || !d_stats || (d_ids && (!d_logp || !d_dlogp))))) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (!a.row_ptr && dlogits_stride < a.n_cols) return fail(XRL_ERR_SHAPE, "%s: dlogits_stride = %lld", who, (long long)dlogits_stride);
  if (d_dlogits == logits->d_logits && !a.row_ptr && dlogits_stride != a.stride)
    return fail(XRL_ERR_SHAPE, "%s: in place, but at another stride", who);
  if (((uintptr_t)d_ids | (uintptr_t)d_logp | (uintptr_t)d_entropy | (uintptr_t)d_stats | (uintptr_t)d_dlogp | (uintptr_t)d_dentropy) % 4 ||
      (uintptr_t)d_dlogits % (logits->type == XRL_PREC_BF16 ? 2 : 4))
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a.ids = d_ids; a.logp = (float *)d_logp; a.entropy = (float *)d_entropy; a.stats = (float *)d_stats; a.dlogp = d_dlogp; a.dentropy = d_dentropy;
  a.dlogits = d_dlogits; a.dstride = dlogits_stride;
  const int64_t cols = a.row_ptr ? a.n_cols / std::max<int64_t>(1, a.n_rows) : a.n_cols, vec = logits->type == XRL_PREC_BF16 ? 8 : 4;
  // Pieces of a thread: us, two / four, 2048 x 50021 in bf16 84 / 78, 4096 x 32000 103 / 95 (eight: 85, 99); 8192 x 16001 in fp32 184 / 198.
  const int64_t per = 256 * vec * (vec == 8 ? 4 : 2);
  // Rows of up to 4 KB have a wave each: us, block / wave, 20000 rows, 200 in bf16 15.7 / 10.3, 1000 22 / 15.4, 1000 in fp32 28.3 / 27.3; 10000 x 2000 in bf16 17.5 /
  // 16.8, in fp32 24.6 / 26.4.
  const bool wave_rows = cols <= 256 * vec;
  const int64_t chunks = wave_rows ? 1 : (cols + per - 1) / per, team_rows = wave_rows ? 4 : 1;
  const bool stream = streams(a.n_cols * (a.row_ptr ? 1 : a.n_rows) * (16 / vec));
  for (a.row0 = 0; a.row0 == 0 || a.row0 < a.n_rows; a.row0 += kMaxBlocks) {
    a.row_blocks = (int)((std::min(a.n_rows - a.row0, kMaxBlocks) + team_rows - 1) / team_rows);
    // blocks for entries that no row covers: 64 entries a thread, at most 512 blocks in all
    a.clear_blocks = a.row_ptr && a.row0 == 0 ? (int)std::max<int64_t>(1, std::min<int64_t>(a.n_cols / (256 * 64), 512) / chunks) : 0;
    const int64_t blocks = a.row_blocks + a.clear_blocks;
    const dim3 grid((unsigned)chunks, (unsigned)std::min<int64_t>(blocks, 32768), (unsigned)((blocks + 32767) / 32768));
    logits->type == XRL_PREC_BF16 ? launch_backward<bf16_t>(c, a, grid, stream, wave_rows) : launch_backward<float>(c, a, grid, stream, wave_rows);
  }
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

}  // extern "C"
