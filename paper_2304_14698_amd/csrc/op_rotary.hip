// The norm of queries and keys per head and the rotation of their columns in pairs by angles position * frequency, in one pass, and its gradients.
//
// Per row x of dim columns: y = x r w, r = (mean x^2 + eps)^-1/2 (without a weight w: y = x); of each pair, z1 = y1 cos a - y2 sin a, z2 = y1 sin a + y2 cos a. With g the
// gradient to z rotated back: dw += g x r, dx = r (g w - x r^2 mean(g w x)).
//
// Bound by memory. A row lies in the lanes of one wave, 16 bytes a lane, so its mean is a few lane moves; the other half of a pair comes from the lane's own piece, or from the
// cache line that a neighbour has just read. A block has up to eight tokens, computes their
// cosines and sines, of angles in 64 bits, once, while its first rows are on their way, and goes over all their heads with the next rows' loads ahead.
//
// 16384 rows of 40 heads of 128 in bf16, half of each rotated: forward 87 to 91 us, 3.8 TB/s; backward 101 to 105 and 5 for the weights' sums, 4.7 TB/s; in fp32 166, and 202 with the sums. (A large copy
// reaches 5.18.) 32 rows: 8.3. Rows at odd addresses, one column a lane at a time: 268 and 366.
#include "op_common.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

using namespace xrl;

namespace {

constexpr int kTokens = 8, kPairs = 128;           // rows of a block, and pairs of a head, at most

struct Heads {
  const void *p;
  int64_t stride, head_stride;
};

struct RotaryArgs {
  int64_t n, block0;            // rows; first block of this launch
  int q_heads, heads, dim, rotary, interleaved;   // heads: of q and k
  int tokens;                   // rows of a block
  float eps;
  const int32_t *positions;
  const float *freqs, *weight[2];
  Heads x[2], z[2], dz[2], dx[2];   // q, k
  float *partial;               // [blocks][2][dim]: sums of the weights' gradients
  float *dweight[2];
  int partials;
};

// Sums over groups of LANES neighbouring lanes, in all of them.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
#define STEP(CTRL) x += __int_as_float(lane_move<CTRL, 0xf>(0, __float_as_int(x)))
  if constexpr (LANES >= 2) STEP(0xB1);
  if constexpr (LANES >= 4) STEP(0x4E);
  if constexpr (LANES >= 8) STEP(0x141);
  if constexpr (LANES >= 16) STEP(0x140);
#undef STEP
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// What a lane has of a row: PIECES pieces of V columns, the first from column `lane in the group` * V on, the others LANES * V further each. V > 1: every piece lies
// wholly in the first half of the pairs, in the second, or behind them.
template <int V, int LANES>
struct Columns {
  int e;                        // first column
  __device__ __forceinline__ int at(int p, int j) const { return e + p * LANES * V + j; }
};
// The pair of column e, its other column, and the sign of that one's sine. Columns behind the pairs: -1.
struct Pair {
  int index, other;
  float sign;
};
__device__ __forceinline__ Pair pair_of(const RotaryArgs &a, int e) {
  if (e >= a.rotary) return {-1, e, 0.f};
  if (a.interleaved) return {e >> 1, e ^ 1, e & 1 ? 1.f : -1.f};
  const int half = a.rotary >> 1;
  return e < half ? Pair{e, e + half, -1.f} : Pair{e - half, e - half, 1.f};
}
// The angle in turns, in 64 bits: a position of 2^31 leaves 2^-22 of a turn's part below it.
__device__ __forceinline__ void angle_of(int position, float freq, float &c, float &s) {
  double t = (double)position * (double)freq * 0.15915494309189533577;
  t -= rint(t);
  sincospif(2.f * (float)t, &s, &c);
}

// V columns of a row as they lie: 16 bytes, or one element.
template <typename T, int V>
struct Raw;
template <>
struct Raw<float, 4> { typedef u32x4 type; };
template <>
struct Raw<bf16_t, 8> { typedef u32x4 type; };
template <>
struct Raw<float, 1> { typedef float type; };
template <>
struct Raw<bf16_t, 1> { typedef bf16_t type; };
template <typename T, int V>
__device__ __forceinline__ float column_of(const typename Raw<T, V>::type &r, int j) {
  if constexpr (V == 1) return (float)r;
  else if constexpr (sizeof(T) == 4) return __uint_as_float(r[j]);
  else return __uint_as_float(j & 1 ? r[j >> 1] & 0xffff0000u : r[j >> 1] << 16);
}
// Columns e on of the row, and of the other halves of their pairs: of its first ones where e lies behind dim (what is not there counts as 0 later). No
// load depends on a condition, so that those of several rows go out together.
template <typename T, int V>
struct Two {
  typename Raw<T, V>::type x, o;
};
template <typename T, int V>
__device__ __forceinline__ typename Raw<T, V>::type load_columns(const T *row, int e, int dim) {
  return *(const typename Raw<T, V>::type *)(row + (e < dim ? e : 0));
}
template <typename T, int V>
__device__ __forceinline__ Two<T, V> load_pair(const RotaryArgs &a, const T *row, int e) {
  Two<T, V> c;
  c.x = load_columns<T, V>(row, e, a.dim);
  if (V > 1 && a.interleaved) c.o = c.x;
  else c.o = load_columns<T, V>(row, pair_of(a, e).other, a.dim);
  return c;
}
// Columns behind the pairs have no other half: 0.
template <typename T, int V>
__device__ __forceinline__ void alone(Two<T, V> &c, bool paired) {
  if constexpr (V > 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c.o[i] = paired ? c.o[i] : 0u;
  } else {
    c.o = paired ? c.o : (T)0.f;
  }
}
template <typename T, int V>
__device__ __forceinline__ float own_of(const Two<T, V> &c, int j) { return column_of<T, V>(c.x, j); }
template <typename T, int V>
__device__ __forceinline__ float other_of(const RotaryArgs &a, const Two<T, V> &c, int j) {
  if constexpr (V > 1) return a.interleaved ? column_of<T, V>(c.o, j ^ 1) : column_of<T, V>(c.o, j);
  else return column_of<T, V>(c.o, j);
}
template <typename T, int V, bool STREAM>
__device__ __forceinline__ void store_columns(T *row, int e, bool there, const float *z) {
  if (!there) return;
  if constexpr (V > 1) store_piece<T, V, STREAM>((T *)__builtin_assume_aligned(row + e, 16), z);
  else row[e] = (T)z[0];
}

// Cosines and sines of a block's tokens, every pair's once: [token][pair].
struct Turns {
  float c[kTokens * kPairs], s[kTokens * kPairs];
};
__device__ __forceinline__ void make_turns(const RotaryArgs &a, Turns &t, int64_t t0, int tokens, float back) {
  const int pairs = a.rotary >> 1;
  for (int i = threadIdx.x; i < tokens * pairs; i += 256) {
    const int token = i / pairs, pair = i % pairs;
    float c, s;
    angle_of(a.positions[t0 + token], a.freqs[pair], c, s);
    t.c[token * kPairs + pair] = c;
    t.s[token * kPairs + pair] = back * s;
  }
  __syncthreads();
}
// Of the lane's V columns from e on: z_e = y_e c + y_other s. Behind the pairs 1 and 0.
template <int V>
__device__ __forceinline__ void turn_of(const RotaryArgs &a, const Turns &t, int token, int e, float (&c)[V], float (&s)[V]) {
  if (e >= a.rotary) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      c[j] = 1.f;
      s[j] = 0.f;
    }
    return;
  }
  if (V > 1 && a.interleaved) {
    const float *tc = t.c + token * kPairs + (e >> 1), *ts = t.s + token * kPairs + (e >> 1);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      c[j] = tc[j >> 1];
      s[j] = j & 1 ? ts[j >> 1] : -ts[j >> 1];
    }
  } else {
    const Pair r = pair_of(a, e);
    const float *tc = t.c + token * kPairs + r.index, *ts = t.s + token * kPairs + r.index;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      c[j] = tc[j];
      s[j] = r.sign * ts[j];
    }
  }
}

// A block's rows of one tensor: token by token, head by head. A group of LANES lanes has every so many-th of them, U at a time.
struct RowAt {
  int token, head;
};
__device__ __forceinline__ RowAt row_at(unsigned i, unsigned rows, unsigned heads) {
  i = i < rows ? i : 0;
  const unsigned t = i / heads;
  return {(int)t, (int)(i - t * heads)};
}

// us, 16384 rows of 32 + 8 heads of 128 in bf16, half of each rotated, when these choices were made, side by side on one machine: 83 (one row at a time 86, four 88, with results that stay in the caches 107,
// without the next rows' loads ahead 110).
template <typename T, int V, int PIECES, int LANES, bool STREAM>
__global__ __launch_bounds__(256) void head_rotary_kernel(const RotaryArgs a) {
  touch_args(a);
  constexpr int GROUPS = 256 / LANES, U = V > 1 ? 2 : 1;
  __shared__ Turns turns;
  const int64_t t0 = (a.block0 + blockIdx.x) * a.tokens;
  const int tokens = (int)(a.n - t0 < a.tokens ? a.n - t0 : a.tokens), group = threadIdx.x / LANES;
  const Columns<V, LANES> col = {(int)threadIdx.x % LANES * V};
  const float mean = 1.f / (float)a.dim;
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const int heads = k ? a.heads - a.q_heads : a.q_heads, rows = tokens * heads;
    const T *x = (const T *)a.x[k].p + t0 * a.x[k].stride;
    T *z = (T *)a.z[k].p + t0 * a.z[k].stride;
    Two<T, V> v[U][PIECES], next[U][PIECES];
    auto load = [&](int first, Two<T, V> (&to)[U][PIECES]) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const RowAt at = row_at(first + i * GROUPS + group, rows, heads);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) to[i][p] = load_pair<T, V>(a, x + at.token * a.x[k].stride + at.head * a.x[k].head_stride, col.at(p, 0));
      }
    };
    if (rows > 0) load(0, v);                          // (on their way while the angles are computed)
    if (k == 0) make_turns(a, turns, t0, tokens, 1.f);
    if (rows == 0) continue;
    const bool norm = a.weight[k] != nullptr;
    float weight[PIECES][V], other[PIECES][V];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int e = col.at(p, j) < a.dim ? col.at(p, j) : 0;
        weight[p][j] = norm ? a.weight[k][e] : 1.f;
        other[p][j] = norm ? a.weight[k][pair_of(a, e).other] : 1.f;
      }
    for (int first = 0; first < rows; first += U * GROUPS) {
      if (first + U * GROUPS < rows) load(first + U * GROUPS, next);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int n = first + i * GROUPS + group;
        const RowAt at = row_at(n, rows, heads);
        float sum = 0.f, r = 1.f;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) alone<T, V>(v[i][p], col.at(p, 0) < a.rotary);
        if (norm) {
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) t = fmaf(own_of(v[i][p], j), own_of(v[i][p], j), t);
            sum += col.at(p, 0) < a.dim ? t : 0.f;
          }
          r = rsqrtf(group_sum<LANES>(sum) * mean + a.eps);
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          float c[V], s[V], y[V];
          turn_of<V>(a, turns, at.token, col.at(p, 0), c, s);
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = r * fmaf(own_of(v[i][p], j) * weight[p][j], c[j], other_of(a, v[i][p], j) * other[p][j] * s[j]);
          store_columns<T, V, STREAM>(z + at.token * a.z[k].stride + at.head * a.z[k].head_stride, col.at(p, 0), n < rows && col.at(p, 0) < a.dim, y);
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) v[i][p] = next[i][p];
      }
    }
  }
}

// Tokens in turn by a fixed number of blocks, each of which leaves one sum of the weights' gradients. The same rows, side by side: 121 us (two rows at a time 158: 149 registers for 110).
template <typename T, int V, int PIECES, int LANES, bool STREAM>
__global__ __launch_bounds__(256) void head_rotary_backward_kernel(const RotaryArgs a) {
  touch_args(a);
  constexpr int GROUPS = 256 / LANES, IN_WAVE = 64 / LANES, U = 1;
  __shared__ Turns turns;
  __shared__ float sums[4][2][LANES * PIECES * V];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = threadIdx.x / LANES;
  const Columns<V, LANES> col = {(int)threadIdx.x % LANES * V};
  float dw[2][PIECES][V];
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[0][p][j] = dw[1][p][j] = 0.f;
  const float mean = 1.f / (float)a.dim;
  for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.n; t0 += (int64_t)gridDim.x * a.tokens) {
    const int tokens = (int)(a.n - t0 < a.tokens ? a.n - t0 : a.tokens);
    auto tensor = [&](auto which) {
      constexpr int k = decltype(which)::value;
      const int heads = k ? a.heads - a.q_heads : a.q_heads, rows = tokens * heads;
      const bool norm = a.weight[k] != nullptr;
      const T *x = (const T *)a.x[k].p + t0 * a.x[k].stride, *dz = (const T *)a.dz[k].p + t0 * a.dz[k].stride;
      T *dx = (T *)a.dx[k].p + t0 * a.dx[k].stride;
      Two<T, V> v[U][PIECES], next[U][PIECES];
      typename Raw<T, V>::type xs[U][PIECES], next_xs[U][PIECES];
      auto load = [&](int first, Two<T, V> (&to)[U][PIECES], typename Raw<T, V>::type (&to_xs)[U][PIECES]) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const RowAt at = row_at(first + i * GROUPS + group, rows, heads);
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            to[i][p] = load_pair<T, V>(a, dz + at.token * a.dz[k].stride + at.head * a.dz[k].head_stride, col.at(p, 0));
            to_xs[i][p] = norm ? load_columns<T, V>(x + at.token * a.x[k].stride + at.head * a.x[k].head_stride, col.at(p, 0), a.dim) : to[i][p].x;
          }
        }
      };
      if (rows > 0) load(0, v, xs);
      if (k == 0) {
        __syncthreads();                               // (the tokens before are done)
        make_turns(a, turns, t0, tokens, -1.f);
      }
      if (rows == 0) return;
      float weight[PIECES][V];
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) weight[p][j] = norm ? a.weight[k][col.at(p, j) < a.dim ? col.at(p, j) : 0] : 1.f;
      for (int first = 0; first < rows; first += U * GROUPS) {
        if (first + U * GROUPS < rows) load(first + U * GROUPS, next, next_xs);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int n = first + i * GROUPS + group;
          const RowAt at = row_at(n, rows, heads);
          float g[PIECES][V], sum = 0.f, dot = 0.f, r = 1.f, along = 0.f;
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            alone<T, V>(v[i][p], col.at(p, 0) < a.rotary);
            float c[V], s[V], t = 0.f, d = 0.f;
            turn_of<V>(a, turns, at.token, col.at(p, 0), c, s);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float y = column_of<T, V>(xs[i][p], j);
              g[p][j] = fmaf(own_of(v[i][p], j), c[j], other_of(a, v[i][p], j) * s[j]);
              t = fmaf(y, y, t);
              d = fmaf(g[p][j] * weight[p][j], y, d);
            }
            sum += col.at(p, 0) < a.dim ? t : 0.f;
            dot += col.at(p, 0) < a.dim ? d : 0.f;
          }
          if (norm) {
            r = rsqrtf(group_sum<LANES>(sum) * mean + a.eps);
            along = group_sum<LANES>(dot) * mean * r * r * r;
            const float counts = n < rows ? r : 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
#pragma unroll
              for (int j = 0; j < V; ++j) {
                const float y = column_of<T, V>(xs[i][p], j);
                dw[k][p][j] = fmaf(g[p][j] * y, counts, dw[k][p][j]);
                g[p][j] = fmaf(-y, along, r * g[p][j] * weight[p][j]);
              }
          }
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            store_columns<T, V, STREAM>(dx + at.token * a.dx[k].stride + at.head * a.dx[k].head_stride, col.at(p, 0), n < rows && col.at(p, 0) < a.dim, g[p]);
            v[i][p] = next[i][p];
            xs[i][p] = next_xs[i][p];
          }
        }
      }
    };
    tensor(std::integral_constant<int, 0>());
    tensor(std::integral_constant<int, 1>());
  }
  if (!a.partial) return;
  // of the wave's groups, then of the block's waves, in order
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float t = dw[k][p][j], u = t;
#pragma unroll
        for (int m = 1; m < IN_WAVE; ++m) u += __shfl(t, (lane + m * LANES) & 63);
        if (lane < LANES) sums[wave][k][col.at(p, j)] = u;
      }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.dim; i += 256) {
    const int k = i / a.dim, e = i % a.dim;
    a.partial[((int64_t)blockIdx.x * 2 + k) * a.dim + e] = sums[0][k][e] + sums[1][k][e] + sums[2][k][e] + sums[3][k][e];
  }
}

// A block of 1024 for 16 columns: 64 sums of every 64th block's, then one of these. (With 16 sums of 2048 blocks' 40 us, a chain of loads.)
__global__ __launch_bounds__(1024) void head_rotary_weights_kernel(const RotaryArgs a) {
  __shared__ float sums[64][17];
  const int i = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
  float t = 0.f;
  if (i < 2 * a.dim)
#pragma unroll 8
    for (int b = part; b < a.partials; b += 64) t += a.partial[(int64_t)b * 2 * a.dim + i];
  sums[part][threadIdx.x & 15] = t;
  __syncthreads();
  if (part || i >= 2 * a.dim) return;
#pragma unroll
  for (int p = 1; p < 64; ++p) t += sums[p][threadIdx.x];
  float *to = a.dweight[i / a.dim];
  if (to) to[i % a.dim] += t;
}

bool lies_apart(const xrl_heads &x, int64_t n, int heads, int dim) {
  const int64_t s = n > 1 ? x.stride : INT64_MAX, h = heads > 1 ? x.head_stride : INT64_MAX;
  const int64_t inner = std::min(s, h), count = s < h ? n : heads, outer = std::max(s, h);
  if (inner != INT64_MAX && inner < dim) return false;
  return outer == INT64_MAX || outer - dim >= (count - 1) * inner;
}

int check_rows(const xrl_heads *x, int64_t n, int heads, int dim, int es, bool written, const char *name, const char *who, Heads &o, bool &aligned) {
  o = {nullptr, 0, 0};
  if (heads == 0 || n == 0) return XRL_OK;
  if (!x || !x->d_data) return fail(XRL_ERR_NULL, "%s: %s is NULL", who, name);
  if ((uintptr_t)x->d_data % es) return fail(XRL_ERR_SHAPE, "%s: %s: a pointer that is no multiple of its elements' size", who, name);
  if (x->stride < 0 || x->head_stride < 0 || (written && !lies_apart(*x, n, heads, dim)))
    return fail(XRL_ERR_SHAPE, "%s: %s: strides %lld and %lld", who, name, (long long)x->stride, (long long)x->head_stride);
  o = {x->d_data, n > 1 ? x->stride : 0, heads > 1 ? x->head_stride : 0};
  aligned = aligned && (uintptr_t)x->d_data % 16 == 0 && o.stride * es % 16 == 0 && o.head_stride * es % 16 == 0;
  return XRL_OK;
}

int check_rotary(const xrl_ctx *c, const xrl_rotary_desc *d, const char *who, RotaryArgs &a, bool &aligned) {
  if (!c || !d) return fail(XRL_ERR_NULL, "%s: ctx or desc is NULL", who);
  if (!op_type_ok(d->type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, d->type);
  if (d->n < 0 || d->q_heads < 0 || d->kv_heads < 0 || d->dim < 1 || d->rotary < 0 || d->rotary > d->dim || d->rotary % 2)
    return fail(XRL_ERR_SHAPE, "%s: %lld rows, %d and %d heads of %d, %d columns rotated", who, (long long)d->n, d->q_heads, d->kv_heads, d->dim, d->rotary);
  if (d->dim > 256 || d->q_heads > 65536 || d->kv_heads > 65536 || d->n > INT32_MAX)
    return fail(XRL_ERR_UNSUPPORTED, "%s: %lld rows, %d and %d heads of %d (at most 256)", who, (long long)d->n, d->q_heads, d->kv_heads, d->dim);
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return fail(XRL_ERR_VALUE, "%s: eps %g", who, (double)d->eps);
  if (d->rotary > 0 && d->n > 0 && (!d->d_positions || !d->d_freqs)) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d->d_positions | (uintptr_t)d->d_freqs | (uintptr_t)d->d_q_weight | (uintptr_t)d->d_k_weight) % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a = RotaryArgs{};
  a.n = d->n; a.q_heads = d->q_heads; a.heads = d->q_heads + d->kv_heads; a.dim = d->dim; a.rotary = d->rotary; a.interleaved = d->interleaved != 0;
  a.eps = d->eps;
  a.positions = d->d_positions; a.freqs = d->d_freqs;
  a.weight[0] = d->d_q_weight; a.weight[1] = d->d_k_weight;
  const int v = d->type == XRL_PREC_BF16 ? 8 : 4;
  aligned = d->dim % v == 0 && (d->interleaved ? d->rotary : d->rotary / 2) % v == 0;
  return XRL_OK;
}

// Rows of a block: as many as leave four blocks for every compute unit, at most eight.
int rows_of_block(const xrl_ctx *c, int64_t n) { return (int)std::min<int64_t>(std::max<int64_t>(1, n / (4 * op_compute_units(c))), kTokens); }

template <typename T, int V, int PIECES, int LANES, bool STREAM>
void launch(const xrl_ctx *c, RotaryArgs &a, bool backward) {
  if (backward) {
    head_rotary_backward_kernel<T, V, PIECES, LANES, STREAM><<<dim3((unsigned)a.partials), dim3(256), 0, op_stream(c)>>>(a);
    return;
  }
  const int64_t blocks = (a.n + a.tokens - 1) / a.tokens;
  for (a.block0 = 0; a.block0 < blocks; a.block0 += kMaxBlocks)
    head_rotary_kernel<T, V, PIECES, LANES, STREAM><<<dim3((unsigned)std::min(blocks - a.block0, kMaxBlocks)), dim3(256), 0, op_stream(c)>>>(a);
}
template <typename T, int V, int LANES>
void launch_whole(const xrl_ctx *c, RotaryArgs &a, bool backward) {
  streams(a.n * a.heads * a.dim * (int)sizeof(T)) ? launch<T, V, 1, LANES, true>(c, a, backward) : launch<T, V, 1, LANES, false>(c, a, backward);
}

// A row in as many lanes as have 16 bytes of it each, at least eight; rows at odd places, or pairs that such pieces would cut, element by element.
int lanes_of(const RotaryArgs &a, int v, bool aligned) {
  if (!aligned) return 64;
  int lanes = 8;
  while (lanes * v < a.dim) lanes *= 2;
  return lanes;
}
template <typename T>
void launch_lanes(const xrl_ctx *c, RotaryArgs &a, bool aligned, int lanes, bool backward) {
  constexpr int V = 16 / (int)sizeof(T);
  if (!aligned) launch<T, 1, 4, 64, false>(c, a, backward);
  else if (lanes == 8) launch_whole<T, V, 8>(c, a, backward);
  else if (lanes == 16) launch_whole<T, V, 16>(c, a, backward);
  else if (lanes == 32 || V * 32 >= 256) launch_whole<T, V, 32>(c, a, backward);
  else if constexpr (V * 32 < 256) launch_whole<T, V, 64>(c, a, backward);
}

}  // namespace

extern "C" {

int xrl_rotary_freqs(int32_t rotary, const xrl_rotary_scaling *s, float *freqs) {
  const char *who = "xrl_rotary_freqs";
  if (!s || (rotary > 0 && !freqs)) return fail(XRL_ERR_NULL, "%s: NULL pointer", who);
  if (rotary < 0 || rotary % 2) return fail(XRL_ERR_SHAPE, "%s: %d columns", who, rotary);
  if (!(s->base > 0.0) || !std::isfinite(s->base) || !(s->factor >= 1.0) || !std::isfinite(s->factor) || !(s->length >= 0.0) || !std::isfinite(s->length) ||
      (s->length > 0.0 && !(s->fast > s->slow && s->slow >= 0.0 && std::isfinite(s->fast))))
    return fail(XRL_ERR_VALUE, "%s: base %g, factor %g, length %g, turns %g to %g", who, s->base, s->factor, s->length, s->slow, s->fast);
  for (int j = 0; j < rotary / 2; ++j) {
    const double f = std::pow(s->base, -2.0 * j / rotary);
    double keep = 0.0;                                 // share of the frequency that stays as it is
    if (s->length > 0.0) {
      const double turns = s->length * f / 6.283185307179586476925;
      keep = std::min(1.0, std::max(0.0, (turns - s->slow) / (s->fast - s->slow)));
    }
    freqs[j] = (float)(f * (keep + (1.0 - keep) / s->factor));
  }
  return XRL_OK;
}

int xrl_head_rotary(xrl_ctx *c, const xrl_rotary_desc *d, const xrl_heads *q, const xrl_heads *k, const xrl_heads *q_out, const xrl_heads *k_out) {
  const char *who = "xrl_head_rotary";
  RotaryArgs a;
  bool aligned;
  if (int rc = check_rotary(c, d, who, a, aligned)) return rc;
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4, v = 16 / es;
  if (int rc = check_rows(q, a.n, d->q_heads, a.dim, es, false, "q", who, a.x[0], aligned)) return rc;
  if (int rc = check_rows(k, a.n, d->kv_heads, a.dim, es, false, "k", who, a.x[1], aligned)) return rc;
  if (int rc = check_rows(q_out, a.n, d->q_heads, a.dim, es, true, "q_out", who, a.z[0], aligned)) return rc;
  if (int rc = check_rows(k_out, a.n, d->kv_heads, a.dim, es, true, "k_out", who, a.z[1], aligned)) return rc;
  if (a.n == 0 || a.heads == 0) return XRL_OK;
  const int lanes = lanes_of(a, v, aligned);
  a.tokens = rows_of_block(c, a.n);
  es == 2 ? launch_lanes<bf16_t>(c, a, aligned, lanes, false) : launch_lanes<float>(c, a, aligned, lanes, false);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

int xrl_head_rotary_backward(xrl_ctx *c, const xrl_rotary_desc *d, const xrl_heads *q, const xrl_heads *k, const xrl_heads *dq_out, const xrl_heads *dk_out,
                             const xrl_heads *dq, const xrl_heads *dk, float *d_dq_weight, float *d_dk_weight) {
  const char *who = "xrl_head_rotary_backward";
  RotaryArgs a;
  bool aligned;
  if (int rc = check_rotary(c, d, who, a, aligned)) return rc;
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4, v = 16 / es;
  if (int rc = check_rows(q, a.n, d->d_q_weight ? d->q_heads : 0, a.dim, es, false, "q", who, a.x[0], aligned)) return rc;
  if (int rc = check_rows(k, a.n, d->d_k_weight ? d->kv_heads : 0, a.dim, es, false, "k", who, a.x[1], aligned)) return rc;
  if (int rc = check_rows(dq_out, a.n, d->q_heads, a.dim, es, false, "dq_out", who, a.dz[0], aligned)) return rc;
  if (int rc = check_rows(dk_out, a.n, d->kv_heads, a.dim, es, false, "dk_out", who, a.dz[1], aligned)) return rc;
  if (int rc = check_rows(dq, a.n, d->q_heads, a.dim, es, true, "dq", who, a.dx[0], aligned)) return rc;
  if (int rc = check_rows(dk, a.n, d->kv_heads, a.dim, es, true, "dk", who, a.dx[1], aligned)) return rc;
  if (((uintptr_t)d_dq_weight | (uintptr_t)d_dk_weight) % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  if (a.n == 0 || a.heads == 0) return XRL_OK;
  a.dweight[0] = d->d_q_weight ? d_dq_weight : nullptr;
  a.dweight[1] = d->d_k_weight ? d_dk_weight : nullptr;
  if (a.dweight[0] && a.dweight[1] && a.dweight[0] != a.dweight[1] && a.dweight[0] < a.dweight[1] + a.dim && a.dweight[1] < a.dweight[0] + a.dim)
    return fail(XRL_ERR_SHAPE, "%s: the weights' gradients lie in a part of each other", who);
  const int lanes = lanes_of(a, v, aligned);
  a.tokens = rows_of_block(c, a.n);
  a.partials = (int)std::min<int64_t>((a.n + a.tokens - 1) / a.tokens, 4 * (int64_t)op_compute_units(c));
  if (a.dweight[0] || a.dweight[1]) {
    char *ws = nullptr;
    if (int rc = op_workspace(c, (size_t)a.partials * 2 * a.dim * 4, &ws, who)) return rc;
    a.partial = (float *)ws;
  }
  es == 2 ? launch_lanes<bf16_t>(c, a, aligned, lanes, true) : launch_lanes<float>(c, a, aligned, lanes, true);
  const bool shared = a.dweight[0] && a.dweight[0] == a.dweight[1];   // one vector for both: in turn, as each entry is read and written
  for (int k = 0; a.partial && k <= (shared ? 1 : 0); ++k) {
    RotaryArgs w = a;
    if (shared) w.dweight[1 - k] = nullptr;
    head_rotary_weights_kernel<<<dim3((unsigned)((2 * a.dim + 15) / 16)), dim3(1024), 0, op_stream(c)>>>(w);
  }
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

}  // extern "C"
