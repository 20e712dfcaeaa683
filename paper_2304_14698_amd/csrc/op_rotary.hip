// The norm of queries and keys per head and the rotation of their columns in pairs by angles position * frequency, in one pass, and its gradients.
//
// Per row x of dim columns: y = x r w, r = (mean x^2 + eps)^-1/2 (without a weight w: y = x); of each pair, z1 = y1 cos a - y2 sin a, z2 = y1 sin a + y2 cos a. With g the
// gradient to z rotated back: dw += g x r, dx = r (g w - x r^2 mean(g w x)).
//
// Bound by memory. A row lies in the lanes of one wave, 16 bytes a lane, so its mean is a few lane moves; the other half of a pair comes from the lane's own piece, or from the
// cache line that a neighbour has just read. A wave keeps its token while it goes over heads: cosines and sines, of an angle in 64 bits, are computed once a token.
#include "op_common.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

using namespace xrl;

namespace {

struct Heads {
  const void *p;
  int64_t stride, head_stride;
};

struct RotaryArgs {
  int64_t n, jobs, job0;        // rows; jobs of a token and some of its heads, and the first one of this launch
  int q_heads, heads, dim, rotary, interleaved;   // heads: of q and k
  int per_job, jobs_a_token;    // heads of one job
  float eps;
  const int32_t *positions;
  const float *freqs, *weight[2];
  Heads x[2], z[2], dz[2], dx[2];   // q, k
  float *partial;               // [jobs' blocks][2][dim]: sums of the weights' gradients
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

// Cosines and sines of the lane's columns at a position: of column e, z_e = y_e c + y_other s. Behind the pairs 1 and 0.
template <int V, int PIECES, int LANES>
__device__ __forceinline__ void turns_of(const RotaryArgs &a, const Columns<V, LANES> &col, int position, float back, float (&c)[PIECES][V], float (&s)[PIECES][V]) {
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      c[p][j] = 1.f;
      s[p][j] = 0.f;
    }
    if (col.at(p, 0) >= a.rotary) continue;
    if (V > 1 && a.interleaved) {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        float x, y;
        angle_of(position, a.freqs[col.at(p, j) >> 1], x, y);
        c[p][j] = c[p][V > 1 ? j + 1 : 0] = x;
        s[p][j] = -back * y;
        s[p][V > 1 ? j + 1 : 0] = back * y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const Pair r = pair_of(a, col.at(p, j));
        float y;
        angle_of(position, a.freqs[r.index], c[p][j], y);
        s[p][j] = back * r.sign * y;
      }
    }
  }
}

// A job's token, first head and number of heads.
struct Job {
  int64_t t;
  int h0, count;
};
__device__ __forceinline__ Job job_of(const RotaryArgs &a, int64_t job) {
  const int64_t t = job / a.jobs_a_token;
  const int h0 = (int)(job % a.jobs_a_token) * a.per_job;
  return {t, h0, a.heads - h0 < a.per_job ? a.heads - h0 : a.per_job};
}

// Rows of a wave at once: their loads are requested together.
template <int V>
constexpr int kRowsAtOnce = V > 1 ? 4 : 1;

template <typename T, int V, int PIECES, int LANES, bool STREAM>
__global__ __launch_bounds__(256) void head_rotary_kernel(const RotaryArgs a) {
  touch_args(a);
  constexpr int GROUPS = 64 / LANES, U = kRowsAtOnce<V>;
  const int64_t job = a.job0 + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= a.jobs) return;
  const Job w = job_of(a, job);
  const int lane = threadIdx.x & 63, group = lane / LANES;
  const Columns<V, LANES> col = {lane % LANES * V};
  float c[PIECES][V], s[PIECES][V];
  turns_of<V, PIECES, LANES>(a, col, a.rotary ? a.positions[w.t] : 0, 1.f, c, s);
  const float mean = 1.f / (float)a.dim;
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    // the job's heads of q, then of k
    const int lo = k ? max(w.h0, a.q_heads) - a.q_heads : w.h0, hi = k ? w.h0 + w.count - a.q_heads : min(w.h0 + w.count, a.q_heads);
    if (lo >= hi) continue;
    const bool norm = a.weight[k] != nullptr;
    float wc[PIECES][V], ws[PIECES][V];                // z_e = r (x_e w_e c + x_other w_other s)
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int e = col.at(p, j) < a.dim ? col.at(p, j) : 0;
        wc[p][j] = norm ? a.weight[k][e] * c[p][j] : c[p][j];
        ws[p][j] = norm ? a.weight[k][pair_of(a, e).other] * s[p][j] : s[p][j];
      }
    const T *x = (const T *)a.x[k].p + w.t * a.x[k].stride;
    T *z = (T *)a.z[k].p + w.t * a.z[k].stride;
    for (int h0 = lo; h0 < hi; h0 += U * GROUPS) {
      Two<T, V> v[U][PIECES];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = h0 + i * GROUPS + group;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) v[i][p] = load_pair<T, V>(a, x + (h < hi ? h : lo) * a.x[k].head_stride, col.at(p, 0));
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = h0 + i * GROUPS + group;
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
          float y[V];
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = r * fmaf(own_of(v[i][p], j), wc[p][j], other_of(a, v[i][p], j) * ws[p][j]);
          store_columns<T, V, STREAM>(z + (h < hi ? h : lo) * a.z[k].head_stride, col.at(p, 0), h < hi && col.at(p, 0) < a.dim, y);
        }
      }
    }
  }
}

// Jobs in turn by a fixed number of blocks, each of which leaves one sum of the weights' gradients.
template <typename T, int V, int PIECES, int LANES, bool STREAM>
__global__ __launch_bounds__(256) void head_rotary_backward_kernel(const RotaryArgs a) {
  touch_args(a);
  constexpr int GROUPS = 64 / LANES, U = V > 1 ? 2 : 1;
  __shared__ float sums[4][2][LANES * PIECES * V];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane / LANES;
  const Columns<V, LANES> col = {lane % LANES * V};
  float dw[2][PIECES][V];
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[0][p][j] = dw[1][p][j] = 0.f;
  const float mean = 1.f / (float)a.dim;
  for (int64_t job = (int64_t)blockIdx.x * 4 + wave; job < a.jobs; job += (int64_t)gridDim.x * 4) {
    const Job w = job_of(a, job);
    float c[PIECES][V], s[PIECES][V];
    turns_of<V, PIECES, LANES>(a, col, a.rotary ? a.positions[w.t] : 0, -1.f, c, s);
    auto heads = [&](auto tensor) {
      constexpr int k = decltype(tensor)::value;
      const int lo = k ? max(w.h0, a.q_heads) - a.q_heads : w.h0, hi = k ? w.h0 + w.count - a.q_heads : min(w.h0 + w.count, a.q_heads);
      if (lo >= hi) return;
      const bool norm = a.weight[k] != nullptr;
      float weight[PIECES][V];
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) weight[p][j] = norm && col.at(p, j) < a.dim ? a.weight[k][col.at(p, j)] : 1.f;
      const T *x = (const T *)a.x[k].p + w.t * a.x[k].stride, *dz = (const T *)a.dz[k].p + w.t * a.dz[k].stride;
      T *dx = (T *)a.dx[k].p + w.t * a.dx[k].stride;
      for (int h0 = lo; h0 < hi; h0 += U * GROUPS) {
        Two<T, V> v[U][PIECES];
        typename Raw<T, V>::type xs[U][PIECES];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int h = h0 + i * GROUPS + group, hh = h < hi ? h : lo;
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            const int e = col.at(p, 0);
            v[i][p] = load_pair<T, V>(a, dz + hh * a.dz[k].head_stride, e);
            xs[i][p] = norm ? load_columns<T, V>(x + hh * a.x[k].head_stride, e, a.dim) : v[i][p].x;
          }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int h = h0 + i * GROUPS + group;
          float g[PIECES][V], sum = 0.f, dot = 0.f, r = 1.f, along = 0.f;
#pragma unroll
          for (int p = 0; p < PIECES; ++p) {
            alone<T, V>(v[i][p], col.at(p, 0) < a.rotary);
            float t = 0.f, d = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float y = column_of<T, V>(xs[i][p], j);
              g[p][j] = fmaf(own_of(v[i][p], j), c[p][j], other_of(a, v[i][p], j) * s[p][j]);
              t = fmaf(y, y, t);
              d = fmaf(g[p][j] * weight[p][j], y, d);
            }
            sum += col.at(p, 0) < a.dim ? t : 0.f;
            dot += col.at(p, 0) < a.dim ? d : 0.f;
          }
          if (norm) {
            r = rsqrtf(group_sum<LANES>(sum) * mean + a.eps);
            along = group_sum<LANES>(dot) * mean * r * r * r;
            const float counts = h < hi ? r : 0.f;
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
          for (int p = 0; p < PIECES; ++p) store_columns<T, V, STREAM>(dx + (h < hi ? h : lo) * a.dx[k].head_stride, col.at(p, 0), h < hi && col.at(p, 0) < a.dim, g[p]);
        }
      }
    };
    heads(std::integral_constant<int, 0>());
    heads(std::integral_constant<int, 1>());
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
        for (int m = 1; m < GROUPS; ++m) u += __shfl(t, (lane + m * LANES) & 63);
        if (group == 0) sums[wave][k][col.at(p, j)] = u;
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

// Heads of a job: all of a token where there are tokens for eight waves a SIMD, else so many that the chip is full, or one round of a wave's.
void share_out(const xrl_ctx *c, RotaryArgs &a, int groups) {
  const int64_t waves = 32 * (int64_t)op_compute_units(c);
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>((waves + a.n - 1) / a.n, (a.heads + groups - 1) / groups));
  a.per_job = (int)((a.heads + parts - 1) / parts + groups - 1) / groups * groups;
  a.jobs_a_token = (a.heads + a.per_job - 1) / a.per_job;
  a.jobs = a.n * a.jobs_a_token;
}

template <typename T, int V, int PIECES, int LANES, bool STREAM>
void launch(const xrl_ctx *c, RotaryArgs &a, bool backward) {
  if (backward) {
    head_rotary_backward_kernel<T, V, PIECES, LANES, STREAM><<<dim3((unsigned)a.partials), dim3(256), 0, op_stream(c)>>>(a);
    return;
  }
  for (a.job0 = 0; a.job0 < a.jobs; a.job0 += 4 * kMaxBlocks)
    head_rotary_kernel<T, V, PIECES, LANES, STREAM><<<dim3((unsigned)((std::min(a.jobs - a.job0, 4 * kMaxBlocks) + 3) / 4)), dim3(256), 0, op_stream(c)>>>(a);
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
  share_out(c, a, 64 / lanes);
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
  const int lanes = lanes_of(a, v, aligned);
  share_out(c, a, 64 / lanes);
  a.partials = (int)std::min<int64_t>((a.jobs + 3) / 4, 4 * (int64_t)op_compute_units(c));
  if (a.dweight[0] || a.dweight[1]) {
    char *ws = nullptr;
    if (int rc = op_workspace(c, (size_t)a.partials * 2 * a.dim * 4, &ws, who)) return rc;
    a.partial = (float *)ws;
  }
  es == 2 ? launch_lanes<bf16_t>(c, a, aligned, lanes, true) : launch_lanes<float>(c, a, aligned, lanes, true);
  if (a.partial) head_rotary_weights_kernel<<<dim3((unsigned)((2 * a.dim + 15) / 16)), dim3(1024), 0, op_stream(c)>>>(a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

}  // extern "C"
