// Momentum with orthogonalised updates: Newton-Schulz steps on every listed matrix of a flat weight vector.
//
// Per matrix, as m x n with m <= n (transposed if it has more rows than columns), X = U / |U|_F and `steps` times
//   A = X X^T,  B = a I + b A + c A A,  X = B X,
// the quintic a X + (b A + c A A) X. All matrices share the launches: 2 + 3 steps in all.
//
// Numbers. The products run on the fp16 matrix cores, which are sixteen times as fast as the fp32 ones, on entries x 2^12 split in two halves
// of 11 bits, hi = fp16(x 2^12) and lo = fp16(x 2^12 - hi), with fp32 sums: hi hi + hi lo + lo hi leaves out 2^-22 of an entry. Entries cannot overflow:
// singular values of X lie in [0, 1.21] in every step (the quintic's largest value on [0, 1.21] is 1.21), so entries of X, A and B are at most 1.21, 1.47
// and 3.45, and 3.45 2^12 < 65504. An entry from 2^-26 down loses bits of lo to the smallest fp16, 2^-36 of the matrix's scale.
//
// Layout. Operands lie in fragment order: 32 rows by 16 of the summed dimension, first hi, then lo, each 64 lanes by 16 bytes, as one matrix
// instruction takes them. Both X (rows m) and X^T (rows n) are kept.
#include "op_common.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

using namespace xrl;

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;
constexpr int kGroup = 32;             // matrices of one launch: their list is a kernel argument
constexpr int kTile = 64;              // a block's output, four waves of 32 x 32
constexpr int kMaxSums = 1024;         // partial sums of squares of a matrix

struct Mat {
  int64_t offset, ws;                  // in the flat vectors; in the workspace (halves)
  int m, n;                            // m <= n
  bool t;                              // the matrix in the vector is n x m
  int chunk;                           // entries of one partial sum of squares
};
struct MuonArgs {
  int count;
  int first[kGroup + 1];               // first block of each matrix in this launch
  Mat mat[kGroup];
  int first_sum[kGroup + 1];           // first partial sum of each
  float *w, *mom;
  const float *g;
  _Float16 *ws;
  double *sums;
  float mu, decay, step;               // step: lr rms (times sqrt(max(rows, cols)))
  bool nesterov;
  int flip;                            // which of the two X^T holds the current one
};

__device__ __forceinline__ int padded(int x) { return (x + kTile - 1) / kTile * kTile; }
// halves of: X, and each X^T; A, and B
__host__ __device__ inline int64_t x_halves(int m, int n) {
  return (int64_t)((m + kTile - 1) / kTile * kTile) * ((n + kTile - 1) / kTile * kTile) * 2;
}
struct Buffers {
  _Float16 *x, *xt[2], *a, *b;
};
__device__ __forceinline__ Buffers buffers(const MuonArgs &p, const Mat &q) {
  const int64_t nx = x_halves(q.m, q.n), na = x_halves(q.m, q.m);
  _Float16 *w = p.ws + q.ws;
  return {w, {w + nx, w + 2 * nx}, w + 3 * nx, w + 3 * nx + na};
}
__device__ __forceinline__ int matrix_of(const MuonArgs &p, int block) {
  int k = 0;
  while (k + 1 < p.count && p.first[k + 1] <= block) ++k;
  return k;
}
__device__ __forceinline__ void split(float y, _Float16 &hi, _Float16 &lo) {
  hi = (_Float16)y;
  lo = (_Float16)(y - (float)hi);
}

// M = mu M + G, and of each chunk the sum of squares of U
__global__ __launch_bounds__(256) void muon_momentum_kernel(const MuonArgs p) {
  const int k = matrix_of(p, blockIdx.x), part = blockIdx.x - p.first[k];
  const Mat &q = p.mat[k];
  const int64_t size = (int64_t)q.m * q.n, i0 = (int64_t)part * q.chunk, i1 = i0 + q.chunk < size ? i0 + q.chunk : size;
  float *mom = p.mom + q.offset;
  const float *g = p.g + q.offset;
  double sum = 0.;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
    const float gi = g[i], mi = p.mu * mom[i] + gi;
    mom[i] = mi;
    const float u = p.nesterov ? gi + p.mu * mi : mi;
    sum += (double)u * (double)u;
  }
  for (int s = 32; s; s /= 2) sum += __shfl_xor(sum, s);
  __shared__ double part_sum[4];
  if ((threadIdx.x & 63) == 0) part_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.sums[p.first_sum[k] + part] = part_sum[0] + part_sum[1] + part_sum[2] + part_sum[3];
}

// X = U / (|U| + 1e-7) in both orders, a 64 x 64 tile a block
__global__ __launch_bounds__(256) void muon_begin_kernel(const MuonArgs p) {
  const int k = matrix_of(p, blockIdx.x), tile = blockIdx.x - p.first[k], t = threadIdx.x, lane = t & 63;
  const Mat &q = p.mat[k];
  const int mp = padded(q.m), np = padded(q.n), ti = tile / (np / kTile), tj = tile % (np / kTile);
  const Buffers buf = buffers(p, q);
  double sum = 0.;
  const int n_sums = p.first_sum[k + 1] - p.first_sum[k];
  for (int i = lane; i < n_sums; i += 64) sum += p.sums[p.first_sum[k] + i];
  for (int s = 32; s; s /= 2) sum += __shfl_xor(sum, s);
  const float inv = (float)(1. / (sqrt(sum) + 1e-7));
  __shared__ float x[kTile][kTile + 1];
  const int ld = q.t ? q.m : q.n;
  for (int s = t; s < kTile * kTile; s += 256) {
    const int a = s / kTile, b = s % kTile, i = ti * kTile + (q.t ? b : a), j = tj * kTile + (q.t ? a : b);
    float u = 0.f;
    if (i < q.m && j < q.n) {
      const int64_t at = q.offset + (q.t ? (int64_t)j * ld + i : (int64_t)i * ld + j);
      const float mi = p.mom[at];
      u = (p.nesterov ? p.g[at] + p.mu * mi : mi) * inv;
    }
    x[q.t ? b : a][q.t ? a : b] = u * kUp;
  }
  __syncthreads();
  for (int s = t; s < 512; s += 256) {
    const int rb = s >> 8, kb = (s >> 6) & 3, row = rb * 32 + (lane & 31), c = kb * 16 + (lane >> 5) * 8;
    f16x8 hi, lo;
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(x[row][c + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16 *o = buf.x + ((int64_t)(ti * 2 + rb) * (np / 16) + tj * 4 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(x[c + e][row], h, l);
      hi[e] = h; lo[e] = l;
    }
    o = buf.xt[0] + ((int64_t)(tj * 2 + rb) * (mp / 16) + ti * 4 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
}

enum { STEP_GRAM, STEP_POLY, STEP_APPLY, STEP_LAST };

// One product of a step. D[i][j] = sum over k of P[i][k] Q[j][k], both in fragment order along k.
template <int STEP>
__global__ __launch_bounds__(256) void muon_product_kernel(const MuonArgs p) {
  const int k = matrix_of(p, blockIdx.x), tile = blockIdx.x - p.first[k], lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Mat &q = p.mat[k];
  const int mp = padded(q.m), np = padded(q.n);
  const Buffers buf = buffers(p, q);
  int ti, tj, kbs;
  const _Float16 *P, *Q;
  if (STEP == STEP_GRAM || STEP == STEP_POLY) {           // symmetric: tiles with tj <= ti
    ti = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    while (ti * (ti + 1) / 2 > tile) --ti;
    tj = tile - ti * (ti + 1) / 2;
    P = Q = STEP == STEP_GRAM ? buf.x : buf.a;
    kbs = (STEP == STEP_GRAM ? np : mp) / 16;
  } else {
    ti = tile / (np / kTile);
    tj = tile % (np / kTile);
    P = buf.b;
    Q = buf.xt[p.flip];
    kbs = mp / 16;
  }
  const int ib = ti * 2 + (wave >> 1), jb = tj * 2 + (wave & 1);
  const _Float16 *pa = P + (int64_t)ib * kbs * 1024 + lane * 8, *qa = Q + (int64_t)jb * kbs * 1024 + lane * 8;
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int kb = 0; kb < kbs; ++kb) {
    const f16x8 ph = *(const f16x8 *)(pa + (int64_t)kb * 1024), pl = *(const f16x8 *)(pa + (int64_t)kb * 1024 + 512);
    const f16x8 qh = *(const f16x8 *)(qa + (int64_t)kb * 1024), ql = *(const f16x8 *)(qa + (int64_t)kb * 1024 + 512);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
  }
  // register r of a lane: D[i][j] with i = ib 32 + 8 (r / 4) + 4 (lane / 32) + r % 4, j = jb 32 + lane % 32
  const int g = lane >> 5, jl = lane & 31;
  if (STEP == STEP_LAST) {
    const int j = jb * 32 + jl;
    const float step = p.step * sqrtf((float)q.n) * (kDown * kDown);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i = ib * 32 + acc_row(r, g);
      if (i < q.m && j < q.n) {
        float *w = p.w + q.offset + (q.t ? (int64_t)j * q.m + i : (int64_t)i * q.n + j);
        *w = p.decay * *w - step * acc[r];
      }
    }
    return;
  }
  float v[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = acc[r] * kDown;
  if (STEP == STEP_POLY) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {                          // A[i][j] = A[j][i]: four i of one j lie side by side
      const _Float16 *at = buf.a + ((int64_t)jb * kbs + ib * 2 + (s >> 1)) * 1024 + (jl + 32 * (s & 1)) * 8 + 4 * g;
      const f16x4 h = *(const f16x4 *)at, l = *(const f16x4 *)(at + 512);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float diag = ib == jb && 8 * s + 4 * g + e == jl ? kNsA * kUp : 0.f;
        v[4 * s + e] = kNsC * v[4 * s + e] + (kNsB * ((float)h[e] + (float)l[e]) + diag);
      }
    }
  }
  // rows j, along i: a lane has four i side by side
  _Float16 *by_j = STEP == STEP_GRAM ? buf.a : STEP == STEP_POLY ? buf.b : buf.xt[p.flip ^ 1];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    f16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(v[4 * s + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16 *o = by_j + ((int64_t)jb * (mp / 16) + ib * 2 + (s >> 1)) * 1024 + (jl + 32 * (s & 1)) * 8 + 4 * g;
    *(f16x4 *)o = hi;
    *(f16x4 *)(o + 512) = lo;
  }
  // rows i, along j: turned round in LDS. (A block on the diagonal of a symmetric product has written both already.)
  if (STEP != STEP_APPLY && ti == tj) return;
  __shared__ float turn[4][32][33];
  float (*x)[33] = turn[wave];
#pragma unroll
  for (int r = 0; r < 16; ++r) x[acc_row(r, g)][jl] = v[r];
  __builtin_amdgcn_wave_barrier();
  __threadfence_block();
  _Float16 *by_i = STEP == STEP_GRAM ? buf.a : STEP == STEP_POLY ? buf.b : buf.x;
  const int kdim = STEP == STEP_APPLY ? np : mp;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(x[jl][kb * 16 + g * 8 + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16 *o = by_i + ((int64_t)ib * (kdim / 16) + jb * 2 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
}

int run_group(xrl_ctx *c, MuonArgs &p, int steps) {
  const hipStream_t stream = op_stream(c);
  // blocks of a launch whose matrix k has of(k) of them
  auto blocks = [&](auto of) {
    int64_t at = 0;
    for (int k = 0; k < p.count; ++k) {
      p.first[k] = (int)at;
      at += of(k);
    }
    p.first[p.count] = (int)at;
    return dim3((unsigned)at);
  };
  auto tiles = [](int x) { return (int64_t)(x + kTile - 1) / kTile; };
  const dim3 all = dim3(256);
  const dim3 sums = blocks([&](int k) { return (int64_t)p.first_sum[k + 1] - p.first_sum[k]; });
  muon_momentum_kernel<<<sums, all, 0, stream>>>(p);
  const dim3 whole = blocks([&](int k) { return tiles(p.mat[k].m) * tiles(p.mat[k].n); });
  muon_begin_kernel<<<whole, all, 0, stream>>>(p);
  for (int s = 0; s < steps; ++s) {
    const dim3 half = blocks([&](int k) { return tiles(p.mat[k].m) * (tiles(p.mat[k].m) + 1) / 2; });
    muon_product_kernel<STEP_GRAM><<<half, all, 0, stream>>>(p);
    muon_product_kernel<STEP_POLY><<<half, all, 0, stream>>>(p);
    blocks([&](int k) { return tiles(p.mat[k].m) * tiles(p.mat[k].n); });
    if (s + 1 < steps) muon_product_kernel<STEP_APPLY><<<whole, all, 0, stream>>>(p);
    else muon_product_kernel<STEP_LAST><<<whole, all, 0, stream>>>(p);
    p.flip ^= 1;
  }
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

}  // namespace

extern "C" {

int xrl_muon_step(xrl_ctx *c, const xrl_muon_desc *desc, int32_t n_matrices, const xrl_matrix *matrices, int64_t n_weights,
                  float *d_weights, const float *d_grads, float *d_momentum) {
  const char *who = "xrl_muon_step";
  if (!c || !desc) return fail(XRL_ERR_NULL, "%s: ctx or desc is NULL", who);
  if (n_matrices < 0 || n_weights < 0) return fail(XRL_ERR_SHAPE, "%s: n_matrices = %d, n_weights = %lld", who, n_matrices, (long long)n_weights);
  if (!std::isfinite(desc->lr) || desc->lr < 0.f || !std::isfinite(desc->momentum) || desc->momentum < 0.f || !std::isfinite(desc->weight_decay) ||
      desc->weight_decay < 0.f || !std::isfinite(desc->rms) || desc->rms < 0.f || desc->steps < 1 || desc->steps > 16)
    return fail(XRL_ERR_VALUE, "%s: lr %g, momentum %g, weight_decay %g, rms %g, steps %d", who, (double)desc->lr, (double)desc->momentum,
                (double)desc->weight_decay, (double)desc->rms, desc->steps);
  if (n_matrices == 0) return XRL_OK;
  if (!matrices) return fail(XRL_ERR_NULL, "%s: matrices is NULL", who);
  for (int k = 0; k < n_matrices; ++k) {
    const xrl_matrix &q = matrices[k];
    if (q.rows < 0 || q.cols < 0 || q.offset < 0) return fail(XRL_ERR_SHAPE, "%s: matrix %d: %lld x %lld at %lld", who, k, (long long)q.rows, (long long)q.cols, (long long)q.offset);
    if (q.rows > 32768 || q.cols > 32768) return fail(XRL_ERR_UNSUPPORTED, "%s: matrix %d: %lld x %lld", who, k, (long long)q.rows, (long long)q.cols);
    if (q.rows * q.cols > n_weights || q.offset > n_weights - q.rows * q.cols)
      return fail(XRL_ERR_SHAPE, "%s: matrix %d ends outside the vector of %lld", who, k, (long long)n_weights);
  }
  std::vector<Mat> list;
  try {
    std::vector<int> order;
    for (int k = 0; k < n_matrices; ++k)
      if (matrices[k].rows > 0 && matrices[k].cols > 0) order.push_back(k);
    std::sort(order.begin(), order.end(), [&](int x, int y) { return matrices[x].offset < matrices[y].offset; });
    for (size_t i = 0; i + 1 < order.size(); ++i) {
      const xrl_matrix &q = matrices[order[i]];
      if (q.offset + q.rows * q.cols > matrices[order[i + 1]].offset) return fail(XRL_ERR_SHAPE, "%s: matrices %d and %d overlap", who, order[i], order[i + 1]);
    }
    for (int k : order) {
      const xrl_matrix &q = matrices[k];
      Mat x = {};
      x.offset = q.offset;
      x.t = q.rows > q.cols;
      x.m = (int)std::min(q.rows, q.cols);
      x.n = (int)std::max(q.rows, q.cols);
      x.chunk = (int)std::max<int64_t>(4096, (q.rows * q.cols + kMaxSums - 1) / kMaxSums);
      list.push_back(x);
    }
  } catch (const std::bad_alloc &) {
    return fail(XRL_ERR_OOM, "%s: out of host memory", who);
  }
  if (list.empty()) return XRL_OK;
  if (!d_weights || !d_grads || !d_momentum) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d_weights | (uintptr_t)d_grads | (uintptr_t)d_momentum) % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of 4", who);
  // the largest group's workspace: every group uses it from the start
  size_t most = 0;
  for (size_t i = 0; i < list.size(); i += kGroup) {
    int64_t halves = 0;
    for (size_t k = i; k < std::min(list.size(), i + kGroup); ++k) {
      list[k].ws = halves;
      halves += 3 * x_halves(list[k].m, list[k].n) + 2 * x_halves(list[k].m, list[k].m);
    }
    most = std::max(most, (size_t)halves * 2);
  }
  const size_t o_sums = op_align(most);
  char *ws = nullptr;
  if (int rc = op_workspace(c, o_sums + (size_t)kGroup * kMaxSums * 8, &ws, who)) return rc;
  for (size_t i = 0; i < list.size(); i += kGroup) {
    MuonArgs p = {};
    p.count = (int)std::min<size_t>(kGroup, list.size() - i);
    for (int k = 0; k < p.count; ++k) {
      p.mat[k] = list[i + k];
      const int64_t size = (int64_t)p.mat[k].m * p.mat[k].n;
      p.first_sum[k + 1] = p.first_sum[k] + (int)((size + p.mat[k].chunk - 1) / p.mat[k].chunk);
    }
    p.w = d_weights; p.mom = d_momentum; p.g = d_grads;
    p.ws = (_Float16 *)ws; p.sums = (double *)(ws + o_sums);
    p.mu = desc->momentum; p.decay = 1.f - desc->lr * desc->weight_decay; p.step = desc->lr * desc->rms; p.nesterov = desc->nesterov != 0;
    if (int rc = run_group(c, p, desc->steps)) return rc;
  }
  return XRL_OK;
}

}  // extern "C"
