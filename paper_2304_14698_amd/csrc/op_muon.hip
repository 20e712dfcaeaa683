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
constexpr int kTile = 64;              // sizes are padded to multiples of this
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
  _Float16 *x, *xt, *next_xt, *a, *b;   // X; X^T as it is, and as the step's last product makes it; A; B
};
__device__ __forceinline__ Buffers buffers(const MuonArgs &p, const Mat &q) {
  const int64_t nx = x_halves(q.m, q.n), na = x_halves(q.m, q.m);
  _Float16 *w = p.ws + q.ws;
  return {w, w + (p.flip ? 2 : 1) * nx, w + (p.flip ? 1 : 2) * nx, w + 3 * nx, w + 3 * nx + na};
}
// The matrix that a block belongs to: a lane looks at one.
__device__ __forceinline__ int matrix_of(const MuonArgs &p, int block) {
  const int lane = threadIdx.x & 63;
  return __popcll(__ballot(lane < p.count && p.first[lane < p.count ? lane : 0] <= block)) - 1;
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
    o = buf.xt + ((int64_t)(tj * 2 + rb) * (mp / 16) + ti * 4 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
}

enum { STEP_GRAM, STEP_POLY, STEP_APPLY, STEP_LAST };

// One product of a step, D[i][j] = sum over k of P[i][k] Q[j][k], both in fragment order along k: the block's tile, of T x T.
struct Product {
  int k, ti, tj, mp, np, kbs;          // matrix; tile; padded sizes; fragments along k
  const _Float16 *P, *Q;
  Buffers buf;
};
template <int STEP, int T>
__device__ __forceinline__ Product product_of(const MuonArgs &p) {
  Product d;
  // Blocks are dealt to the eight XCDs in turn: an XCD takes neighbouring tiles, whose operands its L2 then holds
  const int all = p.first[p.count], xcd = blockIdx.x % 8, per = all / 8, rem = all % 8;
  const int block = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
  d.k = matrix_of(p, block);
  const Mat &q = p.mat[d.k];
  const int tile = block - p.first[d.k];
  d.mp = padded(q.m);
  d.np = padded(q.n);
  d.buf = buffers(p, q);
  if (STEP == STEP_GRAM || STEP == STEP_POLY) {           // symmetric: tiles with tj <= ti
    int ti = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    while (ti * (ti + 1) / 2 > tile) --ti;
    d.ti = ti;
    d.tj = tile - ti * (ti + 1) / 2;
    d.P = d.Q = STEP == STEP_GRAM ? d.buf.x : d.buf.a;
    d.kbs = (STEP == STEP_GRAM ? d.np : d.mp) / 16;
  } else {                                                 // strips of eight tiles' height, column by column
    const int th = (d.mp + T - 1) / T, tw = (d.np + T - 1) / T, strip = tile / (8 * tw), in = tile - strip * 8 * tw;
    const int h = th - strip * 8 < 8 ? th - strip * 8 : 8;
    d.ti = strip * 8 + in % h;
    d.tj = in / h;
    d.P = d.buf.b;
    d.Q = d.buf.xt;
    d.kbs = d.mp / 16;
  }
  return d;
}

// What becomes of a wave's 32 x 32 of a product, block (ib, jb). turn: the wave's own 32 x 33 floats of LDS.
template <int STEP>
__device__ __forceinline__ void put(const MuonArgs &p, const Product &d, const f32x16 &acc, int ib, int jb, float (*turn)[33]) {
  const Mat &q = p.mat[d.k];
  // register r of a lane: D[i][j] with i = ib 32 + 8 (r / 4) + 4 (lane / 32) + r % 4, j = jb 32 + lane % 32
  const int lane = threadIdx.x & 63, g = lane >> 5, jl = lane & 31;
  if (STEP == STEP_LAST) {
    const float step = p.step * sqrtf((float)q.n) * (kDown * kDown);
    float *w = p.w + q.offset;
    if (!q.t) {
      const int j = jb * 32 + jl;
      float old[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = ib * 32 + acc_row(r, g);
        old[r] = i < q.m && j < q.n ? w[(int64_t)i * q.n + j] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = ib * 32 + acc_row(r, g);
        if (i < q.m && j < q.n) w[(int64_t)i * q.n + j] = p.decay * old[r] - step * acc[r];
      }
    } else {                                               // rows j of the vector's matrix, along i
#pragma unroll
      for (int r = 0; r < 16; ++r) turn[acc_row(r, g)][jl] = acc[r];
      __builtin_amdgcn_wave_barrier();
      __threadfence_block();
      const int i = ib * 32 + jl;
      float old[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = jb * 32 + 2 * r + g;
        old[r] = i < q.m && j < q.n ? w[(int64_t)j * q.m + i] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = jb * 32 + 2 * r + g;
        if (i < q.m && j < q.n) w[(int64_t)j * q.m + i] = p.decay * old[r] - step * turn[jl][2 * r + g];
      }
      __threadfence_block();
      __builtin_amdgcn_wave_barrier();
    }
    return;
  }
  float v[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = acc[r] * kDown;
  if (STEP == STEP_POLY) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {                          // A[i][j] = A[j][i]: four i of one j lie side by side
      const _Float16 *at = d.buf.a + ((int64_t)jb * d.kbs + ib * 2 + (s >> 1)) * 1024 + (jl + 32 * (s & 1)) * 8 + 4 * g;
      const f16x4 h = *(const f16x4 *)at, l = *(const f16x4 *)(at + 512);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float diag = ib == jb && 8 * s + 4 * g + e == jl ? kNsA * kUp : 0.f;
        v[4 * s + e] = kNsC * v[4 * s + e] + (kNsB * ((float)h[e] + (float)l[e]) + diag);
      }
    }
  }
  // rows j, along i: a lane has four i side by side
  _Float16 *by_j = STEP == STEP_GRAM ? d.buf.a : STEP == STEP_POLY ? d.buf.b : d.buf.next_xt;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    f16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(v[4 * s + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16 *o = by_j + ((int64_t)jb * (d.mp / 16) + ib * 2 + (s >> 1)) * 1024 + (jl + 32 * (s & 1)) * 8 + 4 * g;
    *(f16x4 *)o = hi;
    *(f16x4 *)(o + 512) = lo;
  }
  // rows i, along j: turned round in LDS. (A block on the diagonal of a symmetric product has written both already.)
  if (STEP != STEP_APPLY && d.ti == d.tj) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) turn[acc_row(r, g)][jl] = v[r];
  __builtin_amdgcn_wave_barrier();
  __threadfence_block();
  _Float16 *by_i = STEP == STEP_GRAM ? d.buf.a : STEP == STEP_POLY ? d.buf.b : d.buf.x;
  const int kdim = STEP == STEP_APPLY ? d.np : d.mp;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(turn[jl][kb * 16 + g * 8 + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16 *o = by_i + ((int64_t)ib * (kdim / 16) + jb * 2 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
  __threadfence_block();
  __builtin_amdgcn_wave_barrier();
}

// Both halves of two factors of a 32 x 32 x 16 product; the small terms first.
__device__ __forceinline__ void add_product(f32x16 &acc, const f16x8 &ph, const f16x8 &pl, const f16x8 &qh, const f16x8 &ql) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
}

// Few tiles: 64 x 64 a block, 32 x 32 a wave, fragments requested in place from L2 and kAhead of them ahead.
template <int STEP>
__global__ __launch_bounds__(256) void muon_product_kernel(const MuonArgs p) {
  constexpr int kAhead = 4;                                // (there are a multiple of four along k)
  __shared__ float turn[4][32][33];
  const Product d = product_of<STEP, kTile>(p);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ib = d.ti * 2 + (wave >> 1), jb = d.tj * 2 + (wave & 1);
  const _Float16 *pa = d.P + (int64_t)ib * d.kbs * 1024 + lane * 8, *qa = d.Q + (int64_t)jb * d.kbs * 1024 + lane * 8;
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  f16x8 ph[kAhead], pl[kAhead], qh[kAhead], ql[kAhead];
  auto request = [&](int u, int kb) {
    const _Float16 *a = pa + (int64_t)kb * 1024, *b = qa + (int64_t)kb * 1024;
    ph[u] = *(const f16x8 *)a; pl[u] = *(const f16x8 *)(a + 512);
    qh[u] = *(const f16x8 *)b; ql[u] = *(const f16x8 *)(b + 512);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) request(u, u);
  __builtin_amdgcn_sched_barrier(0);
  for (int kb = 0; kb < d.kbs; kb += kAhead) {
    const int next = kb + kAhead < d.kbs ? kb + kAhead : kb;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      add_product(acc, ph[u], pl[u], qh[u], ql[u]);
      request(u, next + u);
      __builtin_amdgcn_sched_barrier(0);                   // (else the requests sink to where they are needed)
    }
  }
  put<STEP>(p, d, acc, ib, jb, turn[wave]);
}

// Many tiles: 128 x 128 a block, 64 x 64 a wave. 32 of the summed dimension at a time go from L2 straight into LDS, where two waves each read them;
// while they are multiplied the next 32 are on their way into the other half of the LDS. Two blocks a compute unit.
constexpr int kWide = 128;
constexpr unsigned kStage = 32 * 1024;                     // bytes: 2 factors x 4 blocks of 32 rows x 2 fragments x (hi, lo)
template <int STEP>
__global__ __launch_bounds__(256, 2) void muon_product_wide_kernel(const MuonArgs p) {
  extern __shared__ __align__(16) char lds[];
  const Product d = product_of<STEP, kWide>(p);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wi = wave >> 1, wj = wave & 1;
  const int rows_q = (STEP == STEP_GRAM || STEP == STEP_POLY ? d.mp : d.np) / 32;
  // wave w fills 8 KB of a stage: two blocks of 32 rows of P (w = 0, 1) or Q, 4 KB each, which lie side by side along k. (Rows behind the
  // padded matrix are read from its last block and never stored.)
  const char *src[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int rb = (wave & 1) * 2 + u;
    int at = (wave < 2 ? d.ti : d.tj) * 4 + rb;
    const int last = (wave < 2 ? d.mp / 32 : rows_q) - 1;
    at = at < last ? at : last;
    src[u] = (const char *)((wave < 2 ? d.P : d.Q) + (int64_t)at * d.kbs * 1024) + lane * 16;
  }
  const unsigned base = lds_address(lds), mine = (unsigned)__builtin_amdgcn_readfirstlane(wave) * 8192;
  auto request = [&](int s) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) lds_direct_load16(src[u] + (int64_t)s * 4096 + k * 1024, base + (s & 1) * kStage + mine + u * 4096 + k * 1024);
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
  const int stages = d.kbs / 2;
  request(0);
  for (int s = 0; s < stages; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wave's part of stage s is there, and behind the barrier all of it;
    __syncthreads();                                        // and nobody reads the other half any more
    if (s + 1 < stages) request(s + 1);
    const char *at = lds + (s & 1) * kStage + lane * 16;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f16x8 ph[2], pl[2], qh[2], ql[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const char *a = at + (wi * 2 + u) * 4096 + k * 2048, *b = at + 16384 + (wj * 2 + u) * 4096 + k * 2048;
        ph[u] = *(const f16x8 *)a; pl[u] = *(const f16x8 *)(a + 1024);
        qh[u] = *(const f16x8 *)b; ql[u] = *(const f16x8 *)(b + 1024);
      }
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) add_product(acc[a][b], ph[a], pl[a], qh[b], ql[b]);
    }
  }
  __syncthreads();                                          // the LDS becomes the waves' turning space
  float (*turn)[33] = (float (*)[33])(lds + wave * 32 * 33 * 4);
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int ib = d.ti * 4 + wi * 2 + a, jb = d.tj * 4 + wj * 2 + b;
      if (ib < d.mp / 32 && jb < rows_q) put<STEP>(p, d, acc[a][b], ib, jb, turn);
    }
}

// A launch of product STEP over all matrices.
template <int STEP>
int launch_product(const xrl_ctx *c, MuonArgs &p) {
  auto blocks = [&](int T) {
    int64_t at = 0;
    for (int k = 0; k < p.count; ++k) {
      const int64_t th = (p.mat[k].m + T - 1) / T, tw = (p.mat[k].n + T - 1) / T;
      p.first[k] = (int)at;
      at += STEP == STEP_GRAM || STEP == STEP_POLY ? th * (th + 1) / 2 : th * tw;
    }
    p.first[p.count] = (int)at;
    return at;
  };
  if (blocks(kWide) >= op_compute_units(c)) {
    constexpr int lds = 2 * (int)kStage;
    muon_product_wide_kernel<STEP><<<dim3((unsigned)p.first[p.count]), dim3(256), lds, op_stream(c)>>>(p);
  } else {
    muon_product_kernel<STEP><<<dim3((unsigned)blocks(kTile)), dim3(256), 0, op_stream(c)>>>(p);
  }
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

int run_group(xrl_ctx *c, MuonArgs &p, int steps) {
  for (int k = 0; k <= p.count; ++k) p.first[k] = p.first_sum[k];
  muon_momentum_kernel<<<dim3((unsigned)p.first[p.count]), dim3(256), 0, op_stream(c)>>>(p);
  p.first[0] = 0;
  for (int k = 0; k < p.count; ++k)
    p.first[k + 1] = p.first[k] + (p.mat[k].m + kTile - 1) / kTile * ((p.mat[k].n + kTile - 1) / kTile);
  muon_begin_kernel<<<dim3((unsigned)p.first[p.count]), dim3(256), 0, op_stream(c)>>>(p);
  OP_TRY(hipGetLastError());
  for (int s = 0; s < steps; ++s) {
    if (int rc = launch_product<STEP_GRAM>(c, p)) return rc;
    if (int rc = launch_product<STEP_POLY>(c, p)) return rc;
    if (int rc = s + 1 < steps ? launch_product<STEP_APPLY>(c, p) : launch_product<STEP_LAST>(c, p)) return rc;
    p.flip ^= 1;
  }
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
