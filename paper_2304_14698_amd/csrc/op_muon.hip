// Momentum with orthogonalised updates: Newton-Schulz steps on every listed matrix of a flat weight vector.
//
// Per matrix, as m x n with m <= n (transposed if it has more rows than columns), X = U / |U|_F and `steps` times
//   A = X X^T,  B = a I + b A + c A A,  X = B X,
// the quintic a X + (b A + c A A) X. All matrices share the launches: 2 + 3 steps in all; where every matrix is at most 64 x 512 one launch does all of it.
//
// Numbers. The products run on the fp16 matrix cores, which are sixteen times as fast as the fp32 ones, on entries x 2^12 split in two halves
// of 11 bits, hi = fp16(x 2^12) and lo = fp16((x 2^12 - hi) 2^11), with fp32 sums of their own for hi hi and for hi lo + lo hi, which is added 2^-11 times. That
// leaves out 2^-22 of an entry, fp32 2^-24. Entries cannot overflow: singular values of X lie in [0, 1.21] in every step (the quintic's largest value on
// [0, 1.21] is 1.21), so entries of X, A and B are at most 1.21, 1.47 and 3.45, and 3.45 2^12 < 65504; lo is at most 2^12 times the entry, too. An entry keeps
// its 22 bits down to 2^-26; below, hi and lo together are off by at most 2^-48 (by a subnormal fp16's half, 2^-25, over 2^11 and 2^12). Without the 2^11 lo
// would be subnormal from entries of 2^-15 on, as rows of small size have: of 256 x 512 with row sizes from 1 to 1e-6 the worst row was off by 3e-4 of
// itself so, and is by 4e-6, 6e-6 with fp32 products (from 1 to 1e-8 1.5e-5 and 6e-6).
//
// Layout. Operands lie in fragment order: 32 rows by 16 of the summed dimension, first hi, then lo, each 64 lanes by 16 bytes, as one matrix
// instruction takes them. Both X (rows m) and X^T (rows n) are kept.
#include "op_common.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

using namespace xrl;

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;
constexpr float kLowUp = 2048.f, kLowDown = 1.f / 2048.f;   // of the lower halves besides
constexpr int kGroup = 32;             // matrices of one launch: their list is a kernel argument
constexpr int64_t kGroupHalves = (int64_t)1 << 30;   // operands of a group that has more than one: 2 GB, several times what fills the chip (two 2048^2 and two
                                                    // 2048 x 8192 are 0.5); a model of thirty-two 16384^2 would need 172 GB for them at once
constexpr int kTile = 64;              // sizes are padded to multiples of this
constexpr int kMaxSums = 1024;         // partial sums of squares of a matrix

// A matrix of a launch. A lane of each wave reads one, all at once, and what the block needs of its own matrix is then passed on from that lane: kernel arguments
// lie in host memory, and one look at the list after another took 1.2 to 2.2 us a block.
struct Mat {
  int64_t offset, ws;                  // in the flat vectors; in the workspace (halves)
  int m, n, t;                         // m <= n; t: the matrix in the vector is n x m
  int chunk;                           // entries of one partial sum of squares
  int first_sum;                       // its first partial sum
  int first;                           // its first block in this launch
  int parts;                           // products: parts that the sums of its tiles are cut into, a block each
  int blocks;                          // in this launch
};
struct MuonArgs {
  int count;
  int flip;                            // which of the two X^T holds the current one
  int share[9];                        // products: first block of each XCD's share
  int n_arrived;
  Mat mat[kGroup];
  float *w, *mom;
  const float *g;
  _Float16 *ws;
  double *sums;
  float *partial;                      // [blocks of a launch][T * T] sums of parts
  int *arrived;                        // [blocks of a launch] parts of a tile that are there, zero between launches
  float mu, decay, step;               // step: lr rms (times sqrt(max(rows, cols)))
  int nesterov;
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
__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)x, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// The matrix that block `block` of a launch belongs to.
__device__ __forceinline__ Mat matrix_of(const MuonArgs &p, int block) {
  static_assert(kGroup <= 64, "a lane for each");
  const int lane = threadIdx.x & 63;
  const Mat x = p.mat[lane < kGroup ? lane : 0];
  const int k = __popcll(__ballot(lane < p.count && x.first <= block)) - 1;
  auto of = [&](int v) { return __builtin_amdgcn_readlane(v, k); };
  return {from_lane(x.offset, k), from_lane(x.ws, k), of(x.m), of(x.n), of(x.t), of(x.chunk), of(x.first_sum), of(x.first), of(x.parts), of(x.blocks)};
}
// N values split in two halves each: pairs, so that one instruction rounds two.
template <int N, typename V>
__device__ __forceinline__ void split(const float *y, V &hi, V &lo) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  f16x2 h[N / 2], l[N / 2];
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    const f32x2 x = {y[2 * e], y[2 * e + 1]};
    h[e] = __builtin_convertvector(x, f16x2);
    l[e] = __builtin_convertvector((x - __builtin_convertvector(h[e], f32x2)) * kLowUp, f16x2);
  }
  __builtin_memcpy(&hi, h, sizeof(hi));
  __builtin_memcpy(&lo, l, sizeof(lo));
}

// M = mu M + G, and of each chunk the sum of squares of U. Bound by memory: 42 million entries 81 us, 503 MB at 6.2 TB/s.
__global__ __launch_bounds__(256) void muon_momentum_kernel(const MuonArgs p) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < p.n_arrived; i += gridDim.x * 256) p.arrived[i] = 0;
  const Mat q = matrix_of(p, blockIdx.x);
  const int part = blockIdx.x - q.first;
  const int64_t size = (int64_t)q.m * q.n, i0 = (int64_t)part * q.chunk, i1 = i0 + q.chunk < size ? i0 + q.chunk : size;
  float *mom = p.mom + q.offset;
  const float *g = p.g + q.offset;
  double sum = 0.;
  for (int64_t b = i0; b < i1; b += 4096) {
    const int64_t i = b + threadIdx.x * 4;
    if (b + 4096 <= i1) {                                  // (no load in a branch of its own: eight are on their way together)
      Piece<float, 4> gi[4], mi[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        gi[u] = load_piece<float, 4>(g + i + u * 1024);
        mi[u] = load_piece<float, 4>(mom + i + u * 1024);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float m[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m[e] = p.mu * mi[u].v[e] + gi[u].v[e];
          const float x = p.nesterov ? gi[u].v[e] + p.mu * m[e] : m[e];
          sum += (double)x * (double)x;
        }
        store_piece<float, 4>(mom + i + u * 1024, m);
      }
    } else {
      float gk[16], mk[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const int64_t k = b + u * 256 + threadIdx.x, at = k < i1 ? k : i0;
        gk[u] = g[at];
        mk[u] = mom[at];
      }
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const int64_t k = b + u * 256 + threadIdx.x;
        if (k < i1) {
          const float m = p.mu * mk[u] + gk[u], x = p.nesterov ? gk[u] + p.mu * m : m;
          mom[k] = m;
          sum += (double)x * (double)x;
        }
      }
    }
  }
  for (int s = 32; s; s /= 2) sum += __shfl_xor(sum, s);
  __shared__ double part_sum[4];
  if ((threadIdx.x & 63) == 0) part_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.sums[q.first_sum + part] = part_sum[0] + part_sum[1] + part_sum[2] + part_sum[3];
}

__device__ __forceinline__ int wave_of(int t) { return t >> 6; }

// X = U / (|U| + 1e-7) in both orders, a 64 x 64 tile a block, turned round in LDS. Bound by memory: 42 million entries 143 us, 671 MB at 4.7 TB/s.
__global__ __launch_bounds__(256) void muon_begin_kernel(const MuonArgs p) {
  const Mat q = matrix_of(p, blockIdx.x);
  const int tile = blockIdx.x - q.first, t = threadIdx.x, lane = t & 63;
  const int mp = padded(q.m), np = padded(q.n), ti = tile / (np / kTile), tj = tile % (np / kTile);
  const Buffers buf = buffers(p, q);
  const int ld = q.t ? q.m : q.n;
  float g[kTile * kTile / 256], m[kTile * kTile / 256];
#pragma unroll
  for (int u = 0; u < kTile * kTile / 256; ++u) {         // rows and columns of the tile as the vector has them: lanes along a row
    const int a = wave_of(t) + u * 4, b = lane, i = ti * kTile + (q.t ? b : a), j = tj * kTile + (q.t ? a : b);
    const bool in = i < q.m && j < q.n;
    const int64_t at = q.offset + (q.t ? (int64_t)j * ld + i : (int64_t)i * ld + j);
    m[u] = p.mom[in ? at : q.offset];
    g[u] = p.g[in ? at : q.offset];
    if (!in) m[u] = g[u] = 0.f;
  }
  double sum = 0.;
  const int n_sums = (int)(((int64_t)q.m * q.n + q.chunk - 1) / q.chunk);
  for (int i = lane; i < n_sums; i += 64) sum += p.sums[q.first_sum + i];
  for (int s = 32; s; s /= 2) sum += __shfl_xor(sum, s);
  const float scale = (float)(kUp / (sqrt(sum) + 1e-7));   // (of a norm from 2^126 on 1 / |U| alone would be subnormal)
  __shared__ float x[kTile][kTile + 1];
#pragma unroll
  for (int u = 0; u < kTile * kTile / 256; ++u) {
    const int a = wave_of(t) + u * 4, b = lane;
    x[q.t ? b : a][q.t ? a : b] = (p.nesterov ? g[u] + p.mu * m[u] : m[u]) * scale;
  }
  __syncthreads();
  for (int s = t; s < 512; s += 256) {
    const int rb = s >> 8, kb = (s >> 6) & 3, row = rb * 32 + (lane & 31), c = kb * 16 + (lane >> 5) * 8;
    f16x8 hi, lo;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[row][c + e];
    split<8>(v, hi, lo);
    _Float16 *o = buf.x + ((int64_t)(ti * 2 + rb) * (np / 16) + tj * 4 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[c + e][row];
    split<8>(v, hi, lo);
    o = buf.xt + ((int64_t)(tj * 2 + rb) * (mp / 16) + ti * 4 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
}

enum { STEP_GRAM, STEP_POLY, STEP_APPLY, STEP_LAST };

// One product of a step, D[i][j] = sum over k of P[i][k] Q[j][k], both in fragment order along k: the block's tile, of T x T.
struct Product {
  bool there;
  int ti, tj, mp, np, kbs;             // tile; padded sizes; fragments along k
  int block, part, parts;              // block of the launch, which part of the tile's sums it adds up
  const _Float16 *P, *Q;
  Mat q;
  Buffers buf;
};
template <int STEP, int T>
__device__ __forceinline__ Product product_of(const MuonArgs &p) {
  Product d;
  // Blocks are dealt to the eight XCDs in turn; an XCD takes consecutive tiles, whose operands its L2 then holds
  const int xcd = blockIdx.x % 8, block = p.share[xcd] + (int)(blockIdx.x / 8);
  d.there = block < p.share[xcd + 1];
  d.q = matrix_of(p, block);
  const Mat &q = d.q;
  d.parts = q.parts;
  d.block = block;
  const int tile = (block - q.first) / d.parts;
  d.part = block - q.first - tile * d.parts;
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

// The last product's entries of a lane in its matrix of the vector, lanes along that one's rows (of a matrix taken transposed: along i); -1: none.
// (Sums of products with what depends on the block alone: a choice between the two orders at each entry makes branches. A matrix has at most 2^30 entries.)
struct Entries {
  int first, of_r, of_q, row_r, left;
  bool in;
  __device__ Entries(const Mat &q, int ib, int jb) {
    const int lane = threadIdx.x & 63, g = lane >> 5, jl = lane & 31;
    const int row = q.t ? jb * 32 + g : ib * 32 + 4 * g, col = (q.t ? ib : jb) * 32 + jl, rows = q.t ? q.n : q.m, cols = q.t ? q.m : q.n;
    first = row * cols + col;
    row_r = q.t ? 2 : 1;                                   // register r: 2 r rows on, or 8 (r / 4) + r % 4
    of_r = row_r * cols;
    of_q = 8 * cols;
    left = rows - row;
    in = col < cols;
  }
  __device__ int at(int r) const { return (in & ((r & 3) * row_r + 8 * (r >> 2) < left)) ? first + (r & 3) * of_r + (r >> 2) * of_q : -1; }
};
__device__ __forceinline__ void old_weights(const MuonArgs &p, const Mat &q, int ib, int jb, float *old) {
  const Entries e(q, ib, jb);
  const float *w = p.w + q.offset;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int at = e.at(r);
    old[r] = w[at >= 0 ? at : 0];
  }
}

// What becomes of a wave's 32 x 32 of a product, block (ib, jb). turn: the wave's own 32 x 33 floats of LDS; old: the weights there (last product).
template <int STEP>
__device__ __forceinline__ void put(const MuonArgs &p, const Product &d, const f32x16 &acc, int ib, int jb, float (*turn)[33], const float *old) {
  const Mat &q = d.q;
  // register r of a lane: D[i][j] with i = ib 32 + 8 (r / 4) + 4 (lane / 32) + r % 4, j = jb 32 + lane % 32
  const int lane = threadIdx.x & 63, g = lane >> 5, jl = lane & 31;
  if (STEP == STEP_LAST) {
    const float step = p.step * sqrtf((float)q.n) * (kDown * kDown);
    float y[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = acc[r];
    if (q.t) {
#pragma unroll
      for (int r = 0; r < 16; ++r) turn[acc_row(r, g)][jl] = acc[r];
      __builtin_amdgcn_wave_barrier();
      __threadfence_block();
#pragma unroll
      for (int r = 0; r < 16; ++r) y[r] = turn[jl][2 * r + g];
      __threadfence_block();
      __builtin_amdgcn_wave_barrier();
    }
    float *w = p.w + q.offset;
    const Entries e(q, ib, jb);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int at = e.at(r);
      if (at >= 0) w[at] = p.decay * old[r] - step * y[r];
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
        v[4 * s + e] = kNsC * v[4 * s + e] + (kNsB * ((float)h[e] + kLowDown * (float)l[e]) + diag);
      }
    }
  }
  // rows j, along i: a lane has four i side by side
  _Float16 *by_j = STEP == STEP_GRAM ? d.buf.a : STEP == STEP_POLY ? d.buf.b : d.buf.next_xt;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    f16x4 hi, lo;
    split<4>(v + 4 * s, hi, lo);
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
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = turn[jl][kb * 16 + g * 8 + e];
    split<8>(y, hi, lo);
    _Float16 *o = by_i + ((int64_t)ib * (kdim / 16) + jb * 2 + kb) * 1024 + lane * 8;
    *(f16x8 *)o = hi;
    *(f16x8 *)(o + 512) = lo;
  }
  __threadfence_block();
  __builtin_amdgcn_wave_barrier();
}

// One of the three products of the halves of two factors, 32 x 32 x 16, into NB x NB blocks.
template <int NB>
__device__ __forceinline__ void add_products(f32x16 (*acc)[NB], const f16x8 *p, const f16x8 *q) {
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[a], q[b], acc[a][b], 0, 0, 0);
}

// A block takes T x T of a product, each of its four waves a quarter. 32 of the summed dimension at a time (a stage, two fragments) go from L2 straight into
// LDS, where two waves each read them; while a stage is multiplied those behind it are on their way. Tiles of 64 x 64, which often are alone on a compute
// unit, also read the fragments of each product from LDS while the one before is multiplied, across the barrier between two stages too: a lone block's stage
// 0.25 us, 0.31 without that. (530 clocks, of which the LDS takes 384 to be written and read and the matrix pipes 192.) Of tiles of 128 x 128 two blocks
// fill in for each other: X X^T of two 2048^2 and two 2048 x 8192 342 us so, 331 without. Of these four matrices B X takes 500 us (520 on a machine at
// 1.76 GHz), 515 GF of fp16 products at 1.03 PFLOP/s, bound by the matrix cores; A A 142 and X X^T 330, 0.77 and 0.83: 544 tiles on 512 places, whose last ones
// have the chip to themselves. Of
// smaller matrices a product is bound by the latency of its launch, the first stage and the last: 6 to 12 us for those of a 256-wide agent.
template <int STEP, int T, int STAGES>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(const MuonArgs p) {
  constexpr int NB = T / 64;                               // blocks of 32 of a wave, in each direction
  constexpr int KB = 2;
  constexpr unsigned kRows = KB * 2048, kFactor = T / 32 * kRows, kStage = 2 * kFactor;   // bytes: T / 32 blocks of rows x KB fragments x (hi, lo) of 1 KB
  extern __shared__ __align__(16) char lds[];
  const Product d = product_of<STEP, T>(p);
  if (!d.there) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wi = wave >> 1, wj = wave & 1;
  const int rows_q = (STEP == STEP_GRAM || STEP == STEP_POLY ? d.mp : d.np) / 32;
  // waves 0 and 1 fill in P, 2 and 3 Q, NB blocks of rows each, 4 KB that lie side by side along k. (Rows behind the padded matrix
  // are read from its last block and never stored.)
  const char *src[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    int at = (wave < 2 ? d.ti : d.tj) * (T / 32) + (wave & 1) * NB + u;
    const int last = (wave < 2 ? d.mp / 32 : rows_q) - 1;
    at = at < last ? at : last;
    src[u] = (const char *)((wave < 2 ? d.P : d.Q) + (int64_t)at * d.kbs * 1024) + lane * 16;
  }
  const unsigned base = lds_address(lds) + (unsigned)__builtin_amdgcn_readfirstlane(wave) * (NB * kRows);
  auto request = [&](int s, int buffer) {
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
      for (int k = 0; k < 2 * KB; ++k) lds_direct_load16(src[u] + (int64_t)s * kRows + k * 1024, base + buffer * kStage + u * kRows + k * 1024);
  };
  float old[16];                                           // (of one block: requested now, needed at the end)
  if (STEP == STEP_LAST && NB == 1) old_weights(p, d.q, d.ti * 2 + wi, d.tj * 2 + wj, old);
  f32x16 acc[NB][NB], low[NB][NB];                         // sums of hi hi; of hi lo + lo hi
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = low[a][b][r] = 0.f;
  // this block's part of the sums (kbs is a multiple of four)
  const int per = (d.kbs / KB + d.parts - 1) / d.parts, first = d.part * per, stages = first + per < d.kbs / KB ? per : d.kbs / KB - first;
#pragma unroll
  for (int u = 0; u < NB; ++u) src[u] += (int64_t)first * kRows;
  struct Fragments {
    f16x8 ph[NB], pl[NB], qh[NB], ql[NB];
  };
  auto read = [&](Fragments &f, int buffer, int k) {
    const char *at = lds + buffer * kStage + lane * 16 + k * 2048;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const char *a = at + (wi * NB + u) * kRows, *b = at + kFactor + (wj * NB + u) * kRows;
      f.ph[u] = *(const f16x8 *)a; f.pl[u] = *(const f16x8 *)(a + 1024);
      f.qh[u] = *(const f16x8 *)b; f.ql[u] = *(const f16x8 *)(b + 1024);
    }
  };
  auto multiply = [&](const Fragments &f) {
    add_products<NB>(low, f.ph, f.ql);
    add_products<NB>(acc, f.ph, f.qh);
    add_products<NB>(low, f.pl, f.qh);
  };
  // A stage is there: this wave's part (loads arrive in order; `behind` stages behind it may be on their way still), and behind the barrier all of it;
  // and what was read from LDS before is in registers everywhere
  constexpr int kLoads = (int)(kStage / 4096);             // of a wave and stage
  auto arrive = [&](bool all, auto behind) {
    if (all) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(behind)::value * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");                          // no read of the stage is moved in front of the barrier
  };
  Fragments f0, f1;
  int buffer = 0;
  if constexpr (NB == 1) {
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      if (s < stages) request(s, s);
    arrive(stages < STAGES, std::integral_constant<int, STAGES - 1>());
    read(f0, 0, 0);
    for (int s = 0; s < stages; ++s) {
      read(f1, buffer, 1);
      multiply(f0);
      if (s + 1 < stages) {
        const int next = buffer + 1 == STAGES ? 0 : buffer + 1;
        arrive(s + STAGES - 1 >= stages, std::integral_constant<int, STAGES - 2>());
        if (s + STAGES < stages) request(s + STAGES, buffer);
        read(f0, next, 0);
        buffer = next;
      }
      multiply(f1);
    }
  } else {
    static_assert(NB == 1 || STAGES == 2, "the other half of the LDS");
    request(0, 0);
    for (int s = 0; s < stages; ++s) {
      arrive(true, std::integral_constant<int, 0>());
      if (s + 1 < stages) request(s + 1, buffer ^ 1);
      read(f0, buffer, 0);
      multiply(f0);
      read(f1, buffer, 1);
      multiply(f1);
      buffer ^= 1;
    }
  }
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] += kLowDown * low[a][b][r];
  if (T == 64 && (STEP == STEP_GRAM || STEP == STEP_POLY) && d.parts > 1) {   // (no other sums are cut)
    // The part is laid down, past the L2 that other XCDs do not see; the block that comes last adds up all of them in order.
    constexpr int kTileFloats = T * T;
    const int64_t mine = (int64_t)wave * NB * NB * 1024 + lane;
    float *to = p.partial + (int64_t)d.block * kTileFloats + mine;
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          __hip_atomic_store(to + ((a * NB + b) * 16 + r) * 64, acc[a][b][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __shared__ int last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int *arrived = p.arrived + d.block - d.part;
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == d.parts - 1;
    __syncthreads();
    if (!last) return;
    if (threadIdx.x == 0) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
    for (int k = 0; k < d.parts; ++k) {
      const float *from = p.partial + (int64_t)(d.block - d.part + k) * kTileFloats + mine;
#pragma unroll
      for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[a][b][r] += __hip_atomic_load(from + ((a * NB + b) * 16 + r) * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();                                          // the LDS becomes the waves' turning space
  float (*turn)[33] = (float (*)[33])(lds + wave * 32 * 33 * 4);
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int ib = (d.ti * 2 + wi) * NB + a, jb = (d.tj * 2 + wj) * NB + b;
      if (ib < d.mp / 32 && jb < rows_q) {
        if (STEP == STEP_LAST && NB > 1) old_weights(p, d.q, ib, jb, old);
        put<STEP>(p, d, acc[a][b], ib, jb, turn, old);
      }
    }
}

// ---- matrices of at most 64 x 512: a whole step of one matrix in one block, nothing but the vectors' entries read and written.
// Wave w keeps columns 32 w .. 32 w + 31 of X in registers, as the products leave them: x[b][r] is row 32 b + 8 (r / 4) + 4 (lane / 32) + r % 4 of column
// 32 w + lane % 32, times 2^12, in fp32. For A = X X^T the waves lay X down in LDS in fragment order (turned round on the way) and share out the four
// 32 x 32 blocks of A, a part of the summed columns each; for B X a wave's own columns become its operand by exchanges between the two halves of the wave.
// Bound by latency: 64 x 256 takes 4.3 us a step (turning, X X^T, joining its parts, B, B X with a barrier behind each) and 8 us a call besides, five steps
// 29 us (64 x 64 21, 64 x 512 47). All of the vectors' entries are requested at the start; with the weights requested at the end, and the requests of each half
// of the rows behind the other's stores, this was 2 us more. Sixteen waves have 128 registers each and do it so: with all at the start, and with the entries'
// indices kept for the end, they spilled 116 bytes a lane, and 64 x 512 took 49 us.
constexpr int kSmallRows = 64;
__host__ __device__ constexpr int small_lds(int waves) { return waves * 8192 + 2 * 16384; }   // X, and the parts of A after it; A; B
constexpr int kTurn = 36;              // floats of a row on its way: 16-byte pieces of 8 rows lie in different banks

// 16 floats of a lane, its own row of 32 columns, in the order of columns kb 16 + 8 (lane / 32) ..: turned round from 32 x 32 of a product
__device__ __forceinline__ void turn_round(float (*turn)[kTurn], const float *x, int g, int jl, float (*y)[8]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) turn[acc_row(r, g)][jl] = x[r];
  __builtin_amdgcn_wave_barrier();
  __threadfence_block();
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 v = *(const f32x4 *)&turn[jl][kb * 16 + g * 8 + 4 * u];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[kb][4 * u + e] = v[e];
    }
  __threadfence_block();
  __builtin_amdgcn_wave_barrier();
}
// Four rows of one column, as a lane has them in a product, into a fragment-ordered 64 x 64 matrix: rows along the summed dimension.
__device__ __forceinline__ void put_four(_Float16 *to, int ib, int jb, int s, int lane, const float *v) {
  f16x4 hi, lo;
  split<4>(v, hi, lo);
  _Float16 *o = to + (jb * 4 + ib * 2 + (s >> 1)) * 1024 + ((lane & 31) + 32 * (s & 1)) * 8 + 4 * (lane >> 5);
  *(f16x4 *)o = hi;
  *(f16x4 *)(o + 512) = lo;
}

// The three products of the halves of two factors, 32 x 32 x 16: hi hi to acc, hi lo + lo hi to low; and their sum, in acc.
__device__ __forceinline__ void add_halves(f32x16 &acc, f32x16 &low, const f16x8 &ah, const f16x8 &al, const f16x8 &bh, const f16x8 &bl) {
  low = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, low, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc, 0, 0, 0);
  low = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, low, 0, 0, 0);
}
__device__ __forceinline__ void join_halves(f32x16 &acc, const f32x16 &low) {
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] += kLowDown * low[r];
}

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void muon_small_kernel(const MuonArgs p, int steps) {
  constexpr int PARTS = WAVES / 4;                         // of the sums of a block of A
  constexpr bool EARLY = WAVES == 8;                       // (the weights requested at the start, and all rows at once)
  constexpr int AT_ONCE = EARLY ? 2 : 1;
  extern __shared__ __align__(16) char lds[];
  const Mat q = matrix_of(p, blockIdx.x);
  const int m = q.m, n = q.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, jl = lane & 31;
  const int j = wave * 32 + jl, used = (n + 31) / 32;     // waves that have columns
  _Float16 *X = (_Float16 *)lds, *A = (_Float16 *)(lds + WAVES * 8192), *B = A + 8192;
  f32x4 *parts = (f32x4 *)lds;
  float (*turn)[kTurn] = (float (*)[kTurn])(lds + wave * 8192);
  float *w = p.w + q.offset, *mom = p.mom + q.offset;
  const float *grad = p.g + q.offset;
  // entry (b, r) of a lane in the vector: lanes along its rows, which for a matrix that is taken transposed is another order than x's
  // (Sums of products with what depends on the matrix alone: a choice between the two orders at each entry makes branches.)
  const int of_b = q.t ? 32 : 32 * n, of_r = q.t ? 2 * m : n, of_q = 8 * (q.t ? m : n), row_b = q.t ? 0 : 32, row_r = q.t ? 2 : 1, col_b = q.t ? 32 : 0;
  int first = q.t ? (wave * 32 + g) * m + jl : 4 * g * n + j, rows = q.t ? n - wave * 32 - g : m - 4 * g, cols = q.t ? m - jl : n - j;
  auto at = [&](int b, int r) {
    const bool in = (b * row_b + (r & 3) * row_r + 8 * (r >> 2) < rows) & (b * col_b < cols);
    return in ? first + b * of_b + (r & 3) * of_r + (r >> 2) * of_q : -1;
  };
  // M = mu M + G, U and |U|. (Requests for entries that are not there go to the first one: a request in a branch of its own is waited for there.)
  float x[2][16], old[2][16];
  {
    float gi[2][16], mi[2][16];
    double sum = 0.;
#pragma unroll
    for (int b0 = 0; b0 < 2; b0 += AT_ONCE) {
#pragma unroll
      for (int b = b0; b < b0 + AT_ONCE; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = at(b, r), from = k >= 0 ? k : 0;
          gi[b][r] = grad[from];
          mi[b][r] = mom[from];
          if (EARLY) old[b][r] = w[from];
        }
#pragma unroll
      for (int b = b0; b < b0 + AT_ONCE; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = at(b, r);
          const float mr = p.mu * mi[b][r] + gi[b][r], u = p.nesterov ? gi[b][r] + p.mu * mr : mr;
          if (k >= 0) mom[k] = mr;
          x[b][r] = k >= 0 ? u : 0.f;
          sum += (double)x[b][r] * (double)x[b][r];
        }
    }
    for (int s = 32; s; s /= 2) sum += __shfl_xor(sum, s);
    double *sums = (double *)lds;
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.;
    for (int k = 0; k < WAVES; ++k) sum += sums[k];
    const float scale = (float)(kUp / (sqrt(sum) + 1e-7));
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[b][r] *= scale;
    __syncthreads();
  }
  // 32 x 32 between the vector's order of a transposed matrix and x's, in place; the other way round `back`
  auto reorder = [&](float *v, bool back) {
#pragma unroll
    for (int r = 0; r < 16; ++r) turn[back ? acc_row(r, g) : jl][back ? jl : 2 * r + g] = v[r];
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = turn[back ? jl : acc_row(r, g)][back ? 2 * r + g : jl];
    __threadfence_block();
    __builtin_amdgcn_wave_barrier();
  };
  if (q.t)
#pragma unroll
    for (int b = 0; b < 2; ++b) reorder(x[b], false);
  const int ib = wave / (2 * PARTS), jb = wave / PARTS % 2, part = wave % PARTS;   // the block of A, and part of its sums, that the wave takes
  for (int step = 0; step < steps; ++step) {
    if (wave < used) {
      f16x8 hi[2][2], lo[2][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float y[2][8];
        turn_round(turn, x[b], g, jl, y);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) split<8>(y[kb], hi[b][kb], lo[b][kb]);
      }
      // [wave][kb][row block][hi, lo]
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          _Float16 *o = X + ((wave * 2 + kb) * 2 + b) * 1024 + lane * 8;
          *(f16x8 *)o = hi[b][kb];
          *(f16x8 *)(o + 512) = lo[b][kb];
        }
    }
    __syncthreads();
    f32x16 acc = {}, low = {};
    const int kbs = 2 * used, per = (kbs + PARTS - 1) / PARTS, k0 = part * per, k1 = k0 + per < kbs ? k0 + per : kbs;
    for (int kb = k0; kb < k1; ++kb) {
      const _Float16 *a = X + (kb * 2 + ib) * 1024 + lane * 8, *b = X + (kb * 2 + jb) * 1024 + lane * 8;
      add_halves(acc, low, *(const f16x8 *)a, *(const f16x8 *)(a + 512), *(const f16x8 *)b, *(const f16x8 *)(b + 512));
    }
    join_halves(acc, low);
    __syncthreads();                                       // (the parts take X's place)
#pragma unroll
    for (int s = 0; s < 4; ++s) parts[(wave * 4 + s) * 64 + lane] = f32x4{acc[4 * s], acc[4 * s + 1], acc[4 * s + 2], acc[4 * s + 3]};
    __syncthreads();
#pragma unroll
    for (int s = part * 4 / PARTS; s < (part + 1) * 4 / PARTS; ++s) {   // the same waves: some rows each of the sums of all parts
      f32x4 sum = parts[((wave - part) * 4 + s) * 64 + lane];
#pragma unroll
      for (int k = 1; k < PARTS; ++k) sum += parts[((wave - part + k) * 4 + s) * 64 + lane];
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = sum[e] * kDown;
      put_four(A, ib, jb, s, lane, v);
    }
    __syncthreads();
    if (wave < 4) {                                        // B = a I + b A + c A A, a block a wave
      const int bi = wave >> 1, bj = wave & 1;
      f32x16 low = {};
      acc = f32x16{};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const _Float16 *a = A + (bi * 4 + kb) * 1024 + lane * 8, *b = A + (bj * 4 + kb) * 1024 + lane * 8;
        add_halves(acc, low, *(const f16x8 *)a, *(const f16x8 *)(a + 512), *(const f16x8 *)b, *(const f16x8 *)(b + 512));
      }
      join_halves(acc, low);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const _Float16 *o = A + (bj * 4 + bi * 2 + (s >> 1)) * 1024 + (jl + 32 * (s & 1)) * 8 + 4 * g;
        const f16x4 h = *(const f16x4 *)o, l = *(const f16x4 *)(o + 512);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = kNsC * (acc[4 * s + e] * kDown) + (kNsB * ((float)h[e] + kLowDown * (float)l[e]) + (bi == bj && 8 * s + 4 * g + e == jl ? kNsA * kUp : 0.f));
        put_four(B, bi, bj, s, lane, v);
      }
    }
    __syncthreads();
    if (wave < used) {                                     // X = B X, the wave's columns
      f16x8 xh[4], xl[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        // rows 16 kb .. 16 kb + 15 of the column lie in registers 8 (kb % 2) .. of the lane (rows 0-3 and 8-11) and of its
        // partner in the other half (4-7, 12-15); the operand wants rows 0-7 in the lower half's lane and 8-15 in the upper's
        u32x4 h, l, ph, pl;
        split<8>(x[kb >> 1] + 8 * (kb & 1), h, l);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const auto a = __builtin_amdgcn_permlane32_swap(h[u], h[2 + u], false, false);
          const auto b = __builtin_amdgcn_permlane32_swap(l[u], l[2 + u], false, false);
          ph[u] = a[0]; ph[2 + u] = a[1];
          pl[u] = b[0]; pl[2 + u] = b[1];
        }
        xh[kb] = __builtin_bit_cast(f16x8, ph);
        xl[kb] = __builtin_bit_cast(f16x8, pl);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x16 low = {};
        acc = f32x16{};
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          const _Float16 *o = B + (b * 4 + kb) * 1024 + lane * 8;
          add_halves(acc, low, *(const f16x8 *)o, *(const f16x8 *)(o + 512), xh[kb], xl[kb]);
        }
        join_halves(acc, low);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] = acc[r] * kDown;
      }
    }
    __syncthreads();                                       // (B and the parts are read no more)
  }
  const float step = p.step * sqrtf((float)n) * kDown;
  if (!EARLY) {
    asm volatile("" : "+v"(first), "+v"(rows), "+v"(cols));   // (indices made anew, not kept in registers since the start)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int k = at(b, r);
        old[b][r] = w[k >= 0 ? k : 0];
      }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (q.t) reorder(x[b], true);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int k = at(b, r);
      if (k >= 0) w[k] = p.decay * old[b][r] - step * x[b][r];
    }
  }
}

int64_t put_blocks(Mat &q, int64_t first, int64_t blocks) {
  q.first = (int)first;
  q.blocks = (int)blocks;
  return first + blocks;
}
int all_blocks(const MuonArgs &p) { return p.mat[p.count - 1].first + p.mat[p.count - 1].blocks; }

// The blocks of product `step` of all matrices, in p: tiles of 128 x 128 where they fill the chip, else of 64 x 64; a sum that is long beside what each
// compute unit has to do is cut into parts. Returns the tile's size.
int plan_product(MuonArgs &p, int step, int n_cu) {
  const bool half = step == STEP_GRAM || step == STEP_POLY;
  auto sum_length = [&](int k) { return (int64_t)((step == STEP_GRAM ? p.mat[k].n : p.mat[k].m) + kTile - 1) / kTile * kTile; };
  auto tiles = [&](int k, int T) {
    const int64_t th = (p.mat[k].m + T - 1) / T, tw = (p.mat[k].n + T - 1) / T;
    return half ? th * (th + 1) / 2 : th * tw;
  };
  int64_t wide = 0, work = 0;
  for (int k = 0; k < p.count; ++k) wide += tiles(k, 128);
  // us a call, all products in tiles of 64 / of 128: four 2048^2 2756 / 2404, one 776 / 751 (each as it fits 718), 1500^2 393 / 555, 1024^2 184 / 390
  const int T = wide >= n_cu ? 128 : 64;
  for (int k = 0; k < p.count; ++k) work += tiles(k, T) * sum_length(k);
  // What cutting costs, laying down and adding up, is 2 to 4 us; 64 of a sum take a lone block of 64 x 64 0.8 us. A call of one step
  // of a 1 x 2342 matrix 36 / 26 us, of 2859 x 89 44 / 30. (Tiles of 128 x 128 are cut nowhere: X X^T of 2048 x 8192, three parts, 336 / 392.)
  const int64_t least = std::max<int64_t>(384, work / n_cu);
  int64_t at = 0;
  for (int k = 0; k < p.count; ++k) {
    p.mat[k].parts = half && T == 64 ? (int)std::min<int64_t>(16, std::max<int64_t>(1, sum_length(k) / least)) : 1;
    Mat &q = p.mat[k];
    const int64_t stages = sum_length(k) / 32, per = (stages + q.parts - 1) / q.parts;
    q.parts = (int)((stages + per - 1) / per);             // none is empty
    at = put_blocks(q, at, tiles(k, T) * q.parts);
  }
  return T;
}

// An XCD's share of the blocks is an eighth of the work, in the order of the matrices: a small matrix is one XCD's in all products of a step, a large
// one is cut into few pieces. us a call so / dealt to the XCDs in turn: eight matrices of 256 x 256 and 256 x 512 119 / 123, two 2048^2 and two 2048 x 8192
// 4937 / 5126. Returns the blocks of the launch.
int deal_blocks(MuonArgs &p, int step) {
  constexpr int kFixed = 256;                              // what a block costs beside its products, as a sum's length
  int64_t work = 0, done = 0;
  auto length = [&](int k) { return (int64_t)(step == STEP_GRAM ? p.mat[k].n : p.mat[k].m) / p.mat[k].parts + kFixed; };
  for (int k = 0; k < p.count; ++k) work += p.mat[k].blocks * length(k);
  int x = 1, most = 0;
  for (int k = 0; k < p.count; ++k) {
    const int64_t blocks = p.mat[k].blocks, each = length(k);
    for (; x < 8; ++x) {                                   // share x ends inside matrix k
      const int64_t n = std::max<int64_t>(0, (work * x / 8 - done + each / 2) / each);
      if (n > blocks) break;
      p.share[x] = p.mat[k].first + (int)n;
    }
    done += blocks * each;
  }
  p.share[0] = 0;
  for (; x <= 8; ++x) p.share[x] = all_blocks(p);
  for (int s = 0; s < 8; ++s) most = std::max(most, p.share[s + 1] - p.share[s]);
  return most * 8;
}

template <int STEP>
int launch_product(const xrl_ctx *c, MuonArgs &p) {
  const int T = plan_product(p, STEP, op_compute_units(c));
  const dim3 grid((unsigned)deal_blocks(p, STEP)), block(256);
  if (T == 128) muon_product_kernel<STEP, 128, 2><<<grid, block, 2 * 32 * 1024, op_stream(c)>>>(p);
  else muon_product_kernel<STEP, 64, 3><<<grid, block, 3 * 16 * 1024, op_stream(c)>>>(p);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

template <int WAVES>
int launch_small(const xrl_ctx *c, MuonArgs &p, int steps) {
  static const hipError_t allowed =
      hipFuncSetAttribute((const void *)muon_small_kernel<WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, small_lds(WAVES));
  if (allowed != hipSuccess) return fail(XRL_ERR_HIP, "xrl_muon_step: %d bytes of LDS: %s", small_lds(WAVES), hipGetErrorString(allowed));
  for (int k = 0; k < p.count; ++k) put_blocks(p.mat[k], k, 1);
  muon_small_kernel<WAVES><<<dim3((unsigned)p.count), dim3(WAVES * 64), small_lds(WAVES), op_stream(c)>>>(p, steps);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}

int run_group(xrl_ctx *c, MuonArgs &p, int steps) {
  int rows = 0, cols = 0;
  for (int k = 0; k < p.count; ++k) {
    rows = std::max(rows, p.mat[k].m);
    cols = std::max(cols, p.mat[k].n);
  }
  // us a call of five steps, in launches of their own / a block each of eight waves / of sixteen: 64 x 64 54 / 21 / 26, 64 x 256 65 / 29 / 34, ten of 64 x 128
  // 62 / 24 / 28; 64 x 512 74 / - / 47
  if (rows <= kSmallRows && cols <= 256) return launch_small<8>(c, p, steps);
  if (rows <= kSmallRows && cols <= 512) return launch_small<16>(c, p, steps);
  int64_t at = 0;
  for (int k = 0; k < p.count; ++k) {
    Mat &q = p.mat[k];
    q.first_sum = (int)at;                                 // (one partial sum a block)
    at = put_blocks(q, at, ((int64_t)q.m * q.n + q.chunk - 1) / q.chunk);
  }
  muon_momentum_kernel<<<dim3((unsigned)all_blocks(p)), dim3(256), 0, op_stream(c)>>>(p);
  at = 0;
  for (int k = 0; k < p.count; ++k) at = put_blocks(p.mat[k], at, (int64_t)((p.mat[k].m + kTile - 1) / kTile) * ((p.mat[k].n + kTile - 1) / kTile));
  muon_begin_kernel<<<dim3((unsigned)all_blocks(p)), dim3(256), 0, op_stream(c)>>>(p);
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
    // the longest sums first, so that a launch does not end with them
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) {
      return std::max(matrices[x].rows, matrices[x].cols) > std::max(matrices[y].rows, matrices[y].cols);
    });
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
  // Groups run one after another in the same workspace: operands, sums of squares, parts of sums and their counters
  std::vector<MuonArgs> groups;
  size_t most = 0, floats = 0, counters = 0;
  try {
    for (size_t i = 0; i < list.size();) {
      MuonArgs p = {};
      int64_t halves = 0;
      while (p.count < kGroup && i < list.size()) {
        Mat q = list[i];
        const int64_t more = 3 * x_halves(q.m, q.n) + 2 * x_halves(q.m, q.m);
        if (p.count > 0 && halves + more > kGroupHalves) break;
        q.ws = halves;
        halves += more;
        p.mat[p.count++] = q;
        ++i;
      }
      most = std::max(most, (size_t)halves * 2);
      for (int step : {STEP_GRAM, STEP_POLY}) {
        const int T = plan_product(p, step, op_compute_units(c));
        bool cut = false;
        for (int k = 0; k < p.count; ++k) cut = cut || p.mat[k].parts > 1;
        if (!cut) continue;
        counters = std::max(counters, (size_t)all_blocks(p));
        floats = std::max(floats, (size_t)all_blocks(p) * T * T);
      }
      groups.push_back(p);
    }
  } catch (const std::bad_alloc &) {
    return fail(XRL_ERR_OOM, "%s: out of host memory", who);
  }
  const size_t o_sums = op_align(most), o_part = o_sums + op_align((size_t)kGroup * kMaxSums * 8), o_count = o_part + op_align(floats * 4);
  char *ws = nullptr;
  if (int rc = op_workspace(c, o_count + counters * 4, &ws, who)) return rc;
  for (MuonArgs &p : groups) {
    p.w = d_weights; p.mom = d_momentum; p.g = d_grads;
    p.ws = (_Float16 *)ws; p.sums = (double *)(ws + o_sums);
    p.partial = (float *)(ws + o_part); p.arrived = (int *)(ws + o_count); p.n_arrived = (int)counters;
    p.mu = desc->momentum; p.decay = 1.f - desc->lr * desc->weight_decay; p.step = desc->lr * desc->rms; p.nesterov = desc->nesterov != 0;
    if (int rc = run_group(c, p, desc->steps)) return rc;
  }
  return XRL_OK;
}

}  // extern "C"
