// Attention over packed sequences.
//
// Per sequence and head, s_ij = scale q_i . k_j over the keys j that row i sees, p = softmax of a row, o_i = sum_j p_ij v_j. Scores are computed in tiles of
// 32 x 32 on the matrix cores and never stored: a row's maximum and sum run along. An accumulator tile has one query a lane and keys in its registers, so maxima and sums are taken over
// a lane's own registers, and these are the other operand of the second product as they lie (Tile::across reads the values in the same order). In bf16 the exponentials are rounded to it as that
// operand, half a step of 2^-8 of each: the products of two bf16 numbers are exact, sums and everything else in fp32.
//
// Bound by the matrix cores, and by the exponentials and maxima between their products: 8192 causal rows of 32 heads of 128 in bf16 run 600 us, 916 TFLOP/s of the 4 dim operations a seen pair (a
// library product of 4096^3 reaches 1085); 16 sequences of 330 to 3300 rows with 16 heads of 64 95 us, 625 TFLOP/s. The matrix cores
// are busy for 47 % of the first one's cycles, at 1.8 GHz, the LDS as long. A block of four waves shares the keys' tiles, which come straight into LDS while the
// last ones are worked on.
#include "attn_packed.hip.h"

#include <type_traits>

namespace {

// One block: BM = 32 WAVES rows of one sequence (MIXED: of whatever sequences) and one head, KT keys at a time.
template <typename T, int DP, int WAVES, int KT, bool MIXED>
__global__ __launch_bounds__(WAVES * 64, WAVES == 1 || DP * sizeof(T) > 256 ? 1 : 2) void attention_kernel(const AttnArgs a) {
  using L = Tile<T, DP>;
  using vec = typename L::vec;
  constexpr int BYTES = KT * L::RB, BUFS = kBuffers<WAVES>;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFS * BYTES];
  touch_args(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  Queries w;
  if (!queries_of<WAVES, MIXED>(a, wave, lane, w)) return;
  const int kv = w.head / (a.q_heads / a.kv_heads), keys = w.keys, tiles = (keys + KT - 1) / KT;
  vec q[L::SLABS];
  load_row<T, DP>(q, head_at<T>(a.q, w.row, w.head), w.there, a.dim_in, g);
  const T *k = head_at<T>(a.k, w.key0, kv), *v = head_at<T>(a.v, w.key0, kv);
  const unsigned base = lds_address(lds);
  const float c = a.scale * kLog2e;
  float mc, l;
  auto pass = [&](auto safe, auto &o, int db0) {
    constexpr bool SAFE = decltype(safe)::value;
    mc = kLowest;
    l = 0.f;
    for (auto &x : o) x = zero_acc();
    auto stage = [&](int t) {
      const int64_t j = (int64_t)t * KT;
      const unsigned to = base + t % BUFS * BYTES;
      stage_tile<T, DP, KT, WAVES>(k + j * a.k.stride, keys - (int)j, a.k.stride, a.dim_in, to, wave, lane);
      stage_tile<T, DP, KT, WAVES>(v + j * a.v.stride, keys - (int)j, a.v.stride, a.dim_in, to + BUFS * BYTES, wave, lane);
    };
    if (tiles > 0) stage(0);
    for (int t = 0; t < tiles; ++t) {
      if (MIXED && !__ballot(w.from < t * KT + KT && w.mine > t * KT)) continue;   // (a sequence without queries)
      const unsigned kt = base + t % BUFS * BYTES, vt = kt + BUFS * BYTES;
      if (BUFS == 1 && t > 0) {
        __syncthreads();
        stage(t);
      }
      wait_direct_loads();
      __syncthreads();                              // tile t is there, and t - 1 is read
      if (BUFS == 2 && t + 1 < tiles) stage(t + 1);
      const int j0 = t * KT;
      if (j0 >= w.any_sees) continue;
      const int from = w.from - j0 - 4 * g, mine = w.mine - j0 - 4 * g;
      add_tile<T, DP, KT, SAFE>(kt, vt, q, c, (!MIXED || j0 >= w.all_from) && j0 + KT <= w.all_see, [&](int n) { return n < mine && (!MIXED || n >= from); }, o, mc, l, lane, db0);
    }
    l = half_sum(l);
    store_row<T>(head_at<T>(a.out, w.row, w.head), w.there, a.dim, a.quads, o, l == 0.f ? 0.f : 1.f / l, g, db0);
  };
  f32x16 o[L::BLOCKS];
  pass(std::false_type(), o, 0);
  if (w.there && g == 0) a.lse[w.row * a.q_heads + w.head] = l == 0.f ? -INFINITY : mc * kLn2 + logf(l);
  if (!MIXED && !a.causal) return;
  bool fine = true;
#pragma unroll
  for (int db = 0; db < L::BLOCKS; ++db) fine = fine && all_finite(o[db]);
  if (!__syncthreads_or(!fine)) return;
#pragma unroll 1
  for (int db = 0; db < L::BLOCKS; ++db) {
    __syncthreads();                                // (the last tiles are read)
    f32x16 one[1];
    pass(std::true_type(), one, db);
  }
}

template <typename T, int DP>
void launch(const xrl_ctx *c, AttnArgs &a) {
  // Keys at a time, 32 and 64, us: 8192 rows of 32 heads of 128 in bf16 749 and 680 on one machine, 16 sequences with heads of 64 95 and 99, 16 of 500 rows in fp32, heads of 64, 66 and 68.
  constexpr int KT = sizeof(T) == 2 ? 64 : 32;
  if (mixes(a)) launch_mixed(c, a, attention_kernel<T, DP, 1, 32, true>, a.n_q, a.q_heads);
  else if (few_rows(a, a.n_q)) launch_tiles(c, a, attention_kernel<T, DP, 1, 32, false>, a.n_q, a.q_heads, 32, 64);
  else launch_tiles(c, a, attention_kernel<T, DP, 4, KT, false>, a.n_q, a.q_heads, 128, 256);
}
template <typename T>
void launch_dim(const xrl_ctx *c, AttnArgs &a) {
  a.dim <= 32 ? launch<T, 32>(c, a) : a.dim <= 64 ? launch<T, 64>(c, a) : launch<T, 128>(c, a);
}

}  // namespace

extern "C" int xrl_attention(xrl_ctx *c, const xrl_attention_desc *d, const xrl_heads *q, const xrl_heads *k, const xrl_heads *v, const xrl_heads *out, float *d_lse) {
  const char *who = "xrl_attention";
  AttnArgs a;
  if (int rc = check_attention(c, d, who, a)) return rc;
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4;
  if (int rc = check_heads(q, d->n_q, d->q_heads, d->dim, es, "q", who, a.q)) return rc;
  if (int rc = check_heads(k, d->n_k, d->kv_heads, d->dim, es, "k", who, a.k)) return rc;
  if (int rc = check_heads(v, d->n_k, d->kv_heads, d->dim, es, "v", who, a.v)) return rc;
  if (int rc = check_heads(out, d->n_q, d->q_heads, d->dim, es, "out", who, a.out, &a.quads)) return rc;
  if (d->n_q > 0 && !d_lse) return fail(XRL_ERR_NULL, "%s: d_lse is NULL", who);
  if ((uintptr_t)d_lse % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  if (d->n_q == 0 || d->n_seqs == 0) return XRL_OK;
  a.lse = d_lse;
  Inputs in(d->type, d->dim);
  in.add(a.q, d->n_q, d->q_heads);
  in.add(a.k, d->n_k, d->kv_heads);
  in.add(a.v, d->n_k, d->kv_heads);
  if (in.count) {
    char *ws = nullptr;
    if (int rc = op_workspace(c, in.bytes, &ws, who)) return rc;
    in.copy(c, ws);
  }
  a.dim_in = in.dim_in;
  d->type == XRL_PREC_BF16 ? launch_dim<bf16_t>(c, a) : launch_dim<float>(c, a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}
