// Gradients of attention over packed sequences.
//
// With p from the forward pass's lse and D_i = dout_i . out_i: ds_ij = p_ij (dout_i . v_j - D_i), dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij dout_i. Two kernels, each
// of which computes the scores anew: one has a query a lane and sums over keys, the other a key a lane and sums over queries. That is seven products where one kernel
// would do with five, but no sum is shared by blocks: no float atomics, the same bits from run to run. (bf16: an eighth for the rests of ds, see below.)
//
// Bound by the matrix cores and what feeds them from LDS, each score tile's exponentials between. Two causal sequences of 4096, 32 heads of 128 in bf16: dq 553 to 602 us, dk and dv 672 to
// 736, that is 820 to 900 TFLOP/s of the eight products, the matrix cores busy for 52 and 40 % of the cycles, the LDS for 39 and 65; 16 sequences of 330 to 3300 rows, 16 heads of 64: 169 to 179 and 241 to 256. p and ds are rounded to bf16 as factors of dv and dk, half a step of 2^-8 each.
#include "attn_packed.hip.h"

#include <type_traits>

namespace {

// dq, and of every row what the keys' gradients need besides: lse log2(e) and D. Rows and tiles as in the forward kernel.
//
// bf16: ds is a difference of nearly equal numbers, and rounding it once to the products' 8 bits would cost dq 1.8e-3 of its size, as much as dq's own rounding. So its rest, ds - bf16(ds), is a
// second operand of the same product. D from the rounded out is off as well, by delta_i = sum_j ds_ij, as sum_j p_ij = 1: the keys' gradients take D + delta. For dq, whose sums run before delta is
// known, a pass over the keys takes D = sum_j p_ij (dout_i . v_j) first, where a block has at most kExact of them: what the rounded out does to a row's dq falls as the number of
// keys that it spreads over grows, and the pass would cost half of the kernel's time again.
// Relative errors of dq, a result's rounding alone being 1.66e-3, without any of this, with the rests, and with the pass up to 512 keys, 1024 and all: two sequences of 4096 with heads of 128 2.69e-3,
// 2.08e-3, 1.90e-3, 1.82e-3, 1.66e-3 in 1133, 1200, 1247, 1270 and 1544 us (with dk and dv); 16 episodes of 330 to 3300 with heads of 64 2.90e-3, 2.32e-3, 1.87e-3, 1.75e-3, 1.66e-3; sequences of
// 1 to 24 up to 3.6e-3 without the pass. dk: 2.7e-3, and 2.3e-3 with D + delta (its own rests: 1.7e-3 and 9 % more; left out).
constexpr int kExact = 512;
template <typename T, int DP, int WAVES, int KT, bool MIXED>
__global__ __launch_bounds__(WAVES * 64, 1) void attention_dq_kernel(const AttnArgs a) {
  using L = Tile<T, DP>;
  using vec = typename L::vec;
  constexpr int BYTES = KT * L::RB, BUFS = kBuffers<WAVES>;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFS * BYTES];
  touch_args(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  Queries w;
  if (!queries_of<WAVES, MIXED>(a, wave, lane, w)) return;
  const int kv = w.head / (a.q_heads / a.kv_heads), keys = w.keys, tiles = (keys + KT - 1) / KT;
  vec q[L::SLABS], dout[L::SLABS];
  float delta = 0.f;
  {
    load_row<T, DP>(q, head_at<T>(a.out, w.row, w.head), w.there, a.dim_in, g);
    load_row<T, DP>(dout, head_at<T>(a.dout, w.row, w.head), w.there, a.dim_in, g);
#pragma unroll
    for (int x = 0; x < L::SLABS; ++x)
#pragma unroll
      for (int j = 0; j < L::V; ++j) delta = fmaf((float)q[x][j], (float)dout[x][j], delta);
    delta = half_sum(delta);
  }
  load_row<T, DP>(q, head_at<T>(a.q, w.row, w.head), w.there, a.dim_in, g);
  // (a row without keys, or with scores of -inf alone: every exponential below is 0)
  const float lse = a.lse[w.row * a.q_heads + w.head], lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
  if (w.there && g == 0) a.stat_lse[w.head * a.n_q + w.row] = lse2;
  const T *k = head_at<T>(a.k, w.key0, kv), *v = head_at<T>(a.v, w.key0, kv);
  const unsigned base = lds_address(lds);
  const float c = a.scale * kLog2e;
  constexpr bool REST = sizeof(T) == 2;
  // f(tiles of keys and values, first key, whether all rows of the wave see all of it, whether this lane's row sees its key n + 4 g)
  auto over_keys = [&](auto f) {
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
      f(kt, vt, (!MIXED || j0 >= w.all_from) && j0 + KT <= w.all_see, [&](int n) { return n < mine && (!MIXED || n >= from); });
    }
  };
  // scores, and dout . v, of 32 keys
  auto products = [&](unsigned kt, unsigned vt, int kb, f32x16 &s, f32x16 &dp) {
    s = zero_acc();
    dp = zero_acc();
#pragma unroll
    for (int x = 0; x < L::SLABS; ++x) {
      Operand<T>::mma(L::along(kt, 32 * kb, x, lane), q[x], s);
      Operand<T>::mma(L::along(vt, 32 * kb, x, lane), dout[x], dp);
    }
  };
  if (REST && keys <= kExact) {
    float sum = 0.f;
    over_keys([&](unsigned kt, unsigned vt, bool whole, auto sees) {
#pragma unroll
      for (int kb = 0; kb < KT / 32; ++kb) {
        f32x16 s, dp;
        products(kt, vt, kb, s, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * dp[r];
          sum += whole || sees(32 * kb + acc_row(r, 0)) ? x : 0.f;
        }
      }
    });
    delta = half_sum(sum);
    __syncthreads();                                // (the last tiles are read)
  }
  float more = 0.f;
  auto pass = [&](auto safe, auto &dq, int db0) {
    constexpr bool SAFE = decltype(safe)::value;
    constexpr int NB = sizeof(dq) / sizeof(f32x16);
    for (auto &x : dq) x = zero_acc();
    over_keys([&](unsigned kt, unsigned vt, bool whole, auto sees) {
#pragma unroll
      for (int kb = 0; kb < KT / 32; ++kb) {
        f32x16 s, dp;
        products(kt, vt, kb, s, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * (dp[r] - delta);
        if (!whole) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = sees(32 * kb + acc_row(r, 0)) ? s[r] : 0.f;
        }
        if (REST && !SAFE) {
#pragma unroll
          for (int r = 0; r < 16; ++r) more += s[r];
        }
#pragma unroll
        for (int x = 0; x < 32 / L::STEP; ++x) {
          const vec ds = acc_operand<T>(s, x), rest = acc_rest<T>(s, x, ds);
          if (SAFE && !whole) {
            vec seen;
#pragma unroll
            for (int n = 0; n < L::V; ++n) seen[n] = (T)(sees(32 * kb + acc_row(x * L::V + n, 0)) ? 1.f : 0.f);
#pragma unroll
            for (int db = 0; db < NB; ++db) {
              const vec key = L::across(kt, 32 * kb + x * L::STEP, db0 + db, lane);
              mma_seen<T>(key, ds, seen, dq[db]);
              if (REST) mma_seen<T>(key, rest, seen, dq[db]);
            }
          } else {
#pragma unroll
            for (int db = 0; db < NB; ++db) {
              const vec key = L::across(kt, 32 * kb + x * L::STEP, db0 + db, lane);
              Operand<T>::mma(key, ds, dq[db]);
              if (REST) Operand<T>::mma(key, rest, dq[db]);
            }
          }
        }
      }
    });
    store_row<T>(head_at<T>(a.dq, w.row, w.head), w.there, a.dim, a.quads, dq, a.scale, g, db0);
  };
  f32x16 dq[L::BLOCKS];
  pass(std::false_type(), dq, 0);
  more = half_sum(more);
  if (w.there && g == 0) a.stat_delta[w.head * a.n_q + w.row] = delta + more;
  if (!MIXED && !a.causal) return;
  bool fine = true;
#pragma unroll
  for (int db = 0; db < L::BLOCKS; ++db) fine = fine && all_finite(dq[db]);
  if (!__syncthreads_or(!fine)) return;
#pragma unroll 1
  for (int db = 0; db < L::BLOCKS; ++db) {
    __syncthreads();
    f32x16 one[1];
    pass(std::true_type(), one, db);
  }
}

// n floats from p on into LDS, past the registers, zeros behind them (n at most 64; wave-uniform).
__device__ __forceinline__ void stage_floats(const float *p, int n, unsigned lds, int lane) {
  const u32x4 rows = rows_descriptor(p, n > 0 ? n * 4u : 0u);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(lane * 4), "s"(rows), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
#pragma clang diagnostic pop
}

// A lane's key, and the rows of queries that its block goes over: `rows` of them from row row0 of their tensor on, from the multiple `begin` of QT on. Rows [mine, end) see the
// key, rows [all_see, all_end) all keys of the wave, and rows below any_sees none. A block's keys are key0 + j0 on, of `keys` from key0 on.
struct Keys {
  int head;
  int64_t row, row0, key0;
  bool there;
  int j0, keys, rows, begin, mine, end, any_sees, all_see, all_end;
};
template <int WAVES, bool MIXED>
__device__ __forceinline__ bool keys_of(const AttnArgs &a, int qt, int wave, int lane, Keys &o) {
  constexpr int BM = 32 * WAVES;
  if constexpr (MIXED) {
    static_assert(WAVES == 1);
    const int64_t b = a.block0 + blockIdx.x, tile = b / a.kv_heads;
    const Meets x = meets_of(a, a.k_ptr, a.n_k, a.q_ptr, a.n_q, true, tile, lane);
    o.head = (int)(b % a.kv_heads);
    o.there = x.there;
    o.row = x.there ? 32 * tile + (lane & 31) : 0;
    o.row0 = x.first;
    o.key0 = 32 * tile;
    o.j0 = 0;
    o.keys = a.n_k - o.key0 < 32 ? (int)(a.n_k - o.key0) : 32;
    o.rows = __builtin_amdgcn_readfirstlane(x.last - x.first);
    o.begin = o.any_sees = 0;
    o.mine = x.lo - x.first;
    o.end = x.hi - x.first;
    o.all_see = x.all_lo - x.first;
    o.all_end = x.all_hi - x.first;
    return true;
  } else {
    Place at;
    if (!place_of(a, a.k_ptr, a.n_k, a.kv_heads, BM, false, lane, at)) return false;
    const Span qs = span_of(a.q_ptr, at.seq, a.n_q), ks = span_of(a.k_ptr, at.seq, a.n_k);
    o.j0 = __builtin_amdgcn_readfirstlane(at.tile < (ks.len + BM - 1) / BM ? at.tile * BM : -1);
    if (o.j0 < 0) return false;
    const int len_q = __builtin_amdgcn_readfirstlane(qs.len), off = __builtin_amdgcn_readfirstlane(ks.len - qs.len);
    const int w0 = o.j0 + 32 * wave, j = w0 + (lane & 31);
    // the first row that sees a key
    auto first_of = [&](int j) { const int i = a.causal ? j - off : 0; return i < 0 ? 0 : i < len_q ? i : len_q; };
    o.head = at.head;
    o.there = j < ks.len;
    o.row = ks.begin + (o.there ? j : 0);
    o.row0 = qs.begin;
    o.key0 = ks.begin;
    o.keys = ks.len;
    o.rows = len_q;
    o.begin = __builtin_amdgcn_readfirstlane(first_of(o.j0)) / qt * qt;
    o.any_sees = __builtin_amdgcn_readfirstlane(first_of(w0));
    o.all_see = __builtin_amdgcn_readfirstlane(first_of(w0 + 31));
    o.mine = first_of(j);
    o.end = o.all_end = len_q;
    return true;
  }
}

// dk and dv: one block has 32 WAVES keys of one sequence and one head of keys, a key a lane, and goes over the queries that see them, QT rows at a time, of all
// heads that share the keys, in order. HALVES: so many times WAVES waves each go over their part of these queries, and their sums are added at the end, in order: no sum is taken
// by two blocks. IN_LDS: the block's keys and values stay in LDS, where registers for them as well would leave one wave a SIMD. (Halves, IN_LDS and the order of
// place_of together: 2230 to 1445 us of two sequences of 4096, forward and backward.)
template <typename T, int DP, int WAVES, int QT, int HALVES, bool IN_LDS, bool DK, bool DV, bool MIXED>
__global__ __launch_bounds__(HALVES * WAVES * 64, HALVES) void attention_dkv_kernel(const AttnArgs a) {
  using L = Tile<T, DP>;
  using vec = typename L::vec;
  constexpr int BM = 32 * WAVES, BYTES = QT * L::RB, BUFS = kBuffers<WAVES>, EACH = 2 * BUFS * (BYTES + 256), SUMS = BM * DP * 4;   // of a half: two tiles of q and of dout, and the rows' statistics
  constexpr int KEYS = IN_LDS ? 2 * BM * L::RB : 0, ALL = HALVES * EACH + KEYS, JOIN = HALVES > 1 ? (DK + DV) * SUMS : 0;
  __shared__ __attribute__((aligned(16))) char lds[ALL > JOIN ? ALL : JOIN];
  touch_args(a);
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int half = HALVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES : 0, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WAVES;
  Keys w;
  if (!keys_of<WAVES, MIXED>(a, QT, wave, lane, w)) return;
  const int group = a.q_heads / a.kv_heads, len_q = w.rows, begin = w.begin, j0 = w.j0;
  const bool there = w.there;
  const int per_head = (len_q - begin + QT - 1) / QT, all_tiles = per_head * group, share = (all_tiles + HALVES - 1) / HALVES;
  const int first = half * share, tiles = first < all_tiles ? (all_tiles - first < share ? all_tiles - first : share) : 0;   // of this half
  vec k[L::SLABS], v[L::SLABS];
  const unsigned base = lds_address(lds) + half * EACH, stats = base + 2 * BUFS * BYTES, keys = lds_address(lds) + HALVES * EACH, values = keys + BM * L::RB;
  if constexpr (!IN_LDS) {
    load_row<T, DP>(k, head_at<T>(a.k, w.row, w.head), there, a.dim_in, g);
    if (DK) load_row<T, DP>(v, head_at<T>(a.v, w.row, w.head), there, a.dim_in, g);
  }
  const float c = a.scale * kLog2e;
  auto stage = [&](int e, int i, int b) {             // rows i on of the group's head e
    const int head = w.head * group + e;
    const int64_t row = w.row0 + i;
    stage_tile<T, DP, QT, WAVES>(head_at<T>(a.q, row, head), len_q - i, a.q.stride, a.dim_in, base + b * BYTES, wave, lane);
    stage_tile<T, DP, QT, WAVES>(head_at<T>(a.dout, row, head), len_q - i, a.dout.stride, a.dim_in, base + (BUFS + b) * BYTES, wave, lane);
    const int n = len_q - i < QT ? len_q - i : QT;
    if (wave == 0) stage_floats(a.stat_lse + head * a.n_q + row, n, stats + b * 512, lane);
    if (DK && wave == WAVES - 1) stage_floats(a.stat_delta + head * a.n_q + row, n, stats + b * 512 + 256, lane);
  };
  auto pass = [&](auto safe, auto &dk, auto &dv, int db0) {
    constexpr bool SAFE = decltype(safe)::value;
    constexpr int NB = sizeof(dk) / sizeof(f32x16);
    for (auto &x : dk) x = zero_acc();
    for (auto &x : dv) x = zero_acc();
    const int e0 = per_head > 0 ? first / per_head : 0;
    int next_e = e0, next_i = begin + (first - e0 * per_head) * QT, i = next_i;
    // (without queries nothing is read, and no step below would wait for these loads before the sums go to the places that they write)
    if (IN_LDS && share > 0) {
      stage_tile<T, DP, BM, HALVES * WAVES>(head_at<T>(a.k, w.key0 + j0, w.head), w.keys - j0, a.k.stride, a.dim_in, keys, half * WAVES + wave, lane);
      if (DK) stage_tile<T, DP, BM, HALVES * WAVES>(head_at<T>(a.v, w.key0 + j0, w.head), w.keys - j0, a.v.stride, a.dim_in, values, half * WAVES + wave, lane);
    }
    if (tiles > 0) stage(next_e, next_i, 0);
    for (int t = 0; t < share; ++t) {
      const unsigned qt = base + t % BUFS * BYTES, dt = qt + BUFS * BYTES, st = stats + t % BUFS * 512;
      const int e = next_e;
      i = next_i;
      next_i += QT;
      if (next_i >= len_q) {
        next_i = begin;
        ++next_e;
      }
      if (MIXED && !__ballot(w.mine < i + QT && w.end > i)) continue;   // (a sequence without keys)
      if (BUFS == 1 && t > 0) {
        __syncthreads();
        stage(e, i, 0);
      }
      wait_direct_loads();
      __syncthreads();
      if (BUFS == 2 && t + 1 < tiles) stage(next_e, next_i, (t + 1) & 1);
      if (t >= tiles || i + QT <= w.any_sees) continue;
      const bool whole = i >= w.all_see && i + QT <= (MIXED ? w.all_end : len_q);
      f32x16 s[QT / 32], dp[QT / 32];
#pragma unroll
      for (int qb = 0; qb < QT / 32; ++qb) {
        s[qb] = zero_acc();
        dp[qb] = zero_acc();
#pragma unroll
        for (int x = 0; x < L::SLABS; ++x) {
          Operand<T>::mma(L::along(qt, 32 * qb, x, lane), IN_LDS ? L::along(keys, 32 * wave, x, lane) : k[x], s[qb]);
          if (DK) Operand<T>::mma(L::along(dt, 32 * qb, x, lane), IN_LDS ? L::along(values, 32 * wave, x, lane) : v[x], dp[qb]);
        }
      }
#pragma unroll
      for (int qb = 0; qb < QT / 32; ++qb) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const unsigned at_row = st + (32 * qb + 8 * n + 4 * g) * 4;
          const f32x4 lse2 = *lds_at<const f32x4>(at_row), delta = *lds_at<const f32x4>(at_row + 256);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[qb][4 * n + r], c, -lse2[r]));
            s[qb][4 * n + r] = p;
            if (DK) dp[qb][4 * n + r] = p * (dp[qb][4 * n + r] - delta[r]);
          }
        }
        auto counts = [&](int r) { const int n = 32 * qb + acc_row(r, 0); return n >= w.mine - i - 4 * g && n < (MIXED ? w.end : len_q) - i - 4 * g; };
        if (!whole) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[qb][r] = counts(r) ? s[qb][r] : 0.f;
            if (DK) dp[qb][r] = counts(r) ? dp[qb][r] : 0.f;
          }
        }
#pragma unroll
        for (int x = 0; x < 32 / L::STEP; ++x) {
          const vec p = acc_operand<T>(s[qb], x), ds = acc_operand<T>(dp[qb], x);
          if (SAFE && !whole) {
            vec seen;
#pragma unroll
            for (int n = 0; n < L::V; ++n) seen[n] = (T)(counts(x * L::V + n) ? 1.f : 0.f);
#pragma unroll
            for (int db = 0; db < NB; ++db) {
              if (DV) mma_seen<T>(L::across(dt, 32 * qb + x * L::STEP, db0 + db, lane), p, seen, dv[db]);
              if (DK) mma_seen<T>(L::across(qt, 32 * qb + x * L::STEP, db0 + db, lane), ds, seen, dk[db]);
            }
          } else {
#pragma unroll
            for (int db = 0; db < NB; ++db) {
              if (DV) Operand<T>::mma(L::across(dt, 32 * qb + x * L::STEP, db0 + db, lane), p, dv[db]);
              if (DK) Operand<T>::mma(L::across(qt, 32 * qb + x * L::STEP, db0 + db, lane), ds, dk[db]);
            }
          }
        }
      }
    }
    if constexpr (HALVES > 1) {
      // the second half's sums through LDS to the first
      static_assert(HALVES == 2);
      const unsigned at_dk = lds_address(lds) + (unsigned)(wave * 64 + lane) * 16, at_dv = at_dk + (DK ? SUMS : 0);
      auto exchange = [&](unsigned p, auto &x) {
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            auto *to = lds_at<f32x4>(p + (unsigned)((db * 4 + n) * WAVES * 64 * 16));
            if (half) {
              *to = f32x4{x[db][4 * n], x[db][4 * n + 1], x[db][4 * n + 2], x[db][4 * n + 3]};
            } else {
              const f32x4 y = *to;
#pragma unroll
              for (int r = 0; r < 4; ++r) x[db][4 * n + r] += y[r];
            }
          }
      };
      __syncthreads();                              // (the last tiles are read)
      if (half) {
        if (DK) exchange(at_dk, dk);
        if (DV) exchange(at_dv, dv);
      }
      __syncthreads();
      if (!half) {
        if (DK) exchange(at_dk, dk);
        if (DV) exchange(at_dv, dv);
      }
    }
    if (half) return;
    if (DK) store_row<T>(head_at<T>(a.dk, w.row, w.head), there, a.dim, a.quads, dk, a.scale, g, db0);
    if (DV) store_row<T>(head_at<T>(a.dv, w.row, w.head), there, a.dim, a.quads, dv, 1.f, g, db0);
  };
  f32x16 dk[L::BLOCKS], dv[L::BLOCKS];
  pass(std::false_type(), dk, dv, 0);
  if (!MIXED && !a.causal) return;
  bool fine = true;
#pragma unroll
  for (int db = 0; db < L::BLOCKS; ++db) fine = fine && (!DK || all_finite(dk[db])) && (!DV || all_finite(dv[db]));
  if (!__syncthreads_or(!fine)) return;
#pragma unroll 1
  for (int db = 0; db < L::BLOCKS; ++db) {
    __syncthreads();
    f32x16 one[1], two[1];
    pass(std::true_type(), one, two, db);
  }
}

template <typename T, int DP>
void launch(const xrl_ctx *c, AttnArgs &a) {
  if (mixes(a)) launch_mixed(c, a, attention_dq_kernel<T, DP, 1, 32, true>, a.n_q, a.q_heads);
  else if (few_rows(a, a.n_q)) launch_tiles(c, a, attention_dq_kernel<T, DP, 1, 32, false>, a.n_q, a.q_heads, 32, 64);
  else launch_tiles(c, a, attention_dq_kernel<T, DP, 4, 32, false>, a.n_q, a.q_heads, 128, 256);
  // One launch for both where both sums fit in the registers with their operands, else one for each, which computes the scores once more.
  constexpr bool BOTH = DP * sizeof(T) <= 256, BF16 = sizeof(T) == 2;
  if constexpr (!BOTH) {
    launch_tiles(c, a, attention_dkv_kernel<T, DP, 4, 32, 1, false, true, false, false>, a.n_k, a.kv_heads, 128, 256);
    launch_tiles(c, a, attention_dkv_kernel<T, DP, 4, 32, 1, false, false, true, false>, a.n_k, a.kv_heads, 128, 256);
  } else if (mixes(a)) {
    launch_mixed(c, a, attention_dkv_kernel<T, DP, 1, 32, 1, false, true, true, true>, a.n_k, a.kv_heads);
  } else if (few_rows(a, a.n_k)) {
    launch_tiles(c, a, attention_dkv_kernel<T, DP, 1, 32, 1, false, true, true, false>, a.n_k, a.kv_heads, 32, 64);
  } else {
    launch_tiles(c, a, attention_dkv_kernel<T, DP, 4, BF16 && DP < 128 ? 64 : 32, 2, BF16 && DP == 128, true, true, false>, a.n_k, a.kv_heads, 128, 512);
  }
}
template <typename T>
void launch_dim(const xrl_ctx *c, AttnArgs &a) {
  a.dim <= 32 ? launch<T, 32>(c, a) : a.dim <= 64 ? launch<T, 64>(c, a) : launch<T, 128>(c, a);
}

}  // namespace

extern "C" int xrl_attention_backward(xrl_ctx *c, const xrl_attention_desc *d, const xrl_heads *q, const xrl_heads *k, const xrl_heads *v, const xrl_heads *out,
                                      const float *d_lse, const xrl_heads *dout, const xrl_heads *dq, const xrl_heads *dk, const xrl_heads *dv) {
  const char *who = "xrl_attention_backward";
  AttnArgs a;
  if (int rc = check_attention(c, d, who, a)) return rc;
  const int es = d->type == XRL_PREC_BF16 ? 2 : 4;
  if (int rc = check_heads(q, d->n_q, d->q_heads, d->dim, es, "q", who, a.q)) return rc;
  if (int rc = check_heads(k, d->n_k, d->kv_heads, d->dim, es, "k", who, a.k)) return rc;
  if (int rc = check_heads(v, d->n_k, d->kv_heads, d->dim, es, "v", who, a.v)) return rc;
  if (int rc = check_heads(out, d->n_q, d->q_heads, d->dim, es, "out", who, a.out)) return rc;
  if (int rc = check_heads(dout, d->n_q, d->q_heads, d->dim, es, "dout", who, a.dout)) return rc;
  if (int rc = check_heads(dq, d->n_q, d->q_heads, d->dim, es, "dq", who, a.dq, &a.quads)) return rc;
  if (int rc = check_heads(dk, d->n_k, d->kv_heads, d->dim, es, "dk", who, a.dk, &a.quads)) return rc;
  if (int rc = check_heads(dv, d->n_k, d->kv_heads, d->dim, es, "dv", who, a.dv, &a.quads)) return rc;
  if (d->n_q > 0 && !d_lse) return fail(XRL_ERR_NULL, "%s: d_lse is NULL", who);
  if ((uintptr_t)d_lse % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  if (d->n_seqs == 0 || (d->n_q == 0 && d->n_k == 0)) return XRL_OK;
  a.lse = (float *)d_lse;
  Inputs in(d->type, d->dim);
  const size_t one = op_align((size_t)d->n_q * d->q_heads * 4 + 4);
  in.bytes = 2 * one;
  in.add(a.q, d->n_q, d->q_heads);
  in.add(a.k, d->n_k, d->kv_heads);
  in.add(a.v, d->n_k, d->kv_heads);
  in.add(a.out, d->n_q, d->q_heads);
  in.add(a.dout, d->n_q, d->q_heads);
  char *ws = nullptr;
  if (int rc = op_workspace(c, in.bytes, &ws, who)) return rc;
  in.copy(c, ws);
  a.dim_in = in.dim_in;
  a.stat_lse = (float *)ws;
  a.stat_delta = (float *)(ws + one);
  d->type == XRL_PREC_BF16 ? launch_dim<bf16_t>(c, a) : launch_dim<float>(c, a);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}
