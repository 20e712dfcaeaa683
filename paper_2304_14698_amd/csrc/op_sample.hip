// One entry drawn from every row of logits by a given random number, after temperature, top-k, top-p and min-p.
//
// Weights w = exp((x - largest) / temperature) are computed in 64 bits and held as whole multiples of 2^-S, S = 51 for rows of up to 2048 entries and one less for every
// doubling: sums of them are exact in 64 bits whatever their order, so what is kept and drawn does not depend on how a row is shared out, and differs from exact
// arithmetic only where a border lies within some 2^-S of a sum. (fp32 sums would draw another entry in one row of a few hundred.)
//
// A row's cut (the smallest kept entry, by falling logit, then rising index) comes from a histogram over the distance from the largest logit, of counts for top-k and of
// weights for top-p, and then from the entries of one bin, ranked against each other. Both cuts are monotone in the same order, so that one entry describes
// what is kept.
#include "logits_rows.hip.h"

#include <algorithm>

namespace {

struct SampleArgs {
  const void *logits;
  const int32_t *row_ptr;
  const uint8_t *mask;
  int64_t row0, n_rows, n_cols, stride, mask_stride;   // row0: first row of this launch
  float inv_t;
  double c;                     // log2(e) / temperature
  int top_k;
  double top_p, min_p;
  const float *uniforms;
  int32_t *ids;
  float *logp;
};

constexpr int kBins = 2048, kList = 1024;         // of a histogram; entries that are ranked against each other
constexpr float kBinsATurn = 64.f;                 // bins for a factor e in weight: 32 of these, the last bin has all below

// 2^t, t <= 0, in 64 bits: the integer part by the exponent, the rest in [-1/2, 1/2] by Taylor's sum of thirteen terms, whose rest is below 2^-52. Below 2^-100: of no weight.
__device__ __forceinline__ double exp2_64(double t) {
  t = t > -100.0 ? t : -100.0;
  const double n = rint(t), f = t - n;
  double p = 2.5678435993488206e-11;               // ln(2)^12 / 12!
  p = fma(p, f, 4.4455382718708116e-10);
  p = fma(p, f, 7.054911620801123e-09);
  p = fma(p, f, 1.01780860092397e-07);
  p = fma(p, f, 1.321548679014431e-06);
  p = fma(p, f, 1.5252733804059841e-05);
  p = fma(p, f, 0.0001540353039338161);
  p = fma(p, f, 0.0013333558146428443);
  p = fma(p, f, 0.009618129107628477);
  p = fma(p, f, 0.05550410866482158);
  p = fma(p, f, 0.24022650695910072);
  p = fma(p, f, 0.6931471805599453);
  p = fma(p, f, 1.0);
  return __longlong_as_double(__double_as_longlong(p) + ((long long)(int)n << 52));
}

// A logit's place in the order of all fp32 numbers; zeros of both signs are one.
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned u = __float_as_uint(x + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// Between two entries' exponentials: eight of them side by side take registers that waves to hide the memory's latency need.
__device__ __forceinline__ void apart(int j) {
  if (j & 1) __builtin_amdgcn_sched_barrier(0);
}

struct RowScale {
  float m;                      // largest logit
  double c;
  double one;                   // 2^S
  float bins;
};
__device__ __forceinline__ double weight_of(const RowScale &s, float x) { return exp2_64(((double)x - (double)s.m) * s.c); }
// w as a multiple of 2^-S: in the sum with 2^52 the last place is 1.
__device__ __forceinline__ unsigned long long whole_of(const RowScale &s, double w) {
  return (unsigned long long)__double_as_longlong(fma(w, s.one, 4503599627370496.0)) & 0xfffffffffffffull;
}
// Falls as x rises, so a bin is an interval of keys.
__device__ __forceinline__ int bin_of(const RowScale &s, float x) { return (int)fminf((s.m - x) * s.bins, (float)(kBins - 1)); }

typedef unsigned long long u64;
__device__ __forceinline__ u64 wave_sum64(u64 x) {
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
  return x;
}
__device__ __forceinline__ u64 wave_scan64(u64 x, int lane) {   // of the lanes up to this one
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const u64 y = __shfl_up(x, i);
    x += lane >= i ? y : 0;
  }
  return x;
}

struct Entry {
  u64 w;
  unsigned key;
  int id;
};

template <int WAVES>
struct Shared {
  u64 mass[kBins];
  unsigned count[kBins];
  Entry list[kList];
  u64 sums[WAVES];
  float floats[WAVES];
  unsigned lows[WAVES], highs[WAVES];
  int n, bin;
  u64 before;                   // what lies in front of the bin: counts, or weights
  u64 all;
  unsigned key;
  int id;
  u64 upto;
};

// What is kept of a row: keys above `key`, and of those equal to it the entries up to index `id`.
struct Cut {
  unsigned key;
  int id;
};
__device__ __forceinline__ bool inside(const Cut &c, unsigned key, int id) { return key > c.key || (key == c.key && id <= c.id); }

// A wave's share of the row: columns [begin, end) in steps of 64 VEC; f(col, x) for the lane's piece of each.
template <typename T, typename F>
__device__ __forceinline__ void for_pieces(const Row<T> &row, bool odd, int begin, int end, int lane, F f) {
  constexpr int VEC = 16 / (int)sizeof(T);
  for (int w = begin; w < end; w += 64 * VEC) {
    float x[VEC];
    fetch<T, VEC>(row, odd, w + lane * VEC, end, x);
    f(w + lane * VEC, x);
  }
}

// One block a row.
template <typename T, int WAVES>
struct Sampler {
  static constexpr int VEC = 16 / (int)sizeof(T), STEP = 64 * VEC;
  const SampleArgs &a;
  const Row<T> &row;
  Shared<WAVES> &sh;
  bool odd;
  int lane, wave, begin, end;   // columns of this wave
  RowScale s;

  // Σ of one value a wave, over the waves in front of this one and over all.
  __device__ __forceinline__ u64 over_waves(u64 mine, u64 &all) {
    __syncthreads();
    if (lane == 0) sh.sums[wave] = mine;
    __syncthreads();
    u64 before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      before += w < wave ? sh.sums[w] : 0;
      all += sh.sums[w];
    }
    return before;
  }

  // The bin in which the sum of what lies in front (counts or weights of larger entries) passes `limit`: sh.bin, and sh.before what lies in front of it.
  __device__ __forceinline__ void find_bin(bool by_mass, u64 limit) {
    if (wave == 0) {
      constexpr int EACH = kBins / 64;
      u64 mine = 0;
#pragma unroll 4
      for (int i = 0; i < EACH; ++i) mine += by_mass ? sh.mass[lane * EACH + i] : sh.count[lane * EACH + i];
      const u64 upto = wave_scan64(mine, lane);
      const int at = __ffsll(__ballot(upto >= limit)) - 1;
      if (lane == (at < 0 ? 63 : at)) {
        u64 before = upto - mine;
        int b = lane * EACH;
#pragma unroll 1
        for (; b < lane * EACH + EACH - 1; ++b) {
          const u64 one = by_mass ? sh.mass[b] : sh.count[b];
          if (before + one >= limit) break;
          before += one;
        }
        sh.bin = b;
        sh.before = before;
      }
      if (lane == 63) sh.all = upto;
    }
    __syncthreads();
  }

  __device__ __forceinline__ void clear_bins(bool by_mass) {
    for (int i = threadIdx.x; i < kBins; i += WAVES * 64) {
      sh.count[i] = 0;
      if (by_mass) sh.mass[i] = 0;
    }
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
  }

  // The cut at which the entries in front of it (by_mass: their weights) are fewer than `limit`, from the bins of the first histogram. sh.upto: the weight of all that
  // is kept.
  __device__ __forceinline__ Cut cut_at(bool by_mass, u64 limit) {
    find_bin(by_mass, limit);
    const int bin = sh.bin;
    u64 before = sh.before, mass_before = before;
    if (!by_mass) {                                    // (the weights in front as well: top-p takes its share of them)
      u64 t = 0, all;
      for (int i = threadIdx.x; i < bin; i += WAVES * 64) t += sh.mass[i];
      over_waves(wave_sum64(t), all);
      mass_before = all;
    }
    // its entries, and the range of their keys
    unsigned lo = 0xffffffffu, hi = 0;
    int n = 0;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    for_pieces<T>(row, odd, begin, end, lane, [&](int col, const float *x) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (x[j] == -INFINITY || bin_of(s, x[j]) != bin) continue;
        const unsigned key = key_of(x[j]);
        lo = min(lo, key);
        hi = max(hi, key);
        const int at = atomicAdd(&sh.n, 1);
        if (at < kList) sh.list[at] = {whole_of(s, weight_of(s, x[j])), key, col + j};
        apart(j);
      }
    });
    __syncthreads();
    n = sh.n;
    while (n > kList) {
      // too many: bins over their keys
      lo = block_min(lo);
      hi = ~block_min(~hi);
      if (lo == hi) return cut_of_equal(by_mass, limit, before, mass_before, lo);
      int shift = 0;
      while ((hi - lo) >> shift >= kBins) ++shift;
      clear_bins(true);
      for_pieces<T>(row, odd, begin, end, lane, [&](int, const float *x) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const unsigned key = key_of(x[j]);
          if (x[j] == -INFINITY || key < lo || key > hi) continue;
          atomicAdd(&sh.count[(hi - key) >> shift], 1u);
          atomicAdd(&sh.mass[(hi - key) >> shift], whole_of(s, weight_of(s, x[j])));
          apart(j);
        }
      });
      __syncthreads();
      find_bin(by_mass, limit - before);
      const int b = sh.bin;
      u64 t = 0, all;
      for (int i = threadIdx.x; i < b; i += WAVES * 64) t += sh.mass[i];
      over_waves(wave_sum64(t), all);
      mass_before += all;
      before += sh.before;
      const unsigned top = hi - ((unsigned)b << shift), span = (1u << shift) - 1;
      const unsigned range_lo = top - lo > span ? top - span : lo, range_hi = top;
      __syncthreads();
      if (threadIdx.x == 0) sh.n = 0;
      __syncthreads();
      lo = 0xffffffffu;
      hi = 0;
      for_pieces<T>(row, odd, begin, end, lane, [&](int col, const float *x) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const unsigned key = key_of(x[j]);
          if (x[j] == -INFINITY || key < range_lo || key > range_hi) continue;
          lo = min(lo, key);
          hi = max(hi, key);
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) sh.list[at] = {whole_of(s, weight_of(s, x[j])), key, col + j};
          apart(j);
        apart(j);
        }
      });
      __syncthreads();
      n = sh.n;
    }
    // every entry against all others: what lies in front of it
    for (int i = threadIdx.x; i < n; i += WAVES * 64) {
      const Entry e = sh.list[i];
      u64 count = 0, mass = 0;
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const Entry o = sh.list[k];
        const bool front = o.key > e.key || (o.key == e.key && o.id < e.id);
        count += front ? 1 : 0;
        mass += front ? o.w : 0;
      }
      const u64 from = before + (by_mass ? mass : count), to = from + (by_mass ? e.w : 1);
      if (from < limit && limit <= to) {
        sh.key = e.key;
        sh.id = e.id;
        sh.upto = mass_before + mass + e.w;
      }
    }
    __syncthreads();
    return {sh.key, sh.id};
  }

  __device__ __forceinline__ unsigned block_min(unsigned x) {
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) x = min(x, (unsigned)__shfl_xor((int)x, i));
    __syncthreads();
    if (lane == 0) sh.lows[wave] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x = min(x, sh.lows[w]);
    return x;
  }

  // All entries of the bin are equal: the first so many of them, by index.
  __device__ __forceinline__ Cut cut_of_equal(bool by_mass, u64 limit, u64 before, u64 mass_before, unsigned key) {
    const unsigned bits = key >> 31 ? key ^ 0x80000000u : ~key;
    const u64 w = whole_of(s, weight_of(s, __uint_as_float(bits)));
    const u64 left = limit - before, m = by_mass ? (left + w - 1) / w : left;      // (w > 0: the limit lies inside the bin)
    u64 mine = 0, all;
    for_pieces<T>(row, odd, begin, end, lane, [&](int, const float *x) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) mine += x[j] != -INFINITY && key_of(x[j]) == key ? 1 : 0;
    });
    mine = wave_sum64(mine);
    u64 upto = over_waves(mine, all);
    if (upto < m && m <= upto + mine) {                // in this wave's columns
      bool done = false;
      for_pieces<T>(row, odd, begin, end, lane, [&](int col, const float *x) {
        if (done) return;
        u64 here = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) here += x[j] != -INFINITY && key_of(x[j]) == key ? 1 : 0;
        const u64 scan = wave_scan64(here, lane), step = __shfl(scan, 63);
        if (upto + step < m) {
          upto += step;
          return;
        }
        done = true;
        u64 at = upto + scan - here;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          if (x[j] == -INFINITY || key_of(x[j]) != key) continue;
          if (++at == m) sh.id = col + j;
        }
      });
    }
    if (threadIdx.x == 0) {
      sh.key = key;
      sh.upto = mass_before + m * w;
    }
    __syncthreads();
    return {sh.key, sh.id};
  }
};

template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void token_sample_kernel(const SampleArgs a) {
  touch_args(a);
  using S = Sampler<T, WAVES>;
  constexpr int VEC = S::VEC, STEP = S::STEP;
  __shared__ Shared<WAVES> sh;
  const int64_t r = a.row0 + blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Row<T> row = row_of<T>(a, r);
  const float u = a.uniforms[r];
  const int steps = (row.len + STEP - 1) / STEP, per = (steps + WAVES - 1) / WAVES;
  const int64_t b0 = (int64_t)wave * per * STEP, b1 = b0 + (int64_t)per * STEP;
  S t = {a, row, sh, __builtin_amdgcn_readfirstlane(lead_of(row.x, row.len)) != 0, lane, wave, (int)(b0 < row.len ? b0 : row.len), (int)(b1 < row.len ? b1 : row.len), {}};
  // the largest logit; what is no number or +inf makes itself known
  float m = -INFINITY;
  bool odd_one = false;
  for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int, const float *x) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      m = fmaxf(m, x[j]);
      odd_one = odd_one | !(x[j] < INFINITY);
    }
  });
  m = wave_max(m);
  if (lane == 0) sh.floats[wave] = m;
  odd_one = __syncthreads_or(odd_one);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh.floats[w]);
  if (odd_one || m == -INFINITY) {
    if (threadIdx.x == 0) {
      a.ids[r] = -1;
      a.logp[r] = odd_one ? __builtin_nanf("") : -INFINITY;
    }
    return;
  }
  const int bits = 32 - __clz(row.len - 1);
  t.s = {m, a.c, __longlong_as_double((long long)(1023 + 51 - (bits > 11 ? bits - 11 : 0)) << 52), a.inv_t * kBinsATurn};
  const RowScale s = t.s;
  Cut cut = {0, 0x7fffffff};
  const bool by_k = a.top_k > 0 && a.top_k < row.len, by_p = a.top_p < 1.0;
  if (by_k || by_p) {
    t.clear_bins(true);
    for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int, const float *x) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (x[j] == -INFINITY) continue;
        const int b = bin_of(s, x[j]);
        if (by_k) atomicAdd(&sh.count[b], 1u);
        atomicAdd(&sh.mass[b], whole_of(s, weight_of(s, x[j])));
        apart(j);
      }
    });
    __syncthreads();
    u64 whole = 0;
    if (by_k) {
      u64 n = 0, all;
      for (int i = threadIdx.x; i < kBins; i += WAVES * 64) n += sh.count[i];
      t.over_waves(wave_sum64(n), all);
      if ((u64)a.top_k < all) {
        // (bins over keys may take the histogram's place, which top-p needs after it)
        cut = t.cut_at(false, a.top_k);
        whole = sh.upto;
      }
    }
    if (by_p) {
      if (by_k && whole > 0) {
        __syncthreads();
        t.clear_bins(true);
        for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int, const float *x) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            if (x[j] != -INFINITY) atomicAdd(&sh.mass[bin_of(s, x[j])], whole_of(s, weight_of(s, x[j])));
            apart(j);
          }
        });
        __syncthreads();
      } else {
        u64 n = 0;
        for (int i = threadIdx.x; i < kBins; i += WAVES * 64) n += sh.mass[i];
        t.over_waves(wave_sum64(n), whole);
      }
      const u64 limit = (u64)ceil(a.top_p * (double)whole);
      cut = t.cut_at(true, limit < 1 ? 1 : limit);
    }
  }
  // sums of what is kept, of the waves' shares and, for the log-probability, of all
  u64 kept = 0;
  float sum = 0.f;
  const float c = a.inv_t * kLog2e;
  auto weight = [&](int col, const float *x) {
    u64 k = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (x[j] == -INFINITY || !inside(cut, key_of(x[j]), col + j)) continue;
      const double w = weight_of(s, x[j]);
      if (w >= a.min_p) k += whole_of(s, w);
      apart(j);
    }
    return k;
  };
  for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) {
    kept += weight(col, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum += __builtin_amdgcn_exp2f((x[j] - m) * c);
  });
  kept = wave_sum64(kept);
  u64 all;
  u64 before = t.over_waves(kept, all);
  sum = wave_sum(sum);
  __syncthreads();
  if (lane == 0) sh.floats[wave] = sum;
  // the drawn entry is the first whose sum passes `target`
  const double want = u > 0.f ? floor((double)u * (double)all) : 0.0;
  const u64 target = want < (double)all && (u64)want < all ? (u64)want : all - 1;
  if (before <= target && target < before + kept) {    // in this wave's columns
    sh.bin = t.begin;
    sh.n = t.end;
    sh.before = before;
  }
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) sum += sh.floats[w];
  // those columns shared out once more
  {
    const int first = sh.bin, last = sh.n, n = (last - first + STEP - 1) / STEP, each = (n + WAVES - 1) / WAVES;
    const u64 base = sh.before;
    t.begin = min(first + wave * each * STEP, last);
    t.end = min(t.begin + each * STEP, last);
    kept = 0;
    for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) { kept += weight(col, x); });
    kept = wave_sum64(kept);
    before = base + t.over_waves(kept, all);
  }
  if (!(before <= target && target < before + kept)) return;
  bool done = false;
  for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) {
    if (done) return;
    const u64 mine = weight(col, x), scan = wave_scan64(mine, lane), step = __shfl(scan, 63);
    if (before + step <= target) {
      before += step;
      return;
    }
    done = true;
    u64 at = before + scan - mine;
    if (!(at <= target && target < at + mine)) return;
    bool found = false;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (found || x[j] == -INFINITY || !inside(cut, key_of(x[j]), col + j)) continue;
      const double w = weight_of(s, x[j]);
      if (w >= a.min_p) at += whole_of(s, w);
      if (at <= target) continue;
      found = true;
      a.ids[r] = col + j;
      const float v = (x[j] - m) * a.inv_t - logf(sum);
      a.logp[r] = v < kLowest ? kLowest : v;
    }
  });
}

template <typename T>
void launch(const xrl_ctx *c, SampleArgs &a, bool small) {
  for (a.row0 = 0; a.row0 < a.n_rows; a.row0 += kMaxBlocks) {
    const dim3 grid((unsigned)std::min(a.n_rows - a.row0, kMaxBlocks));
    if (small) token_sample_kernel<T, 4><<<grid, dim3(256), 0, op_stream(c)>>>(a);
    else token_sample_kernel<T, 8><<<grid, dim3(512), 0, op_stream(c)>>>(a);
  }
}

}  // namespace

extern "C" int xrl_token_sample(xrl_ctx *c, const xrl_logits_desc *logits, const xrl_sample_desc *how, const float *d_uniforms, int32_t *d_ids, float *d_logp) {
  const char *who = "xrl_token_sample";
  SampleArgs a;
  if (int rc = check_logits(c, logits, who, a)) return rc;
  if (!how) return fail(XRL_ERR_NULL, "%s: how is NULL", who);
  if (how->top_k < 0 || !(how->top_p > 0.f) || !(how->top_p <= 1.f) || !(how->min_p >= 0.f) || !(how->min_p <= 1.f))
    return fail(XRL_ERR_VALUE, "%s: top_k = %d, top_p = %g, min_p = %g", who, how->top_k, (double)how->top_p, (double)how->min_p);
  if (a.n_rows == 0) return XRL_OK;
  if (!d_uniforms || !d_ids || !d_logp) return fail(XRL_ERR_NULL, "%s: NULL device pointer", who);
  if (((uintptr_t)d_uniforms | (uintptr_t)d_ids | (uintptr_t)d_logp) % 4) return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a.c = 1.4426950408889634 / (double)logits->temperature;
  a.top_k = how->top_k; a.top_p = how->top_p; a.min_p = how->min_p;
  a.uniforms = d_uniforms; a.ids = d_ids; a.logp = d_logp;
  const int64_t cols = a.row_ptr ? a.n_cols / a.n_rows : a.n_cols;
  const bool small = cols <= 4096;
  logits->type == XRL_PREC_BF16 ? launch<bf16_t>(c, a, small) : launch<float>(c, a, small);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}
