// One entry drawn from every row of logits by a given random number, after temperature, top-k, top-p and min-p.
//
// Weights w = exp((x - largest) / temperature) are computed in 64 bits and held as whole multiples of 2^-S, S = 51 for rows of up to 2048 entries and one less for every
// doubling: adding them up is exact in 64 bits whatever their order, so what is kept and drawn does not depend on how a row is shared out. A weight is off by at most 1.5 2^-S: 1/2 for the multiple, 0.38
// for the rest of the exponential's sum and the rest for the roundings of its argument and terms (1.1 is the most of 4 10^7 on the host). A sum of n of them is off by n times that, and with the
// rounding of its product with top_p or the random number what is drawn differs from exact arithmetic only where a border lies within 2 n 2^-S of a sum. (fp32 sums would draw another entry
// in one row of a few hundred.)
//
// A row's cut (the smallest kept entry, by falling logit, then rising index) comes from a histogram over the distance from the largest logit, of counts for top-k and of
// weights for top-p, and then from the entries of one bin, ranked against each other. Both cuts are monotone in the same order, so that one entry describes
// what is kept.
//
// Bound by instructions for many long rows, each entry's exponential in 64 bits first (2048 x 32003 in bf16 with top-p and min-p: 137 us, 58 vector instructions for 64 entries, where reading them takes
// 25), and by a row's chain of barriers and memory round trips for few (8 x 128256, the best 50: 4 + 29 us; 32 rows of 65 slots: 9).
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
  // rows in parts whose groups of entries were looked at before (token_sample_groups_kernel); parts 0: not
  int parts;
  float *group_max;             // [rows][parts][256]
  float *part_stats;            // [rows][parts][2]: the largest logit, and the sum of exponentials relative to it
};

// Bins of a histogram, entries that are ranked against each other, and bins of these: fewer for a row a wave, so that 16 of them fit on a compute unit.
template <int WAVES>
constexpr int kBins = WAVES == 1 ? 256 : 2048;
template <int WAVES>
constexpr int kList = WAVES == 1 ? 256 : 1024;
template <int WAVES>
constexpr int kListBins = kList<WAVES>;
constexpr int kPart = 8192, kGroups = 256;          // entries of a part, and its groups: what one thread has of it
constexpr float kTurns = 32.f;                     // factors of e in weight that the bins cover; the last bin has all below

// 2^t, t <= 0, in 64 bits: the integer part by the exponent, the rest in [-1/2, 1/2] by Taylor's sum of thirteen terms, whose rest is below 2^-52. Below 2^-100: of no weight.
constexpr double kExp2[13] = {2.5678435993488206e-11, 4.4455382718708116e-10, 7.054911620801123e-09, 1.01780860092397e-07, 1.321548679014431e-06, 1.5252733804059841e-05, 0.0001540353039338161, 0.0013333558146428443, 0.009618129107628477, 0.05550410866482158, 0.24022650695910072, 0.6931471805599453, 1.0};   // ln(2)^k / k!, k = 12 .. 0
__device__ __forceinline__ double exp2_64(double t) {
  t = t > -100.0 ? t : -100.0;
  const double n = rint(t), f = t - n;
  double p = kExp2[0];
#pragma unroll
  for (int i = 1; i < 13; ++i) {
    double k = kExp2[i];
    asm("" : "+s"(k));                             // (in scalar registers: as a literal each takes a move more)
    p = fma(p, f, k);
  }
  return __longlong_as_double(__double_as_longlong(p) + ((long long)(int)n << 52));
}

// A logit's place in the order of all fp32 numbers; zeros of both signs are one.
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned u = __float_as_uint(x + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

struct RowScale {
  float m;                      // largest logit
  double c;
  double one;                   // 2^S
  float bins, last;             // bins for a unit of the logits; the last one
};
__device__ __forceinline__ double weight_of(const RowScale &s, float x) { return exp2_64(((double)x - (double)s.m) * s.c); }
// w as a multiple of 2^-S: in the sum with 2^52 the last place is 1.
__device__ __forceinline__ unsigned long long whole_of(const RowScale &s, double w) {
  return (unsigned long long)__double_as_longlong(fma(w, s.one, 4503599627370496.0)) & 0xfffffffffffffull;
}
template <int WAVES>
__device__ __forceinline__ RowScale scale_of(const SampleArgs &a, float m, int len) {
  const int bits = 32 - __clz(len - 1);
  return {m, a.c, __longlong_as_double((long long)(1023 + 51 - (bits > 11 ? bits - 11 : 0)) << 52), a.inv_t * (kBins<WAVES> / kTurns), (float)(kBins<WAVES> - 1)};
}
// Falls as x rises, so a bin is an interval of keys.
__device__ __forceinline__ int bin_of(const RowScale &s, float x) { return (int)fminf((s.m - x) * s.bins, s.last); }

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
  u64 mass[kBins<WAVES>];
  unsigned count[kBins<WAVES>];
  u64 list_mass[kListBins<WAVES>];     // bins over the list
  unsigned list_count[kListBins<WAVES>];
  Entry list[kList<WAVES>];
  int members[64], few;
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

// A wave's share of the row: columns [begin, end) in steps of 64 VEC; f(col, x) for the lane's piece of each. Two steps' loads are on their way while one is worked on: each by
// itself is a round trip to memory of a microsecond or two. The steps' registers move up, and the body stands once: with bodies for four steps side by side the kernel had
// 270 KB of code, of which the instruction cache holds 64 (2048 x 32003 with min-p 580 us for 284 without the list below).
template <typename T, typename F>
__device__ __forceinline__ void for_pieces(const Row<T> &row, bool odd, int begin, int end, int lane, F f) {
  constexpr int VEC = 16 / (int)sizeof(T), STEP = 64 * VEC, AHEAD = 2;
  Piece<T, VEC> v[AHEAD + 1];
  Piece<uint8_t, VEC> k[AHEAD + 1];
  auto request = [&](int w, int at) {
    if (w + STEP > end) return;
    const T *p = row.x + w + lane * VEC;
    v[at] = odd ? load_odd_piece<T, VEC>(p) : load_piece<T, VEC>(p);
    if (row.mask) k[at] = load_piece<uint8_t, VEC>(row.mask + w + lane * VEC);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) request(begin + i * STEP, i);
#pragma unroll 1
  for (int w = begin; w < end; w += STEP) {
    request(w + AHEAD * STEP, AHEAD);
    float x[VEC];
    if (w + STEP <= end) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = row.mask && !k[0].v[j] ? -INFINITY : (float)v[0].v[j];
    } else {
      fetch<T, VEC>(row, odd, w + lane * VEC, end, x);
    }
    f(w + lane * VEC, x);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      v[i] = v[i + 1];
      k[i] = k[i + 1];
    }
  }
}
// f(j, x[j]) for the entries of a piece, two bodies for all of them.
template <int VEC, typename F>
__device__ __forceinline__ void for_entries(const float *x, F f) {
  float y[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) y[j] = x[j];
#pragma unroll 1
  for (int j = 0; j < VEC; j += 2) {
    f(j, y[0]);
    f(j + 1, y[1]);
#pragma unroll
    for (int i = 0; i + 2 < VEC; ++i) y[i] = y[i + 2];
  }
}

// One block a row.
constexpr u64 kBelow = 1ull << 63;                 // beside a listed entry's weight: below min-p
template <typename T, int WAVES>
struct Sampler {
  static constexpr int VEC = 16 / (int)sizeof(T), STEP = 64 * VEC;
  const SampleArgs &a;
  const Row<T> &row;
  Shared<WAVES> &sh;
  bool odd, masses;             // masses: weights are needed, not counts alone
  int lane, wave, begin, end;   // columns of this wave
  RowScale s;
  bool spoiled;                 // bins over keys have taken the first histogram's place

  // The sum of one value a wave, over the waves in front of this one and over all.
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
  template <int BINS>
  __device__ __forceinline__ void find_bin(const unsigned (&counts)[BINS], const u64 (&masses_)[BINS], bool by_mass, u64 limit) {
    constexpr int EACH = BINS / (WAVES * 64);
    u64 v[EACH], mine = 0, all;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      v[i] = by_mass ? masses_[threadIdx.x * EACH + i] : counts[threadIdx.x * EACH + i];
      mine += v[i];
    }
    const u64 scan = wave_scan64(mine, lane), upto = over_waves(__shfl(scan, 63), all) + scan;
    if (upto >= limit && upto - mine < limit) {
      u64 before = upto - mine;
      int at = 0;
#pragma unroll
      for (int i = 0; i < EACH - 1; ++i) {
        const bool on = at == i && before + v[i] < limit;
        before += on ? v[i] : 0;
        at += on ? 1 : 0;
      }
      sh.bin = threadIdx.x * EACH + at;
      sh.before = before;
    }
    __syncthreads();
  }

  template <int BINS>
  __device__ __forceinline__ void clear_bins(unsigned (&counts)[BINS], u64 (&masses_)[BINS]) {
    for (int i = threadIdx.x; i < BINS; i += WAVES * 64) {
      counts[i] = 0;
      masses_[i] = 0;
    }
    __syncthreads();
  }
  // The sum of the bins' weights in front of `bin`.
  __device__ __forceinline__ u64 mass_before(const u64 *masses_, int bin) {
    u64 t = 0, all;
    for (int i = threadIdx.x; i < bin; i += WAVES * 64) t += masses_[i];
    over_waves(wave_sum64(t), all);
    return all;
  }

  // The cut at which the entries in front of it (by_mass: their weights) are fewer than `limit`, from the bins of the first histogram. sh.upto: the weight of all that
  // is kept.
  __device__ __forceinline__ Cut cut_at(bool by_mass, u64 limit) {
    find_bin(sh.count, sh.mass, by_mass, limit);
    const int bin = sh.bin;
    u64 before = sh.before, in_front = before;
    if (!by_mass && masses) in_front = mass_before(sh.mass, bin);   // (the weights in front as well: top-p takes its share of them)
    // its entries, and the range of their keys
    unsigned lo = 0xffffffffu, hi = 0;
    int n = 0;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    for_pieces<T>(row, odd, begin, end, lane, [&](int col, const float *x) {
      for_entries<VEC>(x, [&](int j, float xj) {
        if (xj == -INFINITY || bin_of(s, xj) != bin) return;
        const unsigned key = key_of(xj);
        lo = min(lo, key);
        hi = max(hi, key);
        const int at = atomicAdd(&sh.n, 1);
        if (at < kList<WAVES>) sh.list[at] = {whole_of(s, weight_of(s, xj)), key, col + j};
      });
    });
    __syncthreads();
    n = sh.n;
    while (n > kList<WAVES>) {
      // too many: bins over their keys
      lo = block_min(lo);
      hi = ~block_min(~hi);
      if (lo == hi) return cut_of_equal(by_mass, limit, before, in_front, lo);
      int shift = 0;
      while ((hi - lo) >> shift >= kBins<WAVES>) ++shift;
      clear_bins(sh.count, sh.mass);
      spoiled = true;
      for_pieces<T>(row, odd, begin, end, lane, [&](int, const float *x) {
        for_entries<VEC>(x, [&](int j, float xj) {
          const unsigned key = key_of(xj);
          if (xj == -INFINITY || key < lo || key > hi) return;
          if (!by_mass) atomicAdd(&sh.count[(hi - key) >> shift], 1u);
          if (masses) atomicAdd(&sh.mass[(hi - key) >> shift], whole_of(s, weight_of(s, xj)));
        });
      });
      __syncthreads();
      find_bin(sh.count, sh.mass, by_mass, limit - before);
      const int b = sh.bin;
      if (masses) in_front += mass_before(sh.mass, b);
      before += sh.before;
      const unsigned top = hi - ((unsigned)b << shift), span = (1u << shift) - 1;
      const unsigned range_lo = top - lo > span ? top - span : lo, range_hi = top;
      __syncthreads();
      if (threadIdx.x == 0) sh.n = 0;
      __syncthreads();
      lo = 0xffffffffu;
      hi = 0;
      for_pieces<T>(row, odd, begin, end, lane, [&](int col, const float *x) {
        for_entries<VEC>(x, [&](int j, float xj) {
          const unsigned key = key_of(xj);
          if (xj == -INFINITY || key < range_lo || key > range_hi) return;
          lo = min(lo, key);
          hi = max(hi, key);
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList<WAVES>) sh.list[at] = {whole_of(s, weight_of(s, xj)), key, col + j};
        });
      });
      __syncthreads();
      n = sh.n;
    }
    in_front += select(n, by_mass, false, limit - before, [](int) { return true; });
    if (threadIdx.x == 0) sh.upto = in_front;
    __syncthreads();
    return {sh.key, sh.id};
  }

  // One more entry of the list, if there is room: sh.n counts all.
  __device__ __forceinline__ void push(float x, int id, double w) {
    const int at = atomicAdd(&sh.n, 1);
    if (at < kList<WAVES>) sh.list[at] = {whole_of(s, w) | (w >= a.min_p ? 0 : kBelow), key_of(x), id};
  }

  // Of those of the list's n entries that count(i), in the order of the cuts (by_index: of their indices), the one at which the sum of counts (by_mass: weights) reaches `limit`: its key and
  // index to sh.key and sh.id; returned: the weight up to it and with it. By bins over the entries' places in that order, a range narrower by the number of bins each time until a
  // few are left, which are ranked against each other. (Ranking all against all took 230 us for 200 to 700 entries.)
  template <typename Counts>
  __device__ __forceinline__ u64 select(int n, bool by_mass, bool by_index, u64 limit, Counts counts) {
    constexpr int EACH = kList<WAVES> / (WAVES * 64);
    Entry e[EACH];
    u64 place[EACH];
    bool in[EACH];
    unsigned least = 0xffffffffu, most = 0;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      const int i = threadIdx.x + q * WAVES * 64;
      in[q] = i < n && counts(i);
      e[q] = in[q] ? sh.list[i] : Entry{0, 0, 0};
      e[q].w &= ~kBelow;
      const unsigned first = by_index ? (unsigned)e[q].id : ~e[q].key;
      place[q] = by_index ? first : (u64)first << 32 | (unsigned)e[q].id;
      if (!in[q]) continue;
      least = min(least, first);
      most = max(most, first);
    }
    least = block_min(least);
    most = ~block_min(~most);
    u64 lo = by_index ? least : (u64)least << 32, hi = by_index ? most : (u64)most << 32 | 0xffffffffu, before = 0, mass = 0;
    constexpr int BITS = __builtin_ctz(kListBins<WAVES>);
    for (int step = 0; step < (63 + BITS) / BITS; ++step) {   // (64 bits by BITS each time)
      const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > BITS ? bits - BITS : 0;
      clear_bins(sh.list_count, sh.list_mass);
#pragma unroll
      for (int q = 0; q < EACH; ++q) {
        if (!in[q] || place[q] < lo || place[q] > hi) continue;
        atomicAdd(&sh.list_count[(place[q] - lo) >> shift], 1u);
        atomicAdd(&sh.list_mass[(place[q] - lo) >> shift], e[q].w);
      }
      if (threadIdx.x == 0) sh.few = 0;
      __syncthreads();
      find_bin(sh.list_count, sh.list_mass, by_mass, limit - before);
      const int bin = sh.bin;
      mass += mass_before(sh.list_mass, bin);
      before += sh.before;
      lo += (u64)bin << shift;
      hi = min(hi, lo + (((u64)1 << shift) - 1));
      if (sh.list_count[bin] <= 64) break;
      __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < EACH; ++q)
      if (in[q] && place[q] >= lo && place[q] <= hi) sh.members[atomicAdd(&sh.few, 1)] = threadIdx.x + q * WAVES * 64;
    __syncthreads();
    const int m = sh.few;
    if ((int)threadIdx.x < m) {
      const Entry f = sh.list[sh.members[threadIdx.x]];
      u64 from = before, front = 0;
      for (int k = 0; k < m; ++k) {
        const Entry o = sh.list[sh.members[k]];
        const bool ahead = by_index ? o.id < f.id : o.key > f.key || (o.key == f.key && o.id < f.id);
        front += ahead ? o.w & ~kBelow : 0;
        from += !by_mass && ahead ? 1 : 0;
      }
      from += by_mass ? front : 0;
      const u64 own = by_mass ? f.w & ~kBelow : 1;
      if (from < limit && limit <= from + own) {
        sh.key = f.key;
        sh.id = f.id;
        sh.upto = mass + front + (f.w & ~kBelow);
      }
    }
    __syncthreads();
    const u64 upto = sh.upto;
    __syncthreads();
    return upto;
  }

  // The list's n entries are the row's n first in the order of the cuts, and all that can be kept are among them. sum: of all weights that may be chosen (without top-k, top-p
  // takes its share of `whole`).
  __device__ __forceinline__ void draw_from_list(int64_t r, float u, bool by_k, bool by_p, u64 whole, float sum) {
    constexpr int EACH = kList<WAVES> / (WAVES * 64);
    const int n = sh.n;
    Cut cut = {0, 0x7fffffff};
    auto all_of = [](int) { return true; };
    const bool cut_k = by_k && n > a.top_k;
    u64 kept = 0, all;
    auto kept_weight = [&](int i) {
      const Entry e = sh.list[i];
      return inside(cut, e.key, e.id) ? e.w : 0;
    };
    if (cut_k) {
      whole = select(n, false, false, a.top_k, all_of);
      cut = {sh.key, sh.id};
    } else if (by_k && by_p) {
#pragma unroll
      for (int q = 0; q < EACH; ++q) kept += (int)threadIdx.x + q * WAVES * 64 < n ? sh.list[threadIdx.x + q * WAVES * 64].w & ~kBelow : 0;
      over_waves(wave_sum64(kept), whole);
    }
    if (by_p) {
      const double part = ceil(a.top_p * (double)whole);
      const u64 limit = part < 1.0 ? 1 : (u64)part;
      // (by min-p alone the list may end in front of top-p's cut)
      kept = 0;
#pragma unroll
      for (int q = 0; q < EACH; ++q) kept += (int)threadIdx.x + q * WAVES * 64 < n ? kept_weight(threadIdx.x + q * WAVES * 64) & ~kBelow : 0;
      over_waves(wave_sum64(kept), all);
      __syncthreads();
      if (limit <= all) {
        select(n, true, false, limit, all_of);
        cut = {sh.key, sh.id};
      }
    }
    kept = 0;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      const u64 w = (int)threadIdx.x + q * WAVES * 64 < n ? kept_weight(threadIdx.x + q * WAVES * 64) : kBelow;
      kept += w & kBelow ? 0 : w;
    }
    over_waves(wave_sum64(kept), all);
    __syncthreads();
    select(n, true, true, target_of(u, all) + 1, [&](int i) {
      const u64 w = kept_weight(i);
      return w != 0 && !(w & kBelow);
    });
    if (threadIdx.x == 0) {
      a.ids[r] = sh.id;
      a.logp[r] = log_share(__uint_as_float(sh.key >> 31 ? sh.key ^ 0x80000000u : ~sh.key), sum);
    }
  }
  // From the largest logits of the row's groups: the entries of those groups that can hold one which is kept (of the first top_k, or not below min-p), as a list. false: they are
  // more than the list takes.
  __device__ __forceinline__ bool draw_from_groups(int64_t r, float u, const float *tops, float sum) {
    constexpr int PIECES = kPart / (kGroups * VEC);
    const bool by_k = a.top_k > 0;
    const int groups = a.parts * kGroups;
    unsigned *chosen = (unsigned *)sh.mass;            // [kList<WAVES>]
    clear_bins(sh.count, sh.mass);
    if (threadIdx.x == 0) {
      sh.n = 0;
      sh.few = 0;
      sh.bin = kBins<WAVES> - 1;
    }
    int bin = kBins<WAVES> - 1;
    if (by_k) {
      for (int i = threadIdx.x; i < groups; i += WAVES * 64)
        if (tops[i] > -INFINITY) atomicAdd(&sh.count[bin_of(s, tops[i])], 1u);
      __syncthreads();
      find_bin(sh.count, sh.mass, false, a.top_k);
      bin = sh.bin;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < groups; i += WAVES * 64) {
      if (tops[i] == -INFINITY || bin_of(s, tops[i]) > bin || (!by_k && !(weight_of(s, tops[i]) >= a.min_p))) continue;
      const int at = atomicAdd(&sh.few, 1);
      if (at < kList<WAVES>) chosen[at] = i;
    }
    __syncthreads();
    const int n = sh.few;
    if (n > kList<WAVES>) return false;
    for (int i = threadIdx.x; i < n * PIECES; i += WAVES * 64) {
      const int g = chosen[i / PIECES], col = g / kGroups * kPart + (i % PIECES * kGroups + g % kGroups) * VEC;
      float x[VEC];
      fetch<T, VEC>(row, odd, col, row.len, x);
      for_entries<VEC>(x, [&](int j, float xj) {
        if (xj == -INFINITY || bin_of(s, xj) > bin) return;
        const double w = weight_of(s, xj);
        if (by_k || w >= a.min_p) push(xj, col + j, w);
      });
    }
    __syncthreads();
    if (sh.n > kList<WAVES>) return false;
    draw_from_list(r, u, by_k, a.top_p < 1.0, 0, sum);
    return true;
  }
  static __device__ __forceinline__ u64 target_of(float u, u64 all) {
    const double want = u > 0.f ? floor((double)u * (double)all) : 0.0;
    return want < (double)all && (u64)want < all ? (u64)want : all - 1;
  }
  __device__ __forceinline__ float log_share(float x, float sum) const {
    const float v = (x - s.m) * a.inv_t - logf(sum);
    return v < kLowest ? kLowest : v;
  }
  // The sum of one float a wave.
  __device__ __forceinline__ float block_sum(float x) {
    x = wave_sum(x);
    __syncthreads();
    if (lane == 0) sh.floats[wave] = x;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += sh.floats[w];
    return t;
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
  __device__ __forceinline__ Cut cut_of_equal(bool by_mass, u64 limit, u64 before, u64 in_front, unsigned key) {
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
      sh.upto = in_front + m * w;
    }
    __syncthreads();
    return {sh.key, sh.id};
  }
};

// One block a part of a row: every thread's largest logit, and the part's sum of exponentials. Memory-bound; it spares the kernel behind it all entries but those of the groups
// that can hold one which is kept.
template <typename T>
__global__ __launch_bounds__(256) void token_sample_groups_kernel(const SampleArgs a) {
  touch_args(a);
  constexpr int VEC = 16 / (int)sizeof(T), PIECES = kPart / (kGroups * VEC);
  __shared__ float tops[4], sums[4];
  const int64_t job = a.row0 * a.parts + blockIdx.x, r = job / a.parts;
  const int part = (int)(job % a.parts), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Row<T> row = row_of<T>(a, r);
  const bool odd = __builtin_amdgcn_readfirstlane(lead_of(row.x, row.len)) != 0;
  const int first = part * kPart + threadIdx.x * VEC, end = part * kPart + kPart < row.len ? part * kPart + kPart : row.len;
  float x[PIECES][VEC], m = -INFINITY;
  bool odd_one = false;
  if (end == part * kPart + kPart && !row.mask) {
    Piece<T, VEC> v[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const T *at = row.x + first + p * kGroups * VEC;
      v[p] = odd ? load_odd_piece<T, VEC>(at) : load_piece<T, VEC>(at);
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[p][j] = (float)v[p].v[j];
  } else {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) fetch<T, VEC>(row, odd, first + p * kGroups * VEC, end, x[p]);
  }
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      m = fmaxf(m, x[p][j]);
      odd_one = odd_one | !(x[p][j] < INFINITY);
    }
  a.group_max[job * kGroups + threadIdx.x] = m;
  m = wave_max(m);
  if (lane == 0) tops[wave] = m;
  odd_one = __syncthreads_or(odd_one);
  m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float c = a.inv_t * kLog2e, from = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum += __builtin_amdgcn_exp2f((x[p][j] - from) * c);
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.part_stats[2 * job] = m;
    a.part_stats[2 * job + 1] = odd_one ? __builtin_nanf("") : sums[0] + sums[1] + sums[2] + sums[3];
  }
}

template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 3 : 4) void token_sample_kernel(const SampleArgs a) {
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
  S t = {a, row, sh, __builtin_amdgcn_readfirstlane(lead_of(row.x, row.len)) != 0, a.top_p < 1.0, lane, wave, (int)(b0 < row.len ? b0 : row.len), (int)(b1 < row.len ? b1 : row.len), {}, false};
  const float c = a.inv_t * kLog2e;
  if (a.parts) {
    const float *stats = a.part_stats + 2 * r * a.parts, *tops = a.group_max + r * a.parts * kGroups;
    float m = -INFINITY, sum = 0.f;
    for (int i = 0; i < a.parts; ++i) m = fmaxf(m, stats[2 * i]);
    for (int i = 0; i < a.parts; ++i) sum += __builtin_amdgcn_exp2f((stats[2 * i] - (m == -INFINITY ? 0.f : m)) * c) * stats[2 * i + 1];
    if (!(sum == sum) || m == -INFINITY) {             // (no number, or +inf: a sum that is none)
      if (threadIdx.x == 0) {
        a.ids[r] = -1;
        a.logp[r] = sum == sum ? -INFINITY : __builtin_nanf("");
      }
      return;
    }
    t.s = scale_of<WAVES>(a, m, row.len);
    if (t.draw_from_groups(r, u, tops, sum)) return;
    __syncthreads();
  }
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
  const float mine = m;
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
  t.s = scale_of<WAVES>(a, m, row.len);
  const RowScale s = t.s;
  Cut cut = {0, 0x7fffffff};
  const bool by_k = a.top_k > 0 && a.top_k < row.len, by_p = a.top_p < 1.0;
  u64 whole = 0;                                       // by_p: the weight of all entries that may be chosen
  // Few entries can be kept: a list of them. Of the first top_k, what the threads' largest logits tell: so many entries are at least in the bins up to the one that holds
  // the top_k-th of these.
  const bool few = by_k && a.top_k <= WAVES * 16;
  if (few || a.min_p > 0.0) {
    int bin = kBins<WAVES> - 1;
    t.clear_bins(sh.count, sh.mass);
    if (threadIdx.x == 0) sh.n = 0;
    if (few) {
      if (mine > -INFINITY) atomicAdd(&sh.count[bin_of(s, mine)], 1u);
      if (threadIdx.x == 0) sh.bin = kBins<WAVES> - 1;
      __syncthreads();
      t.find_bin(sh.count, sh.mass, false, a.top_k);                      // (where fewer threads have an entry the last bin stays)
      bin = sh.bin;
    }
    __syncthreads();
    float sum = 0.f;
    if (few) {
      for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) {
        for_entries<VEC>(x, [&](int j, float xj) {
          sum += __builtin_amdgcn_exp2f((xj - m) * c);
          if (xj != -INFINITY && bin_of(s, xj) <= bin) t.push(xj, col + j, weight_of(s, xj));
        });
      });
      sum = t.block_sum(sum);                          // (its barriers: the list is there)
    } else {
      // (four weights at once and one branch for the few that are kept; a masked entry's is 2^-100, whose multiple of 2^-S is 0)
      u64 mass = 0;
      for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) {
        float y[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) y[j] = x[j];
#pragma unroll 1
        for (int j = 0; j < VEC; j += 4) {
          double w[4];
          bool any = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = weight_of(s, y[i]);
            mass += whole_of(s, w[i]);
            any = any | (w[i] >= a.min_p);
          }
          if (any)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (w[i] >= a.min_p && y[i] != -INFINITY) t.push(y[i], col + j + i, w[i]);
#pragma unroll
          for (int i = 0; i + 4 < VEC; ++i) y[i] = y[i + 4];
        }
      });
      t.over_waves(wave_sum64(mass), whole);           // (its barriers as well)
      sum = (float)((double)whole / s.one);
    }
    // (by min-p alone the first top_k have to be there for top-p to take its share of them)
    if (sh.n <= kList<WAVES> && (few || !(by_k && by_p) || sh.n >= a.top_k)) {
      t.draw_from_list(r, u, by_k, by_p, whole, sum);
      return;
    }
    __syncthreads();
    whole = 0;
  }
  auto histogram = [&](bool counts) {
    t.clear_bins(sh.count, sh.mass);
    for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int, const float *x) {
      for_entries<VEC>(x, [&](int j, float xj) {
        if (xj == -INFINITY) return;
        const int b = bin_of(s, xj);
        if (counts) atomicAdd(&sh.count[b], 1u);
        if (by_p) atomicAdd(&sh.mass[b], whole_of(s, weight_of(s, xj)));
      });
    });
    __syncthreads();
  };
  if (by_k || by_p) {
    histogram(by_k);
    if (by_p) whole = t.mass_before(sh.mass, kBins<WAVES>);
    u64 share = whole;                                 // what top-p takes its part of
    if (by_k) {
      u64 n = 0, all;
      for (int i = threadIdx.x; i < kBins<WAVES>; i += WAVES * 64) n += sh.count[i];
      t.over_waves(wave_sum64(n), all);
      if ((u64)a.top_k < all) {
        cut = t.cut_at(false, a.top_k);
        share = sh.upto;
        __syncthreads();
        if (by_p && t.spoiled) histogram(false);
      }
    }
    if (by_p) {
      const u64 limit = (u64)ceil(a.top_p * (double)share);
      cut = t.cut_at(true, limit < 1 ? 1 : limit);
    }
  }
  // sums of what is kept, of the waves' shares and, for the log-probability, of all
  u64 kept = 0;
  float sum = 0.f;
  auto weight = [&](int col, const float *x) {
    u64 k = 0;
    for_entries<VEC>(x, [&](int j, float xj) {
      if (xj == -INFINITY || !inside(cut, key_of(xj), col + j)) return;
      const double w = weight_of(s, xj);
      if (w >= a.min_p) k += whole_of(s, w);
    });
    return k;
  };
  for_pieces<T>(row, t.odd, t.begin, t.end, lane, [&](int col, const float *x) {
    kept += weight(col, x);
    if (!by_p)
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum += __builtin_amdgcn_exp2f((x[j] - m) * c);
  });
  kept = wave_sum64(kept);
  u64 all;
  u64 before = t.over_waves(kept, all);
  sum = by_p ? (float)((double)whole / s.one) : t.block_sum(sum);
  // the drawn entry is the first whose sum passes `target`
  const u64 target = S::target_of(u, all);
  if (before <= target && target < before + kept) {    // in this wave's columns
    sh.bin = t.begin;
    sh.n = t.end;
    sh.before = before;
  }
  __syncthreads();
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
    for_entries<VEC>(x, [&](int j, float xj) {
      if (found || xj == -INFINITY || !inside(cut, key_of(xj), col + j)) return;
      const double w = weight_of(s, xj);
      if (w >= a.min_p) at += whole_of(s, w);
      if (at <= target) return;
      found = true;
      a.ids[r] = col + j;
      a.logp[r] = t.log_share(xj, sum);
    });
  });
}

template <typename T>
void launch(const xrl_ctx *c, SampleArgs &a, int waves) {
  const int64_t most = kMaxBlocks / std::max(1, a.parts);
  for (a.row0 = 0; a.row0 < a.n_rows; a.row0 += most) {
    const dim3 grid((unsigned)std::min(a.n_rows - a.row0, most));
    if (a.parts) token_sample_groups_kernel<T><<<dim3((unsigned)(grid.x * a.parts)), dim3(256), 0, op_stream(c)>>>(a);
    if (waves == 1) token_sample_kernel<T, 1><<<grid, dim3(64), 0, op_stream(c)>>>(a);
    else if (waves == 4) token_sample_kernel<T, 4><<<grid, dim3(256), 0, op_stream(c)>>>(a);
    else if (waves == 8) token_sample_kernel<T, 8><<<grid, dim3(512), 0, op_stream(c)>>>(a);
    else token_sample_kernel<T, 16><<<grid, dim3(1024), 0, op_stream(c)>>>(a);
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
  // A wave a row where rows are short, or so many that they fill the chip; else a block of as many waves as pay for its barriers. us, fp32, no filter and the best 100 with top-p and min-p: 4000 x 64 by
  // a wave 17 and 20, by four 58 and 80; 4000 x 2000 63 and 104, 71 and 202; 32 x 500 10.8 and 27, 10.5 and 23. bf16, top-p alone, by 4, 8 and 16 waves: 200 x 4000 24, 21, 26; 2048 x 16000 224, 169,
  // 279; 200 x 32003 100, 59, 57; 8 x 128256 336, 175, 133.
  const bool many = a.n_rows > 2 * op_compute_units(c);
  const int waves = cols <= 256 || (many && cols <= 2048) ? 1 : cols <= 2048 ? 4 : a.n_rows > op_compute_units(c) || cols <= 16384 ? 8 : 16;
  // Long rows of which few entries can be kept: by groups. us, with top-p, without and with: the best 50 of 8 x 128256 51 and 35, of 2048 x 32003 140 and 118; 20 of 512 x 32003 38 and 35, of
  // 8 x 16384 28 and 30.
  const int64_t parts = (cols + kPart - 1) / kPart;
  if (!a.row_ptr && cols > kPart && (a.top_k > 0 ? (int64_t)a.top_k * 16 <= parts * kGroups : a.top_p == 1.0 && a.min_p > 0.0) && parts <= 1024) {
    const size_t tops = op_align((size_t)a.n_rows * parts * kGroups * 4);
    char *ws = nullptr;
    if (int rc = op_workspace(c, tops + (size_t)a.n_rows * parts * 8, &ws, who)) return rc;
    a.parts = (int)parts;
    a.group_max = (float *)ws;
    a.part_stats = (float *)(ws + tops);
  }
  logits->type == XRL_PREC_BF16 ? launch<bf16_t>(c, a, waves) : launch<float>(c, a, waves);
  OP_TRY(hipGetLastError());
  return XRL_OK;
}
