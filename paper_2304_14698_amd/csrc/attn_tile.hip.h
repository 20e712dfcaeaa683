// Tiles of attention in LDS: 32 or 64 rows (keys, or queries) of DP columns, as the matrix cores read them along a row and across rows.
//
// A tile's row is cut into pieces of 16 bytes, and piece p of row r lies at place p ^ swizzle(r). Read along rows (the contraction runs over columns),
// eight neighbouring lanes read one piece each of eight rows; read across rows (it runs over the rows), sixteen lanes read 32 bytes each of four rows.
// The swizzle spreads both over eight places, 128 bytes; the LDS has banks for 256, and reads still meet in them: with heads of 128 in bf16 conflicts are 46 to 50 % of the LDS's busy
// cycles in the kernels of packed attention, and 38 % in the cache's for single tokens.
#pragma once
#include "op_common.h"

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
#define XRL_LDS __attribute__((address_space(3)))

template <typename T>
using Vec = typename Operand<T>::vec;

// An LDS address as a pointer.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"
template <typename U>
__device__ __forceinline__ XRL_LDS U *lds_at(unsigned address) { return (XRL_LDS U *)address; }
#pragma clang diagnostic pop

template <typename T, int DP>
struct Tile {
  typedef Vec<T> vec;
  static constexpr int ES = (int)sizeof(T), RB = DP * ES, CPR = RB / 16, V = Operand<T>::V;
  static constexpr int SLABS = DP / (2 * V);          // matrix instructions' steps along a row
  static constexpr int STEP = 2 * V;                  // rows that one fragment across rows covers
  static constexpr int BLOCKS = DP / 32;

  static __device__ __forceinline__ int swizzle(int row) { return CPR >= 8 ? ((row & 3) << 1) | ((row >> 2) & 1) : (row & 2) | ((row >> 2) & 1); }

  // Rows r0 .. r0 + 31 (r0 a multiple of 32), columns of slab c: lane l holds row l % 32, columns V (2 c + l / 32) on.
  static __device__ __forceinline__ vec along(unsigned tile, int r0, int c, int lane) {
    const int l32 = lane & 31, x = (lane >> 5) ^ swizzle(l32);
    return *lds_at<const vec>(tile + (unsigned)((r0 + l32) * RB + ((2 * c ^ x) << 4)));
  }

  // Column 32 db + l % 32 of the STEP rows from r0 on (a multiple of STEP): in the order in which an accumulator tile holds its rows, so that 2 V of an
  // accumulator's registers are the other operand as they are. bf16: rows r0 + 4 g + 0 .. 3 and 8 more on; fp32: rows r0 + 4 g + 0 .. 3.
  static __device__ __forceinline__ vec across(unsigned tile, int r0, int db, int lane) {
    const int g = lane >> 5;
    if constexpr (ES == 2) {
      const int row = 4 * g + ((lane & 15) >> 2), piece = (4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swizzle(row);
      const unsigned at = tile + (unsigned)((r0 + row) * RB + (piece << 4) + (lane & 1) * 8);
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(at));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(at + 8 * RB));
      return __builtin_bit_cast(vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      vec x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 4 * g + j, piece = (8 * db + ((lane & 31) >> 2)) ^ swizzle(row);
        x[j] = *lds_at<const float>(tile + (unsigned)((r0 + row) * RB + (piece << 4) + (lane & 3) * 4));
      }
      return x;
    }
  }
};

// The other operand of a product over an accumulator's rows: registers of one slab (8 in bf16, rounded once; 4 in fp32).
template <typename T>
__device__ __forceinline__ Vec<T> acc_operand(const f32x16 &a, int slab) {
  if constexpr (sizeof(T) == 2) {
    const int o = 8 * slab;
    return pack_bf16x8(a[o], a[o + 1], a[o + 2], a[o + 3], a[o + 4], a[o + 5], a[o + 6], a[o + 7]);
  } else {
    const int o = 4 * slab;
    return f32x4{a[o], a[o + 1], a[o + 2], a[o + 3]};
  }
}

// What that operand's rounding left out, rounded in turn (bf16; fp32 leaves nothing out).
template <typename T>
__device__ __forceinline__ Vec<T> acc_rest(const f32x16 &a, int slab, const Vec<T> &rounded) {
  if constexpr (sizeof(T) == 2) {
    float rest[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) rest[n] = a[8 * slab + n] - (float)rounded[n];
    return pack_bf16x8(rest[0], rest[1], rest[2], rest[3], rest[4], rest[5], rest[6], rest[7]);
  } else {
    return rounded;
  }
}

// Rows of a tensor [rows, heads, dim] that a wave's scalar registers describe: loads behind the last one give zeros.
__device__ __forceinline__ u32x4 rows_descriptor(const void *p, unsigned bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  u32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane((unsigned)a);
  d[1] = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32) & 0xffffu);
  d[2] = __builtin_amdgcn_readfirstlane(bytes);
  d[3] = 0x00020000u;
  return d;
}

// 16 bytes a lane from `offset` behind the descriptor's base straight into LDS, lane i's at lds + 16 i. (In assembly for the reason given at lds_direct_load16: whoever
// reads the tile waits for vmcnt(0) and a barrier first.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_direct_rows16(u32x4 rows, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(rows), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ void wait_direct_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ROWS rows from p on (`left` of them are there, `stride` elements apart) into a tile; columns from dim on and rows that are not there as zeros. Every row begins at
// a multiple of 16 bytes and dim is whole pieces. The loads go past the registers: the tile is there behind wait_direct_loads() and a barrier.
template <typename T, int DP, int ROWS, int WAVES>
__device__ __forceinline__ void stage_tile(const T *p, int left, int64_t stride, int dim, unsigned tile, int wave, int lane) {
  using L = Tile<T, DP>;
  constexpr int N = ROWS * L::RB / 1024, EACH = (N + WAVES - 1) / WAVES;
  left = left < 0 ? 0 : left < ROWS ? left : ROWS;
  const unsigned step = (unsigned)stride * L::ES;
  const u32x4 rows = rows_descriptor(p, left > 0 ? (unsigned)(left - 1) * step + (unsigned)dim * L::ES : 0u);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int n = wave + i * WAVES;
    if (N % WAVES && n >= N) break;
    const int e = n * 64 + lane, row = e / L::CPR, piece = (e % L::CPR) ^ L::swizzle(row);
    lds_direct_rows16(rows, piece * L::V < dim ? (unsigned)row * step + (unsigned)piece * 16u : 0x80000000u, __builtin_amdgcn_readfirstlane(tile + n * 1024));
  }
}

// A row's fragments for the other operand: lane l holds columns V (2 c + l / 32) on of its row p (there: whether there is one).
template <typename T, int DP>
__device__ __forceinline__ void load_row(Vec<T> *x, const T *p, bool there, int dim, int g) {
  constexpr int V = Operand<T>::V;
#pragma unroll
  for (int c = 0; c < Tile<T, DP>::SLABS; ++c) {
    const int d = V * (2 * c + g);
    x[c] = Operand<T>::zero();
    if (there && d < dim) __builtin_memcpy(&x[c], __builtin_assume_aligned(p + d, 16), 16);
  }
}

// Accumulator tiles whose columns are rows of the result (lane l % 32: the row at p, registers: NB blocks of 32 of its columns from block db0 on), times f. `quads`: four
// columns may be stored together.
template <typename T, int NB>
__device__ __forceinline__ void store_row(T *p, bool there, int dim, bool quads, const f32x16 (&acc)[NB], float f, int g, int db0 = 0) {
  if (!there) return;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * (db0 + db) + 8 * q + 4 * g;
      const float v[4] = {acc[db][4 * q] * f, acc[db][4 * q + 1] * f, acc[db][4 * q + 2] * f, acc[db][4 * q + 3] * f};
      if (quads) {
        if (d < dim) store4<T>(p + d, v);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (d + j < dim) p[d + j] = (T)v[j];
      }
    }
}

__device__ __forceinline__ f32x16 zero_acc() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// The same value of lane l and lane l ^ 32 together.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What stands in a key or value that a row does not see may reach it through a product with 0. Where results of the ordinary way are not finite, a kernel goes over its keys again with
// such places kept apart (SAFE), 32 columns of the result at a time: that takes few registers, which would otherwise count for every call.
//
// acc += a b where b is 0 at places that do not count: what a holds there reaches nothing, an infinity or NaN neither. `seen` has 1 at the places of b that
// count; an a that is not finite makes NaN of the results that see it.
template <typename T>
__device__ __forceinline__ void mma_seen(Vec<T> a, const Vec<T> &b, const Vec<T> &seen, f32x16 &acc) {
  Vec<T> odd;
#pragma unroll
  for (int j = 0; j < Operand<T>::V; ++j) {
    const float v = (float)a[j];
    const bool fine = fabsf(v) < INFINITY;
    odd[j] = (T)(fine ? 0.f : 1.f);
    a[j] = fine ? a[j] : (T)0.f;
  }
  f32x16 n = zero_acc();
  Operand<T>::mma(odd, seen, n);
  Operand<T>::mma(a, b, acc);
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = n[i] > 0.f ? __builtin_nanf("") : acc[i];
}

__device__ __forceinline__ bool all_finite(const f32x16 &a) {
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) z = fmaf(a[i], 0.f, z);
  return z == 0.f;
}

// One step of a softmax that runs along: KT keys and values in tiles, q the fragments of 32 queries, one a lane. o += sum over the keys n of 2^(s_n c - mc) v_n, l their sum in
// this lane's half of the keys, mc the reference of the exponentials. `whole`: every query of the wave sees all keys, else key
// n + 4 (lane / 32) where sees(n): n is a constant at each place. NB blocks of
// 32 of v's columns, from block db0 on. SAFE: what stands in keys and values that are not seen reaches nothing.
template <typename T, int DP, int KT, bool SAFE, int NB, typename Sees>
__device__ __forceinline__ void add_tile(unsigned kt, unsigned vt, const Vec<T> *q, float c, bool whole, Sees sees, f32x16 (&o)[NB], float &mc, float &l, int lane, int db0 = 0) {
  using L = Tile<T, DP>;
  using vec = Vec<T>;
  const int g = lane >> 5;
  f32x16 s[KT / 32];
#pragma unroll
  for (int kb = 0; kb < KT / 32; ++kb) {
    s[kb] = zero_acc();
#pragma unroll
    for (int x = 0; x < L::SLABS; ++x) Operand<T>::mma(L::along(kt, 32 * kb, x, lane), q[x], s[kb]);
  }
  if (!whole) {
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = sees(32 * kb + acc_row(r, 0)) ? s[kb][r] : -INFINITY;
  }
  float mx = s[0][0];
#pragma unroll
  for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
  mx = half_max(mx) * c;
  // The reference of the exponentials follows the maximum only where that has grown by 2^8: until then sums and results are up to 2^8 times as large, and nothing is
  // multiplied. Each row by its own maximum, whatever shares its wave.
  const bool grown = mx > mc + 8.f;
  if (__ballot(grown)) {
    const float m = grown ? mx : mc, f = __builtin_amdgcn_exp2f(mc - m);
    mc = m;
    l *= f;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] *= f;
  }
#pragma unroll
  for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], c, -mc));
      l += s[kb][r];
    }
#pragma unroll
  for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
    for (int x = 0; x < 32 / L::STEP; ++x) {
      const vec p = acc_operand<T>(s[kb], x);
      if (SAFE && !whole) {
        vec seen;
#pragma unroll
        for (int n = 0; n < L::V; ++n) seen[n] = (T)(sees(32 * kb + acc_row(x * L::V + n, 0)) ? 1.f : 0.f);
#pragma unroll
        for (int db = 0; db < NB; ++db) mma_seen<T>(L::across(vt, 32 * kb + x * L::STEP, db0 + db, lane), p, seen, o[db]);
      } else {
#pragma unroll
        for (int db = 0; db < NB; ++db) Operand<T>::mma(L::across(vt, 32 * kb + x * L::STEP, db0 + db, lane), p, o[db]);
      }
    }
}

// Packed sequences. Tiles of BM rows are counted so that sequence s has the numbers from ptr[s] / BM + s on: no two sequences share one, the last few of a
// sequence may be empty, and n / BM + sequences are enough for all.
struct Span {
  int64_t begin;
  int len;
};
__device__ __forceinline__ int64_t end_at(const int32_t *ptr, int64_t s, int64_t n) {
  const int64_t x = ptr[s];
  return x < 0 ? 0 : x < n ? x : n;
}
__device__ __forceinline__ Span span_of(const int32_t *ptr, int64_t s, int64_t n) {
  const int64_t b = end_at(ptr, s, n), e = end_at(ptr, s + 1, n);
  return {b, e > b ? (int)(e - b) : 0};
}
// The last sequence that begins at a row or in front of it, or -1.
__device__ __forceinline__ int64_t last_begun(const int32_t *ptr, int64_t seqs, int64_t n, int64_t row, int lane) {
  int64_t lo = 0, hi = seqs;
  do {
    const int64_t step = (hi - lo + 63) / 64, p = lo + lane * step;
    const unsigned long long b = __ballot(p < hi && end_at(ptr, p < hi ? p : lo, n) <= row);
    const int c = ~b ? __builtin_ctzll(~b) : 64;
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  } while (hi - lo > 1);
  return lo;
}
// The sequence of a row, or -1.
__device__ __forceinline__ int64_t sequence_of_row(const int32_t *ptr, int64_t seqs, int64_t n, int64_t row, int lane) {
  const int64_t s = last_begun(ptr, seqs, n, row, lane);
  return s >= 0 && row < end_at(ptr, s + 1, n) ? s : -1;
}
// The sequence that tile number u belongs to, or -1; 64 of them are looked at at once.
__device__ __forceinline__ int64_t sequence_of(const int32_t *ptr, int64_t seqs, int64_t n, int bm, int64_t u, int lane) {
  int64_t lo = 0, hi = seqs;
  do {
    const int64_t step = (hi - lo + 63) / 64, p = lo + lane * step;
    const bool before = p < hi && end_at(ptr, p < hi ? p : lo, n) / bm + p <= u;
    const unsigned long long b = __ballot(before);
    const int c = ~b ? __builtin_ctzll(~b) : 64;
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  } while (hi - lo > 1);
  return lo;
}

}  // namespace
