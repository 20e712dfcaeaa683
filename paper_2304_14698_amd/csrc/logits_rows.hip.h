// Rows of logits, dense or ragged, under a mask: where they lie and how a wave reads them.
#pragma once
#include "op_common.h"

#include <cmath>

using namespace xrl;

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.402823466e38f;        // also a maximum that no entry has reached yet: -inf - kLowest is -inf, not NaN

template <typename T>
struct Row {
  const T *x;
  const uint8_t *mask;
  int64_t begin;                // ragged: of the flat arrays
  int len;
};

// Row r. What a row's ends say outside the array counts as not there.
template <typename T, typename Args>
__device__ __forceinline__ Row<T> row_of(const Args &a, int64_t r) {
  Row<T> o;
  if (a.row_ptr) {
    int64_t b = a.row_ptr[r], e = a.row_ptr[r + 1];
    b = b < 0 ? 0 : b;
    e = e > a.n_cols ? a.n_cols : e;
    o.begin = b;
    o.len = e > b ? (int)(e - b) : 0;
    if (o.len == 0) o.begin = 0;
    o.x = (const T *)a.logits + o.begin;
    o.mask = a.mask ? a.mask + o.begin : nullptr;
  } else {
    o.begin = r * a.stride;
    o.len = (int)a.n_cols;
    o.x = (const T *)a.logits + o.begin;
    o.mask = a.mask ? a.mask + r * a.mask_stride : nullptr;
  }
  return o;
}

// bf16 pieces of 16 bytes that lie 2 bytes behind a multiple of 4 take longer than all others, and every second row of an odd length has nothing else: us,
// 4096 rows of 32003 61.5, of 32002 55. Such a row's pieces are read from the element before on, five words, and shifted (then 55.4), which leaves every sum
// its order wherever the row lies; where each entry stands by itself, in the gradient, a row's pieces begin at the element before its first.
template <typename T>
__device__ __forceinline__ int lead_of(const T *p, int len) { return sizeof(T) == 2 && len > 0 ? (int)((uintptr_t)p >> 1 & 1) : 0; }

// VEC elements from such a p. (What is read beside them lies in the same words as the first and the last.)
template <typename T, int VEC>
__device__ __forceinline__ Piece<T, VEC> load_odd_piece(const T *p) {
  Piece<T, VEC> x;
  if constexpr (sizeof(T) == 2) {
    unsigned u[VEC / 2 + 1], s[VEC / 2];
    __builtin_memcpy(u, __builtin_assume_aligned(p - 1, 4), VEC * 2);
    __builtin_memcpy(u + VEC / 2, __builtin_assume_aligned(p - 1 + VEC, 4), 4);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) s[i] = __builtin_amdgcn_alignbit(u[i + 1], u[i], 16);
    __builtin_memcpy(&x, s, sizeof(x));
  } else {
    x = load_piece<T, VEC>(p);
  }
  return x;
}

// Columns col .. col + VEC - 1 of the row as fp32, -inf where nothing may be chosen and from c1 on.
template <typename T, int VEC>
__device__ __forceinline__ void fetch(const Row<T> &row, bool odd, int col, int c1, float *x) {
  if (col + VEC <= c1) {
    const Piece<T, VEC> p = odd ? load_odd_piece<T, VEC>(row.x + col) : load_piece<T, VEC>(row.x + col);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = (float)p.v[j];
    if (row.mask) {
      const Piece<uint8_t, VEC> m = load_piece<uint8_t, VEC>(row.mask + col);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = m.v[j] ? x[j] : -INFINITY;
    }
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = col + j < c1 && (!row.mask || row.mask[col + j]) ? (float)row.x[col + j] : -INFINITY;
  }
}

// Checks the rows of a call and writes what its kernels have of them.
template <typename Args>
int check_logits(const xrl_ctx *c, const xrl_logits_desc *l, const char *who, Args &a) {
  if (!c || !l) return fail(XRL_ERR_NULL, "%s: ctx or logits is NULL", who);
  if (!op_type_ok(l->type)) return fail(XRL_ERR_UNSUPPORTED, "%s: type %d", who, l->type);
  if (!(l->temperature > 0.f) || !std::isfinite(l->temperature)) return fail(XRL_ERR_VALUE, "%s: temperature %g", who, (double)l->temperature);
  if (!std::isfinite(1.f / l->temperature * kLog2e)) return fail(XRL_ERR_VALUE, "%s: temperature %g", who, (double)l->temperature);
  if (l->n_rows < 0 || l->n_cols < 0 || (!l->d_row_ptr && (l->stride < l->n_cols || (l->d_mask && l->mask_stride != 0 && l->mask_stride < l->n_cols))))
    return fail(XRL_ERR_SHAPE, "%s: %lld rows of %lld columns, strides %lld and %lld", who, (long long)l->n_rows, (long long)l->n_cols,
                (long long)l->stride, (long long)l->mask_stride);
  if (l->n_cols > INT32_MAX - 65536 || l->n_rows > INT32_MAX)
    return fail(XRL_ERR_UNSUPPORTED, "%s: %lld rows of %lld columns", who, (long long)l->n_rows, (long long)l->n_cols);
  if (l->n_rows > 0 && l->n_cols > 0 && !l->d_logits) return fail(XRL_ERR_NULL, "%s: d_logits is NULL", who);
  if ((uintptr_t)l->d_logits % (l->type == XRL_PREC_BF16 ? 2 : 4) || (uintptr_t)l->d_row_ptr % 4)
    return fail(XRL_ERR_SHAPE, "%s: a pointer that is no multiple of its elements' size", who);
  a = Args{};
  a.logits = l->d_logits; a.row_ptr = l->d_row_ptr; a.mask = l->d_mask;
  a.n_rows = l->n_rows; a.n_cols = l->n_cols; a.stride = l->stride; a.mask_stride = l->mask_stride;
  a.inv_t = 1.f / l->temperature;
  return XRL_OK;
}

}  // namespace
