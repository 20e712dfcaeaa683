// What the operators' translation units share: the context's stream and workspace, and small pieces of kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mma.hip.h"
#include "xrl_internal.h"

#define OP_TRY(expr)                                                                          \
  do {                                                                                        \
    hipError_t e_ = (expr);                                                                   \
    if (e_ != hipSuccess)                                                                     \
      return xrl::fail(XRL_ERR_HIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, __LINE__); \
  } while (0)

namespace xrl {
// Implemented in the device translation unit.
hipStream_t op_stream(const xrl_ctx *c);
int op_compute_units(const xrl_ctx *c);
// The operators' workspace of at least `bytes` bytes. It grows only; memory that a captured call was given stays until the context goes,
// and a capture that needs more than there is is refused.
int op_workspace(xrl_ctx *c, size_t bytes, char **ws, const char *who);
}  // namespace xrl

namespace {

constexpr int64_t kMaxBlocks = 1 << 22;   // of one launch: a grid's threads are counted in 32 bits

inline size_t op_align(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

inline bool op_type_ok(int32_t type) { return type == XRL_PREC_FP32 || type == XRL_PREC_BF16; }

// Whether rows of `stride` elements of `elem` bytes from p on all begin at multiples of 16 bytes.
inline bool rows_aligned(const void *p, int64_t stride, int elem) { return ((uintptr_t)p | (uintptr_t)(stride * elem)) % 16 == 0; }

// N elements from p, which may lie at any multiple of the element's size.
template <typename T, int N>
struct Piece {
  T v[N];
};
template <typename T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T *p) {
  Piece<T, N> x;
  __builtin_memcpy(&x, p, sizeof(x));
  return x;
}
template <typename T, int N>
__device__ __forceinline__ void store_piece(T *p, const float *v) {
  Piece<T, N> x;
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
    unsigned u[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) u[i] = cvt_pk_bf16(v[2 * i], v[2 * i + 1]);
    __builtin_memcpy(&x, u, sizeof(x));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x.v[i] = (T)v[i];
  }
  __builtin_memcpy(p, &x, sizeof(x));
}

}  // namespace
