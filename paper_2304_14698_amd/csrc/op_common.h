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

// N elements from p, which may lie at any multiple of the element's size. STREAM: what is read for the last time, 16-byte pieces that leave no copy in
// the caches.
template <typename T, int N>
struct Piece {
  T v[N];
};
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename T, int N, bool STREAM = false>
__device__ __forceinline__ Piece<T, N> load_piece(const T *p) {
  Piece<T, N> x;
  if constexpr (STREAM) {
    u32x4 u[sizeof(x) / 16];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(x) / 16); ++i) u[i] = __builtin_nontemporal_load((const u32x4_any *)p + i);
    __builtin_memcpy(&x, u, sizeof(x));
  } else {
    __builtin_memcpy(&x, p, sizeof(x));
  }
  return x;
}
// N floats to p, rounded to T. STREAM: stores that leave no copy in the caches (16-byte pieces), for results that are larger than these.
template <typename T, int N, bool STREAM = false>
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
  if constexpr (STREAM) {
    u32x4 u[sizeof(x) / 16];
    __builtin_memcpy(u, &x, sizeof(x));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(x) / 16); ++i) __builtin_nontemporal_store(u[i], (u32x4_any *)p + i);
  } else {
    __builtin_memcpy(p, &x, sizeof(x));
  }
}
// Results of more bytes than all L2s together hold (eight of 4 MB) are stored past the caches.
inline bool streams(int64_t bytes) { return bytes > (int64_t)32 << 20; }

// Reductions over a wave by lane moves within the vector registers (a row of 16 lanes, then rows onto the next), the result in all lanes.
// A shuffle goes through the LDS, about 100 clocks each way: six of them for a maximum, two dozen for a row's sums.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_move(int old, int x) { return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xf, false); }
constexpr int kShr1 = 0x111, kShr2 = 0x112, kShr4 = 0x114, kShr8 = 0x118, kBcast15 = 0x142, kBcast31 = 0x143, kWaveShr1 = 0x138;
__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ float wave_max(float x) {
#define STEP(CTRL) x = fmaxf(x, __int_as_float(lane_move<CTRL, 0xf>(__float_as_int(x), __float_as_int(x))))
  STEP(kShr1); STEP(kShr2); STEP(kShr4); STEP(kShr8); STEP(kBcast15); STEP(kBcast31);
#undef STEP
  return last_lane(x);
}
__device__ __forceinline__ int wave_min(int x) {
#define STEP(CTRL) { const int o = lane_move<CTRL, 0xf>(x, x); x = o < x ? o : x; }
  STEP(kShr1) STEP(kShr2) STEP(kShr4) STEP(kShr8) STEP(kBcast15) STEP(kBcast31)
#undef STEP
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ float wave_sum(float x) {
#define STEP(CTRL, ROWS) x += __int_as_float(lane_move<CTRL, ROWS>(0, __float_as_int(x)))
  STEP(kShr1, 0xf); STEP(kShr2, 0xf); STEP(kShr4, 0xf); STEP(kShr8, 0xf); STEP(kBcast15, 0xa); STEP(kBcast31, 0xc);
#undef STEP
  return last_lane(x);
}

}  // namespace
