// Shared by the operators of the recurrent block (scan.hip, block_norm.hip, quant.hip):
// argument checks, vector accesses and the arithmetic they have in common.
#pragma once

#include "internal.h"

namespace spz {

// Sets the calling thread's error message ("call: what") and returns `code`.
int op_error(int code, const char* call, const char* what) noexcept;

// ----------------------------------------------------------------------------- checks
constexpr int64_t OP_MAX_EXTENT = (int64_t)1 << 31;   // extents are below this
constexpr int64_t OP_MAX_STRIDE = (int64_t)1 << 42;   // strides in bytes do not wrap

inline bool op_prec_ok(int32_t prec) { return prec == SPZ_PREC_FP32 || prec == SPZ_PREC_BF16; }
inline int op_size(int32_t prec) { return prec == SPZ_PREC_BF16 ? 2 : 4; }
inline bool op_extent_ok(int64_t n) { return n >= 0 && n < OP_MAX_EXTENT; }
__host__ __device__ inline bool op_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool op_in_stride_ok(int64_t s) { return s >= 0 && s < OP_MAX_STRIDE; }
// Rows of `width` elements at stride s do not overlap (one row: any stride).
inline bool op_out_stride_ok(int64_t rows, int64_t width, int64_t s) {
  return op_in_stride_ok(s) && (rows <= 1 || s >= width);
}
// Elements of a [n0, n1, width] output do not overlap, for either order of the outer two.
inline bool op_out_strides_ok(int64_t n0, int64_t n1, int64_t width, int64_t s0, int64_t s1) {
  if (n0 == 0 || n1 == 0 || width == 0) return op_in_stride_ok(s0) && op_in_stride_ok(s1);
  if (!op_out_stride_ok(n0, width, s0) || !op_out_stride_ok(n1, width, s1)) return false;
  if (n0 <= 1 || n1 <= 1) return true;
  // The inner dimension's span, (n - 1) strides and a row, fits between two elements of the outer one. (By
  // division, as the product may wrap; the strides are at least `width` here.)
  return s0 >= s1 ? (s0 - width) / s1 >= n1 - 1 : (s1 - width) / s0 >= n0 - 1;
}

inline int64_t op_div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// launch(first, grid) over `blocks` workgroups of `threads`, as many dispatches as it takes. A dispatch counts its
// work-items in 32 bits: of a grid with more of them only a part runs, and no call reports it.
constexpr int64_t OP_DISPATCH = (int64_t)1 << 31;
template <typename F> void op_dispatch(int64_t blocks, int64_t threads, F&& launch) {
  const int64_t most = OP_DISPATCH / threads;
  for (int64_t first = 0; first < blocks; first += most)
    launch(first, dim3((unsigned)(blocks - first < most ? blocks - first : most)));
}

inline int op_launched(const char* call) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPZ_OK : op_error(SPZ_EHIP, call, hipGetErrorString(e));
}

// ----------------------------------------------------------------------------- vectors
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements of one 16-byte access.
template <typename T> constexpr int OP_VEC = 16 / (int)sizeof(T);

__device__ inline void unpack(const u32x4& w, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = w[i];   // a bit_cast of w[i] itself would take the vector's first element
    x[i] = __builtin_bit_cast(float, u);
  }
}
__device__ inline void unpack(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
  }
}
__device__ inline u32x4 pack(const float (&x)[4]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, x[i]);
  return w;
}
__device__ inline u32x4 pack(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  return w;
}

// Sixteen bytes at any alignment of the element type (the hardware takes 16-byte accesses of global
// memory at any address; ones that straddle cache lines cost an access more), or the first n < OP_VEC
// elements of them, with zeros behind.
template <typename T> __device__ inline u32x4 load16(const T* p) {
  u32x4 w;
  __builtin_memcpy(&w, p, 16);
  return w;
}
template <typename T> __device__ inline void store16(T* p, const u32x4& w) { __builtin_memcpy(p, &w, 16); }
template <typename T> __device__ inline u32x4 load_part(const T* p, int n) {
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < OP_VEC<T> - 1; ++i)
    if (i < n) {
      if (sizeof(T) == 4) w[i & 3] = __builtin_bit_cast(uint32_t, to_f<T>(p[i]));
      else w[(i / 2) & 3] |= (__builtin_bit_cast(uint32_t, to_f<T>(p[i])) >> 16) << (16 * (i & 1));
    }
  return u32x4{w[0], w[1], w[2], w[3]};
}
template <typename T> __device__ inline void store_part(T* p, const u32x4& v, int n) {
  const uint32_t w[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int i = 0; i < OP_VEC<T> - 1; ++i)
    if (i < n) {
      const uint32_t bits = sizeof(T) == 4 ? w[i & 3] : (i & 1) ? w[(i / 2) & 3] & 0xFFFF0000u : w[(i / 2) & 3] << 16;
      p[i] = from_f<T>(__builtin_bit_cast(float, bits));   // exact: the value is one of T
    }
}

// ----------------------------------------------------------------------------- arithmetic
// a = 1 / (1 + exp(-x)) and b = 1 - a, each to 7 units of 2^-24 of itself: with e = exp(-|x|), which cannot overflow, the
// larger one is 1 / (1 + e) and the other one e / (1 + e). The hardware's exponential and reciprocal (1 ulp) serve. The
// exponential's argument t = -|x| log2(e) would lose |t| 2^-24 to its rounding (62 units at |x| = 80), so what e lacks, the
// factor exp(s), s = -|x| - t ln 2, is put back as 1 + s. The constant is two ulp above log2(e), so that s >= 0 whatever t's
// rounding: held to [0, 1], which costs no instruction, it is 0 instead of NaN where x is infinite.
__device__ inline void sigmoid2(float x, float& a, float& b) {
  constexpr float LOG2E_ABOVE = 0x1.71547ap+0f, LN2 = 0x1.62e43p-1f, LN2_LOW = -0x1.05c61p-29f;
  const float m = __builtin_fabsf(x), t = m * -LOG2E_ABOVE;
  const float s = __builtin_amdgcn_fmed3f(fmaf(t, -LN2_LOW, fmaf(t, -LN2, -m)), 0.0f, 1.0f);
  const float p = __builtin_amdgcn_exp2f(t), e = fmaf(p, s, p);
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  a = x < 0.0f ? small : big;
  b = x < 0.0f ? big : small;
}

// Dropout's 16-bit words of elements 8 blk .. 8 blk + 7 (two to a word, low half first).
constexpr uint32_t P_DROP = 5;
// philox() with each round's two products as one 32 x 32 -> 64 instruction and its two exclusive ors as
// one three-operand instruction: these rounds are a fifth of what a fused kernel computes.
__device__ inline U4 drop_words(uint64_t blk, uint64_t seed, uint32_t step, uint32_t tensor) {
  uint32_t c0 = (uint32_t)blk, c1 = step, c2 = P_DROP + ((uint32_t)(blk >> 32) << 8), c3 = tensor;
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c1, k0, 0x96);
    c1 = (uint32_t)p1;
    c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c3, k1, 0x96);
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return U4{c0, c1, c2, c3};
}
__device__ inline uint32_t drop_half(const U4& w, int i) {
  const uint32_t v = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
  return (i & 1) ? v >> 16 : v & 0xFFFFu;
}
// p as 65536ths, rounded to nearest, ties to even (p in [0, 1]).
inline uint32_t drop_threshold(float p) { return (uint32_t)__builtin_nearbyint((double)p * 65536.0); }
inline float drop_gain(uint32_t d) { return d < 65536u ? (float)(65536.0 / (65536.0 - d)) : 0.0f; }

}  // namespace spz
