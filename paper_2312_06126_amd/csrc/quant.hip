// The 8-bit integer product with a scale for each row of the input and each output channel
// (spz_quant_*).
//
//   y[m, n] = s[m] w_scale[n] sum_k q[m, k] w[n, k] + bias[n],   s[m] = max_k |x[m, k]| / 127
//
// Both operands are kept as fragments: 1 KB pieces of 32 rows by 32 bytes of k in the order in which
// one wave feeds v_mfma_i32_32x32x32_i8 (lane l: 16 bytes of row l % 32, k from 16 (l / 32)), zeros
// past the edges, k innermost. A wave's loads are then whole, contiguous kilobytes.
#include "ops.h"

namespace spz {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
constexpr int64_t QUANT_MAX_INNER = 131072;   // 127^2 of these still fit 32 bits
constexpr int FRAG = 1024;

inline int64_t frag_blocks(int64_t n) { return op_div_up(n, 32); }

__device__ inline uint32_t wave_max(uint32_t m) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_xor(m, d);
    m = o > m ? o : m;
  }
  return m;
}
// The row's scale from the largest |x| as bits, and whether the row quantises to zeros: infinity and
// NaN have the largest bits.
__device__ inline float row_scale(uint32_t bits, bool& zero) {
  const float s = bits >= 0x7F800000u ? __builtin_nanf("") : __builtin_bit_cast(float, bits) / 127.0f;
  zero = !(s > 0.0f);
  return s;
}
__device__ inline int quantised(float x, float s) {
  const float q = rintf(x / s);
  return (int)fminf(fmaxf(q, -127.0f), 127.0f);
}

// Rows of integers: one wave a row, which it reads twice. q [rows, width] at q_row, or (FRAGS) as
// fragments over 32 * frag_blocks(rows) rows.
template <typename T, bool FRAGS>
__global__ __launch_bounds__(256) void quant_rows(const T* x, int64_t x_row, int64_t rows, int64_t width, int8_t* q,
                                                  int64_t q_row, float* scale) {
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  const int64_t steps = (width + 31) / 32;
  if (row >= (FRAGS ? (rows + 31) / 32 * 32 : rows)) return;
  const T* p = x + row * x_row;
  uint32_t m = 0;
  if (row < rows)
    for (int64_t c = lane; c < width; c += 64) {
      const uint32_t b = __builtin_bit_cast(uint32_t, to_f<T>(p[c])) & 0x7FFFFFFFu;
      m = b > m ? b : m;
    }
  bool zero;
  const float s = row_scale(wave_max(m), zero);
  if (lane == 0 && row < rows) scale[row] = s;
  for (int64_t c = lane; c < (FRAGS ? steps * 32 : width); c += 64) {
    const int v = c < width && row < rows && !zero ? quantised(to_f<T>(p[c]), s) : 0;
    if (FRAGS) q[(row / 32 * steps + c / 32) * FRAG + (c % 32 / 16 * 32 + row % 32) * 16 + c % 16] = (int8_t)v;
    else q[row * q_row + c] = (int8_t)v;
  }
}

__global__ __launch_bounds__(256) void quant_pack(const int8_t* q, int64_t q_row, int64_t outer, int64_t inner, int8_t* image) {
  const int64_t steps = (inner + 31) / 32, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (outer + 31) / 32 * steps * FRAG) return;
  const int64_t frag = i / FRAG, lane = i % FRAG / 16;
  const int64_t n = frag / steps * 32 + lane % 32, k = frag % steps * 32 + lane / 32 * 16 + i % 16;
  image[i] = n < outer && k < inner ? q[n * q_row + k] : (int8_t)0;
}

// One wave a 32 x 32 tile of y.
template <typename T>
__global__ __launch_bounds__(256) void quant_product(const int8_t* x, const int8_t* w, const float* xs, const float* ws,
                                                     const float* bias, T* y, int64_t y_row, int64_t rows, int64_t outer,
                                                     int64_t steps) {
  const int64_t nb = (outer + 31) / 32, tile = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (tile >= (rows + 31) / 32 * nb) return;
  const int lane = threadIdx.x % 64;
  const i32x4* a = reinterpret_cast<const i32x4*>(x) + tile / nb * steps * 64 + lane;
  const i32x4* b = reinterpret_cast<const i32x4*>(w) + tile % nb * steps * 64 + lane;
  i32x16 acc = {};
  for (int64_t s = 0; s < steps; ++s) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[s * 64], b[s * 64], acc, 0, 0, 0);
  const int64_t n = tile % nb * 32 + lane % 32;
  if (n >= outer) return;
  const float sw = ws[n], bn = bias ? bias[n] : 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t m = tile / nb * 32 + i / 4 * 8 + lane / 32 * 4 + i % 4;
    if (m < rows) y[m * y_row + n] = from_f<T>((float)acc[i] * (xs[m] * sw) + bn);
  }
}

const char* quant_check(int32_t prec, int64_t rows, int64_t outer, int64_t inner) {
  if (!op_prec_ok(prec)) return "unknown precision";
  if (!op_extent_ok(rows) || !op_extent_ok(outer) || !op_extent_ok(inner)) return "extent out of range";
  if (inner > QUANT_MAX_INNER) return "inner above 131072";
  if (outer && rows > ((int64_t)1 << 40) / outer) return "rows * outer out of range";
  return nullptr;
}
int64_t quant_workspace(int64_t rows, int64_t inner) {   // q as fragments, then the scales
  return frag_blocks(rows) * frag_blocks(inner) * FRAG + op_div_up(rows, 4) * 16;
}

template <typename T>
void quant_launch(int64_t rows, int64_t outer, int64_t inner, const void* x, int64_t x_row, const void* image,
                  const float* w_scale, const float* bias, void* y, int64_t y_row, void* ws, hipStream_t s) {
  const int64_t mb = frag_blocks(rows), nb = frag_blocks(outer), steps = frag_blocks(inner);
  int8_t* q = static_cast<int8_t*>(ws);
  float* xs = reinterpret_cast<float*>(q + mb * steps * FRAG);
  quant_rows<T, true><<<dim3((unsigned)op_div_up(mb * 32, 4)), 256, 0, s>>>(static_cast<const T*>(x), x_row, rows, inner, q, 0, xs);
  quant_product<T><<<dim3((unsigned)op_div_up(mb * nb, 4)), 256, 0, s>>>(q, static_cast<const int8_t*>(image), xs, w_scale, bias,
                                                                       static_cast<T*>(y), y_row, rows, outer, steps);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int spz_quant_rows(int32_t prec, int64_t rows, int64_t width, const void* x, int64_t x_row, int8_t* q, int64_t q_row,
                   float* scale, void* hip_stream) {
  const char* call = "spz_quant_rows";
  if (!op_prec_ok(prec)) return op_error(SPZ_EINVAL, call, "unknown precision");
  if (!op_extent_ok(rows) || !op_extent_ok(width)) return op_error(SPZ_EINVAL, call, "extent out of range");
  if (width && rows > ((int64_t)1 << 44) / width) return op_error(SPZ_EINVAL, call, "extents out of range");
  if (rows > 0 && (!scale || (width > 0 && (!x || !q)))) return op_error(SPZ_EINVAL, call, "NULL array");
  if (!op_aligned(x, op_size(prec)) || !op_aligned(scale, 4)) return op_error(SPZ_EINVAL, call, "array not aligned to its type");
  if (!op_in_stride_ok(x_row)) return op_error(SPZ_EINVAL, call, "input stride out of range");
  if (!op_out_stride_ok(rows, width, q_row)) return op_error(SPZ_EINVAL, call, "rows of q overlap");
  if (rows == 0) return SPZ_OK;
  const dim3 grid((unsigned)op_div_up(rows, 4));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (prec == SPZ_PREC_BF16)
    quant_rows<bf16_t, false><<<grid, 256, 0, s>>>(static_cast<const bf16_t*>(x), x_row, rows, width, q, q_row, scale);
  else
    quant_rows<float, false><<<grid, 256, 0, s>>>(static_cast<const float*>(x), x_row, rows, width, q, q_row, scale);
  return op_launched(call);
}

int64_t spz_quant_image_bytes(int64_t outer, int64_t inner) {
  const char* bad = quant_check(SPZ_PREC_FP32, 0, outer, inner);
  if (bad) return op_error(SPZ_EINVAL, "spz_quant_image_bytes", bad);
  return frag_blocks(outer) * frag_blocks(inner) * FRAG;
}

int spz_quant_pack(int64_t outer, int64_t inner, const int8_t* q, int64_t q_row, void* image, void* hip_stream) {
  const char* call = "spz_quant_pack";
  const char* bad = quant_check(SPZ_PREC_FP32, 0, outer, inner);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const int64_t bytes = frag_blocks(outer) * frag_blocks(inner) * FRAG;
  if (bytes > 0 && (!q || !image)) return op_error(SPZ_EINVAL, call, "NULL array");
  if (!op_aligned(image, 16)) return op_error(SPZ_EINVAL, call, "image not aligned to 16 bytes");
  if (!op_in_stride_ok(q_row)) return op_error(SPZ_EINVAL, call, "input stride out of range");
  if (bytes / 256 >= OP_MAX_EXTENT) return op_error(SPZ_EINVAL, call, "extents out of range");
  if (bytes == 0) return SPZ_OK;
  quant_pack<<<dim3((unsigned)op_div_up(bytes, 256)), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(
      q, q_row, outer, inner, static_cast<int8_t*>(image));
  return op_launched(call);
}

int64_t spz_quant_linear_workspace(int32_t prec, int64_t rows, int64_t outer, int64_t inner) {
  const char* bad = quant_check(prec, rows, outer, inner);
  if (bad) return op_error(SPZ_EINVAL, "spz_quant_linear_workspace", bad);
  return quant_workspace(rows, inner);
}

int spz_quant_linear(int32_t prec, int64_t rows, int64_t outer, int64_t inner, const void* x, int64_t x_row,
                     const void* image, const float* w_scale, const float* bias, void* y, int64_t y_row,
                     void* workspace, int64_t workspace_bytes, void* hip_stream) {
  const char* call = "spz_quant_linear";
  const char* bad = quant_check(prec, rows, outer, inner);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const bool some = rows > 0 && outer > 0;
  if (some && (!w_scale || !y || (inner > 0 && (!x || !image)))) return op_error(SPZ_EINVAL, call, "NULL array");
  if (!op_aligned(x, op_size(prec)) || !op_aligned(y, op_size(prec)) || !op_aligned(w_scale, 4) || !op_aligned(bias, 4))
    return op_error(SPZ_EINVAL, call, "array not aligned to its type");
  if (!op_aligned(image, 16)) return op_error(SPZ_EINVAL, call, "image not aligned to 16 bytes");
  if (!op_in_stride_ok(x_row)) return op_error(SPZ_EINVAL, call, "input stride out of range");
  if (!op_out_stride_ok(rows, outer, y_row)) return op_error(SPZ_EINVAL, call, "rows of y overlap");
  const int64_t need = quant_workspace(rows, inner);
  if (need > 0 && (!workspace || workspace_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
  if (need > 0 && !op_aligned(workspace, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
  if (!some) return SPZ_OK;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (prec == SPZ_PREC_BF16)
    quant_launch<bf16_t>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s);
  else
    quant_launch<float>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s);
  return op_launched(call);
}

}  // extern "C"
