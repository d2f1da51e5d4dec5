// Linear attention with a decay for each head: forward, backward and single steps.
//
// Four results are one recurrence in four roles. With R_p = d R_{p-1} + in b_p^T c_p and o_p = out a_p R_p,
//     y  = o(a, b, c = query, key, value), forward in time, R = S;
//     dq = o(dy, value, key), forward in time, R = S^T (both: in = 1, out = scale);
//     dk = o(value, dy, query) and dv = o(key, query, dy), backward in time, R = G^T and G (in = scale, out = 1),
// where the gradient to the last state is not decayed on its way in, and the one to the first is on its way out.
#include "ops.h"

namespace spz {
namespace {

constexpr int LIN_MAX_WIDTH = 256;

struct LinRole {
  const void *a, *b, *c; void* out;          // [batch, steps, heads, ka], ka, nc, nc
  int64_t a_batch, a_step, a_head, b_batch, b_step, b_head, c_batch, c_step, c_head, out_batch, out_step, out_head;
  const float* init; float* last;            // [batch, heads, ka x nc] at row_stride, col_stride, or NULL
  int64_t row_stride, col_stride;
  int ka, nc;
  bool back;
  float in, out_scale;
};
struct LinArgs {
  LinRole role[3];
  int roles;
  int64_t batch, steps, heads, first;
  const float* rate;
  const uint8_t* reset; int64_t reset_batch, reset_step;
  const int32_t* lengths;
};

__device__ inline int64_t lin_length(const LinArgs& g, int64_t b) {
  if (!g.lengths) return g.steps;
  const int64_t n = g.lengths[b];
  return n < 0 ? 0 : (n < g.steps ? n : g.steps);
}
// exp(-rate n); an infinite rate forgets within a step.
__device__ inline float lin_decay(float rate, int n) { return n == 0 ? 1.0f : expf(-rate * (float)n); }

// Step by step: a workgroup holds 64 columns of a head's state, thread (column group, row group) rows
// row, row + 16, .. of four columns.
constexpr int STEP_THREADS = 256, STEP_COLS = 64;
template <typename T, int KR> __global__ __launch_bounds__(STEP_THREADS) void lin_steps(LinArgs g) {
  const LinRole& r = g.role[blockIdx.y];
  const int64_t slices = (r.nc + STEP_COLS - 1) / STEP_COLS;
  const int64_t at = g.first + blockIdx.x;
  if (at >= g.batch * g.heads * slices) return;
  const int64_t sl = at % slices, h = at / slices % g.heads, b = at / slices / g.heads;
  const int c0 = (int)sl * STEP_COLS + 4 * (threadIdx.x & 15), row0 = threadIdx.x >> 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = lin_length(g, b);
  const float d = lin_decay(g.rate ? g.rate[h] : 0.0f, 1);
  const T* pa = static_cast<const T*>(r.a) + b * r.a_batch + h * r.a_head;
  const T* pb = static_cast<const T*>(r.b) + b * r.b_batch + h * r.b_head;
  const T* pc = static_cast<const T*>(r.c) + b * r.c_batch + h * r.c_head;
  T* po = static_cast<T*>(r.out) + b * r.out_batch + h * r.out_head;
  __shared__ float part[2][4][STEP_COLS];
  float S[KR][4];
  const int64_t st = (b * g.heads + h) * r.ka * r.nc;
#pragma unroll
  for (int i = 0; i < KR; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 16 * i;
      S[i][j] = r.init && row < r.ka && c0 + j < r.nc ? r.init[st + row * r.row_stride + (c0 + j) * r.col_stride] : 0.0f;
    }
  for (int64_t p = 0; p < n; ++p) {
    const int64_t t = r.back ? n - 1 - p : p;
    const int64_t flag = r.back ? t + 1 : t;   // the step whose start cuts the state off
    const bool cut = g.reset && flag < n && g.reset[b * g.reset_batch + flag * g.reset_step] != 0;
    const float keep = r.back && p == 0 ? 1.0f : d;
    float c[4], o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = c0 + j < r.nc && r.c ? to_f<T>(pc[t * r.c_step + c0 + j]) : 0.0f;
#pragma unroll
    for (int i = 0; i < KR; ++i) {
      const int row = row0 + 16 * i;
      const float x = row < r.ka && r.a ? to_f<T>(pa[t * r.a_step + row]) : 0.0f, y = row < r.ka && r.b ? to_f<T>(pb[t * r.b_step + row]) : 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        S[i][j] = row < r.ka ? fmaf(r.in * y, c[j], cut ? 0.0f : keep * S[i][j]) : 0.0f;
        o[j] = fmaf(x, S[i][j], o[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[j] += __shfl_xor(o[j], 16);
      o[j] += __shfl_xor(o[j], 32);
      if (lane < 16) part[p & 1][wave][4 * lane + j] = o[j];
    }
    __syncthreads();
    const int col = (int)sl * STEP_COLS + threadIdx.x;
    if (threadIdx.x < STEP_COLS && col < r.nc) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) s += part[p & 1][k][threadIdx.x];
      po[t * r.out_step + col] = from_f<T>(r.out_scale * s);
    }
  }
  for (int64_t t = n; t < g.steps; ++t)
    if (threadIdx.x < STEP_COLS && (int)sl * STEP_COLS + (int)threadIdx.x < r.nc)
      po[t * r.out_step + sl * STEP_COLS + threadIdx.x] = from_f<T>(0.0f);
  if (!r.last) return;
  const bool cut = r.back && n > 0 && g.reset && g.reset[b * g.reset_batch] != 0;
  const float keep = r.back && n > 0 ? d : 1.0f;
#pragma unroll
  for (int i = 0; i < KR; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + 16 * i;
      if (row < r.ka && c0 + j < r.nc)
        r.last[st + row * r.row_stride + (c0 + j) * r.col_stride] = cut ? 0.0f : keep * S[i][j];
    }
}

// The elements of a [n0, n1, n2, width] output do not overlap: from the smallest stride up, each dimension's
// stride is at least the span of those inside it.
bool lin_out_strides_ok(int64_t n0, int64_t n1, int64_t n2, int64_t width, int64_t s0, int64_t s1, int64_t s2) {
  if (!op_in_stride_ok(s0) || !op_in_stride_ok(s1) || !op_in_stride_ok(s2)) return false;
  if (n0 == 0 || n1 == 0 || n2 == 0 || width == 0) return true;
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (s[j] > s[j + 1]) {
        const int64_t t = s[j], u = n[j];
        s[j] = s[j + 1]; n[j] = n[j + 1];
        s[j + 1] = t; n[j + 1] = u;
      }
  int64_t span = width;   // below 2^42 and more than any span inside it, or the check ends
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < span) return false;
    if (n[i] - 1 > (((int64_t)1 << 60) - span) / s[i]) return false;   // no address space holds it
    span += (n[i] - 1) * s[i];
  }
  return true;
}

const char* lin_check(const spz_linear_attention_args* p) {
  if (!p) return "NULL arguments";
  const spz_linear_attention_args& a = *p;
  if (!op_prec_ok(a.prec)) return "unknown precision";
  if (!op_extent_ok(a.batch) || !op_extent_ok(a.steps) || !op_extent_ok(a.heads)) return "extent out of range";
  if (a.key_width < 0 || a.key_width > LIN_MAX_WIDTH || a.value_width < 0 || a.value_width > LIN_MAX_WIDTH) return "width out of range (256 at most)";
  // No device holds more; keeps every index and count within 62 bits.
  const int64_t state = a.key_width * a.value_width;
  if (a.batch && a.heads > ((int64_t)1 << 38) / a.batch / (state ? state : 1)) return "batch * heads out of range";
  if (a.batch && a.heads && a.steps > ((int64_t)1 << 44) / (a.batch * a.heads) / LIN_MAX_WIDTH) return "extents out of range";
  if (!(__builtin_fabsf(a.scale) <= 3.0e38f)) return "scale is not finite";
  return nullptr;
}

const char* lin_check_arrays(const spz_linear_attention_args& a, bool back) {
  const size_t e = op_size(a.prec);
  const bool heads = a.batch > 0 && a.heads > 0, rows = heads && a.steps > 0, kw = rows && a.key_width > 0, vw = rows && a.value_width > 0;
  if ((kw && (!a.q || !a.k)) || (vw && !a.v)) return "NULL q, k or v";
  if (vw && !back && !a.y) return "NULL y";
  if (back && ((kw && (!a.dq || !a.dk)) || (vw && !a.dv))) return "NULL dq, dk or dv";
  for (const void* p : {a.q, a.k, a.v, (const void*)a.y, a.dy, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
    if (!op_aligned(p, e)) return "array not aligned to its type";
  for (const void* p : {(const void*)a.rate, (const void*)a.lengths, (const void*)a.state, (const void*)a.last, (const void*)a.dlast, (const void*)a.dstate})
    if (!op_aligned(p, 4)) return "state, rate or lengths not aligned to 4 bytes";
  for (int64_t s : {a.q_batch, a.q_step, a.q_head, a.k_batch, a.k_step, a.k_head, a.v_batch, a.v_step, a.v_head, a.reset ? a.reset_batch : 0,
                    a.reset ? a.reset_step : 0, back && a.dy ? a.dy_batch : 0, back && a.dy ? a.dy_step : 0, back && a.dy ? a.dy_head : 0})
    if (!op_in_stride_ok(s)) return "input stride out of range";
  if (!back && !lin_out_strides_ok(a.batch, a.steps, a.heads, a.value_width, a.y_batch, a.y_step, a.y_head)) return "rows of y overlap";
  if (back && !lin_out_strides_ok(a.batch, a.steps, a.heads, a.key_width, a.dq_batch, a.dq_step, a.dq_head)) return "rows of dq overlap";
  if (back && !lin_out_strides_ok(a.batch, a.steps, a.heads, a.key_width, a.dk_batch, a.dk_step, a.dk_head)) return "rows of dk overlap";
  if (back && !lin_out_strides_ok(a.batch, a.steps, a.heads, a.value_width, a.dv_batch, a.dv_step, a.dv_head)) return "rows of dv overlap";
  return nullptr;
}

template <typename T> void lin_steps_launch(const LinArgs& g, hipStream_t s) {
  int64_t blocks = 0;
  int ka = 0;
  for (int i = 0; i < g.roles; ++i) {
    const int64_t n = g.batch * g.heads * op_div_up(g.role[i].nc, STEP_COLS);
    blocks = n > blocks ? n : blocks;
    ka = g.role[i].ka > ka ? g.role[i].ka : ka;
  }
  op_dispatch(blocks, STEP_THREADS * 3, [&](int64_t first, dim3 grid) {
    LinArgs part = g;
    part.first = first;
    grid.y = (unsigned)g.roles;
    if (ka <= 16) lin_steps<T, 1><<<grid, STEP_THREADS, 0, s>>>(part);
    else if (ka <= 64) lin_steps<T, 4><<<grid, STEP_THREADS, 0, s>>>(part);
    else if (ka <= 128) lin_steps<T, 8><<<grid, STEP_THREADS, 0, s>>>(part);
    else lin_steps<T, 16><<<grid, STEP_THREADS, 0, s>>>(part);
  });
}

int lin_run(const char* call, const spz_linear_attention_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = lin_check(args);
  if (!bad) bad = lin_check_arrays(*args, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const spz_linear_attention_args& a = *args;
  const int64_t need = spz_linear_attention_workspace(args, back);
  if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
  if (need > 0 && !op_aligned(ws, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
  LinArgs g{};
  g.batch = a.batch;
  g.steps = a.steps;
  g.heads = a.heads;
  g.rate = a.rate;
  g.reset = a.reset;
  g.reset_batch = a.reset_batch;
  g.reset_step = a.reset_step;
  g.lengths = a.lengths;
  const int K = (int)a.key_width, V = (int)a.value_width;
  const auto role = [&](const void* x, int64_t x0, int64_t x1, int64_t x2, const void* y, int64_t y0, int64_t y1, int64_t y2, const void* z,
                        int64_t z0, int64_t z1, int64_t z2, void* o, int64_t o0, int64_t o1, int64_t o2, const float* init, float* last,
                        int64_t rs, int64_t cs, int ka, int nc, bool rev) {
    if (nc > 0)
      g.role[g.roles++] = LinRole{x, y, z, o, x0, x1, x2, y0, y1, y2, z0, z1, z2, o0, o1, o2, init, last, rs, cs, ka, nc, rev, rev ? a.scale : 1.0f, rev ? 1.0f : a.scale};
  };
  if (!back) {
    role(a.q, a.q_batch, a.q_step, a.q_head, a.k, a.k_batch, a.k_step, a.k_head, a.v, a.v_batch, a.v_step, a.v_head, a.y, a.y_batch, a.y_step,
         a.y_head, a.state, a.last, V, 1, K, V, false);
  } else {
    role(a.dy, a.dy_batch, a.dy_step, a.dy_head, a.v, a.v_batch, a.v_step, a.v_head, a.k, a.k_batch, a.k_step, a.k_head, a.dq, a.dq_batch, a.dq_step,
         a.dq_head, a.state, nullptr, 1, V, V, K, false);
    role(a.v, a.v_batch, a.v_step, a.v_head, a.dy, a.dy_batch, a.dy_step, a.dy_head, a.q, a.q_batch, a.q_step, a.q_head, a.dk, a.dk_batch, a.dk_step,
         a.dk_head, a.dlast, nullptr, 1, V, V, K, true);
    role(a.k, a.k_batch, a.k_step, a.k_head, a.q, a.q_batch, a.q_step, a.q_head, a.dy, a.dy_batch, a.dy_step, a.dy_head, a.dv, a.dv_batch, a.dv_step,
         a.dv_head, a.dlast, a.dstate, V, 1, K, V, true);
  }
  if (g.roles == 0 || a.batch == 0 || a.heads == 0) return SPZ_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.prec == SPZ_PREC_BF16) lin_steps_launch<bf16_t>(g, s);
  else lin_steps_launch<float>(g, s);
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_linear_attention_workspace(const spz_linear_attention_args* args, int32_t backward) {
  (void)backward;
  const char* bad = lin_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_linear_attention_workspace", bad);
  return 0;
}

int spz_linear_attention_forward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return lin_run("spz_linear_attention_forward", args, false, workspace, workspace_bytes, hip_stream);
}

int spz_linear_attention_backward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return lin_run("spz_linear_attention_backward", args, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
