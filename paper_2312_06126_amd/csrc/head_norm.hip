// Norms of each head of queries and keys, and their rotation by position, in one pass.
//
// A wave takes heads of rows one after the other: lane l holds columns l, l + 64, .. and, of columns that turn,
// the partner's value as well, which it normalises itself, so that nothing crosses lanes but the two sums.
#include "ops.h"

namespace spz {
namespace {

constexpr int HEAD_MAX_DIM = 1024, HEAD_THREADS = 256, HEAD_WAVES = HEAD_THREADS / 64;
constexpr int64_t HEAD_BLOCKS = 2048;   // most workgroups of a backward call: each leaves a row of partial sums

// Queries or keys.
struct HeadPart {
  const void* x; int64_t x_row, x_head;
  const float *w, *b;
  const void* dy; int64_t dy_row, dy_head;   // backward
  void* out; int64_t out_row, out_head;      // forward: y; backward: dx
  int64_t heads, items;                      // items: rows * heads
  int64_t first, blocks;                     // its workgroups
};
struct HeadArgs {
  HeadPart part[2];
  const int32_t* positions;
  const double* freqs;
  const uint8_t* valid;
  float* sums;                               // backward: [workgroups, 2, dim]
  int dim, pairs, norm, layout;
  float eps;
};

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

// Cosine and sine of pos * freq: the angle in turns less the nearest whole number of them, in 64 bits, so that
// only a part of a turn is rounded to 32.
__device__ inline void turn_of(int32_t pos, double freq, float& c, float& s) {
  constexpr double TURNS = 0.15915494309189533577;   // 1 / (2 pi)
  const double t = (double)pos * freq * TURNS;
  sincospif(2.0f * (float)(t - rint(t)), &s, &c);
}

// Column c's partner of its pair, and the pair (-1: the column stays). second: c is the pair's second column.
__device__ inline int partner_of(const HeadArgs& g, int c, int& pair, bool& second) {
  if (c >= 2 * g.pairs) { pair = -1; second = false; return c; }
  if (g.layout == SPZ_PAIRS_HALVES) {
    second = c >= g.pairs;
    pair = second ? c - g.pairs : c;
    return second ? pair : c + g.pairs;
  }
  second = c & 1;
  pair = c >> 1;
  return c ^ 1;
}

template <typename T, int K, bool BACK> __global__ __launch_bounds__(HEAD_THREADS) void head_norm(HeadArgs g, int64_t first) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t blk = first + blockIdx.x;
  const HeadPart& p = g.part[blk >= g.part[1].first];
  const int D = g.dim;
  const float inv = 1.0f / (float)D;
  float w[K], b[K], wp[K], bp[K], dw[K], db[K];
  int pair[K], other[K];
  bool second[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = lane + 64 * i;
    pair[i] = -1; other[i] = c; second[i] = false;
    w[i] = wp[i] = 1.0f; b[i] = bp[i] = dw[i] = db[i] = 0.0f;
    if (c >= D) continue;
    other[i] = partner_of(g, c, pair[i], second[i]);
    if (p.w) { w[i] = p.w[c]; wp[i] = p.w[other[i]]; }
    if (p.b) { b[i] = p.b[c]; bp[i] = p.b[other[i]]; }
  }
  for (int64_t it = (blk - p.first) * HEAD_WAVES + wave; it < p.items; it += p.blocks * HEAD_WAVES) {
    const int64_t row = it / p.heads, head = it - row * p.heads;
    T* out = static_cast<T*>(p.out) + row * p.out_row + head * p.out_head;
    if (g.valid && !g.valid[row]) {
      if (p.out)
        for (int c = lane; c < D; c += 64) out[c] = from_f<T>(0.0f);
      continue;
    }
    const T* x = static_cast<const T*>(p.x) + row * p.x_row + head * p.x_head;
    float n[K], q[K];
    float s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int c = lane + 64 * i;
      n[i] = c < D ? to_f<T>(x[c]) : 0.0f;
      q[i] = !BACK && pair[i] >= 0 ? to_f<T>(x[other[i]]) : 0.0f;
      s1 += n[i];
    }
    float r = 1.0f;
    if (g.norm != SPZ_NORM_NONE) {
      const float mean = g.norm == SPZ_NORM_LAYER ? wave_sum(s1) * inv : 0.0f;
      float s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < K; ++i) {
        n[i] -= mean;
        q[i] -= mean;
        s2 += lane + 64 * i < D ? n[i] * n[i] : 0.0f;
      }
      r = 1.0f / sqrtf(wave_sum(s2) * inv + g.eps);
    }
    if constexpr (!BACK) {
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int c = lane + 64 * i;
        if (c >= D) continue;
        float y = fmaf(n[i] * r, w[i], b[i]);
        if (pair[i] >= 0) {
          float co, si;
          turn_of(g.positions[row], g.freqs[pair[i]], co, si);
          const float z = fmaf(q[i] * r, wp[i], bp[i]);
          y = y * co + (second[i] ? z * si : -(z * si));
        }
        out[c] = from_f<T>(y);
      }
    } else {
      const T* dy = static_cast<const T*>(p.dy) + row * p.dy_row + head * p.dy_head;
      float d[K], a1 = 0.0f, a2 = 0.0f;
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int c = lane + 64 * i;
        d[i] = 0.0f;
        if (c >= D) continue;
        n[i] *= r;
        d[i] = to_f<T>(dy[c]);
        if (pair[i] >= 0) {   // turned back
          float co, si;
          turn_of(g.positions[row], g.freqs[pair[i]], co, si);
          const float z = to_f<T>(dy[other[i]]);
          d[i] = d[i] * co + (second[i] ? -(z * si) : z * si);
        }
        dw[i] = fmaf(d[i], n[i], dw[i]);
        db[i] += d[i];
        d[i] *= w[i];
        a1 += d[i];
        a2 = fmaf(d[i], n[i], a2);
      }
      if (p.out) {
        if (g.norm != SPZ_NORM_NONE) {
          a1 = g.norm == SPZ_NORM_LAYER ? wave_sum(a1) * inv : 0.0f;
          a2 = wave_sum(a2) * inv;
        } else {
          a1 = a2 = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const int c = lane + 64 * i;
          if (c < D) out[c] = from_f<T>(r * (d[i] - fmaf(n[i], a2, a1)));
        }
      }
    }
  }
  if constexpr (BACK) {
    __shared__ float part[HEAD_WAVES][2][64 * K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
      part[wave][0][lane + 64 * i] = dw[i];
      part[wave][1][lane + 64 * i] = db[i];
    }
    __syncthreads();
    float* to = g.sums + blk * 2 * D;
    for (int c = threadIdx.x; c < 2 * D; c += HEAD_THREADS) {
      const int v = c >= D, col = c - v * D;
      float s = 0.0f;
      for (int k = 0; k < HEAD_WAVES; ++k) s += part[k][v][col];
      to[c] = s;
    }
  }
}

// The workgroups' partial sums, in a fixed order: thread (column, group) takes every 4th row.
constexpr int HSUM_COLS = 64, HSUM_GROUPS = 4;
struct HeadSums { float* out[2][2]; int64_t first[2], blocks[2]; };
__global__ __launch_bounds__(HSUM_COLS* HSUM_GROUPS) void head_sums(const float* sums, HeadSums o, int dim) {
  __shared__ float part[HSUM_GROUPS][HSUM_COLS];
  const int c = blockIdx.x * HSUM_COLS + threadIdx.x % HSUM_COLS, grp = threadIdx.x / HSUM_COLS;
  const int which = blockIdx.y >> 1, v = blockIdx.y & 1;
  float* out = o.out[which][v];
  float s = 0.0f;
  if (out && c < dim)
    for (int64_t k = grp; k < o.blocks[which]; k += HSUM_GROUPS) s += sums[((o.first[which] + k) * 2 + v) * dim + c];
  part[grp][threadIdx.x % HSUM_COLS] = s;
  __syncthreads();
  if (grp == 0 && out && c < dim) {
    for (int k = 1; k < HSUM_GROUPS; ++k) s += part[k][threadIdx.x];
    out[c] = s;
  }
}

int64_t head_blocks(int64_t items, bool back) {
  const int64_t n = op_div_up(items, HEAD_WAVES);
  return back && n > HEAD_BLOCKS ? HEAD_BLOCKS : n;
}

const char* head_check(const spz_head_norm_args* p) {
  if (!p) return "NULL arguments";
  const spz_head_norm_args& a = *p;
  if (!op_prec_ok(a.prec)) return "unknown precision";
  if (!op_extent_ok(a.rows) || !op_extent_ok(a.heads_q) || !op_extent_ok(a.heads_k)) return "extent out of range";
  if (a.dim < 0 || a.dim > HEAD_MAX_DIM) return "dim out of range";
  if (a.pairs < 0 || 2 * a.pairs > a.dim) return "more pairs than columns";
  const int64_t wide = (a.heads_q + a.heads_k) * (a.dim ? a.dim : 1);
  if (wide && a.rows > ((int64_t)1 << 42) / wide) return "extents out of range";
  if (a.norm < SPZ_NORM_NONE || a.norm > SPZ_NORM_LAYER) return "unknown norm";
  if (a.layout != SPZ_PAIRS_HALVES && a.layout != SPZ_PAIRS_NEIGHBOURS) return "unknown layout of pairs";
  if (!(a.eps >= 1.2e-38f) || !(a.eps < 3.0e38f)) return "eps out of range";
  return nullptr;
}

const char* head_check_arrays(const spz_head_norm_args& a, bool back) {
  const bool some = a.rows > 0 && a.dim > 0, q = some && a.heads_q > 0, k = some && a.heads_k > 0;
  const size_t e = op_size(a.prec);
  if ((q && !a.q) || (k && !a.k)) return "NULL q or k";
  if ((q || k) && a.pairs > 0 && (!a.positions || !a.freqs)) return "NULL positions or freqs";
  if (!back && ((q && !a.q_out) || (k && !a.k_out))) return "NULL output";
  for (const void* p : {a.q, a.k, (const void*)a.q_out, (const void*)a.k_out, a.dq_out, a.dk_out, (const void*)a.dq, (const void*)a.dk})
    if (!op_aligned(p, e)) return "array not aligned to its type";
  for (const float* p : {a.w_q, a.b_q, a.w_k, a.b_k, (const float*)a.dw_q, (const float*)a.db_q, (const float*)a.dw_k, (const float*)a.db_k})
    if (!op_aligned(p, 4)) return "vector not aligned to 4 bytes";
  if (!op_aligned(a.positions, 4)) return "positions not aligned to 4 bytes";
  if (!op_aligned(a.freqs, 8)) return "freqs not aligned to 8 bytes";
  for (int64_t s : {a.q_row, a.q_head, a.heads_k ? a.k_row : 0, a.heads_k ? a.k_head : 0, back && a.dq_out ? a.dq_out_row : 0,
                    back && a.dq_out ? a.dq_out_head : 0, back && a.dk_out ? a.dk_out_row : 0, back && a.dk_out ? a.dk_out_head : 0})
    if (!op_in_stride_ok(s)) return "input stride out of range";
  if (!back) {
    if (!op_out_strides_ok(a.rows, a.heads_q, a.dim, a.q_out_row, a.q_out_head)) return "rows of q_out overlap";
    if (a.heads_k && !op_out_strides_ok(a.rows, a.heads_k, a.dim, a.k_out_row, a.k_out_head)) return "rows of k_out overlap";
    return nullptr;
  }
  if (a.dq && !op_out_strides_ok(a.rows, a.heads_q, a.dim, a.dq_row, a.dq_head)) return "rows of dq overlap";
  if (a.dk && a.heads_k && !op_out_strides_ok(a.rows, a.heads_k, a.dim, a.dk_row, a.dk_head)) return "rows of dk overlap";
  return nullptr;
}

// The work of a call: without a gradient of its outputs, a part's gradients are zeros, which its kernel does not compute.
void head_parts(const spz_head_norm_args& a, bool back, HeadArgs& g) {
  g.part[0] = {a.q, a.q_row, a.q_head, a.w_q, a.b_q, a.dq_out, a.dq_out_row, a.dq_out_head,
               back ? a.dq : a.q_out, back ? a.dq_row : a.q_out_row, back ? a.dq_head : a.q_out_head, a.heads_q, a.rows * a.heads_q, 0, 0};
  g.part[1] = {a.k, a.k_row, a.k_head, a.w_k, a.b_k, a.dk_out, a.dk_out_row, a.dk_out_head,
               back ? a.dk : a.k_out, back ? a.dk_row : a.k_out_row, back ? a.dk_head : a.k_out_head, a.heads_k, a.rows * a.heads_k, 0, 0};
  int64_t at = 0;
  for (HeadPart& p : g.part) {
    p.first = at;
    p.blocks = head_blocks(p.items, back);
    at += p.blocks;
  }
}

template <typename T> __global__ void head_zero(HeadPart p, int dim, int64_t first) {
  const int64_t i = (first + blockIdx.x) * HEAD_THREADS + threadIdx.x;
  if (i >= p.items * dim) return;
  const int64_t it = i / dim, row = it / p.heads;
  static_cast<T*>(p.out)[row * p.out_row + (it - row * p.heads) * p.out_head + (i - it * dim)] = from_f<T>(0.0f);
}

template <typename T, bool BACK> void head_launch(const HeadArgs& g, hipStream_t s) {
  const int64_t blocks = g.part[1].first + g.part[1].blocks;
  const auto go = [&](auto k) {
    op_dispatch(blocks, HEAD_THREADS, [&](int64_t first, dim3 grid) {
      head_norm<T, decltype(k)::value, BACK><<<grid, HEAD_THREADS, 0, s>>>(g, first);
    });
  };
  using std::integral_constant;
  if (g.dim <= 64) go(integral_constant<int, 1>{});
  else if (g.dim <= 128) go(integral_constant<int, 2>{});
  else if (g.dim <= 256) go(integral_constant<int, 4>{});
  else if (g.dim <= 512) go(integral_constant<int, 8>{});
  else go(integral_constant<int, 16>{});
}

int head_run(const char* call, const spz_head_norm_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = head_check(args);
  if (!bad) bad = head_check_arrays(*args, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const spz_head_norm_args& a = *args;
  HeadArgs g{};
  head_parts(a, back, g);
  g.positions = a.positions;
  g.freqs = a.freqs;
  g.valid = a.valid;
  g.dim = (int)a.dim;
  g.pairs = (int)a.pairs;
  g.norm = a.norm;
  g.layout = a.layout;
  g.eps = a.eps;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (back) {
    const int64_t need = spz_head_norm_workspace(args);
    if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
    if (need > 0 && !op_aligned(ws, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
    g.sums = static_cast<float*>(ws);
    for (HeadPart& p : g.part)
      if (!p.dy && p.items > 0) {   // no gradient comes in
        if (p.out && a.dim > 0)
          op_dispatch(op_div_up(p.items * a.dim, HEAD_THREADS), HEAD_THREADS, [&](int64_t first, dim3 grid) {
            if (a.prec == SPZ_PREC_BF16) head_zero<bf16_t><<<grid, HEAD_THREADS, 0, s>>>(p, g.dim, first);
            else head_zero<float><<<grid, HEAD_THREADS, 0, s>>>(p, g.dim, first);
          });
        p.items = 0;
      }
    int64_t at = 0;
    for (HeadPart& p : g.part) {
      p.first = at;
      p.blocks = head_blocks(p.items, back);
      at += p.blocks;
    }
  }
  const int64_t blocks = g.part[1].first + g.part[1].blocks;
  if (a.dim == 0 || (!back && blocks == 0)) return SPZ_OK;
  if (blocks > 0) {
    if (a.prec == SPZ_PREC_BF16) {
      if (back) head_launch<bf16_t, true>(g, s);
      else head_launch<bf16_t, false>(g, s);
    } else {
      if (back) head_launch<float, true>(g, s);
      else head_launch<float, false>(g, s);
    }
  }
  if (back && (a.dw_q || a.db_q || a.dw_k || a.db_k)) {
    const HeadSums o{{{a.dw_q, a.db_q}, {a.dw_k, a.db_k}}, {g.part[0].first, g.part[1].first}, {g.part[0].blocks, g.part[1].blocks}};
    head_sums<<<dim3((unsigned)op_div_up(a.dim, HSUM_COLS), 4), HSUM_COLS * HSUM_GROUPS, 0, s>>>(g.sums, o, g.dim);
  }
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_head_norm_workspace(const spz_head_norm_args* args) {
  const char* bad = head_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_head_norm_workspace", bad);
  HeadArgs g{};
  head_parts(*args, true, g);
  return (g.part[1].first + g.part[1].blocks) * 2 * args->dim * 4;
}

int spz_head_norm_forward(const spz_head_norm_args* args, void* hip_stream) {
  return head_run("spz_head_norm_forward", args, false, nullptr, 0, hip_stream);
}

int spz_head_norm_backward(const spz_head_norm_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return head_run("spz_head_norm_backward", args, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
