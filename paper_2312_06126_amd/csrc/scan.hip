// Gated linear recurrence over sequences (spz_scan_*): forward, backward and single steps.
//
//   h_t = a_t k_t h_{t-1} + (1 - a_t) v_t,  a_t = sigmoid(f_t), k_t = 0 at an episode start.
//
// Both directions are bound by HBM: 3 elements moved a step and channel forward, 5 backward
// (f, v, dy, df, dv), for some 15 and 40 instructions. A thread owns SCAN_V adjacent channels of
// one sequence (8 or 16 bytes a step, so a wave reads whole cache lines) and walks time with the
// next steps' loads in flight; states stay in registers in float32.
//
// A step is the affine map h -> A h + H, and maps compose, so where batch and width alone give too
// few threads time is cut into pieces: each piece's map is taken first (scan_piece), the maps
// are joined into the state in front of every piece (scan_join), then every piece is walked
// (scan_forward, scan_backward). The second reading of f and v comes mostly from the 256 MB
// last-level cache. An episode start inside a piece makes its map independent of the state: such a
// map is marked by A = -1 (A is a product of sigmoids, else >= 0), so that a state that is not
// finite does not pass it as 0 * inf.
//
// Backward the same with time reversed: c -> P c + Q is the gradient handed from step to step.
// h_{t-1} is not stored by the forward pass: `saved` holds the state in front of every SEG-th step
// (3% of the bytes moved), from which a thread recomputes SEG steps in registers.
#include "ops.h"

namespace spz {
namespace {

constexpr int SCAN_THREADS = 256;
constexpr int SCAN_V = 4;                    // channels a thread, where rows are aligned for it
template <typename T> constexpr int SEG = 32 / (int)sizeof(T);   // bf16 16, float32 8 (registers)
constexpr int JOIN_CH = 16, JOIN_GROUPS = 16;

struct ScanArgs {
  spz_scan_args a;
  int64_t chunks;       // of V channels
  int64_t pieces, len;  // time pieces and their steps (a multiple of SEG)
  float *map_a, *map_h; // [pieces, batch, width]: maps; map_h then the carries
};

// V elements at p, as floats.
template <typename T, int V> __device__ inline void load_v(const T* p, float (&x)[V]) {
  if constexpr (V == 1) {
    x[0] = to_f<T>(*p);
  } else if constexpr (sizeof(T) == 4) {
    unpack(*reinterpret_cast<const u32x4*>(p), x);
  } else {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
    }
  }
}
template <typename T, int V> __device__ inline void store_v(T* p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = from_f<T>(x[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<u32x4*>(p) = pack(x);
  } else {
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  }
}
// V floats of a [.., width] state array: its rows are aligned only where width is.
template <int V> __device__ inline void load_s(const float* p, bool vec, float (&x)[V]) {
  if (V == 4 && vec) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = w[i & 3];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = p[i];
  }
}
template <int V> __device__ inline void store_s(float* p, bool vec, const float (&x)[V]) {
  if (V == 4 && vec) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1 % V], x[2 % V], x[3 % V]};
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = x[i];
  }
}
__device__ inline bool op_aligned16(const void* p) { return op_aligned(p, 16); }

struct ScanPos { int64_t b, c, p; };
template <int V> __device__ inline bool scan_pos(const ScanArgs& g, ScanPos& q) {
  const int64_t i = (int64_t)blockIdx.x * SCAN_THREADS + threadIdx.x;
  if (i >= g.chunks * g.a.batch * g.pieces) return false;
  q.c = i % g.chunks * V;
  q.b = i / g.chunks % g.a.batch;
  q.p = i / g.chunks / g.a.batch;
  return true;
}
__device__ inline int64_t scan_length(const spz_scan_args& a, int64_t b) {
  if (!a.lengths) return a.steps;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : (n < a.steps ? n : a.steps);
}
__device__ inline bool cut_at(const spz_scan_args& a, int64_t b, int64_t t) {
  return a.reset && a.reset[b * a.reset_batch + t * a.reset_step] != 0;
}

// The affine map of each piece: BACK = false (f, v), true (f, dy; from the piece's end).
template <typename T, int V, bool BACK> __global__ __launch_bounds__(SCAN_THREADS) void scan_piece(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b), t1 = n < end ? n : end;
  float A[V], H[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { A[i] = 1.0f; H[i] = 0.0f; }
  const T* f = static_cast<const T*>(a.f) + q.b * a.f_batch + q.c;
  const T* v = static_cast<const T*>(BACK ? a.dy : a.v) + q.b * (BACK ? a.dy_batch : a.v_batch) + q.c;
  const int64_t v_step = BACK ? a.dy_step : a.v_step;
  bool cut = false;
  for (int64_t s = t0; s < t1; ++s) {
    const int64_t t = BACK ? t1 - 1 - (s - t0) : s;
    float x[V], w[V];
    load_v<T, V>(f + t * a.f_step, x);
    if (BACK && !a.dy) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = 0.0f;
    } else {
      load_v<T, V>(v + t * v_step, w);
    }
    const bool k = cut_at(a, q.b, t);
    cut |= k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float al, be;
      sigmoid2(x[i], al, be);
      if (BACK) {
        H[i] = k ? 0.0f : al * (H[i] + w[i]);
      } else {
        H[i] = fmaf(be, w[i], k ? 0.0f : al * H[i]);
      }
      A[i] *= al;
    }
  }
  if (cut) {
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = -1.0f;
  }
  const int64_t o = (q.p * a.batch + q.b) * a.width + q.c;
  const bool vec = a.width % 4 == 0;
  store_s<V>(g.map_a + o, vec, A);
  store_s<V>(g.map_h + o, vec, H);
}

// map_h[p] <- the state in front of piece p (backward: behind it), from the maps and the first
// state (`first`, NULL: zeros). 16 channels a workgroup; 16 groups of threads each join a range of
// pieces, then walk it from the ranges' joint maps.
__global__ __launch_bounds__(JOIN_CH * JOIN_GROUPS) void scan_join(const float* map_a, float* map_h, const float* first,
                                                                   int64_t channels, int64_t pieces, bool back) {
  __shared__ float sa[JOIN_GROUPS][JOIN_CH], sh[JOIN_GROUPS][JOIN_CH];
  const int c = threadIdx.x % JOIN_CH, gr = threadIdx.x / JOIN_CH;
  const int64_t ch = (int64_t)blockIdx.x * JOIN_CH + c;
  const bool on = ch < channels;
  const int64_t per = (pieces + JOIN_GROUPS - 1) / JOIN_GROUPS;
  const int64_t p0 = gr * per < pieces ? gr * per : pieces, p1 = p0 + per < pieces ? p0 + per : pieces;
  float A = 1.0f, H = 0.0f;
  for (int64_t p = p0; on && p < p1; ++p) {
    const int64_t o = (back ? pieces - 1 - p : p) * channels + ch;
    const float ma = map_a[o], mh = map_h[o];
    if (ma == -1.0f) {
      A = -1.0f;
      H = mh;
    } else {
      A = A == -1.0f ? -1.0f : A * ma;
      H = fmaf(ma, H, mh);
    }
  }
  sa[gr][c] = A;
  sh[gr][c] = H;
  __syncthreads();
  if (!on) return;
  float h = first ? first[ch] : 0.0f;
  for (int j = 0; j < gr; ++j) h = sa[j][c] == -1.0f ? sh[j][c] : fmaf(sa[j][c], h, sh[j][c]);
  for (int64_t p = p0; p < p1; ++p) {
    const int64_t o = (back ? pieces - 1 - p : p) * channels + ch;
    const float ma = map_a[o], mh = map_h[o];
    map_h[o] = h;
    h = ma == -1.0f ? mh : fmaf(ma, h, mh);
  }
}

template <typename T, int V> __global__ __launch_bounds__(SCAN_THREADS) void scan_forward(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const bool vec = a.width % 4 == 0;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b);
  const int64_t t2 = end < a.steps ? end : a.steps, t1 = n < t2 ? n : t2;
  const int64_t st = q.b * a.width + q.c;
  const T* f = static_cast<const T*>(a.f) + q.b * a.f_batch + q.c;
  const T* v = static_cast<const T*>(a.v) + q.b * a.v_batch + q.c;
  T* y = static_cast<T*>(a.y) + q.b * a.y_batch + q.c;
  const int64_t segs = (a.steps + SEG<T> - 1) / SEG<T>;
  float h[V];
  if (g.pieces > 1) {
    load_s<V>(g.map_h + q.p * a.batch * a.width + st, vec, h);
  } else if (a.h0) {
    load_s<V>(a.h0 + st, vec && op_aligned16(a.h0), h);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = 0.0f;
  }
  for (int64_t t = t0; t < t1; ++t) {
    if (a.saved && t % SEG<T> == 0) store_s<V>(a.saved + ((q.b * segs + t / SEG<T>) * a.width + q.c), vec && op_aligned16(a.saved), h);
    float x[V], w[V];
    load_v<T, V>(f + t * a.f_step, x);
    load_v<T, V>(v + t * a.v_step, w);
    const bool k = cut_at(a, q.b, t);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float al, be;
      sigmoid2(x[i], al, be);
      h[i] = fmaf(be, w[i], k ? 0.0f : al * h[i]);
    }
    store_v<T, V>(y + t * a.y_step, h);
  }
  float zero[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = t1 > t0 ? t1 : t0; t < t2; ++t) store_v<T, V>(y + t * a.y_step, zero);
  if (a.hT && q.p == g.pieces - 1) store_s<V>(a.hT + st, vec && op_aligned16(a.hT), h);
}

template <typename T, int V> __global__ __launch_bounds__(SCAN_THREADS) void scan_backward(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const bool vec = a.width % 4 == 0;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b);
  const int64_t t2 = end < a.steps ? end : a.steps, t1 = n < t2 ? n : t2;
  const int64_t st = q.b * a.width + q.c;
  const T* f = static_cast<const T*>(a.f) + q.b * a.f_batch + q.c;
  const T* v = static_cast<const T*>(a.v) + q.b * a.v_batch + q.c;
  const T* dy = a.dy ? static_cast<const T*>(a.dy) + q.b * a.dy_batch + q.c : nullptr;
  T* df = static_cast<T*>(a.df) + q.b * a.df_batch + q.c;
  T* dv = static_cast<T*>(a.dv) + q.b * a.dv_batch + q.c;
  const int64_t segs = (a.steps + SEG<T> - 1) / SEG<T>;
  float zero[V], c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = t1 > t0 ? t1 : t0; t < t2; ++t) {
    store_v<T, V>(df + t * a.df_step, zero);
    store_v<T, V>(dv + t * a.dv_step, zero);
  }
  if (g.pieces > 1) {
    load_s<V>(g.map_h + q.p * a.batch * a.width + st, vec, c);
  } else if (a.dhT) {
    load_s<V>(a.dhT + st, vec && op_aligned16(a.dhT), c);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = 0.0f;
  }
  for (int64_t ts = t1 > t0 ? t0 + (t1 - 1 - t0) / SEG<T> * SEG<T> : t0 - 1; ts >= t0; ts -= SEG<T>) {
    const int cnt = (int)(t1 - ts < SEG<T> ? t1 - ts : SEG<T>);
    // Forward through the segment: before[i] = k_t h_{t-1}.
    float before[SEG<T>][V], h[V];
    load_s<V>(a.saved + ((q.b * segs + ts / SEG<T>) * a.width + q.c), vec && op_aligned16(a.saved), h);
#pragma unroll
    for (int j = 0; j < SEG<T>; ++j) {
      if (j >= cnt) continue;
      const int64_t t = ts + j;
      float x[V], w[V];
      load_v<T, V>(f + t * a.f_step, x);
      load_v<T, V>(v + t * a.v_step, w);
      const bool k = cut_at(a, q.b, t);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float al, be;
        sigmoid2(x[i], al, be);
        before[j][i] = k ? 0.0f : h[i];
        h[i] = fmaf(be, w[i], al * before[j][i]);
      }
    }
#pragma unroll
    for (int j = SEG<T> - 1; j >= 0; --j) {
      if (j >= cnt) continue;
      const int64_t t = ts + j;
      float x[V], w[V], d[V], of[V], ov[V];
      load_v<T, V>(f + t * a.f_step, x);
      load_v<T, V>(v + t * a.v_step, w);
      if (dy) load_v<T, V>(dy + t * a.dy_step, d);
      const bool k = cut_at(a, q.b, t);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float al, be;
        sigmoid2(x[i], al, be);
        const float gr = dy ? d[i] + c[i] : c[i];
        ov[i] = gr * be;
        of[i] = ov[i] * al * (before[j][i] - w[i]);
        c[i] = k ? 0.0f : al * gr;
      }
      store_v<T, V>(df + t * a.df_step, of);
      store_v<T, V>(dv + t * a.dv_step, ov);
    }
  }
  if (a.dh0 && q.p == 0) store_s<V>(a.dh0 + st, vec && op_aligned16(a.dh0), c);
}

// Time pieces: one where the channels alone give SCAN_FILL threads (eight waves a compute unit),
// else enough for as many, of at least SCAN_MIN_LEN steps each.
constexpr int64_t SCAN_FILL = 131072, SCAN_MIN_LEN = 32;
struct ScanPlan { int64_t pieces, len; };
ScanPlan scan_plan(const spz_scan_args& a) {
  const int64_t threads = a.batch * op_div_up(a.width, SCAN_V);
  int64_t pieces = threads > 0 ? op_div_up(SCAN_FILL, threads) : 1;
  const int64_t most = a.steps / SCAN_MIN_LEN;
  if (threads * 2 > SCAN_FILL || most < 2) return {1, a.steps};
  if (pieces > most) pieces = most;
  const int64_t len = op_div_up(op_div_up(a.steps, pieces), 16) * 16;
  return {op_div_up(a.steps, len), len};
}

const char* scan_check(const spz_scan_args* a) {
  if (!a) return "NULL arguments";
  if (!op_prec_ok(a->prec)) return "unknown precision";
  if (!op_extent_ok(a->batch) || !op_extent_ok(a->steps) || !op_extent_ok(a->width)) return "extent out of range";
  // Bounds every index and the grid.
  if (a->width && a->batch && a->batch > ((int64_t)1 << 38) / a->width) return "batch * width out of range";
  if (a->width && a->batch && a->steps > ((int64_t)1 << 44) / (a->batch * a->width)) return "extents out of range";
  return nullptr;
}

const char* scan_check_arrays(const spz_scan_args& a, bool back, int64_t ws_bytes, const void* ws, int64_t need) {
  const size_t e = op_size(a.prec);
  const bool some = a.batch > 0 && a.width > 0, rows = some && a.steps > 0;
  if (rows && (!a.f || !a.v)) return "NULL f or v";
  if (rows && !back && !a.y) return "NULL y";
  if (rows && back && (!a.df || !a.dv)) return "NULL df or dv";
  if (rows && back && !a.saved) return "NULL saved";
  for (const void* p : {a.f, a.v, (const void*)a.y, a.dy, (const void*)a.df, (const void*)a.dv})
    if (!op_aligned(p, e)) return "array not aligned to its type";
  for (const void* p : {(const void*)a.h0, (const void*)a.hT, (const void*)a.saved, (const void*)a.dhT, (const void*)a.dh0, (const void*)a.lengths})
    if (!op_aligned(p, 4)) return "state or lengths not aligned to 4 bytes";
  for (int64_t s : {a.f_batch, a.f_step, a.v_batch, a.v_step, a.reset ? a.reset_batch : 0, a.reset ? a.reset_step : 0,
                    back && a.dy ? a.dy_batch : 0, back && a.dy ? a.dy_step : 0})
    if (!op_in_stride_ok(s)) return "input stride out of range";
  if (!back && !op_out_strides_ok(a.batch, a.steps, a.width, a.y_batch, a.y_step)) return "rows of y overlap";
  if (back && !op_out_strides_ok(a.batch, a.steps, a.width, a.df_batch, a.df_step)) return "rows of df overlap";
  if (back && !op_out_strides_ok(a.batch, a.steps, a.width, a.dv_batch, a.dv_step)) return "rows of dv overlap";
  if (need > 0 && ws && !op_aligned(ws, 16)) return "workspace not aligned to 16 bytes";
  return nullptr;
}

template <typename T, int V> void scan_launch(const ScanArgs& g, bool back, hipStream_t s) {
  const int64_t threads = g.chunks * g.a.batch * g.pieces;
  const dim3 grid((unsigned)op_div_up(threads, SCAN_THREADS));
  if (g.pieces > 1) {
    const int64_t channels = g.a.batch * g.a.width;
    if (back) scan_piece<T, V, true><<<grid, SCAN_THREADS, 0, s>>>(g);
    else scan_piece<T, V, false><<<grid, SCAN_THREADS, 0, s>>>(g);
    scan_join<<<dim3((unsigned)op_div_up(channels, JOIN_CH)), JOIN_CH * JOIN_GROUPS, 0, s>>>(
        g.map_a, g.map_h, back ? g.a.dhT : g.a.h0, channels, g.pieces, back);
  }
  if (back) scan_backward<T, V><<<grid, SCAN_THREADS, 0, s>>>(g);
  else scan_forward<T, V><<<grid, SCAN_THREADS, 0, s>>>(g);
}

int64_t scan_workspace(const spz_scan_args& a) {
  const ScanPlan p = scan_plan(a);
  return p.pieces > 1 ? 2 * p.pieces * a.batch * a.width * 4 + 16 : 0;
}

int scan_run(const char* call, const spz_scan_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = scan_check(args);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const spz_scan_args& a = *args;
  const int64_t need = scan_workspace(a);
  bad = scan_check_arrays(a, back, ws_bytes, ws, need);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
  if (a.batch == 0 || a.width == 0) return SPZ_OK;
  const ScanPlan plan = scan_plan(a);
  ScanArgs g{};
  g.a = a;
  g.pieces = plan.pieces;
  g.len = plan.pieces > 1 ? plan.len : a.steps;
  if (plan.pieces > 1) {
    const int64_t n = plan.pieces * a.batch * a.width;
    g.map_a = static_cast<float*>(ws);
    g.map_h = g.map_a + op_div_up(n, 4) * 4;
  }
  // Vectors of SCAN_V channels need every touched row aligned for them.
  const int e = op_size(a.prec);
  const auto vec = [&](const void* p, int64_t s0, int64_t s1) {
    return !p || (op_aligned(p, SCAN_V * e) && s0 % SCAN_V == 0 && s1 % SCAN_V == 0);
  };
  const bool v4 = a.width % SCAN_V == 0 && vec(a.f, a.f_batch, a.f_step) && vec(a.v, a.v_batch, a.v_step) &&
                  (back ? vec(a.dy, a.dy_batch, a.dy_step) && vec(a.df, a.df_batch, a.df_step) && vec(a.dv, a.dv_batch, a.dv_step)
                        : vec(a.y, a.y_batch, a.y_step));
  g.chunks = v4 ? a.width / SCAN_V : a.width;
  if (op_div_up(g.chunks * a.batch * g.pieces, SCAN_THREADS) >= OP_MAX_EXTENT)
    return op_error(SPZ_EINVAL, call, "extents out of range");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.prec == SPZ_PREC_BF16) {
    if (v4) scan_launch<bf16_t, SCAN_V>(g, back, s);
    else scan_launch<bf16_t, 1>(g, back, s);
  } else {
    if (v4) scan_launch<float, SCAN_V>(g, back, s);
    else scan_launch<float, 1>(g, back, s);
  }
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_scan_saved(const spz_scan_args* args) {
  const char* bad = scan_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_scan_saved", bad);
  const int64_t seg = args->prec == SPZ_PREC_BF16 ? SEG<bf16_t> : SEG<float>;
  return args->batch * op_div_up(args->steps, seg) * args->width;
}

int64_t spz_scan_workspace(const spz_scan_args* args, int32_t backward) {
  (void)backward;   // both directions keep the same maps
  const char* bad = scan_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_scan_workspace", bad);
  return scan_workspace(*args);
}

int spz_scan_forward(const spz_scan_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return scan_run("spz_scan_forward", args, false, workspace, workspace_bytes, hip_stream);
}

int spz_scan_backward(const spz_scan_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return scan_run("spz_scan_backward", args, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
