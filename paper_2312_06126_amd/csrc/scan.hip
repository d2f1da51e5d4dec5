// Gated linear recurrence over sequences (spz_scan_*): forward, backward and single steps.
//
//   h_t = a_t k_t h_{t-1} + (1 - a_t) v_t,  a_t = sigmoid(f_t), k_t = 0 at an episode start.
//
// Forward moves 3 elements a step and channel, backward 5 (f, v, dy, df, dv), for some 20 and 45 instructions, which
// take nearly as long: bound by HBM where enough steps are in flight, in pieces by both. A thread owns SCAN_V adjacent channels of
// one sequence (8 or 16 bytes a step, so a wave reads whole cache lines) and walks time with the
// next steps' loads in flight; states stay in registers in float32.
//
// A step is the affine map h -> A h + H, and maps compose, so where batch and width alone give too
// few threads time is cut into pieces: each piece's map is taken first (scan_piece), the maps
// are joined into the state in front of every piece (scan_join), then every piece is walked
// (scan_forward, scan_backward). The second reading of f and v comes mostly from the 256 MB
// last-level cache. Maps are kept in 64 bits: a state that a map gives is a sum of terms that may
// cancel, and then has to be as near as the one that steps in a row give. An episode start inside a
// piece makes its map independent of the state: such a map is marked by A = -1 (A is a product of
// sigmoids, else >= 0), so that a state that is not finite does not pass it as 0 * inf.
//
// Backward the same with time reversed: c -> P c + Q is the gradient handed from step to step.
// h_{t-1} is not stored by the forward pass: `saved` holds the state in front of every SEG-th step
// (6% of the bytes moved in bf16), from which a thread recomputes SEG steps in registers.
//
// Measured, on arrays that come from memory (in brackets: on the same arrays again and again, which the last-level cache
// holds in part or, in tiles, whole): 2048 x 50 x 256 bf16, serially: forward 49 us, backward 72 (39, 71; 3.2 and
// 3.6 TB/s), with lengths of half as many steps 39 and 57 (28, 49). 64 x 1000 x 200 float32 in tiles: forward 49 us,
// 3.2 TB/s (41); backward 74, 3.5 TB/s (74).
// 1 x 65536 x 512 bf16 in pieces: forward 42 + 10 + 40 us (36 + 10 + 41; scan_piece, scan_join, scan_forward), backward
// 37 + 10 + 82 (39 + 10 + 83).
#include <type_traits>

#include "../../include/spz_testing.h"
#include "ops.h"

namespace spz {
namespace {

constexpr int SCAN_THREADS = 256;
constexpr int SCAN_V = 4, SCAN_V_BACK = 2;   // channels a thread, where rows are aligned for them
                                             // (backward: more values a step, in 256 registers)
constexpr int SEG = 8;                        // steps in registers at once, and between saved states
constexpr int JOIN_CH = 8, JOIN_GROUPS = 128;

struct ScanArgs {
  spz_scan_args a;
  int64_t chunks;       // of V channels
  int64_t first;        // workgroup of the call that the dispatch starts with (scan_pos)
  int64_t pieces, len;  // time pieces and their steps (a multiple of SEG)
  double *map_a, *map_h; // [pieces, batch, width]: maps; map_h then the states between the pieces
};

// V elements of an array as they are stored, and as floats.
template <typename T, int V> struct Raw;
template <> struct Raw<float, 4> { u32x4 w; };
template <> struct Raw<bf16_t, 4> { u32x2 w; };
template <> struct Raw<float, 2> { u32x2 w; };
template <> struct Raw<bf16_t, 2> { uint32_t w; };
template <typename T> struct Raw<T, 1> { T w; };
template <typename T, int V> __device__ inline void load_raw(const T* p, Raw<T, V>& r) {
  r.w = *reinterpret_cast<const decltype(r.w)*>(p);
}
template <typename T, int V> __device__ inline void floats(const Raw<T, V>& r, float (&x)[V]) {
  if constexpr (V == 1) {
    x[0] = to_f<T>(r.w);
  } else {
    uint32_t w[V * sizeof(T) / 4];
    __builtin_memcpy(w, &r.w, sizeof(w));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (sizeof(T) == 4) x[i] = __builtin_bit_cast(float, w[i % (V * sizeof(T) / 4)]);
      else x[i] = __builtin_bit_cast(float, (i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
  }
}
template <typename T, int V> __device__ inline void store_v(T* p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = from_f<T>(x[0]);
  } else {
    Raw<T, V> r;
    uint32_t w[V * sizeof(T) / 4];
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) {
      if (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, x[i]);
      else w[i] = pack_bf16x2(x[(2 * i) % V], x[(2 * i + 1) % V]);
    }
    __builtin_memcpy(&r.w, w, sizeof(w));
    *reinterpret_cast<decltype(r.w)*>(p) = r.w;
  }
}
// V floats of a [.., width] state array: its rows are aligned only where width is.
template <int V> __device__ inline void load_s(const float* p, bool vec, float (&x)[V]) {
  typedef float vf __attribute__((ext_vector_type(V)));
  if (V > 1 && vec) {
    const vf w = *reinterpret_cast<const vf*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = w[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = p[i];
  }
}
template <int V> __device__ inline void store_s(float* p, bool vec, const float (&x)[V]) {
  typedef float vf __attribute__((ext_vector_type(V)));
  if (V > 1 && vec) {
    vf w;
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = x[i];
    *reinterpret_cast<vf*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = x[i];
  }
}
__device__ inline bool op_aligned16(const void* p) { return op_aligned(p, 16); }

struct ScanPos { int64_t b, c, p; };
template <int V> __device__ inline bool scan_pos(const ScanArgs& g, ScanPos& q) {
  const int64_t i = (g.first + blockIdx.x) * SCAN_THREADS + threadIdx.x;
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
// The same number, of which the compiler cannot know that it grows by a constant from segment to
// segment: else it keeps a pointer of its own for every access of a segment in registers (80 of them).
__device__ inline int64_t opaque(int64_t x) {
  asm("" : "+v"(x));
  return x;
}

// SEG steps of N arrays of a thread's channels and of the episode starts, as loaded: the next
// segment's loads are issued before the present one is worked on, so that each thread keeps
// N SEG accesses in flight. Steps past the last one (`last`, which exists) load that one again.
template <typename T, int V, int N> struct Segment {
  Raw<T, V> x[N][SEG];
  uint32_t cut;   // bit j: step j starts an episode
  __device__ void load(const spz_scan_args& a, int64_t b, const T* const (&p)[N], const int64_t (&step)[N], int64_t ts,
                       int64_t last) {
    ts = opaque(ts);
    const int n = (int)(last - ts);
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (p[k]) {
        const T* q = p[k] + ts * step[k];
        if (n >= SEG - 1) {
#pragma unroll
          for (int j = 0; j < SEG; ++j) load_raw<T, V>(q + j * step[k], x[k][j]);
        } else {
#pragma unroll
          for (int j = 0; j < SEG; ++j) load_raw<T, V>(q + (j < n ? j : n) * step[k], x[k][j]);
        }
      }
    cut = 0;
    if (!a.reset) return;
    const uint8_t* r = a.reset + b * a.reset_batch + ts * a.reset_step;
    if (a.reset_step == 1 && n >= SEG - 1) {
      uint64_t w;
      __builtin_memcpy(&w, r, SEG);
      // Bit 8 j + 7 of the sum: byte j is not 0.
      w = ((w & 0x7F7F7F7F7F7F7F7Full) + 0x7F7F7F7F7F7F7F7Full) | w;
#pragma unroll
      for (int j = 0; j < SEG; ++j) cut |= (uint32_t)(w >> (8 * j + 7) & 1) << j;
    } else {
#pragma unroll
      for (int j = 0; j < SEG; ++j) cut |= (uint32_t)(r[(j < n ? j : n) * a.reset_step] != 0) << j;
    }
  }
};

// step(j, k) over the `cnt` steps of a segment, from the last one where BACK, k: step j starts an
// episode. Whole segments without a start, nearly all of them, run without a branch or select.
template <bool BACK, typename F> __device__ inline void walk(int cnt, uint32_t cut, F&& step) {
  if (cnt == SEG && cut == 0) {
#pragma unroll
    for (int j = 0; j < SEG; ++j) step(BACK ? SEG - 1 - j : j, false);
  } else {
#pragma unroll
    for (int jj = 0; jj < SEG; ++jj) {
      const int j = BACK ? SEG - 1 - jj : jj;
      if (j < cnt) step(j, (cut >> j & 1) != 0);
    }
  }
}

// The affine map of each piece: BACK = false (f, v), true (f, dy; from the piece's end).
template <typename T, int V, bool BACK> __global__ __launch_bounds__(SCAN_THREADS, 2) void scan_piece(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b), t1 = n < end ? n : end;
  double A[V], H[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { A[i] = 1.0; H[i] = 0.0; }
  const T* f = static_cast<const T*>(a.f) + q.b * a.f_batch + q.c;
  const T* w = static_cast<const T*>(BACK ? a.dy : a.v);
  if (w) w += q.b * (BACK ? a.dy_batch : a.v_batch) + q.c;
  const T* const p[2] = {f, w};
  const int64_t step[2] = {a.f_step, BACK ? a.dy_step : a.v_step};
  uint32_t cut = 0;
  if (t1 > t0) {
    const int64_t segs = (t1 - t0 + SEG - 1) / SEG;
    Segment<T, V, 2> now, next;
    now.load(a, q.b, p, step, t0 + (BACK ? segs - 1 : 0) * SEG, t1 - 1);
    for (int64_t s = 0; s < segs; ++s) {
      const int64_t ts = t0 + (BACK ? segs - 1 - s : s) * SEG;
      if (s + 1 < segs) next.load(a, q.b, p, step, BACK ? ts - SEG : ts + SEG, t1 - 1);
      const int cnt = (int)(t1 - ts < SEG ? t1 - ts : SEG);
      cut |= now.cut & ((1u << cnt) - 1);
      walk<BACK>(cnt, now.cut, [&](int j, bool k) {
        float x[V], y[V];
        floats<T, V>(now.x[0][j], x);
        if (w) floats<T, V>(now.x[1][j], y);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float al, be;
          sigmoid2(x[i], al, be);
          if (BACK) H[i] = k ? 0.0 : (double)al * (w ? H[i] + (double)y[i] : H[i]);
          else H[i] = k ? (double)(be * y[i]) : fma((double)al, H[i], (double)(be * y[i]));
          A[i] *= (double)al;
        }
      });
      now = next;
    }
  }
  if (cut) {
#pragma unroll
    for (int i = 0; i < V; ++i) A[i] = -1.0;
  }
  const int64_t o = (q.p * a.batch + q.b) * a.width + q.c;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    g.map_a[o + i] = A[i];
    g.map_h[o + i] = H[i];
  }
}

// (A, H) after (A1, H1): the map that applies (A1, H1) first.
__device__ inline void join_maps(double A1, double H1, double& A, double& H) {
  const bool cut = A == -1.0;
  H = cut ? H : fma(A, H1, H);
  A = cut || A1 == -1.0 ? -1.0 : A * A1;
}
__device__ inline double apply_map(double A, double H, double h) { return A == -1.0 ? H : fma(A, h, H); }

// map_h[p] <- the state in front of piece p (backward: behind it), from the maps and the first
// state (`first`, NULL: zeros). 8 channels a workgroup; 128 groups of threads each join a range of
// pieces, the ranges' maps are joined by doubling, then each range is walked from its first state. Bound by
// latency: 1024 pieces of 512 channels 10 us, with ranges of up to U kept in registers (12 when read again;
// 4 or 2 channels a workgroup: 15, 16).
__global__ __launch_bounds__(JOIN_CH * JOIN_GROUPS) void scan_join(const double* map_a, double* map_h, const float* first,
                                                                   int64_t channels, int64_t pieces, bool back) {
  __shared__ double sa[JOIN_GROUPS][JOIN_CH], sh[JOIN_GROUPS][JOIN_CH];
  const int c = threadIdx.x % JOIN_CH, gr = threadIdx.x / JOIN_CH;
  const int64_t ch = (int64_t)blockIdx.x * JOIN_CH + c;
  const bool on = ch < channels;
  const int64_t per = (pieces + JOIN_GROUPS - 1) / JOIN_GROUPS;
  const int64_t p0 = gr * per < pieces ? gr * per : pieces, p1 = on ? (p0 + per < pieces ? p0 + per : pieces) : p0;
  const auto at = [&](int64_t p) { return (back ? pieces - 1 - p : p) * channels + ch; };
  constexpr int U = 8;   // maps loaded at once
  double ma[U], mh[U];
  const auto load = [&](int64_t p) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t o = at(p + j < p1 ? p + j : p1 - 1);
      ma[j] = map_a[o];
      mh[j] = map_h[o];
    }
  };
  double A = 1.0, H = 0.0;
  for (int64_t p = p0; p < p1; p += U) {
    load(p);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (p + j >= p1) continue;
      double A2 = ma[j], H2 = mh[j];
      join_maps(A, H, A2, H2);
      A = A2;
      H = H2;
    }
  }
  for (int d = 1; d < JOIN_GROUPS; d *= 2) {
    sa[gr][c] = A;
    sh[gr][c] = H;
    __syncthreads();
    if (gr >= d) join_maps(sa[gr - d][c], sh[gr - d][c], A, H);
    __syncthreads();
  }
  sa[gr][c] = A;
  sh[gr][c] = H;
  __syncthreads();
  if (!on) return;
  double h = first ? first[ch] : 0.0;
  if (gr) h = apply_map(sa[gr - 1][c], sh[gr - 1][c], h);
  for (int64_t p = p0; p < p1; p += U) {
    if (per > U) load(p);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (p + j >= p1) continue;
      map_h[at(p + j)] = h;
      h = apply_map(ma[j], mh[j], h);
    }
  }
}

template <typename T, int V> __global__ __launch_bounds__(SCAN_THREADS, 2) void scan_forward(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const bool vec = a.width % 4 == 0;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b);
  const int64_t t2 = end < a.steps ? end : a.steps, t1 = n < t2 ? n : t2;
  const int64_t st = q.b * a.width + q.c;
  const T* const p[2] = {static_cast<const T*>(a.f) + q.b * a.f_batch + q.c, static_cast<const T*>(a.v) + q.b * a.v_batch + q.c};
  const int64_t step[2] = {a.f_step, a.v_step};
  T* y = static_cast<T*>(a.y) + q.b * a.y_batch + q.c;
  const int64_t saves = (a.steps + SEG - 1) / SEG;
  const bool vs = vec && op_aligned16(a.saved);
  float h[V];
  if (g.pieces > 1) {
    const double* m = g.map_h + q.p * a.batch * a.width + st;
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = (float)m[i];
  } else if (a.h0) {
    load_s<V>(a.h0 + st, vec && op_aligned16(a.h0), h);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = 0.0f;
  }
  if (t1 > t0) {
    Segment<T, V, 2> now, next;
    now.load(a, q.b, p, step, t0, t1 - 1);
    for (int64_t ts = t0; ts < t1; ts += SEG) {
      if (ts + SEG < t1) next.load(a, q.b, p, step, ts + SEG, t1 - 1);
      if (a.saved) store_s<V>(a.saved + (q.b * saves + ts / SEG) * a.width + q.c, vs, h);
      const int cnt = (int)(t1 - ts < SEG ? t1 - ts : SEG);
      T* const out = y + opaque(ts) * a.y_step;
      walk<false>(cnt, now.cut, [&](int j, bool k) {
        float x[V], w[V];
        floats<T, V>(now.x[0][j], x);
        floats<T, V>(now.x[1][j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float al, be;
          sigmoid2(x[i], al, be);
          h[i] = fmaf(be, w[i], k ? 0.0f : al * h[i]);
        }
        store_v<T, V>(out + j * a.y_step, h);
      });
      now = next;
    }
  }
  float zero[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = t1 > t0 ? t1 : t0; t < t2; ++t) store_v<T, V>(y + t * a.y_step, zero);
  // hT from the piece with the last step (the joint maps' state behind it may differ in its last bits); h0 without steps.
  if (a.hT && (n ? t0 < n && n <= end : q.p == 0)) store_s<V>(a.hT + st, vec && op_aligned16(a.hT), h);
}

template <typename T, int V> __global__ __launch_bounds__(SCAN_THREADS, 2) void scan_backward(ScanArgs g) {
  ScanPos q;
  if (!scan_pos<V>(g, q)) return;
  const spz_scan_args& a = g.a;
  const bool vec = a.width % 4 == 0;
  const int64_t t0 = q.p * g.len, end = t0 + g.len, n = scan_length(a, q.b);
  const int64_t t2 = end < a.steps ? end : a.steps, t1 = n < t2 ? n : t2;
  const int64_t st = q.b * a.width + q.c;
  const T* const p[3] = {static_cast<const T*>(a.f) + q.b * a.f_batch + q.c, static_cast<const T*>(a.v) + q.b * a.v_batch + q.c,
                         a.dy ? static_cast<const T*>(a.dy) + q.b * a.dy_batch + q.c : nullptr};
  const int64_t step[3] = {a.f_step, a.v_step, a.dy_step};
  T* df = static_cast<T*>(a.df) + q.b * a.df_batch + q.c;
  T* dv = static_cast<T*>(a.dv) + q.b * a.dv_batch + q.c;
  const float* saved = a.saved + q.b * ((a.steps + SEG - 1) / SEG) * a.width + q.c;
  const bool vs = vec && op_aligned16(a.saved);
  float zero[V], c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = t1 > t0 ? t1 : t0; t < t2; ++t) {
    store_v<T, V>(df + t * a.df_step, zero);
    store_v<T, V>(dv + t * a.dv_step, zero);
  }
  if (g.pieces > 1) {
    const double* m = g.map_h + q.p * a.batch * a.width + st;
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = (float)m[i];
  } else if (a.dhT) {
    load_s<V>(a.dhT + st, vec && op_aligned16(a.dhT), c);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = 0.0f;
  }
  if (t1 > t0) {
    Segment<T, V, 3> now, next;
    float h[V], h_next[V];
    int64_t ts = t0 + (t1 - 1 - t0) / SEG * SEG;
    now.load(a, q.b, p, step, ts, t1 - 1);
    load_s<V>(saved + ts / SEG * a.width, vs, h);
    for (; ts >= t0; ts -= SEG) {
      if (ts > t0) {
        next.load(a, q.b, p, step, ts - SEG, t1 - 1);
        load_s<V>(saved + (ts / SEG - 1) * a.width, vs, h_next);
      }
      const int cnt = (int)(t1 - ts < SEG ? t1 - ts : SEG);
      // Forward through the segment: the sigmoids, and k_t h_{t-1} - v_t times a_t.
      float al[SEG][V], be[SEG][V], gap[SEG][V];
      walk<false>(cnt, now.cut, [&](int j, bool k) {
        float x[V], w[V];
        floats<T, V>(now.x[0][j], x);
        floats<T, V>(now.x[1][j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sigmoid2(x[i], al[j][i], be[j][i]);
          const float before = k ? 0.0f : h[i];
          gap[j][i] = al[j][i] * (before - w[i]);
          h[i] = fmaf(be[j][i], w[i], al[j][i] * before);
        }
      });
      T* const out_f = df + opaque(ts) * a.df_step;
      T* const out_v = dv + opaque(ts) * a.dv_step;
      walk<true>(cnt, now.cut, [&](int j, bool k) {
        float d[V], of[V], ov[V];
        if (p[2]) floats<T, V>(now.x[2][j], d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float gr = p[2] ? d[i] + c[i] : c[i];
          ov[i] = gr * be[j][i];
          of[i] = ov[i] * gap[j][i];
          c[i] = k ? 0.0f : al[j][i] * gr;
        }
        store_v<T, V>(out_f + j * a.df_step, of);
        store_v<T, V>(out_v + j * a.dv_step, ov);
      });
      now = next;
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = h_next[i];
    }
  }
  if (a.dh0 && q.p == 0) store_s<V>(a.dh0 + st, vec && op_aligned16(a.dh0), c);
}

// ----------------------------------------------------------------------------- tiles of time
// One workgroup a sequence and CL chunks of channels: its TILE_WAVES waves of 64 / CL time lanes
// each take SEG steps at once (CL = 16: 256 steps), join their maps within the workgroup, and go on
// to the next steps from the joint state, with its loads in flight. Everything is read once, in one
// launch. Order position (wave, time lane) runs with time, backward against it.
constexpr int TILE_THREADS = 256, TILE_WAVES = TILE_THREADS / 64;

// Workgroup b runs on XCD b % 8: neighbours in width, whose 128 bytes a step share cache lines where rows
// are not whole lines, on the same one (64 x 1000 x 200 float32, in the last-level cache: 39 against 48 us).
__device__ inline int64_t tile_block() { return blockIdx.x % 8 * (int64_t)(gridDim.x / 8) + blockIdx.x / 8; }

template <int V, int CL, bool BACK> struct Tile {
  static constexpr int TL = 64 / CL, LANES = TILE_WAVES * TL;
  double (*maps)[TILE_WAVES][CL][2 * V];   // [2]: the waves' maps, two buffers in turn
  int wave, tl, cl, slot = 0;
  // From each thread's map: the state in front of its steps; carry becomes the one behind the tile.
  __device__ void join(double (&A)[V], double (&H)[V], double (&carry)[V], float (&h)[V]) {
    double eA[V], eH[V];
#pragma unroll
    for (int d = 1; d < TL; d *= 2)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const double A1 = __shfl_up(A[i], d * CL), H1 = __shfl_up(H[i], d * CL);
        if (tl >= d) join_maps(A1, H1, A[i], H[i]);
      }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      eA[i] = TL > 1 ? __shfl_up(A[i], CL) : 1.0;
      eH[i] = TL > 1 ? __shfl_up(H[i], CL) : 0.0;
      if (tl == 0) { eA[i] = 1.0; eH[i] = 0.0; }
    }
    double* mine = maps[slot][wave][cl];
    if (tl == TL - 1)
#pragma unroll
      for (int i = 0; i < V; ++i) { mine[i] = A[i]; mine[V + i] = H[i]; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TILE_WAVES; ++w) {
      const double* m = maps[slot][w][cl];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (w == wave) h[i] = (float)apply_map(eA[i], eH[i], carry[i]);
        carry[i] = apply_map(m[i], m[V + i], carry[i]);
      }
    }
    slot ^= 1;   // a wave that writes this buffer again has passed the other one's barrier
  }
};

template <typename T, int V, int CL> __global__ __launch_bounds__(TILE_THREADS, 2) void scan_tile_forward(ScanArgs g) {
  const spz_scan_args& a = g.a;
  using Ti = Tile<V, CL, false>;
  __shared__ double maps[2][TILE_WAVES][CL][2 * V];
  Ti tile{maps, (int)threadIdx.x / 64, (int)threadIdx.x % 64 / CL, (int)threadIdx.x % CL};
  const int64_t groups = (g.chunks + CL - 1) / CL, at = tile_block(), b = at / groups;
  const int64_t chunk = at % groups * CL + tile.cl, c = chunk * V;
  if (b >= a.batch) return;
  const bool on = chunk < g.chunks, vec = a.width % 4 == 0;
  const int64_t n = scan_length(a, b), saves = (a.steps + SEG - 1) / SEG, st = b * a.width + c;
  const T* const p[2] = {static_cast<const T*>(a.f) + b * a.f_batch + c, static_cast<const T*>(a.v) + b * a.v_batch + c};
  const int64_t step[2] = {a.f_step, a.v_step};
  T* y = static_cast<T*>(a.y) + b * a.y_batch + c;
  const bool vs = vec && op_aligned16(a.saved);
  double carry[V];
  float h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = 0.0f;
  if (on && a.h0) load_s<V>(a.h0 + st, vec && op_aligned16(a.h0), h);
#pragma unroll
  for (int i = 0; i < V; ++i) carry[i] = h[i];
  Segment<T, V, 2> now, next;
  int64_t ts = (int64_t)(tile.wave * Ti::TL + tile.tl) * SEG;
  if (on && ts < n) now.load(a, b, p, step, ts, n - 1);
  for (int64_t t0 = 0; t0 < n; t0 += Ti::LANES * SEG, ts += Ti::LANES * SEG) {
    const int64_t ahead = ts + Ti::LANES * SEG;
    if (on && ahead < n) next.load(a, b, p, step, ahead, n - 1);
    const int cnt = !on || ts >= n ? 0 : (int)(n - ts < SEG ? n - ts : SEG);
    float al[SEG][V], bw[SEG][V];
    double A[V], H[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { A[i] = 1.0; H[i] = 0.0; }
    if (cnt) {
      walk<false>(cnt, now.cut, [&](int j, bool k) {
        float x[V], w[V];
        floats<T, V>(now.x[0][j], x);
        floats<T, V>(now.x[1][j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float be;
          sigmoid2(x[i], al[j][i], be);
          bw[j][i] = be * w[i];
          H[i] = k ? (double)bw[j][i] : fma((double)al[j][i], H[i], (double)bw[j][i]);
          A[i] *= (double)al[j][i];
        }
      });
      if (now.cut & ((1u << cnt) - 1)) {
#pragma unroll
        for (int i = 0; i < V; ++i) A[i] = -1.0;
      }
    }
    tile.join(A, H, carry, h);
    if (cnt) {
      if (a.saved) store_s<V>(a.saved + (b * saves + ts / SEG) * a.width + c, vs, h);
      T* const out = y + opaque(ts) * a.y_step;
      walk<false>(cnt, now.cut, [&](int j, bool k) {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = k ? bw[j][i] : fmaf(al[j][i], h[i], bw[j][i]);
        store_v<T, V>(out + j * a.y_step, h);
      });
      // The last state comes from its own steps, not from the joint maps, whose sums may cancel.
      if (a.hT && ts + SEG >= n) store_s<V>(a.hT + st, vec && op_aligned16(a.hT), h);
    }
    now = next;
  }
  if (!on) return;
  float zero[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = n + tile.wave * Ti::TL + tile.tl; t < a.steps; t += Ti::LANES) store_v<T, V>(y + t * a.y_step, zero);
  if (a.hT && n == 0 && threadIdx.x < CL) store_s<V>(a.hT + st, vec && op_aligned16(a.hT), h);
}

template <typename T, int V, int CL> __global__ __launch_bounds__(TILE_THREADS, 2) void scan_tile_backward(ScanArgs g) {
  const spz_scan_args& a = g.a;
  using Ti = Tile<V, CL, true>;
  __shared__ double maps[2][TILE_WAVES][CL][2 * V];
  Ti tile{maps, (int)threadIdx.x / 64, (int)threadIdx.x % 64 / CL, (int)threadIdx.x % CL};
  const int64_t groups = (g.chunks + CL - 1) / CL, at = tile_block(), b = at / groups;
  const int64_t chunk = at % groups * CL + tile.cl, c0 = chunk * V;
  if (b >= a.batch) return;
  const bool on = chunk < g.chunks, vec = a.width % 4 == 0;
  const int64_t n = scan_length(a, b), st = b * a.width + c0;
  const T* const p[3] = {static_cast<const T*>(a.f) + b * a.f_batch + c0, static_cast<const T*>(a.v) + b * a.v_batch + c0,
                         a.dy ? static_cast<const T*>(a.dy) + b * a.dy_batch + c0 : nullptr};
  const int64_t step[3] = {a.f_step, a.v_step, a.dy_step};
  T* df = static_cast<T*>(a.df) + b * a.df_batch + c0;
  T* dv = static_cast<T*>(a.dv) + b * a.dv_batch + c0;
  const float* saved = a.saved + b * ((a.steps + SEG - 1) / SEG) * a.width + c0;
  const bool vs = vec && op_aligned16(a.saved);
  double carry[V];
  float c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) c[i] = 0.0f;
  if (on && a.dhT) load_s<V>(a.dhT + st, vec && op_aligned16(a.dhT), c);
#pragma unroll
  for (int i = 0; i < V; ++i) carry[i] = c[i];
  Segment<T, V, 3> now, next;
  float h[V], h_next[V];
  const int64_t tiles = (n + Ti::LANES * SEG - 1) / (Ti::LANES * SEG);
  int64_t ts = (tiles * Ti::LANES - 1 - (tile.wave * Ti::TL + tile.tl)) * SEG;
  if (on && tiles && ts < n) {
    now.load(a, b, p, step, ts, n - 1);
    load_s<V>(saved + ts / SEG * a.width, vs, h);
  }
  for (int64_t k = 0; k < tiles; ++k, ts -= Ti::LANES * SEG) {
    if (on && k + 1 < tiles) {   // the tiles in front of the last one are whole
      next.load(a, b, p, step, ts - Ti::LANES * SEG, n - 1);
      load_s<V>(saved + (ts / SEG - Ti::LANES) * a.width, vs, h_next);
    }
    const int cnt = !on || ts >= n ? 0 : (int)(n - ts < SEG ? n - ts : SEG);
    float al[SEG][V], be[SEG][V], gap[SEG][V];
    double P[V], Q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) { P[i] = 1.0; Q[i] = 0.0; }
    if (cnt) {
      walk<false>(cnt, now.cut, [&](int j, bool cut) {
        float x[V], w[V];
        floats<T, V>(now.x[0][j], x);
        floats<T, V>(now.x[1][j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sigmoid2(x[i], al[j][i], be[j][i]);
          const float before = cut ? 0.0f : h[i];
          gap[j][i] = al[j][i] * (before - w[i]);
          h[i] = fmaf(be[j][i], w[i], al[j][i] * before);
          P[i] *= (double)al[j][i];
        }
      });
      walk<true>(cnt, now.cut, [&](int j, bool cut) {
        float d[V];
        if (p[2]) floats<T, V>(now.x[2][j], d);
#pragma unroll
        for (int i = 0; i < V; ++i) Q[i] = cut ? 0.0 : (double)al[j][i] * (p[2] ? Q[i] + (double)d[i] : Q[i]);
      });
      if (now.cut & ((1u << cnt) - 1)) {
#pragma unroll
        for (int i = 0; i < V; ++i) P[i] = -1.0;
      }
    }
    tile.join(P, Q, carry, c);
    if (cnt) {
      T* const out_f = df + opaque(ts) * a.df_step;
      T* const out_v = dv + opaque(ts) * a.dv_step;
      walk<true>(cnt, now.cut, [&](int j, bool cut) {
        float d[V], of[V], ov[V];
        if (p[2]) floats<T, V>(now.x[2][j], d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float gr = p[2] ? d[i] + c[i] : c[i];
          ov[i] = gr * be[j][i];
          of[i] = ov[i] * gap[j][i];
          c[i] = cut ? 0.0f : al[j][i] * gr;
        }
        store_v<T, V>(out_f + j * a.df_step, of);
        store_v<T, V>(out_v + j * a.dv_step, ov);
      });
      if (a.dh0 && ts == 0) store_s<V>(a.dh0 + st, vec && op_aligned16(a.dh0), c);   // as hT forward
    }
    now = next;
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = h_next[i];
  }
  if (!on) return;
  float zero[V];
#pragma unroll
  for (int i = 0; i < V; ++i) zero[i] = 0.0f;
  for (int64_t t = n + tile.wave * Ti::TL + tile.tl; t < a.steps; t += Ti::LANES) {
    store_v<T, V>(df + t * a.df_step, zero);
    store_v<T, V>(dv + t * a.dv_step, zero);
  }
  if (a.dh0 && n == 0 && threadIdx.x < CL) store_s<V>(a.dh0 + st, vec && op_aligned16(a.dh0), c);
}

// How a call is spread over the threads, by its sizes alone, from what the ways cost (microseconds
// forward, both sides measured from 16 x 40 x 256 to 27 x 13250 x 56):
//   serial: a thread walks the whole sequence: 0.26 a step, as long as there are threads for it;
//   tiles: a workgroup walks it in tiles of time, 512 workgroups at a time: 3 a round and 3.7 a tile of it
//     (64 x 64 x 256: 7 against 17 serially; 270 x 23 x 536: 64 against 12);
//   pieces: time cut into pieces, for SCAN_FILL threads but of at least SCAN_MIN_LEN steps each: 24 for
//     three launches and 1.6 a million elements for reading twice (1 x 4096 x 256: 26 against 59 in
//     tiles; 8 x 2216 x 624: 54 against 43).
constexpr int64_t SCAN_FILL = 131072, SCAN_MIN_LEN = 32;
enum ScanWay { SCAN_SERIAL, SCAN_TILED, SCAN_PIECES };
struct ScanPlan { ScanWay way; int64_t pieces, len; };
ScanPlan scan_plan(const spz_scan_args& a) {
  const int64_t threads = a.batch * op_div_up(a.width, SCAN_V);
  const bool narrow = a.width <= 8, vectors = a.width % SCAN_V == 0;
  const int64_t tile = (narrow ? 1024 : 256) / (vectors ? 1 : SCAN_V);   // steps of one
  const int64_t rounds = op_div_up(a.batch * op_div_up(a.width, narrow ? 8 : 32), 512);
  const int64_t turns = rounds * op_div_up(a.steps, tile);
  if (threads * 2 > SCAN_FILL || a.steps <= 14 * turns + 11 * rounds) return {SCAN_SERIAL, 1, a.steps};
  const int64_t millions = a.batch * a.steps * a.width >> 20;
  if (turns <= 6 + millions / 2 || a.steps < 2 * SCAN_MIN_LEN) return {SCAN_TILED, 1, a.steps};
  int64_t pieces = op_div_up(SCAN_FILL, threads);
  const int64_t most = a.steps / SCAN_MIN_LEN;
  if (pieces > most) pieces = most;
  const int64_t len = op_div_up(op_div_up(a.steps, pieces), SEG) * SEG;
  return {SCAN_PIECES, op_div_up(a.steps, len), len};
}

const char* scan_check(const spz_scan_args* a) {
  if (!a) return "NULL arguments";
  if (!op_prec_ok(a->prec)) return "unknown precision";
  if (!op_extent_ok(a->batch) || !op_extent_ok(a->steps) || !op_extent_ok(a->width)) return "extent out of range";
  // No device holds more; keeps every index and count within 62 bits.
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

template <typename T, int V, bool BACK> void scan_launch(const ScanArgs& g, ScanWay way, hipStream_t s) {
  if (way == SCAN_TILED) {
    const auto tiles = [&](auto lanes) {
      constexpr int CL = decltype(lanes)::value;
      const dim3 grid((unsigned)(op_div_up(g.a.batch * op_div_up(g.chunks, CL), 8) * 8));
      if constexpr (BACK) scan_tile_backward<T, V, CL><<<grid, TILE_THREADS, 0, s>>>(g);
      else scan_tile_forward<T, V, CL><<<grid, TILE_THREADS, 0, s>>>(g);
    };
    // 32 channels a workgroup; with 8 or fewer, the lanes that they leave are better used in time.
    if (g.chunks <= 8 / V) tiles(std::integral_constant<int, 8 / V>{});
    else tiles(std::integral_constant<int, 32 / V>{});
    return;
  }
  const int64_t blocks = op_div_up(g.chunks * g.a.batch * g.pieces, SCAN_THREADS);
  if (way == SCAN_PIECES) {   // SCAN_FILL threads or some more: one dispatch
    const dim3 grid((unsigned)blocks);
    const int64_t channels = g.a.batch * g.a.width;
    scan_piece<T, V, BACK><<<grid, SCAN_THREADS, 0, s>>>(g);
    scan_join<<<dim3((unsigned)op_div_up(channels, JOIN_CH)), JOIN_CH * JOIN_GROUPS, 0, s>>>(
        g.map_a, g.map_h, BACK ? g.a.dhT : g.a.h0, channels, g.pieces, BACK);
  }
  op_dispatch(blocks, SCAN_THREADS, [&](int64_t first, dim3 grid) {
    ScanArgs part = g;
    part.first = first;
    if constexpr (BACK) scan_backward<T, V><<<grid, SCAN_THREADS, 0, s>>>(part);
    else scan_forward<T, V><<<grid, SCAN_THREADS, 0, s>>>(part);
  });
}

template <typename T> void scan_dispatch(const ScanArgs& g, ScanWay way, bool back, bool vectors, hipStream_t s) {
  if (back && vectors) scan_launch<T, SCAN_V_BACK, true>(g, way, s);
  else if (back) scan_launch<T, 1, true>(g, way, s);
  else if (vectors) scan_launch<T, SCAN_V, false>(g, way, s);
  else scan_launch<T, 1, false>(g, way, s);
}

// Vectors of channels need every touched row aligned for them.
bool scan_vectors(const spz_scan_args& a, bool back) {
  const int e = op_size(a.prec), v = back ? SCAN_V_BACK : SCAN_V;
  const auto vec = [&](const void* p, int64_t s0, int64_t s1) {
    return !p || (op_aligned(p, v * e) && s0 % v == 0 && s1 % v == 0);
  };
  return a.width % v == 0 && vec(a.f, a.f_batch, a.f_step) && vec(a.v, a.v_batch, a.v_step) &&
         (back ? vec(a.dy, a.dy_batch, a.dy_step) && vec(a.df, a.df_batch, a.df_step) && vec(a.dv, a.dv_batch, a.dv_step)
               : vec(a.y, a.y_batch, a.y_step));
}

int64_t scan_workspace(const spz_scan_args& a) {
  const ScanPlan p = scan_plan(a);
  return p.way == SCAN_PIECES ? 2 * p.pieces * a.batch * a.width * 8 : 0;
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
  g.len = plan.len;
  if (plan.way == SCAN_PIECES) {
    g.map_a = static_cast<double*>(ws);
    g.map_h = g.map_a + plan.pieces * a.batch * a.width;
  }
  const int v = back ? SCAN_V_BACK : SCAN_V;
  const bool vectors = scan_vectors(a, back);
  g.chunks = vectors ? a.width / v : a.width;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.prec == SPZ_PREC_BF16) scan_dispatch<bf16_t>(g, plan.way, back, vectors, s);
  else scan_dispatch<float>(g, plan.way, back, vectors, s);
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_scan_saved(const spz_scan_args* args) {
  const char* bad = scan_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_scan_saved", bad);
  return args->batch * op_div_up(args->steps, SEG) * args->width;
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

int spzt_scan_way(const spz_scan_args* args, int32_t backward) {
  if (scan_check(args)) return SPZ_EINVAL;
  return (int)scan_plan(*args).way + (scan_vectors(*args, backward != 0) ? 4 : 0);
}

}  // extern "C"
