// Norms before and after a block with its gate, dropout and residual scale in one pass over the
// rows (spz_block_norm_*), and dropout by itself (spz_dropout).
//
//   n = post(h) w_post + b_post,  o = drop(gate(z) n),  x' = x + scale o,  u = pre(x') w_pre + b_pre
//
// Bound by HBM: forward 3 arrays read and 2 written, backward 5 read and 3 written, for about 30
// and 90 instructions an element. A row stays in the registers of TPR threads (16 lanes to a
// workgroup, by its width) from its loads to its stores, so the statistics of both norms and their
// gradients are sums over registers and nothing is read twice; variances are of the centred values.
// The backward pass recomputes the forward one from x, h and z (cheaper than reading x' and the
// statistics back). Its rows are walked with a stride, the next row's loads in flight; parameter
// vectors and the column sums of their gradients stay in registers, which is why a thread has only
// eight elements of a row there. A workgroup adds its rows in LDS, norm_sums the workgroups in order: no
// atomics, the same bits on every run. Rows wider than the registers hold take norm_wide, which
// reads them again for each statistic.
//
// Measured at 65536 x 1024 bf16: norm_forward 120 us (5.6 TB/s), norm_backward 253 to 266 (4.2 to 4.0), norm_sums 5;
// without a block in front (h NULL) 51, 107 (from memory; 5.3 and 3.8 TB/s) and 5. At 5000 x 393 float32, rows
// that no access of 16 bytes fits: 15, 29 and 4 us from memory.
#include <type_traits>

#include "ops.h"

namespace spz {
namespace {

constexpr int NORM_THREADS = 256;
constexpr int NORM_VECTORS = 5;          // dw_post, db_post, dscale, dw_pre, db_pre
constexpr int64_t NORM_MAX_WAVES = 2048; // of the backward pass: eight a compute unit (16: 31 against 27
                                         // us at 5000 x 393 float32, and twice the sums to add)
constexpr int NORM_CHUNK = 8;            // adjacent elements of a thread: one Philox block

struct Drop { uint32_t d; float gain; bool on; };

struct NormArgs {
  spz_block_norm_args a;
  Drop drop;
  int64_t first;      // workgroup of the forward call that the dispatch starts with
  float* part;        // backward: [blocks, NORM_VECTORS, width]
  bool wants[NORM_VECTORS];
};

// ----------------------------------------------------------------------------- sums over a row
// Sums over the TPR threads of a row. More than a wave: through LDS, two buffers in turn so that one
// barrier a sum is enough (a wave that writes a buffer again has passed the other one's barrier).
template <int TPR> struct RowSum {
  __device__ float operator()(float x) { return TPR == 16 ? sum16(x) : TPR == 32 ? sum32(x) : sum64(x); }
};
template <int TPR> struct WideSum {
  float (*buf)[TPR / 64];
  int slot = 0;
  __device__ float operator()(float x) {
    x = sum64(x);
    if (threadIdx.x % 64 == 0) buf[slot][threadIdx.x / 64] = x;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) s += buf[slot][i];
    slot ^= 1;
    return s;
  }
};

// ----------------------------------------------------------------------------- a row in registers
// Thread `lane` of TPR holds K chunks of NORM_CHUNK adjacent elements, chunk j from column
// (j TPR + lane) NORM_CHUNK on, in 16-byte accesses at whatever alignment the rows have. EVEN: the width
// is a multiple of the chunk; else the row's last chunk has a part of its elements.
template <typename T, bool EVEN, int TPR, int K> struct RowMap {
  static constexpr int VW = NORM_CHUNK, N = K * VW, E = OP_VEC<T>, P = VW / E;
  static constexpr int MASK = TPR * K + 2;   // bytes of a row's dropout mask: its Philox blocks
  uint32_t lane, D;
  __device__ uint32_t col(int j, int i) const { return (j * TPR + lane) * VW + i; }
  // Element i of chunk j exists.
  __device__ bool in(int j, int i) const { return col(j, EVEN ? 0 : i) < D; }
  // Element c of a row. The row's address is the same for a whole wave (where it is one): with a 32-bit
  // byte offset beside it no thread needs 64-bit arithmetic or registers for its addresses.
  template <typename V> static __device__ V* at(V* row, uint32_t c) {
    return reinterpret_cast<V*>(reinterpret_cast<char*>(const_cast<typename std::remove_const<V>::type*>(row)) + c * (uint32_t)sizeof(V));
  }
  // The thread's part of a row as it is stored. Elements past the width are set to zero once (clear)
  // and never loaded, so that they add nothing to a sum.
  struct Raw {
    u32x4 w[K * P];
    __device__ void clear() {
#pragma unroll
      for (int i = 0; i < K * P; ++i) w[i] = u32x4{0, 0, 0, 0};
    }
  };
  // access(index, first column, elements) over the thread's accesses.
  template <typename F> __device__ void each(F&& access) const {
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const uint32_t c = col(j, k * E);
        if (c < D) access(j * P + k, c, EVEN || c + E <= D ? E : (int)(D - c));
      }
  }
  __device__ void load(const T* p, Raw& r) const {
    each([&](int i, uint32_t c, int n) {
      if (n == E) r.w[i] = load16(at(p, c));
      else r.w[i] = load_part(at(p, c), n);
    });
  }
  __device__ void floats(const Raw& r, float (&x)[N]) const {
#pragma unroll
    for (int k = 0; k < N / E; ++k) {
      float t[E];
      unpack(r.w[k], t);
#pragma unroll
      for (int i = 0; i < E; ++i) x[k * E + i] = t[i];
    }
  }
  __device__ void load(const T* p, float (&x)[N]) const {
    Raw r;
    r.clear();
    load(p, r);
    floats(r, x);
  }
  __device__ void store(T* p, const float (&x)[N]) const {
    each([&](int i, uint32_t c, int n) {
      float t[E];
#pragma unroll
      for (int k = 0; k < E; ++k) t[k] = x[i * E + k];
      if (n == E) store16(at(p, c), pack(t));
      else store_part(at(p, c), pack(t), n);
    });
  }
  // A parameter vector; NULL: `other`, also past the width.
  __device__ void vec(const float* p, float other, float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = other;
    if (!p) return;
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int i = 0; i < VW; i += 4) {
        const uint32_t c = col(j, i);
        if (EVEN ? c < D : c + 4 <= D) {
          const u32x4 w = load16(at(p, c));
          float t[4];
          unpack(w, t);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[j * VW + i + k] = t[k];
        } else if (!EVEN) {
#pragma unroll
          for (int k = 0; k < 3; ++k)
            if (c + k < D) x[j * VW + i + k] = *at(p, c + k);
        }
      }
  }
  // Dropout of the thread's elements. EVEN: a chunk is one Philox block, whose words are kept. Else it lies
  // across two, and the row's threads take a block each and hand its bits over through LDS (`mask`,
  // MASK bytes, a buffer that no thread of the row reads any more; one barrier where the row is more
  // than a wave).
  struct Kept {
    U4 w[EVEN ? K : 1];
    uint32_t bits;   // bit j VW + i
    uint32_t d;
    __device__ float pass(int e, float x) const {
      const bool keep = EVEN ? drop_half(w[e / VW], e % VW) >= d : (bits >> e & 1) != 0;
      return keep ? x : 0.0f;
    }
  };
  __device__ void kept(const spz_block_norm_args& a, uint32_t d, int64_t row, uint8_t* mask, Kept& q) const {
    const uint64_t e0 = (uint64_t)row * D;
    q.d = d;
    q.bits = 0;
    if constexpr (EVEN) {
#pragma unroll
      for (int j = 0; j < K; ++j) q.w[j] = drop_words((e0 + col(j, 0)) >> 3, a.seed, a.step, a.tensor);
    } else {
      const uint64_t b0 = e0 >> 3, b1 = (e0 + D - 1) >> 3;
      for (uint32_t k = lane; k <= (uint32_t)(b1 - b0); k += TPR) {
        const U4 w = drop_words(b0 + k, a.seed, a.step, a.tensor);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m |= (uint32_t)(drop_half(w, i) >= d) << i;
        mask[k] = (uint8_t)m;
      }
      if (TPR > 64) {
        __syncthreads();
      } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
#pragma unroll
      for (int j = 0; j < K; ++j) {
        const uint32_t c = (uint32_t)(e0 & 7) + (in(j, 0) ? col(j, 0) : 0);
        const uint32_t two = mask[c >> 3] | (uint32_t)mask[(c >> 3) + 1] << 8;
        q.bits |= (two >> (c & 7) & 0xFFu) << (j * VW);
      }
    }
  }
  // Normalised in place; returns the factor 1 / sqrt(var + eps) (1 where the norm is none).
  template <typename SUM> __device__ float norm(int kind, float eps, float inv_d, SUM& sum, float (&x)[N]) const {
    if (kind == SPZ_NORM_NONE) return 1.0f;
    if (kind == SPZ_NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) s += x[i];
      const float mean = sum(s) * inv_d;
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < VW; ++i) x[j * VW + i] = in(j, i) ? x[j * VW + i] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(x[i], x[i], s);
    const float r = __builtin_amdgcn_rsqf(fmaf(sum(s), inv_d, eps));
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= r;
    return r;
  }
  // dn (gradient to the normalised n, times its weight) -> gradient to the norm's input.
  template <typename SUM>
  __device__ void norm_back(int kind, float r, float inv_d, SUM& sum, const float (&n)[N], float (&dn)[N]) const {
    if (kind == SPZ_NORM_NONE) return;
    float s = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s = fmaf(dn[i], n[i], s);
      q += dn[i];
    }
    s = sum(s) * inv_d;
    if (kind == SPZ_NORM_LAYER) {
      q = sum(q) * inv_d;
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < VW; ++i) dn[j * VW + i] -= in(j, i) ? q : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) dn[i] = r * fmaf(-n[i], s, dn[i]);
  }
};

// gate(z) and its slope, of kind SIGMOID or SILU.
template <int KIND> __device__ inline void gate_of(float z, float& g, float& slope) {
  float s, t;
  sigmoid2(z, s, t);
  if (KIND == SPZ_GATE_SIGMOID) {
    g = s;
    slope = s * t;
  } else {
    // z = +-inf: z sigmoid(z) and z (1 - sigmoid(z)) are 0 where the sigmoid is, not inf * 0.
    g = s == 0.0f ? 0.0f : z * s;
    slope = t == 0.0f ? s : fmaf(g, t, s);
  }
}
__device__ inline void gate_value(int kind, float z, float& g, float& slope) {
  if (kind == SPZ_GATE_SIGMOID) {
    gate_of<SPZ_GATE_SIGMOID>(z, g, slope);
  } else if (kind == SPZ_GATE_SILU) {
    gate_of<SPZ_GATE_SILU>(z, g, slope);
  } else {
    g = 1.0f;
    slope = 0.0f;
  }
}
// Of a row's elements: the choice is made once.
template <int N> __device__ inline void gate_row(int kind, const float (&z)[N], float (&g)[N], float (&slope)[N]) {
  if (kind == SPZ_GATE_SIGMOID) {
#pragma unroll
    for (int i = 0; i < N; ++i) gate_of<SPZ_GATE_SIGMOID>(z[i], g[i], slope[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) gate_of<SPZ_GATE_SILU>(z[i], g[i], slope[i]);
  }
}

// The first row of a thread in workgroup b: uniform over its wave where the row fills one.
template <int TPR> __device__ inline int64_t first_row(int64_t b) {
  constexpr int GROUPS = TPR > 64 ? 1 : NORM_THREADS / TPR;
  if constexpr (GROUPS == 1) return b;
  const int sub = threadIdx.x / TPR;
  return b * GROUPS + (TPR == 64 ? __builtin_amdgcn_readfirstlane(sub) : sub);
}

// Workgroups: rows of more than a wave have one to themselves (its barriers are the row's).
template <int TPR> constexpr int norm_threads = TPR > 64 ? TPR : NORM_THREADS;

// The threads' sums over a row, and its place in LDS.
#define NORM_ROW_SUM()                                                                                  \
  __shared__ float buf[2][TPR > 64 ? TPR / 64 : 1];                                                     \
  typename std::conditional<(TPR > 64), WideSum<(TPR > 64 ? TPR : 128)>, RowSum<TPR>>::type sum{};      \
  if constexpr (TPR > 64) sum.buf = buf;                                                                \
  __shared__ uint8_t masks[2][EVEN ? 1 : GROUPS][EVEN ? 1 : M::MASK]

template <typename T, bool EVEN, int TPR, int K>
__global__ __launch_bounds__(norm_threads<TPR>) void norm_forward(NormArgs g) {
  using M = RowMap<T, EVEN, TPR, K>;
  constexpr int N = M::N, GROUPS = norm_threads<TPR> / TPR;
  const spz_block_norm_args& a = g.a;
  const M m{threadIdx.x % TPR, (uint32_t)a.width};
  const int64_t row = first_row<TPR>(g.first + blockIdx.x);
  if (row >= a.rows) return;
  T* xo = a.h ? static_cast<T*>(a.x_out) + row * a.x_out_row : nullptr;
  T* u = a.pre != SPZ_NORM_NONE ? static_cast<T*>(a.u) + row * a.u_row : nullptr;
  float x[N], h[N], z[N], w[N];
  if (a.valid && !a.valid[row]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.0f;
    if (xo) m.store(xo, x);
    if (u) m.store(u, x);
    return;
  }
  const float inv_d = 1.0f / (float)a.width;
  NORM_ROW_SUM();
  m.load(static_cast<const T*>(a.x) + row * a.x_row, x);
  if (a.h) {
    m.load(static_cast<const T*>(a.h) + row * a.h_row, h);
    if (a.gate != SPZ_GATE_NONE) m.load(static_cast<const T*>(a.z) + row * a.z_row, z);
    typename M::Kept kept;
    if (g.drop.on) m.kept(a, g.drop.d, row, masks[0][EVEN ? 0 : threadIdx.x / TPR], kept);
    m.norm(a.post, a.eps, inv_d, sum, h);
    if (a.post != SPZ_NORM_NONE) {
      if (a.w_post) {
        m.vec(a.w_post, 1.0f, w);
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] *= w[i];
      }
      if (a.b_post) {
        m.vec(a.b_post, 0.0f, w);
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] += w[i];
      }
    }
    if (a.gate != SPZ_GATE_NONE) {
      float slope[N];
      gate_row(a.gate, z, w, slope);
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] *= w[i];
    }
    if (g.drop.on) {
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = kept.pass(i, h[i] * g.drop.gain);
    }
    m.vec(a.scale, 1.0f, w);
    // Past the width h is 0: the loads, the normalised values, and b_post as vec() fills it.
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(w[i], h[i], x[i]);
    m.store(xo, x);
  }
  if (!u) return;
  m.norm(a.pre, a.eps, inv_d, sum, x);
  if (a.w_pre) {
    m.vec(a.w_pre, 1.0f, w);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= w[i];
  }
  if (a.b_pre) {
    m.vec(a.b_pre, 0.0f, w);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += w[i];
  }
  m.store(u, x);
}

template <typename T, bool EVEN, int TPR, int K>
__global__ __launch_bounds__(norm_threads<TPR>, 2) void norm_backward(NormArgs g) {
  using M = RowMap<T, EVEN, TPR, K>;
  constexpr int N = M::N, GROUPS = norm_threads<TPR> / TPR;
  const spz_block_norm_args& a = g.a;
  const M m{threadIdx.x % TPR, (uint32_t)a.width};
  const float inv_d = 1.0f / (float)a.width;
  NORM_ROW_SUM();
  int slot = 0;
  const bool gated = a.h && a.gate != SPZ_GATE_NONE, has_du = a.du && a.pre != SPZ_NORM_NONE;
  // More than a chunk a thread (rows above 4096): registers hold the sums, but neither the vectors nor a
  // second row beside them (with both, 600 of them spilled: 461 against 292 us at 4096 x 6000 bf16).
  constexpr bool LEAN = K > 1;
  float acc[NORM_VECTORS][N], kept_w[4][LEAN ? 1 : N];
#pragma unroll
  for (int k = 0; k < NORM_VECTORS; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[k][i] = 0.0f;
  const bool post = a.post != SPZ_NORM_NONE;
  const float* const params[4] = {post ? a.w_post : nullptr, post ? a.b_post : nullptr, a.scale, a.w_pre};
  constexpr int WQ = 0, BQ = 1, SC = 2, WP = 3;
  if constexpr (!LEAN)
#pragma unroll
    for (int k = 0; k < 4; ++k) m.vec(params[k], k == BQ ? 0.0f : 1.0f, kept_w[k]);
  const auto vec = [&](int k, float (&w)[N]) {
    if constexpr (LEAN) m.vec(params[k], k == BQ ? 0.0f : 1.0f, w);
    else
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = kept_w[k][i];
  };

  struct Rows { typename M::Raw x, h, z, d, du; bool on; };
  const auto load = [&](int64_t row, Rows& r) {
    r.on = !a.valid || a.valid[row];
    if (!r.on) return;
    m.load(static_cast<const T*>(a.x) + row * a.x_row, r.x);
    if (a.h) m.load(static_cast<const T*>(a.h) + row * a.h_row, r.h);
    if (gated) m.load(static_cast<const T*>(a.z) + row * a.z_row, r.z);
    if (a.dx_out) m.load(static_cast<const T*>(a.dx_out) + row * a.dx_out_row, r.d);
    if (has_du) m.load(static_cast<const T*>(a.du) + row * a.du_row, r.du);
  };
  const auto take = [&](int64_t row, const Rows& now) {
    float x[N];
    if (!now.on) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = 0.0f;
      if (a.dx) m.store(static_cast<T*>(a.dx) + row * a.dx_row, x);
      if (a.h && a.dh) m.store(static_cast<T*>(a.dh) + row * a.dh_row, x);
      if (gated && a.dz) m.store(static_cast<T*>(a.dz) + row * a.dz_row, x);
      return;
    }
    // Forward: n in h, gate and its slope, x' in x. Past the width all of them are 0 (but the gate).
    float h[N], gt[N], slope[N], rh = 1.0f;
    typename M::Kept kept;
    m.floats(now.x, x);
    if (a.h) {
      if (g.drop.on) {
        m.kept(a, g.drop.d, row, masks[slot][EVEN ? 0 : threadIdx.x / TPR], kept);
        slot ^= 1;
      }
      m.floats(now.h, h);
      rh = m.norm(a.post, a.eps, inv_d, sum, h);
      if (gated) {
        float z[N];
        m.floats(now.z, z);
        gate_row(a.gate, z, gt, slope);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) { gt[i] = 1.0f; slope[i] = 0.0f; }
      }
      float wq[N], bq[N], sc[N];
      vec(WQ, wq);
      vec(BQ, bq);
      vec(SC, sc);
      if (g.drop.on) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(sc[i], kept.pass(i, gt[i] * fmaf(h[i], wq[i], bq[i]) * g.drop.gain), x[i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(sc[i], gt[i] * fmaf(h[i], wq[i], bq[i]), x[i]);
      }
    }
    // Through the pre norm: d becomes the gradient to x'.
    float d[N];
    if (a.dx_out) m.floats(now.d, d);
    else
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = 0.0f;
    if (has_du) {
      float du[N];
      m.floats(now.du, du);
      const float rx = m.norm(a.pre, a.eps, inv_d, sum, x);
      float wp[N];
      vec(WP, wp);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        acc[3][i] = fmaf(du[i], x[i], acc[3][i]);
        acc[4][i] += du[i];
        du[i] *= wp[i];
      }
      m.norm_back(a.pre, rx, inv_d, sum, x, du);
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] += du[i];
    }
    if (a.dx) m.store(static_cast<T*>(a.dx) + row * a.dx_row, d);
    if (!a.h) return;
    if (g.drop.on) {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = kept.pass(i, d[i] * g.drop.gain);
    }
    float wq[N], bq[N], sc[N];
    vec(WQ, wq);
    vec(BQ, bq);
    vec(SC, sc);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = fmaf(h[i], wq[i], bq[i]);
      acc[2][i] = fmaf(d[i], gt[i] * t, acc[2][i]);
      d[i] *= sc[i];          // gradient to gate(z) n
      slope[i] *= d[i] * t;   // to z
      d[i] *= gt[i];          // to n w + b
    }
    if (gated && a.dz) m.store(static_cast<T*>(a.dz) + row * a.dz_row, slope);
    if (post) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        acc[0][i] = fmaf(d[i], h[i], acc[0][i]);
        acc[1][i] += d[i];
        d[i] *= wq[i];
      }
    }
    if (!a.dh) return;
    m.norm_back(a.post, rh, inv_d, sum, h, d);
    m.store(static_cast<T*>(a.dh) + row * a.dh_row, d);
  };
  const int64_t stride = (int64_t)gridDim.x * GROUPS;
  const auto clear = [](Rows& r) {
    for (typename M::Raw* w : {&r.x, &r.h, &r.z, &r.d, &r.du}) w->clear();
  };
  if constexpr (LEAN) {
    Rows r;
    clear(r);
    for (int64_t row = first_row<TPR>(blockIdx.x); row < a.rows; row += stride) {
      load(row, r);
      take(row, r);
    }
  } else {
    // Two rows in turn, so that none is copied: the other one's loads are in flight.
    Rows r0, r1;
    clear(r0);
    clear(r1);
    int64_t row = first_row<TPR>(blockIdx.x);
    if (row < a.rows) load(row, r0);
    while (row < a.rows) {
      if (row + stride < a.rows) load(row + stride, r1);
      take(row, r0);
      row += stride;
      if (row >= a.rows) break;
      if (row + stride < a.rows) load(row + stride, r0);
      take(row, r1);
      row += stride;
    }
  }

  // Column sums of the workgroup's rows, in their order.
  float* part = g.part + (int64_t)blockIdx.x * NORM_VECTORS * a.width;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int k = 0; k < NORM_VECTORS; ++k) {
      if (!g.wants[k]) continue;
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < M::VW; ++i)
          if (m.in(j, i)) part[k * a.width + m.col(j, i)] = acc[k][j * M::VW + i];
    }
  } else {
    __shared__ float sums[GROUPS][TPR * N];
#pragma unroll
    for (int k = 0; k < NORM_VECTORS; ++k) {
      if (!g.wants[k]) continue;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) sums[threadIdx.x / TPR][i * TPR + m.lane] = acc[k][i];
      __syncthreads();
      for (int e = threadIdx.x; e < TPR * N; e += norm_threads<TPR>) {
        const M me{(uint32_t)e % TPR, m.D};
        const uint32_t c = me.col(e / TPR / M::VW, e / TPR % M::VW);
        if (c >= m.D) continue;
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < GROUPS; ++r) s += sums[r][e];
        part[k * a.width + c] = s;
      }
    }
  }
}

// out[k][c] = sum over the workgroups b of part[b][k][c]: 32 threads a column take every 32nd each.
struct SumArgs { float* out[NORM_VECTORS]; };
constexpr int SUM_COLS = 32, SUM_GROUPS = 32;
__global__ __launch_bounds__(SUM_COLS * SUM_GROUPS) void norm_sums(const float* part, SumArgs o, int64_t width, int blocks,
                                                                   int64_t first) {
  __shared__ float s[SUM_GROUPS][SUM_COLS];
  const int c = threadIdx.x % SUM_COLS, gr = threadIdx.x / SUM_COLS;
  const int64_t block = first + blockIdx.x;
  const int k = (int)(block % NORM_VECTORS);
  float* out = o.out[k];
  if (!out) return;
  const int64_t col = block / NORM_VECTORS * SUM_COLS + c;
  float x = 0.0f;
  if (col < width) {
    const float* p = part + k * width + col;
    constexpr int U = 8;
    for (int b = gr; b < blocks; b += U * SUM_GROUPS) {
      float v[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int q = b + j * SUM_GROUPS;
        v[j] = q < blocks ? p[(int64_t)q * NORM_VECTORS * width] : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < U; ++j) x += v[j];
    }
  }
  s[gr][c] = x;
  __syncthreads();
  if (gr || col >= width) return;
#pragma unroll
  for (int i = 1; i < SUM_GROUPS; ++i) x += s[i][c];
  out[col] = x;
}

// ----------------------------------------------------------------------------- rows of any width
// One workgroup a row, which reads it once for every statistic (from L2 after the first time): forward
// 291 us at 1024 x 20000 bf16, backward 1363 at 1024 x 16384. The simple form, for rows that no
// network here has.
constexpr int WIDE_THREADS = 1024;
template <typename T, bool BACK> __global__ __launch_bounds__(WIDE_THREADS) void norm_wide(NormArgs g) {
  const spz_block_norm_args& a = g.a;
  __shared__ float buf[2][WIDE_THREADS / 64];
  WideSum<WIDE_THREADS> sum{buf};
  const int64_t D = a.width;
  const float inv_d = 1.0f / (float)D;
  float* part = BACK ? g.part + (int64_t)blockIdx.x * NORM_VECTORS * D : nullptr;
  if (BACK)
    for (int64_t c = threadIdx.x; c < D; c += WIDE_THREADS)
      for (int k = 0; k < NORM_VECTORS; ++k) part[k * D + c] = 0.0f;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const bool on = !a.valid || a.valid[row];
    const bool has_du = BACK && a.du && a.pre != SPZ_NORM_NONE;
    const auto at = [&](const void* p, int64_t stride, int64_t c) { return to_f<T>(static_cast<const T*>(p)[row * stride + c]); };
    const auto put = [&](void* p, int64_t stride, int64_t c, float v) {
      if (p) static_cast<T*>(p)[row * stride + c] = from_f<T>(v);
    };
    const auto w = [&](const float* p, float other, int64_t c) { return p ? p[c] : other; };
    if (!on) {
      for (int64_t c = threadIdx.x; c < D; c += WIDE_THREADS) {
        if (BACK) {
          put(a.dx, a.dx_row, c, 0.0f);
          if (a.h) put(a.dh, a.dh_row, c, 0.0f);
          if (a.h && a.gate != SPZ_GATE_NONE) put(a.dz, a.dz_row, c, 0.0f);
        } else {
          if (a.h) put(a.x_out, a.x_out_row, c, 0.0f);
          if (a.pre != SPZ_NORM_NONE) put(a.u, a.u_row, c, 0.0f);
        }
      }
      continue;
    }
    float mh = 0.0f, rh = 1.0f, mx = 0.0f, rx = 1.0f;
    struct El { float n, t, gt, slope, f, x; };
    const auto value = [&](int64_t c) {   // the element's forward values up to x'
      El e{0.0f, 0.0f, 1.0f, 0.0f, 1.0f, at(a.x, a.x_row, c)};
      if (!a.h) return e;
      e.n = (at(a.h, a.h_row, c) - mh) * rh;
      e.t = a.post != SPZ_NORM_NONE ? fmaf(e.n, w(a.w_post, 1.0f, c), w(a.b_post, 0.0f, c)) : e.n;
      if (a.gate != SPZ_GATE_NONE) gate_value(a.gate, at(a.z, a.z_row, c), e.gt, e.slope);
      if (g.drop.on) {
        const uint64_t i = (uint64_t)row * D + c;
        const U4 v = drop_words(i >> 3, a.seed, a.step, a.tensor);
        const uint32_t q = (i & 4) ? ((i & 2) ? v.w : v.z) : ((i & 2) ? v.y : v.x);
        e.f = ((i & 1) ? q >> 16 : q & 0xFFFFu) >= g.drop.d ? g.drop.gain : 0.0f;
      }
      if (e.f != 0.0f) e.x = fmaf(w(a.scale, 1.0f, c), e.gt * e.t * e.f, e.x);
      return e;
    };
    const auto total = [&](auto&& term) {
      float s = 0.0f;
      for (int64_t c = threadIdx.x; c < D; c += WIDE_THREADS) s += term(c);
      return sum(s);
    };
    if (a.h && a.post != SPZ_NORM_NONE) {
      if (a.post == SPZ_NORM_LAYER) mh = total([&](int64_t c) { return at(a.h, a.h_row, c); }) * inv_d;
      rh = 1.0f / sqrtf(total([&](int64_t c) { const float v = at(a.h, a.h_row, c) - mh; return v * v; }) * inv_d + a.eps);
    }
    if (BACK ? has_du : a.pre != SPZ_NORM_NONE) {
      if (a.pre == SPZ_NORM_LAYER) mx = total([&](int64_t c) { return value(c).x; }) * inv_d;
      rx = 1.0f / sqrtf(total([&](int64_t c) { const float v = value(c).x - mx; return v * v; }) * inv_d + a.eps);
    }
    if (!BACK) {
      for (int64_t c = threadIdx.x; c < D; c += WIDE_THREADS) {
        const El e = value(c);
        if (a.h) put(a.x_out, a.x_out_row, c, e.x);
        if (a.pre != SPZ_NORM_NONE) put(a.u, a.u_row, c, fmaf((e.x - mx) * rx, w(a.w_pre, 1.0f, c), w(a.b_pre, 0.0f, c)));
      }
      continue;
    }
    float s1 = 0.0f, s2 = 0.0f, q1 = 0.0f, q2 = 0.0f;
    if (has_du) {
      s1 = total([&](int64_t c) { return at(a.du, a.du_row, c) * w(a.w_pre, 1.0f, c) * ((value(c).x - mx) * rx); }) * inv_d;
      if (a.pre == SPZ_NORM_LAYER) s2 = total([&](int64_t c) { return at(a.du, a.du_row, c) * w(a.w_pre, 1.0f, c); }) * inv_d;
    }
    const auto grad = [&](int64_t c, const El& e) {   // to x'
      float d = a.dx_out ? at(a.dx_out, a.dx_out_row, c) : 0.0f;
      if (has_du) d += rx * (at(a.du, a.du_row, c) * w(a.w_pre, 1.0f, c) - fmaf((e.x - mx) * rx, s1, s2));
      return d;
    };
    const auto grad_t = [&](int64_t c, const El& e) {   // to n w_post + b_post
      return e.f == 0.0f ? 0.0f : grad(c, e) * e.f * w(a.scale, 1.0f, c) * e.gt;
    };
    if (a.h && a.dh && a.post != SPZ_NORM_NONE) {
      q1 = total([&](int64_t c) { const El e = value(c); return grad_t(c, e) * w(a.w_post, 1.0f, c) * e.n; }) * inv_d;
      if (a.post == SPZ_NORM_LAYER)
        q2 = total([&](int64_t c) { const El e = value(c); return grad_t(c, e) * w(a.w_post, 1.0f, c); }) * inv_d;
    }
    for (int64_t c = threadIdx.x; c < D; c += WIDE_THREADS) {
      const El e = value(c);
      const float d = grad(c, e), dt = grad_t(c, e);
      put(a.dx, a.dx_row, c, d);
      if (has_du) {
        const float u = at(a.du, a.du_row, c);
        part[3 * D + c] += u * ((e.x - mx) * rx);
        part[4 * D + c] += u;
      }
      if (!a.h) continue;
      const float gd = e.f == 0.0f ? 0.0f : d * e.f;
      if (a.post != SPZ_NORM_NONE) {
        part[0 * D + c] += dt * e.n;
        part[1 * D + c] += dt;
      }
      part[2 * D + c] += gd * (e.gt * e.t);
      if (a.gate != SPZ_GATE_NONE) put(a.dz, a.dz_row, c, gd * w(a.scale, 1.0f, c) * e.t * e.slope);
      if (a.dh)
        put(a.dh, a.dh_row, c, a.post != SPZ_NORM_NONE ? rh * (dt * w(a.w_post, 1.0f, c) - fmaf(e.n, q1, q2)) : dt);
    }
  }
}

// ----------------------------------------------------------------------------- dropout
// Eight elements a thread: one Philox block. FLAT: rows follow each other without a gap, so that they
// are one row of eights with a ragged end. 88 us at 131072 x 1024 bf16: 6.1 TB/s, HBM's rate. Else each element by itself:
// 71 us at 131072 rows of 256 out of 768 bf16 (1.9 TB/s; rows without gaps 22).
template <typename T, bool FLAT>
__global__ __launch_bounds__(256) void dropout(const T* x, int64_t x_row, T* y, int64_t y_row, int64_t width, int64_t n,
                                               Drop d, uint64_t seed, uint32_t step, uint32_t tensor, int64_t first) {
  constexpr int VW = OP_VEC<T>;
  const int64_t blk = (first + blockIdx.x) * 256 + threadIdx.x, i0 = blk * 8;
  if (i0 >= n) return;
  if (FLAT && i0 + 8 <= n) {
    float v[8 / VW][VW];
#pragma unroll
    for (int j = 0; j < 8 / VW; ++j) unpack(load16(x + i0 + j * VW), v[j]);
    const U4 w = drop_words((uint64_t)blk, seed, step, tensor);
#pragma unroll
    for (int j = 0; j < 8 / VW; ++j) {
#pragma unroll
      for (int i = 0; i < VW; ++i) v[j][i] = drop_half(w, j * VW + i) >= d.d ? v[j][i] * d.gain : 0.0f;
      store16(y + i0 + j * VW, pack(v[j]));
    }
    return;
  }
  const U4 w = drop_words((uint64_t)blk, seed, step, tensor);
  int64_t r = i0 / width, c = i0 - r * width;
  float v[8];
  int64_t to[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    to[i] = -1;
    if (i0 + i < n) {
      v[i] = drop_half(w, i) >= d.d ? to_f<T>(x[r * x_row + c]) * d.gain : 0.0f;
      to[i] = r * y_row + c;
    }
    if (++c == width) { c = 0; ++r; }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (to[i] >= 0) y[to[i]] = from_f<T>(v[i]);
}

// ----------------------------------------------------------------------------- launches
// How a row is held: TPR threads with K chunks each (0: norm_wide). Forward up to four chunks,
// so that rows of up to 2048 stay within a wave, without barriers; backward one (two above 4096: 256 registers
// do not hold more).
struct NormWay { int tpr, k; };
NormWay norm_way(int64_t width, bool back) {
  const int64_t c = op_div_up(width, NORM_CHUNK);
  if (c <= 16) return {16, 1};
  if (c <= 32) return {32, 1};
  if (c <= 64) return {64, 1};
  if (back) return c <= 128 ? NormWay{128, 1} : c <= 256 ? NormWay{256, 1} : c <= 512 ? NormWay{512, 1} : c <= 1024 ? NormWay{512, 2} : NormWay{0, 0};
  return c <= 128 ? NormWay{64, 2} : c <= 256 ? NormWay{64, 4} : c <= 512 ? NormWay{256, 2} : c <= 1024 ? NormWay{256, 4} : c <= 2048 ? NormWay{1024, 2} : NormWay{0, 0};
}
int64_t norm_blocks(const spz_block_norm_args& a) {   // of the backward pass
  const int tpr = norm_way(a.width, true).tpr;
  const int64_t threads = tpr == 0 ? WIDE_THREADS : tpr > 64 ? tpr : NORM_THREADS;
  const int64_t n = op_div_up(a.rows, tpr == 0 || tpr > 64 ? 1 : threads / tpr), most = NORM_MAX_WAVES * 64 / threads;
  return n < most ? n : most;
}

template <typename T, bool EVEN> void norm_dispatch(const NormArgs& g, bool back, int64_t blocks, hipStream_t s) {
  const NormWay way = norm_way(g.a.width, back);
  const auto go = [&](auto tpr, auto k) {
    constexpr int TPR = decltype(tpr)::value, K = decltype(k)::value;
    if constexpr (K == 1 || TPR == 512) {
      if (back) {
        norm_backward<T, EVEN, TPR, K><<<dim3((unsigned)blocks), norm_threads<TPR>, 0, s>>>(g);
        return;
      }
    }
    if constexpr ((K > 1 && TPR != 512) || TPR <= 64)
      op_dispatch(op_div_up(g.a.rows, norm_threads<TPR> / TPR), norm_threads<TPR>, [&](int64_t first, dim3 grid) {
        NormArgs part = g;
        part.first = first;
        norm_forward<T, EVEN, TPR, K><<<grid, norm_threads<TPR>, 0, s>>>(part);
      });
  };
  using std::integral_constant;
  const auto is = [&](int tpr, int k) { return way.tpr == tpr && way.k == k; };
  const integral_constant<int, 1> k1{};
  const integral_constant<int, 2> k2{};
  const integral_constant<int, 4> k4{};
  if (is(16, 1)) go(integral_constant<int, 16>{}, k1);
  else if (is(32, 1)) go(integral_constant<int, 32>{}, k1);
  else if (is(64, 1)) go(integral_constant<int, 64>{}, k1);
  else if (is(64, 2)) go(integral_constant<int, 64>{}, k2);
  else if (is(64, 4)) go(integral_constant<int, 64>{}, k4);
  else if (is(128, 1)) go(integral_constant<int, 128>{}, k1);
  else if (is(256, 1)) go(integral_constant<int, 256>{}, k1);
  else if (is(256, 2)) go(integral_constant<int, 256>{}, k2);
  else if (is(256, 4)) go(integral_constant<int, 256>{}, k4);
  else if (is(512, 1)) go(integral_constant<int, 512>{}, k1);
  else if (is(512, 2)) go(integral_constant<int, 512>{}, k2);
  else if (is(1024, 2)) go(integral_constant<int, 1024>{}, k2);
  else if (back) norm_wide<T, true><<<dim3((unsigned)blocks), WIDE_THREADS, 0, s>>>(g);
  else norm_wide<T, false><<<dim3((unsigned)(g.a.rows < 65536 ? g.a.rows : 65536)), WIDE_THREADS, 0, s>>>(g);
}

const char* norm_check(const spz_block_norm_args* p) {
  if (!p) return "NULL arguments";
  const spz_block_norm_args& a = *p;
  if (!op_prec_ok(a.prec)) return "unknown precision";
  if (!op_extent_ok(a.rows) || !op_extent_ok(a.width)) return "extent out of range";
  if (a.width && a.rows > ((int64_t)1 << 44) / a.width) return "extents out of range";
  if (a.post < SPZ_NORM_NONE || a.post > SPZ_NORM_LAYER || a.pre < SPZ_NORM_NONE || a.pre > SPZ_NORM_LAYER)
    return "unknown norm";
  if (a.gate < SPZ_GATE_NONE || a.gate > SPZ_GATE_SILU) return "unknown gate";
  if (!(a.eps >= 1.2e-38f) || !(a.eps < 3.0e38f)) return "eps out of range";
  if (!(a.drop_p >= 0.0f && a.drop_p <= 1.0f)) return "drop_p outside [0, 1]";
  return nullptr;
}

const char* norm_check_arrays(const spz_block_norm_args& a, bool back) {
  const bool some = a.rows > 0 && a.width > 0, z = a.h && a.gate != SPZ_GATE_NONE, pre = a.pre != SPZ_NORM_NONE;
  const size_t e = op_size(a.prec);
  if (some && !a.x) return "NULL x";
  if (some && !a.h && !pre) return "neither a block nor a pre norm";
  if (some && z && !a.z) return "NULL z";
  if (some && !back && ((a.h && !a.x_out) || (pre && !a.u))) return "NULL output";
  for (const void* p : {a.x, a.h, a.z, a.dx_out, a.du, (const void*)a.x_out, (const void*)a.u, (const void*)a.dx,
                        (const void*)a.dh, (const void*)a.dz})
    if (!op_aligned(p, e)) return "array not aligned to its type";
  for (const float* p : {a.w_post, a.b_post, a.scale, a.w_pre, a.b_pre, (const float*)a.dw_post, (const float*)a.db_post,
                         (const float*)a.dscale, (const float*)a.dw_pre, (const float*)a.db_pre})
    if (!op_aligned(p, 4)) return "vector not aligned to 4 bytes";
  if (!op_in_stride_ok(a.x_row) || (a.h && !op_in_stride_ok(a.h_row)) || (z && !op_in_stride_ok(a.z_row)))
    return "input stride out of range";
  if (!back) {
    if (a.h && !op_out_stride_ok(a.rows, a.width, a.x_out_row)) return "rows of x_out overlap";
    if (pre && !op_out_stride_ok(a.rows, a.width, a.u_row)) return "rows of u overlap";
    return nullptr;
  }
  if ((a.dx_out && !op_in_stride_ok(a.dx_out_row)) || (a.du && pre && !op_in_stride_ok(a.du_row))) return "input stride out of range";
  if (a.dx && !op_out_stride_ok(a.rows, a.width, a.dx_row)) return "rows of dx overlap";
  if (a.h && a.dh && !op_out_stride_ok(a.rows, a.width, a.dh_row)) return "rows of dh overlap";
  if (z && a.dz && !op_out_stride_ok(a.rows, a.width, a.dz_row)) return "rows of dz overlap";
  return nullptr;
}

int norm_run(const char* call, const spz_block_norm_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = norm_check(args);
  if (!bad) bad = norm_check_arrays(*args, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  NormArgs g{};
  g.a = *args;
  const spz_block_norm_args& a = g.a;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t blocks = back ? norm_blocks(a) : 0;
  if (back) {
    const int64_t need = spz_block_norm_workspace(args);
    if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
    if (need > 0 && !op_aligned(ws, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
    g.part = static_cast<float*>(ws);
  }
  if (a.width == 0) return SPZ_OK;
  g.drop.d = drop_threshold(a.drop_p);
  g.drop.gain = drop_gain(g.drop.d);
  g.drop.on = g.drop.d > 0;
  const bool even = a.width % NORM_CHUNK == 0;
  const SumArgs o{{a.dw_post, a.db_post, a.dscale, a.dw_pre, a.db_pre}};
  for (int k = 0; k < NORM_VECTORS; ++k) g.wants[k] = o.out[k] != nullptr;
  if (a.rows > 0) {
    if (a.prec == SPZ_PREC_BF16) {
      if (even) norm_dispatch<bf16_t, true>(g, back, blocks, s);
      else norm_dispatch<bf16_t, false>(g, back, blocks, s);
    } else {
      if (even) norm_dispatch<float, true>(g, back, blocks, s);
      else norm_dispatch<float, false>(g, back, blocks, s);
    }
  }
  if (back) {
    if (a.dw_post || a.db_post || a.dscale || a.dw_pre || a.db_pre)
      op_dispatch(op_div_up(a.width, SUM_COLS) * NORM_VECTORS, SUM_COLS * SUM_GROUPS, [&](int64_t first, dim3 grid) {
        norm_sums<<<grid, SUM_COLS * SUM_GROUPS, 0, s>>>(g.part, o, a.width, (int)blocks, first);
      });
  }
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_block_norm_workspace(const spz_block_norm_args* args) {
  const char* bad = norm_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_block_norm_workspace", bad);
  return norm_blocks(*args) * NORM_VECTORS * args->width * 4;
}

int spz_block_norm_forward(const spz_block_norm_args* args, void* hip_stream) {
  return norm_run("spz_block_norm_forward", args, false, nullptr, 0, hip_stream);
}

int spz_block_norm_backward(const spz_block_norm_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return norm_run("spz_block_norm_backward", args, true, workspace, workspace_bytes, hip_stream);
}

int spz_dropout(int32_t prec, int64_t rows, int64_t width, const void* x, int64_t x_row, void* y, int64_t y_row,
                float p, uint64_t seed, uint32_t step, uint32_t tensor, void* hip_stream) {
  const char* call = "spz_dropout";
  if (!op_prec_ok(prec)) return op_error(SPZ_EINVAL, call, "unknown precision");
  if (!op_extent_ok(rows) || !op_extent_ok(width)) return op_error(SPZ_EINVAL, call, "extent out of range");
  if (width && rows > ((int64_t)1 << 41) / width) return op_error(SPZ_EINVAL, call, "extents out of range");
  if (!(p >= 0.0f && p <= 1.0f)) return op_error(SPZ_EINVAL, call, "p outside [0, 1]");
  const int64_t n = rows * width;
  if (n > 0 && (!x || !y)) return op_error(SPZ_EINVAL, call, "NULL array");
  const int e = op_size(prec);
  if (!op_aligned(x, e) || !op_aligned(y, e)) return op_error(SPZ_EINVAL, call, "array not aligned to its type");
  if (!op_in_stride_ok(x_row) || !op_out_stride_ok(rows, width, y_row))
    return op_error(SPZ_EINVAL, call, "stride out of range");
  if (n == 0) return SPZ_OK;
  const Drop d{drop_threshold(p), drop_gain(drop_threshold(p)), true};
  const bool flat = rows == 1 || (x_row == width && y_row == width);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const auto go = [&](auto kernel, auto tag) {
    using T = decltype(tag);
    op_dispatch(op_div_up(op_div_up(n, 8), 256), 256, [&](int64_t first, dim3 grid) {
      kernel<<<grid, 256, 0, s>>>(static_cast<const T*>(x), x_row, static_cast<T*>(y), y_row, width, n, d, seed, step, tensor, first);
    });
  };
  if (prec == SPZ_PREC_BF16) {
    if (flat) go(dropout<bf16_t, true>, bf16_t{});
    else go(dropout<bf16_t, false>, bf16_t{});
  } else {
    if (flat) go(dropout<float, true>, float{});
    else go(dropout<float, false>, float{});
  }
  return op_launched(call);
}

}  // extern "C"
