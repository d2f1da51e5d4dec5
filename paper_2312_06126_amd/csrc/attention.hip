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
constexpr int64_t LIN_MAX_HEADS = 65536;

struct LinRole {
  const void *a, *b, *c; void* out;          // [batch, steps, heads, ka], ka, nc, nc
  int64_t a_batch, a_step, a_head, b_batch, b_step, b_head, c_batch, c_step, c_head, out_batch, out_step, out_head;
  const float* init; float* last;            // [batch, heads, ka x nc] at row_stride, col_stride, or NULL
  int64_t row_stride, col_stride;
  int ka, nc;
  bool back;
  float in, out_scale;
};
// x / d for x < 2^31 by a multiplication: 2^(31 + l) / d rounded up, l = ceil(log2 d).
struct Divisor { uint32_t mul; int shift; };
__device__ inline uint32_t divided(uint32_t x, const Divisor& d) { return (uint32_t)(((uint64_t)x * d.mul) >> d.shift); }
Divisor divisor(uint32_t d) {
  int l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  return {(uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), 31 + l};
}

struct LinArgs {
  LinRole role[3];
  int roles, units, slices[3];               // units: workgroups of a piece of a head, slices: of it for a role
  uint32_t groups;                           // of a launch: pieces of heads, or (step by step) sequences
  Divisor by_units, by_pieces, by_heads;
  bool far;                                  // 32 bits do not hold 16 steps of an output
  int64_t batch, steps, heads, first;        // first: sequence that the launch starts with
  int64_t pieces, len;                       // of time, len steps each
  const float* inits[3];                     // states in front of the pieces [batch, heads, pieces, ..], or NULL
  float *adds[2], *keeps[2];                 // what the pieces add to the states of the first two roles, and the factor that
                                             // they keep of them (-1: an episode starts in the piece)
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
// row, row + 16, .. of four columns. vec[role]: a thread's four columns are one access of the state's arrays. Bound by the
// states' bytes: 4096 x 8 heads of 64 x 64, one step, 199 us, 5.5 TB/s (with a wait behind each operand's load 312).
constexpr int STEP_THREADS = 256, STEP_COLS = 64;
struct StepArgs { Divisor by_slices[3], by_heads; bool vec[3]; };
template <typename T, int KR> __global__ __launch_bounds__(STEP_THREADS) void lin_steps(LinArgs g, StepArgs f) {
  const LinRole& r = g.role[blockIdx.y];
  const int slices = (r.nc + STEP_COLS - 1) / STEP_COLS;
  const uint32_t at = blockIdx.x, seq = divided(at, f.by_slices[blockIdx.y]), bq = divided(seq, f.by_heads);
  if (bq >= g.groups) return;
  const int sl = (int)(at - seq * (uint32_t)slices);
  const int64_t h = seq - bq * (uint32_t)g.heads, b = g.first + bq;
  const int c0 = sl * STEP_COLS + 4 * (threadIdx.x & 15), row0 = threadIdx.x >> 4, left = r.nc - c0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool vec = f.vec[blockIdx.y];
  __shared__ float part[2][4][STEP_COLS];
  f32x4 S[KR];
  const int rs = (int)r.row_stride, cs = (int)r.col_stride, ka = r.ka;
  const int64_t st = (b * g.heads + h) * ka * r.nc;
  const float* init = r.init ? r.init + st : nullptr;
  const int64_t n = lin_length(g, b);
  const T* pa = r.a ? static_cast<const T*>(r.a) + b * r.a_batch + h * r.a_head : nullptr;
  const T* pb = r.b ? static_cast<const T*>(r.b) + b * r.b_batch + h * r.b_head : nullptr;
  const T* pc = r.c ? static_cast<const T*>(r.c) + b * r.c_batch + h * r.c_head : nullptr;
  T* po = static_cast<T*>(r.out) + b * r.out_batch + h * r.out_head;
  // The operands of a step, read before the step in front of it is worked on. Rows and columns that do not exist read the
  // last one, so that no load waits behind a branch.
  T xa[KR] = {}, xb[KR] = {}, xc[4] = {};
  bool cut = false;
  const auto fetch = [&](int64_t p) {
    const int64_t t = r.back ? n - 1 - p : p;
    const int64_t flag = r.back ? t + 1 : t;   // the step whose start cuts the state off
    if (pa) {
#pragma unroll
      for (int i = 0; i < KR; ++i) xa[i] = pa[t * r.a_step + (row0 + 16 * i < ka ? row0 + 16 * i : ka - 1)];
    }
    if (pb) {
#pragma unroll
      for (int i = 0; i < KR; ++i) xb[i] = pb[t * r.b_step + (row0 + 16 * i < ka ? row0 + 16 * i : ka - 1)];
    }
    if (pc) {
#pragma unroll
      for (int j = 0; j < 4; ++j) xc[j] = pc[t * r.c_step + (j < left ? c0 + j : r.nc - 1)];
    }
    cut = g.reset && flag < n && g.reset[b * g.reset_batch + flag * g.reset_step] != 0;
  };
  if (n > 0 && ka > 0) fetch(0);
#pragma unroll
  for (int i = 0; i < KR; ++i) {
    const int row = row0 + 16 * i;
    S[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (init && row < ka && left > 0) {
      if (vec) {
        S[i] = *reinterpret_cast<const f32x4*>(init + row * rs + c0);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left) S[i][j] = init[row * rs + (c0 + j) * cs];
      }
    }
  }
  const float d = lin_decay(g.rate ? g.rate[h] : 0.0f, 1);
  for (int64_t p = 0; p < n; ++p) {
    const int64_t t = r.back ? n - 1 - p : p;
    const float keep = r.back && p == 0 ? 1.0f : d;
    const bool cuts = cut;
    float x[KR], y[KR], c[4], o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < KR; ++i) {
      x[i] = row0 + 16 * i < ka ? to_f<T>(xa[i]) : 0.0f;
      y[i] = row0 + 16 * i < ka ? r.in * to_f<T>(xb[i]) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = j < left ? to_f<T>(xc[j]) : 0.0f;
    if (p + 1 < n && ka > 0) fetch(p + 1);
#pragma unroll
    for (int i = 0; i < KR; ++i)
      if (row0 + 16 * i < ka) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          S[i][j] = fmaf(y[i], c[j], cuts ? 0.0f : keep * S[i][j]);
          o[j] = fmaf(x[i], S[i][j], o[j]);
        }
      }
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = add32(add16(o[j]));
    if (lane < 16) *reinterpret_cast<f32x4*>(&part[p & 1][wave][4 * lane]) = f32x4{o[0], o[1], o[2], o[3]};
    __syncthreads();
    const int col = sl * STEP_COLS + threadIdx.x;
    if (threadIdx.x < STEP_COLS && col < r.nc) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) s += part[p & 1][k][threadIdx.x];
      po[t * r.out_step + col] = from_f<T>(r.out_scale * s);
    }
  }
  for (int64_t t = n; t < g.steps; ++t)
    if (threadIdx.x < STEP_COLS && sl * STEP_COLS + (int)threadIdx.x < r.nc) po[t * r.out_step + sl * STEP_COLS + threadIdx.x] = from_f<T>(0.0f);
  if (!r.last) return;
  const bool gone = r.back && n > 0 && g.reset && g.reset[b * g.reset_batch] != 0;
  const float keep = r.back && n > 0 ? d : 1.0f;
  float* last = r.last + st;
#pragma unroll
  for (int i = 0; i < KR; ++i) {
    const int row = row0 + 16 * i;
    if (row >= ka || left <= 0) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) S[i][j] = gone ? 0.0f : keep * S[i][j];
    if (vec) {
      *reinterpret_cast<f32x4*>(last + row * rs + c0) = S[i];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < left) last[row * rs + (c0 + j) * cs] = S[i][j];
    }
  }
}

// ----------------------------------------------------------------------------- chunks of steps
// CL steps at a time on the matrix cores. Within a chunk, with s <= t steps of one episode, e(n) = exp(-rate n) and
// n the chunk's steps:
//     o_t = out (sum_s e(t - s) in (a_t b_s) c_s + e(t + 1) a_t R),   R' = e(n) R + sum_s e(n - 1 - s) in b_s^T c_s.
// A workgroup of four waves holds the state of 64 columns in the matrix instructions' accumulators, a wave 16 of them.
// The scores a_t b_s are shared through LDS; everything else is a wave's own. All products are taken so that a lane
// ends with four consecutive elements of what it stores (o as its transpose), and the accumulators of the state are
// operands of the next product as they stand: the order of the contraction is the same for both operands.
// bfloat16 operands: the scores, the state and the weighted c enter a product as three bfloat16 numbers each, which hold all
// 24 bits, so that a state is float32 in a product too. (Scores and states as two, with 16 bits: 1 x 65536 x 8 x 64 x 128 training 689 us
// and not 729, 2048 x 50 x 4 x 64 x 64 284 and not 291; their errors, 2^-17 of a term, show where terms cancel.)
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int CHUNK_THREADS = 256, CHUNK_COLS = 64;

template <typename T> struct Mat;
template <> struct Mat<bf16_t> {
  static constexpr int KB = 32, PAD = 8;               // contraction of one instruction; LDS elements behind a row
  static constexpr int PARTS = 3;                      // numbers that a float32 one enters a product as
  typedef bf16x8 frag;
  static constexpr int N = 8;                          // elements of a lane's fragment
  static __device__ inline void mma(f32x4& acc, const frag& a, const frag& b) { acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
  // Row row0 + lane % 16, columns k0 + 8 (lane / 16) ..
  static __device__ inline frag row(const bf16_t* p, int pitch, int row0, int k0, int i, int g) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + (row0 + i) * pitch + k0 + 8 * g));
  }
  // The same row, in the state's order: columns k0 + 4 (lane / 16) .. and the same 16 further.
  static __device__ inline frag row_state(const bf16_t* p, int pitch, int row0, int k0, int i, int g) {
    const bf16_t* q = p + (row0 + i) * pitch + k0 + 4 * g;
    const u32x2 lo = *reinterpret_cast<const u32x2*>(q), hi = *reinterpret_cast<const u32x2*>(q + 16);
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  }
  // Column col0 + lane % 16, rows k0 + 8 (lane / 16) ..: 16 lanes read four rows of 16 elements, each lane four of one
  // row, and the instruction hands lane i column i.
  static __device__ inline frag col(const bf16_t* p, int pitch, int k0, int col0, int i, int g) {
    const bf16_t* q = p + (k0 + 8 * g + (i >> 2)) * pitch + col0 + 4 * (i & 3);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(q));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(q + 4 * pitch));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ inline float at(const frag& f, int j) { return (float)f[j]; }
  // x as fragments whose sum it is (8 bits more with each).
  static __device__ inline void split(const float (&x)[8], frag (&f)[PARTS]) {
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j] = pack_bf16x2(r[2 * j], r[2 * j + 1]);
        r[2 * j] -= __builtin_bit_cast(float, w[j] << 16);
        r[2 * j + 1] -= __builtin_bit_cast(float, w[j] & 0xFFFF0000u);
      }
      f[k] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
    }
  }
  // Scores of row lane % 16, columns 4 (lane / 16) .. of tile `si`, to each of the parts' arrays of its block.
  static __device__ inline void put(bf16_t* block, int part_size, int si, int i, int q, const f32x4& x) {
    bf16_t* p = block + ((2 * (si & 1) + (q >> 1)) * 16 + i) * N + 4 * (q & 1);
    float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const u32x2 w = {pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3])};
      *reinterpret_cast<u32x2*>(p + k * part_size) = w;
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] -= __builtin_bit_cast(float, j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
  }
  // Largest magnitudes of two elements a word, as their bits.
  static __device__ inline uint32_t most(uint32_t m, uint32_t w) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
  }
  static __device__ inline bool finite(uint32_t m) { return (m & 0xFFFFu) < 0x7F80u && (m >> 16) < 0x7F80u; }
};
template <> struct Mat<float> {
  static constexpr int KB = 16, PAD = 4;
  static constexpr int PARTS = 1;
  typedef f32x4 frag;
  static constexpr int N = 4;
  static __device__ inline void mma(f32x4& acc, const frag& a, const frag& b) {   // four instructions of four elements
#pragma unroll
    for (int r = 0; r < 4; ++r) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], acc, 0, 0, 0);
  }
  static __device__ inline frag row(const float* p, int pitch, int row0, int k0, int i, int g) {
    return *reinterpret_cast<const f32x4*>(p + (row0 + i) * pitch + k0 + 4 * g);
  }
  static __device__ inline frag row_state(const float* p, int pitch, int row0, int k0, int i, int g) { return row(p, pitch, row0, k0, i, g); }
  static __device__ inline frag col(const float* p, int pitch, int k0, int col0, int i, int g) {
    const float* q = p + (k0 + 4 * g) * pitch + col0 + i;
    return f32x4{q[0], q[pitch], q[2 * pitch], q[3 * pitch]};
  }
  static __device__ inline float at(const frag& f, int j) { return f[j]; }
  static __device__ inline void split(const float (&x)[4], frag (&f)[PARTS]) { f[0] = f32x4{x[0], x[1], x[2], x[3]}; }
  static __device__ inline void put(float* block, int, int, int i, int q, const f32x4& x) { *reinterpret_cast<f32x4*>(block + (q * 16 + i) * N) = x; }
  static __device__ inline uint32_t most(uint32_t m, uint32_t w) {
    w &= 0x7FFFFFFFu;
    return w > m ? w : m;
  }
  static __device__ inline bool finite(uint32_t m) { return m < 0x7F800000u; }
};

// The scores in LDS: blocks of 16 rows and one instruction's contraction of columns, those that have an element on or below the
// diagonal, row by row. Within a block a lane's fragment follows the one of the lane in front, so no bank is asked twice. (In
// bfloat16 as many bytes with three parts as whole rows, padded, took with two: 18 KB at 64 places.)
template <typename T> __device__ constexpr int score_block(int ti, int kk) {
  constexpr int PER = Mat<T>::KB / 16;                 // tiles of a block
  const int u = ti / PER;
  return PER * u * (u + 1) / 2 + (ti - PER * u) * (u + 1) + kk;
}

// The same number, of which the compiler does not know that it stays from chunk to chunk: else it keeps everything that
// follows from it in registers throughout (1 x 65536 x 8 x 64 x 128 bfloat16 without: forward 281 us and not 205, backward 729 and not 514).
__device__ inline int opaque(int x) {
  asm("" : "+v"(x));
  return x;
}
template <typename I> __device__ inline I opaque_scalar(I x) {
  asm("" : "+s"(x));
  return x;
}

// CL steps of W columns (zeros past `width` and past the sequence) on their way from memory to LDS. A thread's vectors
// are of one column group and RI rows apart, so that one 32-bit offset from scalar addresses serves them all.
struct Walk { int n; bool back; };   // place p of a walk is step p, or n - 1 - p
template <typename T, int W, int CL> struct Tile {
  static constexpr int VW = OP_VEC<T>, VR = W / VW, RI = CHUNK_THREADS / VR, N = CL / RI, PITCH = W + Mat<T>::PAD;
  static_assert(CL % RI == 0, "whole vectors a thread");
  u32x4 v[N];
  const char* at;            // of the next chunk's place that comes first in memory, were the chunk whole
  int64_t step;              // in bytes, forward in the walk
  int width, cnt;
  bool some, plain;          // plain: rows of a vector and more, and 32 bits hold a chunk's offsets
  __device__ inline void init(const T* p, int64_t stride, int columns, const Walk& w, int begin) {
    some = p != nullptr;
    step = stride * (int)sizeof(T);
    width = columns;
    plain = width >= VW && step < (int64_t)1 << 26;
    at = reinterpret_cast<const char*>(p) + (w.back ? w.n - begin - CL : begin) * step;
    if (w.back) step = -step;
    cnt = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = u32x4{0, 0, 0, 0};
  }
  // Where a vector is read: the last one of a row that ends inside it is read whole, from further in front.
  __device__ inline int column(int col) const { return col + VW <= width ? col : col < width ? width - VW : 0; }
  // The next chunk, of which `count` > 0 places exist. Rows behind the last one read that one again.
  __device__ inline void load(uint32_t tid, bool back, int count) {
    cnt = count;
    if (!some) return;
    const int64_t step = opaque_scalar(this->step);
    if (plain) {
      const int row = tid / VR;
      const uint32_t c = column(tid % VR * VW) * (int)sizeof(T), up = (uint32_t)(back ? -step : step);
      if (count == CL) {
        const char* from = at;
        const uint32_t off = (back ? CL - 1 - row : row) * up + c;
#pragma unroll
        for (int j = 0; j < N; ++j, from += RI * step) v[j] = load16(reinterpret_cast<const T*>(from + off));
      } else {
        const char* from = back ? at - (CL - count) * step : at;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int r = row + j * RI < count ? row + j * RI : count - 1;
          v[j] = load16(reinterpret_cast<const T*>(from + ((uint32_t)(back ? count - 1 - r : r) * up + c)));
        }
      }
    }
    at += CL * step;
  }
  // Zeros where nothing is, and the ragged end of a row in its place.
  __device__ inline void trim(int row, int col) {
    if (!some) return;
    if (width < W) {
      const int part = col < width && col + VW > width ? col - (width - VW) : 0;   // elements to shift down
      const bool none = col >= width;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (width % VW != 0) {
          constexpr int WORD = 4 / (int)sizeof(T);
          if (WORD == 2 && part & 1) {
            uint32_t u[4] = {v[j][0], v[j][1], v[j][2], v[j][3]};
            v[j] = u32x4{u[0] >> 16 | u[1] << 16, u[1] >> 16 | u[2] << 16, u[2] >> 16 | u[3] << 16, u[3] >> 16};
          }
          if (part / WORD & 1) v[j] = u32x4{v[j][1], v[j][2], v[j][3], 0};
          if (part / WORD & 2) v[j] = u32x4{v[j][2], v[j][3], 0, 0};
        }
        if (none) v[j] = u32x4{0, 0, 0, 0};
      }
    }
    if (cnt < CL) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (row + j * RI >= cnt) v[j] = u32x4{0, 0, 0, 0};
    }
  }
  // To LDS; returns the largest of the magnitudes and m. Rows that are not `plain` come from memory only here.
  __device__ inline uint32_t store(uint32_t tid, T* lds, bool back, uint32_t m) {
    if (some && !plain) {
      const char* from = at - CL * step + (back ? -(CL - 1) * step : 0);   // of the chunk's first place
#pragma unroll 1
      for (int e = tid; e < CL * W; e += CHUNK_THREADS) {
        const int r = e / W, c = e % W;
        T x = from_f<T>(0.0f);
        if (r < cnt && c < width) x = reinterpret_cast<const T*>(from + r * step)[c];
        lds[r * PITCH + c] = x;
        m = Mat<T>::most(m, __builtin_bit_cast(uint32_t, to_f<T>(x)));   // a bfloat16 is the high half of its float32
      }
      return m;
    }
    const int row = tid / VR, col = tid % VR * VW;
    if (width < W || cnt < CL) trim(row, col);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      *reinterpret_cast<u32x4*>(lds + (row + j * RI) * PITCH + col) = v[j];
#pragma unroll
      for (int k = 0; k < 4; ++k) m = Mat<T>::most(m, v[j][k]);
    }
    return m;
  }
};

// log2 of d, kept finite, so that no steps are a factor of 1 at an infinite rate too (NaN stays).
__device__ inline float lin_log2(float rate) {
  const float x = rate * -1.44269504088896341f;
  return x < -1e30f ? -1e30f : x > 1e30f ? 1e30f : x;
}
__device__ inline float lin_power(float log2d, int n) { return __builtin_amdgcn_exp2f(log2d * (float)n); }

// A lane's part of a state at row and column strides rs and cs: rows 16 k + 4 q .. of column c.
template <int TILES>
__device__ inline void state_load(const float* p, f32x4 (&S)[TILES], bool full, bool mine, int ka, int rs, int cs, int c, int q) {
#pragma unroll
  for (int k = 0; k < TILES; ++k) S[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (!p) return;
  const uint32_t at = 4 * q * rs + c * cs;
  if (full && rs == 1) {
#pragma unroll
    for (int k = 0; k < TILES; ++k) __builtin_memcpy(&S[k], p + 16 * k + at, 16);
  } else if (full) {
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[k][e] = (p + (16 * k + e) * rs)[at];
  } else if (mine) {
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * k + 4 * q + e < ka) S[k][e] = (p + (16 * k + e) * rs)[at];
  }
}
template <int TILES>
__device__ inline void state_store(float* p, const f32x4 (&S)[TILES], bool full, bool mine, int ka, int rs, int cs, int c, int q) {
  rs = opaque_scalar(rs);
  const uint32_t at = 4 * q * rs + c * cs;
  if (full && rs == 1) {
#pragma unroll
    for (int k = 0; k < TILES; ++k) __builtin_memcpy(p + 16 * k + at, &S[k], 16);
  } else if (full) {
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) (p + (16 * k + e) * rs)[at] = S[k][e];
  } else if (mine) {
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * k + 4 * q + e < ka) (p + (16 * k + e) * rs)[at] = S[k][e];
  }
}

// KP: rows of the state that are worked on, a multiple of the contraction's (48 instead of 64 for heads of 40 x 39 in float32,
// 64 x 1000 x 5: 157 us against 178, backward 278 against 316).
// Workgroups a compute unit is to hold, which bounds their registers (three and not two in float32 up to 64 rows: 256 x 500 x 4 x
// 64 x 64 backward 453 us against 511).
template <typename T, int KP> constexpr int chunk_waves = KP > 64 ? 1 : sizeof(T) == 4 ? 3 : 4;

// A workgroup: slice of a role, head, sequence, piece of time. STATE: only what the piece adds to the state. ONE: no
// sequence is longer than a chunk. The scores take the place of c, of which each wave has its columns in registers by then.
// The slices of all roles of a piece of a head follow each other on one XCD, whose L2 holds what they share.
// 65536 steps x 8 heads of 64 x 128 bf16 in 64 pieces take 158 us, 2.6 TB/s: 732 vector instructions a wave and chunk at 64 rows, issued in 59%
// of the cycles that a compute unit is busy, and 71 matrix instructions, which run in 23%. Of the vector instructions some 270 split
// scores, states and weighted values into bfloat16 parts; the others are addresses, predicates, trimming, the test for values that
// are not finite, and scalars (117 do not fit) read back from lanes. The rest of the time waits: three barriers and products that
// follow from each other a chunk. Short sequences are bound by the states' bytes: 2048 x 4 heads of 64 x 64, 50 steps, ragged, 96 us.
template <typename T, int KP, int CL, bool STATE, bool ONE> __global__ __launch_bounds__(CHUNK_THREADS, (chunk_waves<T, KP>)) void lin_chunks(LinArgs g) {
  using M = Mat<T>;
  typedef typename M::frag frag;
  constexpr int W = KP <= 32 ? 32 : KP <= 64 ? 64 : KP <= 128 ? 128 : 256;   // columns of a and b in LDS
  constexpr int TILES = KP / 16, ROWS = CL / 16, PA = W + M::PAD, PC = CHUNK_COLS + M::PAD, BLOCK = 16 * M::KB, SCORES = score_block<T>(ROWS, 0) * BLOCK;
  constexpr int LOWER = ROWS * (ROWS + 1) / 2;         // tiles of scores on and below the diagonal
  __shared__ __align__(16) T lds_a[STATE ? 1 : CL * PA];
  __shared__ __align__(16) T lds_b[CL * PA];
  __shared__ __align__(16) T lds_c[STATE || M::PARTS * SCORES < CL * PC ? CL * PC : M::PARTS * SCORES];
  T* const lds_p = lds_c;
  __shared__ int odd[2];
  __shared__ __align__(16) float fade[CL], enter[CL];    // of a place's c in the state behind the chunk, of the state in front in a place's o
  __shared__ int start[CL];                              // first place of a place's episode within the chunk
  const uint32_t block = (uint32_t)blockIdx.x, eighth = block / 8, set = divided(eighth, g.by_units);
  const uint32_t group = set * 8 + block % 8;
  if (group >= g.groups) return;
  int unit = (int)(eighth - set * (uint32_t)g.units), which = 0;
  while (unit >= g.slices[which]) unit -= g.slices[which++];
  const LinRole& r = g.role[which];
  const uint32_t seq = divided(group, g.by_pieces), bq = divided(seq, g.by_heads);
  const int64_t piece = group - seq * (uint32_t)g.pieces, h = seq - bq * (uint32_t)g.heads, b = g.first + bq;
  const int c0 = unit * CHUNK_COLS, cols = r.nc - c0 < CHUNK_COLS ? r.nc - c0 : CHUNK_COLS, ka = r.ka;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i0 = lane & 15, q0 = lane >> 4;
  const int n = (int)lin_length(g, b), begin = (int)(piece * g.len), stop = n - begin > (int)g.len ? begin + (int)g.len : n;
  const bool back = r.back;
  const Walk walk{n, back};
  const float log2d = lin_log2(g.rate ? g.rate[h] : 0.0f);
  const uint8_t* flags = g.reset ? g.reset + b * g.reset_batch : nullptr;
  // Whether place p starts an episode in the order of the walk (backward: whether the step behind it does).
  const auto starts = [&](int64_t p) {
    if (!flags || p >= stop) return 0;
    if (back) return p == 0 ? 0 : (int)flags[(n - p) * g.reset_step];
    return (int)flags[p * g.reset_step];
  };

  Tile<T, W, CL> ta, tb;
  Tile<T, CHUNK_COLS, CL> tc;
  if constexpr (!STATE) ta.init(r.a ? static_cast<const T*>(r.a) + b * r.a_batch + h * r.a_head : nullptr, r.a_step, ka, walk, begin);
  tb.init(r.b ? static_cast<const T*>(r.b) + b * r.b_batch + h * r.b_head : nullptr, r.b_step, ka, walk, begin);
  tc.init(r.c ? static_cast<const T*>(r.c) + b * r.c_batch + h * r.c_head + c0 : nullptr, r.c_step, cols, walk, begin);
  int flag = 0;
  const auto fetch = [&](int p0) {
    const int count = stop - p0 < CL ? stop - p0 : CL, tid = opaque(threadIdx.x);
    if constexpr (!STATE) ta.load(tid, back, count);
    tb.load(tid, back, count);
    tc.load(tid, back, count);
    flag = lane < CL ? starts((int64_t)p0 + lane) : 0;
  };
  if (begin < stop) fetch(begin);
  // The next place's row of o, or of 16 places the one that comes first in memory.
  const int64_t o_step = STATE ? 0 : r.out_step * (int)sizeof(T);
  T* const po = STATE ? nullptr : static_cast<T*>(r.out) + b * r.out_batch + h * r.out_head + c0;
  char* out = reinterpret_cast<char*>(po) + (back ? (int64_t)n - 16 - begin : (int64_t)begin) * o_step;

  f32x4 S[TILES];
  const int col = 16 * wave + i0;
  const bool mine = col < cols;
  const int rs = (int)r.row_stride, cs = (int)r.col_stride, size = ka * r.nc;
  const bool full = ka == KP && cols == CHUNK_COLS;   // every lane's part of the state exists
  {
    const float* init = nullptr;
    if constexpr (!STATE)
      init = g.inits[which] ? g.inits[which] + ((b * g.heads + h) * g.pieces + piece) * size : r.init ? r.init + (b * g.heads + h) * size : nullptr;
    state_load<TILES>(init, S, full, mine, ka, rs, cs, c0 + col, q0);
  }
  if (threadIdx.x < 2) odd[threadIdx.x] = 0;
  float keep = 1.0f;   // STATE: what is left of the state in front of the piece, but for
  bool opens = false;  // an episode's start, behind which nothing is
  // Weights of the scores in a tile on the diagonal and in the one below it.
  float on[4], below[4];
  const float score = r.in * r.out_scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    on[e] = score * lin_power(log2d, i0 >= 4 * q0 + e ? i0 - 4 * q0 - e : 0);
    below[e] = score * lin_power(log2d, 16 + i0 - 4 * q0 - e);
  }
  const float two = lin_power(log2d, 16);
  __syncthreads();
  int turn = 0;
  for (int left = stop - begin; left > 0; left -= CL, turn ^= 1, out += CL * (back ? -o_step : o_step)) {   // (31 bits do not hold the place behind the last chunk)
    const int tid = opaque(threadIdx.x), lane = tid & 63, i = lane & 15, q = lane >> 4;
    const int64_t out_step = opaque_scalar(o_step), out_walk = back ? -out_step : out_step;
    const int p0 = stop - left, cnt = left < CL ? left : CL;
    const int lead = back && p0 == 0 ? 0 : 1;   // steps between the state in front and the first place
    if constexpr (!STATE) ta.store(tid, lds_a, back, 0);
    if (!M::finite(tc.store(tid, lds_c, back, tb.store(tid, lds_b, back, 0)))) odd[turn] = 1;
    const uint64_t cuts = __ballot(flag != 0);
    if (wave == 0 && lane < CL) {
      const uint64_t before = cuts & ((2ull << lane) - 1);
      const int ahead = cnt - 1 - lane;
      const float f = r.in * lin_power(log2d, ahead > 0 ? ahead : 0), o = r.out_scale * lin_power(log2d, lane + lead);
      fade[lane] = ahead >= 0 && !(cuts >> lane >> 1) ? f : 0.0f;
      enter[lane] = o;
      start[lane] = before ? 63 - __builtin_clzll(before) : 0;
    }
    const int first = cuts ? __builtin_ctzll(cuts) : CL;
    __syncthreads();
    if (!ONE && left > CL) fetch(p0 + CL);
    const bool slow = __builtin_amdgcn_readfirstlane(odd[turn]) != 0;
    frag v[CL / M::KB];
    if (16 * wave < cols) {
#pragma unroll
      for (int kk = 0; kk < CL / M::KB; ++kk) v[kk] = M::col(lds_c, PC, M::KB * kk, 16 * wave, i, q);
    }
    if constexpr (!STATE) {
      __syncthreads();
      if (!slow) {   // the scores below the diagonal, tile by tile
#pragma unroll
        for (int k = 0; k < (LOWER + ROWS / 2 + 3) / 4; ++k) {
          const int tile = wave + 4 * k;
          const int ti = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0, si = tile - ti * (ti + 1) / 2;
          if (M::KB == 32 && tile >= LOWER && tile < LOWER + ROWS / 2) {   // above it, but in one instruction with the tile on it
            const int u = 2 * (tile - LOWER);
            M::put(lds_p + score_block<T>(u, u / 2) * BLOCK, SCORES, u + 1, i, q, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
          }
          if (tile < LOWER && 16 * ti < cnt) {
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < KP; kk += M::KB)
              M::mma(acc, M::row(lds_b, PA, 16 * si, kk, i, q), M::row(lds_a, PA, 16 * ti, kk, i, q));
            const int t = 16 * ti + i, s = 16 * si + 4 * q;
            if (ti == si) {
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[e] = 4 * q + e <= i ? acc[e] * on[e] : 0.0f;
            } else {
              const float f = ti - si == 1 ? 1.0f : ti - si == 2 ? two : two * two;
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[e] *= below[e] * f;
            }
            if (cuts) {
              const int from = start[t];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[e] = s + e >= from ? acc[e] : 0.0f;
            }
            M::put(lds_p + score_block<T>(ti, si / (M::KB / 16)) * BLOCK, SCORES, si, i, q, acc);
          }
        }
      }
      __syncthreads();
    }
    if (!slow && 16 * wave < cols) {
      if constexpr (!STATE) {
        f32x4 o[ROWS];
#pragma unroll
        for (int ti = 0; ti < ROWS; ++ti) o[ti] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (first > 0) {
#pragma unroll
          for (int kk = 0; kk < KP / M::KB; ++kk) {
            float x[M::N];
#pragma unroll
            for (int e = 0; e < M::N; ++e) x[e] = S[kk * (M::KB / 16) + e / 4][e % 4];
            frag f[M::PARTS];
            M::split(x, f);
#pragma unroll
            for (int ti = 0; ti < ROWS; ++ti) {
              const frag a = M::row_state(lds_a, PA, 16 * ti, M::KB * kk, i, q);
#pragma unroll
              for (int k = M::PARTS - 1; k >= 0; --k) M::mma(o[ti], f[k], a);
            }
          }
        }
        const int wide = cols - 16 * wave - 4 * q;
#pragma unroll
        for (int ti = 0; ti < ROWS; ++ti) {
          const int t = 16 * ti + i;
          if (16 * ti >= cnt) continue;
          const float f = enter[t];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[ti][e] *= f;
          if (cuts) {   // (a state that is not finite does not pass a start either)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[ti][e] = t < first ? o[ti][e] : 0.0f;
          }
#pragma unroll
          for (int kk = 0; kk < CL / M::KB; ++kk)
            if (M::KB * kk <= 16 * ti) {
#pragma unroll
              for (int k = M::PARTS - 1; k >= 0; --k)
                M::mma(o[ti], v[kk], *reinterpret_cast<const frag*>(lds_p + k * SCORES + score_block<T>(ti, kk) * BLOCK + M::N * lane));
            }
          if (t < cnt && wide > 0) {
            const int up = back ? 15 - i : i;
            char* to = out + 16 * ti * out_walk + (g.far ? up * out_step : (int64_t)(uint32_t)(up * (uint32_t)out_step));
            T* y = reinterpret_cast<T*>(to) + 16 * wave + 4 * q;
            if (wide >= 4) {
              if constexpr (sizeof(T) == 2) {
                const u32x2 w = {pack_bf16x2(o[ti][0], o[ti][1]), pack_bf16x2(o[ti][2], o[ti][3])};
                __builtin_memcpy(y, &w, 8);
              } else {
                __builtin_memcpy(y, &o[ti], 16);
              }
            } else {
#pragma unroll
              for (int e = 0; e < 3; ++e)
                if (e < wide) y[e] = from_f<T>(o[ti][e]);
            }
          }
        }
      }
      if (!STATE && !r.last && left <= CL) {
        // Nobody asks for the state behind it.
      } else {
        const float whole = lin_power(log2d, cnt - 1 + lead);
#pragma unroll
        for (int k = 0; k < TILES; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[k][e] *= whole;
        if (cuts) {
#pragma unroll
          for (int k = 0; k < TILES; ++k) S[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        keep *= whole;
        opens = opens || cuts;
#pragma unroll
        for (int kk = 0; kk < CL / M::KB; ++kk) {
          if (M::KB * kk >= cnt) continue;
          float x[M::N];
#pragma unroll
          for (int e = 0; e < M::N; e += 4) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(fade + M::KB * kk + M::N * q + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[e + j] = M::at(v[kk], e + j) * w[j];
          }
          frag f[M::PARTS];
          M::split(x, f);
#pragma unroll
          for (int k = 0; k < TILES; ++k) {
            const frag a = M::col(lds_b, PA, M::KB * kk, 16 * k, i, q);
#pragma unroll
            for (int e = M::PARTS - 1; e >= 0; --e) M::mma(S[k], a, f[e]);
          }
        }
      }
    } else if (slow) {
      // A value that is not finite: step by step, as a product with a weight of 0 would spread it.
      for (int p = 0; p < cnt; ++p) {
        const bool cut = (cuts >> p & 1) != 0;
        const float d = p == 0 && lead == 0 ? 1.0f : lin_power(log2d, 1), c = mine ? to_f<T>(lds_c[p * PC + col]) : 0.0f;
        float o = 0.0f;
#pragma unroll
        for (int k = 0; k < TILES; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = 16 * k + 4 * q + e;
            if (row < ka) {
              S[k][e] = fmaf(r.in * to_f<T>(lds_b[p * PA + row]), c, cut ? 0.0f : d * S[k][e]);
              if constexpr (!STATE) o = fmaf(to_f<T>(lds_a[p * PA + row]), S[k][e], o);
            }
          }
        keep *= d;
        opens = opens || cut;
        if constexpr (!STATE) {
          o = add32(add16(o));
          if (q == 0 && mine) reinterpret_cast<T*>(out + (back ? 15 * out_step : 0) + p * out_walk)[col] = from_f<T>(r.out_scale * o);
        }
      }
    }
    if (ONE) break;
    __syncthreads();
    if (slow && threadIdx.x == 0) odd[turn] = 0;
  }
  if constexpr (STATE) {
    const int64_t at = (b * g.heads + h) * g.pieces + piece;
    state_store<TILES>(g.adds[which] + at * size, S, full, mine, ka, r.nc, 1, c0 + col, q0);
    if (unit == 0 && threadIdx.x == 0) g.keeps[which][at] = opens ? -1.0f : keep;
  } else {
    // Steps behind the sequence.
    const int64_t end = begin + g.len < g.steps ? begin + g.len : g.steps;
    for (int64_t t = (begin > n ? begin : n) + threadIdx.x / CHUNK_COLS; t < end; t += CHUNK_THREADS / CHUNK_COLS)
      if ((int)threadIdx.x % CHUNK_COLS < cols) po[t * r.out_step + threadIdx.x % CHUNK_COLS] = from_f<T>(0.0f);
    if (r.last && stop == n && (begin < n || piece == 0)) {
      const bool cut = back && n > 0 && flags && flags[0] != 0;
      const float d = back && n > 0 ? lin_power(log2d, 1) : 1.0f;
      float* to = r.last + (b * g.heads + h) * size;
#pragma unroll
      for (int k = 0; k < TILES; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[k][e] = cut ? 0.0f : S[k][e] * d;
      state_store<TILES>(to, S, full, mine, ka, rs, cs, c0 + col, q0);
    }
  }
}

// The state in front of each piece, in the place of what the piece adds to it: a thread an element.
constexpr int JOIN_THREADS = 256, JOIN_AHEAD = 16;
__global__ __launch_bounds__(JOIN_THREADS) void lin_join(LinArgs g) {
  const int which = blockIdx.y;
  const int64_t size = (int64_t)g.role[which].ka * g.role[which].nc;
  const int64_t at = (int64_t)blockIdx.x * JOIN_THREADS + threadIdx.x;
  if (at >= g.batch * g.heads * size) return;
  const int64_t head = at / size, e = at - head * size;
  float* u = g.adds[which] + head * g.pieces * size + e;
  const float* keep = g.keeps[which] + head * g.pieces;
  float s = g.role[which].init ? g.role[which].init[at] : 0.0f;
  for (int64_t p = 0; p < g.pieces; p += JOIN_AHEAD) {
    float x[JOIN_AHEAD], k[JOIN_AHEAD];
#pragma unroll
    for (int j = 0; j < JOIN_AHEAD; ++j) {
      const bool on = p + j < g.pieces;
      x[j] = on ? u[(p + j) * size] : 0.0f;
      k[j] = on ? keep[p + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < JOIN_AHEAD; ++j)
      if (p + j < g.pieces) {
        u[(p + j) * size] = s;
        s = k[j] < 0.0f ? x[j] : fmaf(k[j], s, x[j]);   // nothing passes an episode's start, finite or not (a factor of 0 does not stop a NaN)
      }
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
  if (!op_extent_ok(a.batch) || !op_extent_ok(a.steps) || !op_extent_ok(a.heads) || a.heads > LIN_MAX_HEADS) return "extent out of range";
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

// Arrays that workgroups of one launch read and write in any order. (y in the place of v is sound: a workgroup has read the columns of a
// step before it writes them, and no other one reads them.)
const char* lin_check_shares(const spz_linear_attention_args& a, bool back) {
  const int64_t K = a.key_width, V = a.value_width;
  const int e = op_size(a.prec);
  const auto rows = [&](const void* p, int64_t w, int64_t s0, int64_t s1, int64_t s2) { return OpArray{p, w, {a.batch, a.steps, a.heads}, {s0, s1, s2}}; };
  const auto states = [&](const float* x, const float* y) {
    return op_shares(4, OpArray{x, K * V, {a.batch, a.heads, 1}, {a.heads * K * V, K * V, 0}}, OpArray{y, K * V, {a.batch, a.heads, 1}, {a.heads * K * V, K * V, 0}});
  };
  const OpArray q = rows(a.q, K, a.q_batch, a.q_step, a.q_head), k = rows(a.k, K, a.k_batch, a.k_step, a.k_head), v = rows(a.v, V, a.v_batch, a.v_step, a.v_head);
  if (!back) {
    const OpArray y = rows(a.y, V, a.y_batch, a.y_step, a.y_head);
    if (op_shares(e, y, q) || op_shares(e, y, k) || (!op_same(y, v) && op_shares(e, y, v))) return "y shares elements with q, k or other places of v";
    return a.last != a.state && states(a.last, a.state) ? "last shares elements with other places of state" : nullptr;
  }
  const OpArray dy = rows(a.dy, V, a.dy_batch, a.dy_step, a.dy_head);
  const OpArray outs[3] = {rows(a.dq, K, a.dq_batch, a.dq_step, a.dq_head), rows(a.dk, K, a.dk_batch, a.dk_step, a.dk_head), rows(a.dv, V, a.dv_batch, a.dv_step, a.dv_head)};
  for (int i = 0; i < 3; ++i) {
    if (op_shares(e, outs[i], outs[(i + 1) % 3])) return "dq, dk and dv share elements";
    for (const OpArray* x : {&q, &k, &v, &dy})
      if (op_shares(e, outs[i], *x)) return "dq, dk or dv shares elements with q, k, v or dy";
  }
  return states(a.dstate, a.dlast) || states(a.dstate, a.state) ? "dstate shares elements with dlast or state" : nullptr;
}

template <typename T> void lin_steps_launch(LinArgs g, hipStream_t s) {
  StepArgs f{};
  int64_t slices = 1;
  int ka = 0;
  for (int i = 0; i < g.roles; ++i) {
    const LinRole& r = g.role[i];
    const int64_t n = op_div_up(r.nc, STEP_COLS);
    slices = n > slices ? n : slices;
    ka = r.ka > ka ? r.ka : ka;
    f.by_slices[i] = divisor((uint32_t)n);
    f.vec[i] = r.col_stride == 1 && r.nc % 4 == 0 && op_aligned(r.init, 16) && op_aligned(r.last, 16);
  }
  f.by_heads = divisor((uint32_t)g.heads);
  // Sequences whose workgroups one dispatch counts (heads are limited).
  const int64_t most = OP_DISPATCH / (STEP_THREADS * 3) / (g.heads * slices);
  const auto go = [&](auto kr) {
    for (int64_t first = 0; first < g.batch; first += most) {
      const int64_t count = g.batch - first < most ? g.batch - first : most;
      g.first = first;
      g.groups = (uint32_t)count;
      lin_steps<T, decltype(kr)::value><<<dim3((unsigned)(count * g.heads * slices), (unsigned)g.roles), STEP_THREADS, 0, s>>>(g, f);
    }
  };
  using std::integral_constant;
  if (ka <= 16) go(integral_constant<int, 1>{});
  else if (ka <= 64) go(integral_constant<int, 4>{});
  else if (ka <= 128) go(integral_constant<int, 8>{});
  else go(integral_constant<int, 16>{});
}

// The rows of states that the kernels come in.
template <typename T> int lin_rows(int ka) {
  for (const int kp : {32, 48, 64, 96, 128})
    if (ka <= kp && kp % Mat<T>::KB == 0) return kp;
  return 256;
}
// Microseconds of a launch of n workgroups of `chunks` chunks each: a compute unit holds `most` of them at once, and a
// workgroup's start counts as a chunk. A chunk takes 5 and 1 more for each workgroup of the unit (64 x 64 heads, 1 to 4 a unit: 5.3,
// 6.3, 7.5 and 9.2 measured), in float32 5 and 3 (1 to 3 a unit: 7.7, 10.7 and 14.0). Other heads count as these, by their workgroups.
template <typename T> int64_t lin_time(int ka, int64_t n, int64_t chunks) {
  const int kp = lin_rows<T>(ka);
  const int64_t most = kp > 128 ? 1 : kp > 64 ? (sizeof(T) == 2 ? 2 : 1) : sizeof(T) == 2 ? 4 : 3;
  const int64_t each = op_div_up(n, 256), rounds = op_div_up(each, most);
  return (chunks + 1) * (5 * rounds + (sizeof(T) == 2 ? 1 : 3) * each);
}
// How a call is spread, by its sizes and whether it has a gradient to the last state (microseconds a call, both sides measured, bfloat16
// unless said, steps against chunks):
//   steps: a thread keeps its part of the state and walks: up to 2 steps, in float32 4 (2048 x 4 heads of 64 x 64: 4 steps 81 against 66; in
//     float32 4 steps 90 against 110, 8 steps 143 against 111);
//   chunks: a workgroup walks in chunks on the matrix cores; up to 2 steps of bfloat16 too where they are faster, which takes widths that fill
//     the tiles (others' states are read element by element: 2048 x 4 x 100 x 100, 1 step 286 against 407, backward 505 against 768):
//     forward heads of 128 rows, which leave a thread of the step kernel twice the registers, and states past the last-level cache
//       (1 step, 128 x 128: 16 x 4 7.2 against 9.0, 256 x 4 33 against 42, 1024 x 4 132 against 136, 2 steps 160 against 142; 2048 x 4 314
//       against 272, 2 steps 350 against 275; 128 x 64: 1024 x 4 58 against 67, 4096 x 8 615 against 527);
//     backward from 1024 heads on, with a gradient to the last state (4096 x 8 x 64 x 64 670 against 586, 2048 x 4 x 128 x 128 1012 against 677,
//       256 x 4 108 against 88, 16 x 4 8.7 against 10.8), or without it at 128 rows or columns, but for one step of 128 x 128 (2048 x 4, 1 step: 128 x 64 366
//       against 294, 64 x 128 334 against 313, 128 x 128 596 against 615, 64 x 64 105 against 137; 2 steps 460 against 296, 411 against 313, 730
//       against 617, 125 against 140);
//   pieces: time cut into pieces of 64 steps and more whose sums are joined first, two launches and a second reading of keys and
//     values more, where the model above says that it pays (in pieces against whole, forward: 1 x 1000 x 4 18 against 80, in float32
//     20 against 112; 1 x 300 x 16 18 against 29; 8 x 1000 x 8 39 against 84; 64 x 1000 x 4 70 against 89). The two launches count
//     as 12: as 8 the model cuts 32 x 256 x 4 (31 against 24), as 16 it leaves 4 x 200 x 4 in float32 whole (30 against 20).
struct LinPlan { bool chunks; int64_t pieces, len; };
constexpr int64_t LAST_LEVEL = (int64_t)1 << 28;   // bytes of the last-level cache
template <typename T> bool lin_in_steps(const spz_linear_attention_args& a, bool back, bool dlast) {
  const int64_t K = a.key_width, V = a.value_width, heads = a.batch * a.heads;
  if (a.steps == 0 || K == 0 || V == 0) return true;
  if (a.steps > (sizeof(T) == 4 ? 4 : 2)) return false;
  if (sizeof(T) == 4) return true;
  if (!back) return !(K == 128 && V % CHUNK_COLS == 0 && 4 * heads * K * V >= LAST_LEVEL);
  const auto fills = [](int64_t w) { return w == 64 || w == 128; };
  return !(fills(K) && fills(V) && heads >= 1024 && (dlast || (K + V > 128 && (a.steps == 2 || K != V))));
}
// dlast: whether a backward call has that gradient. A call of steps needs no workspace, one of so few steps in chunks neither.
template <typename T> LinPlan lin_plan_of(const spz_linear_attention_args& a, bool back, bool dlast) {
  const int K = (int)a.key_width, V = (int)a.value_width;
  if (lin_in_steps<T>(a, back, dlast)) return {false, 1, a.steps};
  const int64_t k = op_div_up(K, CHUNK_COLS), v = op_div_up(V, CHUNK_COLS), heads = a.batch * a.heads;
  LinPlan best{true, 1, a.steps};
  if (heads == 0 || a.steps <= 128 || heads > 2048) return best;
  // Workgroups of a launch: by key rows (y; dv), by value rows (dq and dk), or all in one; and of the pieces' sums.
  const bool same = lin_rows<T>(K) == lin_rows<T>(V);
  const int64_t by_k = v + (back && same ? 2 * k : 0), by_v = back && !same ? 2 * k : 0, sums = back ? 2 * v : v;
  int64_t least = 0;
  for (const int64_t pieces : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 80, 96, 128}) {
    const int64_t len = op_div_up(op_div_up(a.steps, pieces), 64) * 64, chunks = len / 64;
    if (pieces > 1 && op_div_up(a.steps, len) != pieces) continue;
    int64_t time = lin_time<T>(K, heads * pieces * by_k, chunks) + (by_v ? lin_time<T>(V, heads * pieces * by_v, chunks) : 0);
    if (pieces > 1) time += lin_time<T>(K, heads * pieces * sums, chunks) / 2 + 12 + pieces / 8;   // the launches and the join, 3, 10 and 15 us for 16, 64 and 128 pieces of 8 heads
    if (pieces == 1 || time < least) {
      least = time;
      best = {true, pieces, pieces > 1 ? len : a.steps};
    }
  }
  return best;
}
LinPlan lin_plan(const spz_linear_attention_args& a, bool back, bool dlast) {
  return a.prec == SPZ_PREC_BF16 ? lin_plan_of<bf16_t>(a, back, dlast) : lin_plan_of<float>(a, back, dlast);
}
// Floats of one state of all pieces, and of what they keep, each at 16 bytes.
int64_t lin_states(const spz_linear_attention_args& a, const LinPlan& p) {
  return op_div_up(a.batch * a.heads * p.pieces * a.key_width * a.value_width, 4) * 4;
}
int64_t lin_keeps(const spz_linear_attention_args& a, const LinPlan& p) { return op_div_up(a.batch * a.heads * p.pieces, 4) * 4; }

template <typename T, int KP, int CL, bool STATE, bool ONE> void lin_chunks_go(LinArgs g, hipStream_t s) {
  g.units = 0;
  g.far = false;
  for (int i = 0; i < g.roles; ++i) {
    g.units += g.slices[i] = (g.role[i].nc + CHUNK_COLS - 1) / CHUNK_COLS;
    g.far = g.far || g.role[i].out_step > (int64_t)1 << 24;
  }
  g.by_units = divisor((uint32_t)g.units);
  g.by_pieces = divisor((uint32_t)g.pieces);
  g.by_heads = divisor((uint32_t)g.heads);
  // Sequences whose workgroups one dispatch counts (a sequence has fewer than that: heads and pieces are limited).
  const int64_t each = g.heads * g.pieces, most = (OP_DISPATCH / CHUNK_THREADS / g.units - 8) / each;
  for (int64_t first = 0; first < g.batch; first += most) {
    const int64_t count = g.batch - first < most ? g.batch - first : most;
    g.first = first;
    g.groups = (uint32_t)(count * each);
    lin_chunks<T, KP, CL, STATE, ONE><<<dim3((unsigned)(op_div_up(count * each, 8) * 8 * g.units)), CHUNK_THREADS, 0, s>>>(g);
  }
}
// Roles of one number of rows in a launch.
template <typename T, bool STATE> void lin_chunks_launch(const LinArgs& all, hipStream_t s) {
  for (const int kp : {32, 48, 64, 96, 128, 256}) {
    LinArgs g = all;
    g.roles = 0;
    for (int i = 0; i < all.roles; ++i)
      if (lin_rows<T>(all.role[i].ka) == kp) {
        g.role[g.roles] = all.role[i];
        g.inits[g.roles++] = all.inits[i];
      }
    if (g.roles == 0) continue;
    const auto go = [&](auto one) {
      constexpr bool ONE = decltype(one)::value, BF16 = sizeof(T) == 2;
      if (kp == 32) lin_chunks_go<T, 32, 64, STATE, ONE>(g, s);
      else if (kp == 48) lin_chunks_go<T, BF16 ? 64 : 48, 64, STATE, ONE>(g, s);
      else if (kp == 64) lin_chunks_go<T, 64, 64, STATE, ONE>(g, s);
      else if (kp == 96) lin_chunks_go<T, 96, 64, STATE, ONE && BF16>(g, s);
      else if (kp == 128) lin_chunks_go<T, 128, 64, STATE, ONE && BF16>(g, s);
      else lin_chunks_go<T, 256, BF16 ? 64 : 32, STATE, ONE && BF16>(g, s);
    };
    if constexpr (!STATE) {
      if (g.steps <= 64) {
        go(std::true_type{});
        continue;
      }
    }
    go(std::false_type{});
  }
}

template <typename T> void lin_launch(LinArgs& g, const LinPlan& plan, const spz_linear_attention_args& a, bool back, void* ws, hipStream_t s) {
  if (!plan.chunks) return lin_steps_launch<T>(g, s);
  g.pieces = plan.pieces;
  g.len = plan.len;
  if (plan.pieces > 1) {
    LinArgs u = g;
    u.roles = 1;
    float* at = static_cast<float*>(ws);
    const int K = (int)a.key_width, V = (int)a.value_width;
    const auto state = [&](LinRole& r, int i, const void* x, int64_t x0, int64_t x1, int64_t x2, const void* y, int64_t y0, int64_t y1, int64_t y2,
                           const float* init, bool rev) {
      r = LinRole{};
      r.b = x; r.b_batch = x0; r.b_step = x1; r.b_head = x2;
      r.c = y; r.c_batch = y0; r.c_step = y1; r.c_head = y2;
      r.init = init; r.row_stride = V; r.col_stride = 1; r.ka = K; r.nc = V; r.back = rev; r.in = rev ? a.scale : 1.0f;
      u.adds[i] = at;
      u.keeps[i] = at + lin_states(a, plan);
      at += lin_states(a, plan) + lin_keeps(a, plan);
    };
    state(u.role[0], 0, a.k, a.k_batch, a.k_step, a.k_head, a.v, a.v_batch, a.v_step, a.v_head, a.state, false);
    if (back) {
      u.roles = 2;
      state(u.role[1], 1, a.q, a.q_batch, a.q_step, a.q_head, a.dy, a.dy_batch, a.dy_step, a.dy_head, a.dlast, true);
    }
    lin_chunks_launch<T, true>(u, s);
    lin_join<<<dim3((unsigned)op_div_up(a.batch * a.heads * K * V, JOIN_THREADS), (unsigned)u.roles), JOIN_THREADS, 0, s>>>(u);
    for (int i = 0; i < g.roles; ++i) g.inits[i] = u.adds[g.role[i].back ? 1 : 0];
  }
  lin_chunks_launch<T, false>(g, s);
}

int lin_run(const char* call, const spz_linear_attention_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = lin_check(args);
  if (!bad) bad = lin_check_arrays(*args, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const spz_linear_attention_args& a = *args;
  const int64_t need = spz_linear_attention_workspace(args, back);
  if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
  if (need > 0 && !op_aligned(ws, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
  bad = lin_check_shares(a, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
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
  const LinPlan plan = lin_plan(a, back, back && a.dlast);
  if (a.prec == SPZ_PREC_BF16) lin_launch<bf16_t>(g, plan, a, back, ws, s);
  else lin_launch<float>(g, plan, a, back, ws, s);
  return op_launched(call);
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int64_t spz_linear_attention_workspace(const spz_linear_attention_args* args, int32_t backward) {
  const char* bad = lin_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_linear_attention_workspace", bad);
  const LinPlan plan = lin_plan(*args, backward != 0, false);
  return plan.pieces > 1 ? 4 * (backward ? 2 : 1) * (lin_states(*args, plan) + lin_keeps(*args, plan)) : 0;
}

int spz_linear_attention_forward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return lin_run("spz_linear_attention_forward", args, false, workspace, workspace_bytes, hip_stream);
}

int spz_linear_attention_backward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return lin_run("spz_linear_attention_backward", args, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
