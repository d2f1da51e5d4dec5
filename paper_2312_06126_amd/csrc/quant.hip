// The 8-bit integer product with a scale for each row of the input and each output channel
// (spz_quant_*).
//
//   y[m, n] = s[m] w_scale[n] sum_k q[m, k] w[n, k] + bias[n],   s[m] = max_k |x[m, k]| float32(1 / 127)
//
// Weights are kept as fragments: 1 KB pieces of 32 channels by 32 bytes of k in the order in which
// one wave feeds v_mfma_i32_32x32x32_i8 (lane l: 16 bytes of channel l % 32, k from 16 (l / 32)), zeros
// past the edges, k innermost: a wave's load is one contiguous kilobyte, straight to registers.
//
// Up to QUANT_LDS_INNER inputs a workgroup keeps its rows of x, quantised as they arrive, in LDS for
// the whole product (quant_wide, quant_few), so x is read once and its integers never leave the
// compute unit: large calls are bound by reading x and writing y, small ones by latency. Longer
// rows go through the workspace (quant_rows, quant_product).
#include <atomic>
#include <type_traits>

#include "ops.h"

namespace spz {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
constexpr int64_t QUANT_MAX_INNER = 131072;   // 127^2 of these still fit 32 bits
constexpr int FRAG = 1024;

inline int64_t frag_blocks(int64_t n) { return op_div_up(n, 32); }

template <int CTRL> __device__ inline uint32_t dpp_max(uint32_t x) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
  return o > x ? o : x;
}
__device__ inline uint32_t max16(uint32_t x) {   // of 16 lanes
  x = dpp_max<0xB1>(x);    // neighbours, pairs, the halves of 16 lanes mirrored, the 16 mirrored
  x = dpp_max<0x4E>(x);
  x = dpp_max<0x141>(x);
  return dpp_max<0x140>(x);
}
__device__ inline uint32_t max32(uint32_t x) {   // of 32 lanes
  x = max16(x);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return r[0] > r[1] ? r[0] : r[1];
}
__device__ inline uint32_t wave_max(uint32_t x) {
  x = max32(x);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return r[0] > r[1] ? r[0] : r[1];
}
// A scale is the row's largest |x| times the float32 next to 1 / 127: what dividing a float32 tensor on the GPU by the
// number 127 gives in torch, so that a quantisation written there rounds the same elements up. In 5% of rows it is an ulp from
// the rounded quotient max |x| / 127, which moves elements that lie at a tie: of a million normal ones (rows of 512) less than
// 0.1 in float32, but 40 to 80 in bfloat16, where ties are common.
constexpr float QUANT_STEP = 1.0f / 127.0f;
// The row's scale from the largest |x| as bits, and whether the row quantises to zeros: infinity and
// NaN have the largest bits.
__device__ inline float row_scale(uint32_t bits, bool& zero) {
  const float s = bits >= 0x7F800000u ? __builtin_nanf("") : __builtin_bit_cast(float, bits) * QUANT_STEP;
  zero = !(s > 0.0f);
  return s;
}
__device__ inline int quantised(float x, float s) {
  const float q = rintf(x / s);
  return (int)fminf(fmaxf(q, -127.0f), 127.0f);
}

// Rows of integers: one wave a row, which it reads twice (bound by HBM and its latency; weights, once). q [rows, width]
// at q_row, or (FRAGS) as fragments over 32 * frag_blocks(rows) rows.
template <typename T, bool FRAGS>
__global__ __launch_bounds__(256) void quant_rows(const T* x, int64_t x_row, int64_t rows, int64_t width, int8_t* q,
                                                  int64_t q_row, float* scale, int64_t first) {
  const int64_t row = (first + blockIdx.x) * 4 + threadIdx.x / 64;
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

// A byte of the image a thread, zeros past the edges: 5 us at 1024 x 1024, once for the weights.
__global__ __launch_bounds__(256) void quant_pack(const int8_t* q, int64_t q_row, int64_t outer, int64_t inner, int8_t* image,
                                                  int64_t first) {
  const int64_t steps = (inner + 31) / 32, i = (first + blockIdx.x) * 256 + threadIdx.x;
  if (i >= (outer + 31) / 32 * steps * FRAG) return;
  const int64_t frag = i / FRAG, lane = i % FRAG / 16;
  const int64_t n = frag / steps * 32 + lane % 32, k = frag % steps * 32 + lane / 32 * 16 + i % 16;
  image[i] = n < outer && k < inner ? q[n * q_row + k] : (int8_t)0;
}

// Rows above QUANT_LDS_INNER inputs, the simple form: one wave a 32 x 32 tile of y, fragments straight from
// L2, which bounds it. With quant_rows 160 us at 4096 x 8192 x 1024 bf16 (0.43 POP/s), 220 where all comes from memory.
template <typename T>
__global__ __launch_bounds__(256) void quant_product(const int8_t* x, const int8_t* w, const float* xs, const float* ws,
                                                     const float* bias, T* y, int64_t y_row, int64_t rows, int64_t outer,
                                                     int64_t steps, int64_t first) {
  const int64_t nb = (outer + 31) / 32, tile = (first + blockIdx.x) * 4 + threadIdx.x / 64;
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

// ----------------------------------------------------------------------------- rows in LDS
constexpr int64_t QUANT_LDS_INNER = 4096;
constexpr int QUANT_THREADS = 512, QUANT_WAVES = QUANT_THREADS / 64;
constexpr int QUANT_SCRATCH = 2560;   // bytes of LDS a wave beside the rows

struct QuantArgs {
  const void* x; int64_t x_row;
  const int8_t* image; const float* w_scale; const float* bias;
  void* y; int64_t y_row;
  int64_t rows, outer;
  int inner, steps;         // steps of 32 inputs
  int row_tiles, parts, units;  // quant_wide: units of 64 channels, shared out over `parts` workgroups
};

// Sixteen elements over s, rounded to integers, as bytes. r is 1 / s correctly rounded; then, with q = x r
// (within an ulp of the quotient) and its exact remainder x - q s, q + remainder * r is the correctly
// rounded quotient (Markstein, 1990) in three operations. Ties are common where x is bfloat16
// (127 x / max |x| is a ratio of small integers), so an estimate would not do. Where s is so tiny that
// the remainder could underflow, x and s are first multiplied by 2^64, and quotients are held to 127
// (a subnormal s is a coarse one).
constexpr float QUANT_MAGIC = 12582912.0f;   // 1.5 * 2^23: the sum's low byte is the rounded integer
constexpr float QUANT_TINY = 1e-30f, QUANT_LIFT = 18446744073709551616.0f;
struct RowScale { float s, r; bool tiny; };
__device__ inline RowScale row_factors(float s) {
  const bool tiny = s < QUANT_TINY;
  const float t = tiny ? s * QUANT_LIFT : s;
  return RowScale{t, 1.0f / t, tiny};
}
__device__ inline u32x4 quantise16(float (&x)[16], const RowScale& f) {
  float t[16];
  if (f.tiny) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= QUANT_LIFT;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float q = x[i] * f.r;
    t[i] = fmaf(fmaf(-q, f.s, x[i]), f.r, q);
  }
  if (f.tiny) {
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = fminf(fmaxf(t[i], -127.0f), 127.0f);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) t[i] += QUANT_MAGIC;
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __builtin_bit_cast(uint32_t, t[4 * j + i]);
    w[j] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) | __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
  }
  return w;
}

// The larger of m and the magnitudes in w, as bits (bfloat16: of each half by itself).
template <typename T> __device__ inline uint32_t largest(const u32x4& w, uint32_t m) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = w[i];
    if constexpr (sizeof(T) == 2) {
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v & 0x7FFF7FFFu), __builtin_bit_cast(u16x2, m)));
    } else {
      m = (v & 0x7FFFFFFFu) > m ? v & 0x7FFFFFFFu : m;
    }
  }
  return m;
}

// Rows of x as a wave loads them: LPR lanes a row (64; 16 or 32 for up to 256 or 512 inputs: four or two
// rows at once), R times, NU units of 16 inputs a lane (up to 16 LPR NU inputs); and their way into LDS: unit k of the
// workgroup's row r at k RT + (r ^ (k & 7)), so that 32 rows of a unit are contiguous for the products and
// eight units of a row fall on different banks here. What lies past a row's inputs within its last
// step meets zero weights; what lies past the rows is not stored.
template <typename T, int R, int NU, int LPR> struct RowChunk {
  static constexpr int E = OP_VEC<T>, W = 16 / E, ROWS = R * (64 / LPR);
  u32x4 raw[R][NU][W];

  static __device__ int row_of(int j) { return LPR == 64 ? j : j * (64 / LPR) + (int)(threadIdx.x % 64) / LPR; }

  __device__ void load(const QuantArgs& g, int64_t row0) {
    const int lane = threadIdx.x % LPR;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t want = row0 + row_of(j), row = want < g.rows ? want : g.rows - 1;
      const T* p = static_cast<const T*>(g.x) + row * g.x_row;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          raw[j][u][k] = u32x4{0, 0, 0, 0};
          const int c = (u * LPR + lane) * 16 + k * E;
          if (c + E <= g.inner) raw[j][u][k] = load16(p + (uint32_t)c);
        }
      // The last elements of a row of no whole number of accesses: one lane's, one access.
      if (g.inner % E) {
        const int last = g.inner / E, u0 = last / W, k0 = last % W;
        if (u0 % LPR == lane) {
          const u32x4 w = load_part(p + last * E, g.inner % E);
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int k = 0; k < W; ++k)
              if (u == u0 / LPR && k == k0) raw[j][u][k] = w;
        }
      }
    }
  }

  // The rows' scales and their integers, 16 bytes a unit of the lane (the inputs as load() took them).
  __device__ void quantise(float (&scale)[R], u32x4 (&q)[R][NU]) const {
    uint32_t m[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      m[j] = 0;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int k = 0; k < W; ++k) m[j] = largest<T>(raw[j][u][k], m[j]);
      if (sizeof(T) == 2) m[j] = (m[j] << 16) > (m[j] & 0xFFFF0000u) ? m[j] << 16 : m[j] & 0xFFFF0000u;
      if (LPR == 64) m[j] = __builtin_amdgcn_readfirstlane(wave_max(m[j]));
      else m[j] = LPR == 32 ? max32(m[j]) : max16(m[j]);
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      bool zero;
      scale[j] = row_scale(m[j], zero);
      const RowScale f = row_factors(scale[j]);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float v[16];
#pragma unroll
        for (int k = 0; k < W; ++k) {
          float t[E];
          unpack(raw[j][u][k], t);
#pragma unroll
          for (int i = 0; i < E; ++i) v[k * E + i] = t[i];
        }
        q[j][u] = zero ? u32x4{0, 0, 0, 0} : quantise16(v, f);
      }
    }
  }

  // One unit of a row's integers to its place: unit u of the lane, row r of the RT.
  template <int RT> static __device__ void place(const QuantArgs& g, u32x4* a, int r, int u, const u32x4& q) {
    const int k = u * LPR + threadIdx.x % LPR;
    if (k < 2 * g.steps) a[k * RT + (r ^ (k & 7))] = q;
  }
};

// Rows row0 .. row0 + RT - 1 into LDS by WAVES waves, 64 registers of them at a time.
template <typename T, int RT, int NU, int LPR, int WAVES>
__device__ inline void quantise_rows(const QuantArgs& g, int64_t row0, u32x4* a, float* scale) {
  constexpr int PER = RT / WAVES, TIMES = PER / (64 / LPR), MOST = 16 / (int)sizeof(T) / NU, R = MOST < 1 ? 1 : MOST < TIMES ? MOST : TIMES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  using C = RowChunk<T, R, NU, LPR>;
  for (int j = 0; j < PER; j += C::ROWS) {
    if (row0 + wave * PER + j >= g.rows) break;
    C c;
    c.load(g, row0 + wave * PER + j);
    float sc[R];
    u32x4 q[R][NU];
    c.quantise(sc, q);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = wave * PER + j + C::row_of(i);
      if (threadIdx.x % LPR == 0) scale[r] = sc[i];
#pragma unroll
      for (int u = 0; u < NU; ++u) C::template place<RT>(g, a, r, u, q[i][u]);
    }
  }
}

// y of RB blocks of 32 rows by 64 channels a wave: lane l holds row l % 32 and, of each 32 channels, those
// of which bit 2 is l / 32; they go through 2 KB of LDS a wave to leave as 64-byte pieces of rows. wl, bl:
// the scale and bias of channel `lane` of the 64, handed out through the last 512 bytes of LDS.
template <typename T, int RB>
__device__ inline void quant_store(const QuantArgs& g, const i32x16 (&acc)[RB][2], const float (&xs)[RB], int64_t row0, int64_t n0,
                                   float wl, float bl, uint8_t* scratch) {
  const int lane = threadIdx.x % 64, l = lane % 32, h = lane / 32, turn = l >> 2 & 3;
  constexpr int E = OP_VEC<T>, COLS = 4 * E, Q = COLS / 8;   // channels of a piece, and its groups of 8
  const auto settle = []() {   // LDS between the lanes of the wave
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  float* channel = reinterpret_cast<float*>(scratch + 2048);
  channel[lane] = wl;
  channel[64 + lane] = bl;
  settle();
  // A piece's rows are read back while the next one is computed, and stored after that.
  u32x4 held[2];
  const auto flush = [&](int piece, int rb) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t row = row0 + rb * 32 + i * 16 + lane / 4, n = n0 + piece * COLS + lane % 4 * E;
      T* p = static_cast<T*>(g.y) + row * g.y_row + n;
      if (row < g.rows && n + E <= g.outer) store16(p, held[i]);
      else if (row < g.rows && n < g.outer) store_part(p, held[i], (int)(g.outer - n));
    }
  };
#pragma unroll
  for (int piece = 0; piece < 64 / COLS; ++piece) {
    float sw[Q][4], bn[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(channel + piece * COLS + q * 8 + h * 4);
      const f32x4 b = *reinterpret_cast<const f32x4*>(channel + 64 + piece * COLS + q * 8 + h * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { sw[q][i] = w[i]; bn[q][i] = b[i]; }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int of = piece * Q + q;   // group of 8 channels of the 64
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf((float)acc[rb][of / 4][of % 4 * 4 + i], xs[rb] * sw[q][i], bn[q][i]);
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<u32x2*>(scratch + l * 64 + (q ^ turn) * 16 + h * 8) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else
          *reinterpret_cast<u32x4*>(scratch + l * 64 + ((2 * q + h) ^ turn) * 16) = pack(v);
      }
      settle();
      if (piece + rb > 0) flush(rb ? piece : piece - 1, rb ? rb - 1 : RB - 1);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = i * 16 + lane / 4, unit = lane % 4;
        held[i] = *reinterpret_cast<const u32x4*>(scratch + r * 64 + (unit ^ (r >> 2 & 3)) * 16);
      }
      settle();
    }
  }
  flush(64 / COLS - 1, RB - 1);
}

// One wave: RB blocks of 32 rows in LDS by the units of 64 channels unit0, unit0 + by, ... below unit1.
// Weights are loaded DEPTH steps ahead (L2's latency under load), the next unit's before the present
// one is stored, rows XD - 1. A unit goes through whole turns of DEPTH steps: past the last step the
// weights read as zeros (buffer loads, whose bounds end there; the step's offset is a scalar, so the
// loop computes no addresses), and the rows whatever lies in LDS behind them: up to three steps, 6 RT units.
template <typename T, int RB>
__device__ inline void quant_units(const QuantArgs& g, const u32x4* lds, int unit0, int unit1, int by, const float (&xs)[RB],
                                   int64_t row0, uint8_t* scratch) {
  constexpr int RT = RB * 32, DEPTH = 8, XD = 4;
  const int lane = threadIdx.x % 64, l = lane % 32, h = lane / 32, nb = (int)((g.outer + 31) / 32);
  if (unit0 >= unit1) return;
  // Rows of step 4 s + j: unit 8 s + 2 j + h.
  const u32x4* ax[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) ax[j] = lds + (2 * j + h) * RT + (l ^ (2 * j + h));
  __amdgpu_buffer_rsrc_t w[2];
  i32x4 b[DEPTH][2], x[XD][RB];
  const auto start = [&](int unit) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int n = unit * 2 + c < nb ? unit * 2 + c : nb - 1;
      w[c] = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.image) + (int64_t)n * g.steps * FRAG, 0, g.steps * FRAG, 0x00027000);
    }
  };
  const auto weights = [&](int c, int s) {
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(w[c], lane * 16, s * FRAG, 0));
  };
  const int last4 = (g.steps - 1) / 4 * 4;
  const auto rows = [&](int s4, int j, int to) {   // of step s4 + j, s4 a multiple of 4
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) x[to][rb] = __builtin_bit_cast(i32x4, ax[j][(s4 < last4 ? s4 : last4) * 2 * RT + rb * 32]);
  };
  const auto first = [&]() {
#pragma unroll
    for (int j = 0; j < DEPTH; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) b[j][c] = weights(c, j);
  };
  start(unit0);
  first();
  for (int unit = unit0; unit < unit1; unit += by) {
    const int64_t n = (int64_t)unit * 64 + lane, in = n < g.outer ? n : g.outer - 1;
    const float wl = g.w_scale[in], bl = g.bias ? g.bias[in] : 0.0f;
    i32x16 acc[RB][2] = {};
#pragma unroll
    for (int j = 0; j < XD - 1; ++j) rows(0, j, j);
    for (int s = 0; s < g.steps; s += DEPTH) {
#pragma unroll
      for (int j = 0; j < DEPTH; ++j) {
        rows(s + (j + XD - 1) / 4 * 4, (j + XD - 1) % 4, (j + XD - 1) % XD);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            acc[rb][c] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[j][c], x[j % XD][rb], acc[rb][c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 2; ++c) b[j][c] = weights(c, s + j + DEPTH);
        __builtin_amdgcn_sched_barrier(0);   // the order above is the order of issue
      }
    }
    if (unit + by < unit1) {
      start(unit + by);
      first();
    }
    __builtin_amdgcn_sched_barrier(0);
    quant_store<T, RB>(g, acc, xs, row0, (int64_t)unit * 64, wl, bl, scratch);
  }
}

// A workgroup: RT rows and its part of the channels, 64 a wave at a time, each wave on its own once the
// rows are in LDS. Bound by its phases: all workgroups read and quantise, multiply and write at about the
// same time, so neither HBM nor the matrix instructions are always busy; two workgroups a compute unit
// cover some of it. 131072 x 1024 x 1024 bf16: 200 us at the least, 1.37 POP/s (the matrix instructions alone take a
// third), 232 in the median of calls without a pause; 131072 x 256 x 256: 39 us, 3.4 TB/s, from memory. Waves of the workgroup that load the next tile of 128 rows
// while the others multiply were as fast at the first (197 to 211) and slower elsewhere
// (65536 x 1024 x 4096: 482 against 368).
template <typename T, int RB, int NU, int LPR, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void quant_wide(QuantArgs g) {
  extern __shared__ u32x4 lds[];
  constexpr int RT = RB * 32;
  // Workgroup b runs on XCD b % 8: there are the workgroups of the same channels (eight parts or more:
  // few rows, to which the weights are the larger part) or of the same rows.
  const bool many = g.parts >= 8;
  const int tile = many ? blockIdx.x / g.parts : blockIdx.x % 8 + blockIdx.x / 8 / g.parts * 8;
  const int part = many ? blockIdx.x % g.parts : blockIdx.x / 8 % g.parts;
  if (tile >= g.row_tiles) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 32;
  uint8_t* scratch = reinterpret_cast<uint8_t*>(lds + 2 * g.steps * RT);
  float* scale = reinterpret_cast<float*>(scratch);
  const int64_t row0 = (int64_t)tile * RT;
  quantise_rows<T, RT, NU, LPR, WAVES>(g, row0, lds, scale);
  __syncthreads();
  float xs[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) xs[rb] = scale[rb * 32 + l];
  __syncthreads();   // the scratch holds the scales until here
  const int per = (g.units + g.parts - 1) / g.parts, u1 = (part + 1) * per < g.units ? (part + 1) * per : g.units;
  quant_units<T, RB>(g, lds, part * per + wave, u1, WAVES, xs, row0, scratch + wave * QUANT_SCRATCH);
}

// Few rows: 32 rows by 32 channels a workgroup, whose waves share the inputs out (every eighth step each) and add
// their sums in LDS: the weights' loads of a call are spread over the whole device and are in flight
// while the rows are quantised (by every workgroup for itself, from L2). Bound by latency: 16 x 1024 x 1024 bf16
// 5.4 us, of which an empty launch takes about half.
template <typename T, int NU, int LPR>
__global__ __launch_bounds__(QUANT_THREADS, 2) void quant_few(QuantArgs g) {
  extern __shared__ u32x4 lds[];
  const int nb = (int)((g.outer + 31) / 32), lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t row0 = (int64_t)(blockIdx.x / nb) * 32, n0 = (int64_t)(blockIdx.x % nb) * 32;
  const u32x4* w = reinterpret_cast<const u32x4*>(g.image) + (n0 / 32) * g.steps * 64 + lane;
  constexpr int U = 4;
  u32x4 b[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int s = wave + j * QUANT_WAVES;
    b[j] = w[(s < g.steps ? s : 0) * 64];
  }
  float* scale = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(lds) + (g.steps > QUANT_WAVES * 4 ? g.steps : QUANT_WAVES * 4) * 1024);
  quantise_rows<T, 32, NU, LPR, QUANT_WAVES>(g, row0, lds, scale);
  __syncthreads();
  i32x16 acc = {};
  for (int s0 = 0; s0 < g.steps; s0 += U * QUANT_WAVES) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int s = s0 + wave + j * QUANT_WAVES;
      if (s >= g.steps) continue;
      const u32x4 now = b[j];
      if (s + U * QUANT_WAVES < g.steps) b[j] = w[(s + U * QUANT_WAVES) * 64];
      const int k = 2 * s + lane / 32;
      const u32x4 x = lds[k * 32 + ((lane % 32) ^ (k & 7))];
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, now), __builtin_bit_cast(i32x4, x), acc, 0, 0, 0);
    }
  }
  __syncthreads();   // the rows are done with: their place takes the sums, [wave][row][channel]
  int32_t* sums = reinterpret_cast<int32_t*>(lds);
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<i32x4*>(sums + wave * 1024 + (lane % 32) * 32 + (((2 * q + lane / 32) ^ (lane & 7)) * 4)) =
        i32x4{acc[q * 4], acc[q * 4 + 1], acc[q * 4 + 2], acc[q * 4 + 3]};
  __syncthreads();
#pragma unroll
  for (int e = threadIdx.x; e < 1024; e += QUANT_THREADS) {
    const int r = e / 32, c = e % 32;
    int32_t t = 0;
#pragma unroll
    for (int i = 0; i < QUANT_WAVES; ++i) t += sums[i * 1024 + r * 32 + (((c / 4) ^ (r & 7)) * 4) + c % 4];
    const int64_t row = row0 + r, n = n0 + c;
    if (row < g.rows && n < g.outer)
      static_cast<T*>(g.y)[row * g.y_row + n] = from_f<T>(fmaf((float)t, scale[r] * g.w_scale[n], g.bias ? g.bias[n] : 0.0f));
  }
}

// A kernel's LDS limit, raised on each device once.
template <auto KERNEL> hipError_t quant_lds_limit() {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || (dev < 64 && (done.load() >> dev & 1))) return e;
  e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (e == hipSuccess && dev < 64) done.fetch_or((uint64_t)1 << dev);
  return e;
}

const char* quant_check(int32_t prec, int64_t rows, int64_t outer, int64_t inner) {
  if (!op_prec_ok(prec)) return "unknown precision";
  if (!op_extent_ok(rows) || !op_extent_ok(outer) || !op_extent_ok(inner)) return "extent out of range";
  if (inner > QUANT_MAX_INNER) return "inner above 131072";
  if (outer && rows > ((int64_t)1 << 40) / outer) return "rows * outer out of range";
  return nullptr;
}
// Calls whose rows stay in LDS (no inputs at all: the general path's loops, which then load nothing).
bool quant_in_lds(int64_t inner) { return inner > 0 && inner <= QUANT_LDS_INNER; }
int64_t quant_workspace(int64_t rows, int64_t inner) {   // q as fragments, then the scales
  if (quant_in_lds(inner)) return 0;
  return frag_blocks(rows) * frag_blocks(inner) * FRAG + op_div_up(rows, 4) * 16;
}

template <auto KERNEL> hipError_t quant_go(int64_t grid, size_t bytes, const QuantArgs& g, hipStream_t s, int threads = QUANT_THREADS) {
  if (bytes > 65536) {
    const hipError_t e = quant_lds_limit<KERNEL>();
    if (e != hipSuccess) return e;
  }
  KERNEL<<<dim3((unsigned)grid), threads, bytes, s>>>(g);
  return hipGetLastError();
}

// Rows of up to QUANT_LDS_INNER inputs, by what a compute unit gets (microseconds, bf16, both sides
// measured):
//   quant_few, while its 32 x 32 tiles are at most one a compute unit (64 x 2048 x 2048: 12 against 15 of
//     quant_wide; 512 x 512 x 2048, four each: 15 against 7);
//   quant_wide of 64 rows, two workgroups of four waves a compute unit (above 1024 inputs one of eight),
//     where LDS holds them and every compute unit gets rows or some 2^27 multiplications
//     (8192 x 1024 x 4096: 48 against 57 of 32 rows; 16384 x 2048 x 512: 33 against 45);
//   else of 32 rows (5000 x 1024 x 800: 16 against 19).
// Its channels are shared out over as many workgroups as run at once: one more a tile would be a second
// round (2000 x 4096 x 4001: 57 in 4 parts, 100 in 5).
template <typename T> hipError_t quant_launch_lds(QuantArgs g, hipStream_t s) {
  constexpr int64_t CUS = 256;
  const int64_t t32 = op_div_up(g.rows, 32), nb = op_div_up(g.outer, 32);
  const size_t unit32 = (size_t)g.steps * 1024;   // bytes of 32 rows
  if (t32 * nb <= CUS) {
    const size_t bytes = (g.steps > QUANT_WAVES * 4 ? g.steps : QUANT_WAVES * 4) * 1024 + 128;
    if (g.inner <= 256) return quant_go<quant_few<T, 1, 16>>(t32 * nb, bytes, g, s);
    if (g.inner <= 512) return quant_go<quant_few<T, 1, 32>>(t32 * nb, bytes, g, s);
    if (g.inner <= 1024) return quant_go<quant_few<T, 1, 64>>(t32 * nb, bytes, g, s);
    return quant_go<quant_few<T, 4, 64>>(t32 * nb, bytes, g, s);
  }
  g.units = (int)op_div_up(g.outer, 64);
  const bool two = g.inner <= 2048 && (g.rows > 64 * (CUS - 1) || t32 * g.units * g.steps >= 512 * CUS);
  const bool four = two && g.inner <= 1024;   // waves
  const int64_t tiles = op_div_up(g.rows, two ? 64 : 32), at_once = four ? 2 * CUS : CUS;
  g.row_tiles = (int)tiles;
  const int64_t most = at_once / tiles < g.units ? at_once / tiles : g.units, tiles8 = op_div_up(tiles, 8) * 8;
  g.parts = (int)(most >= 8 ? most / 8 * 8 : most < at_once / tiles8 ? most : at_once / tiles8);
  if (g.parts < 1) g.parts = 1;
  const int64_t grid = (g.parts >= 8 ? tiles : tiles8) * g.parts;
  const size_t bytes = unit32 * (two ? 2 : 1) + QUANT_SCRATCH * (four ? 4 : QUANT_WAVES);
  if (four && g.inner <= 256) return quant_go<quant_wide<T, 2, 1, 16, 4>>(grid, bytes, g, s, 256);
  if (four && g.inner <= 512) return quant_go<quant_wide<T, 2, 1, 32, 4>>(grid, bytes, g, s, 256);
  if (four) return quant_go<quant_wide<T, 2, 1, 64, 4>>(grid, bytes, g, s, 256);
  if (two) return quant_go<quant_wide<T, 2, 2, 64, QUANT_WAVES>>(grid, bytes, g, s);
  if (g.inner <= 256) return quant_go<quant_wide<T, 1, 1, 16, QUANT_WAVES>>(grid, bytes, g, s);
  if (g.inner <= 512) return quant_go<quant_wide<T, 1, 1, 32, QUANT_WAVES>>(grid, bytes, g, s);
  if (g.inner <= 1024) return quant_go<quant_wide<T, 1, 1, 64, QUANT_WAVES>>(grid, bytes, g, s);
  return quant_go<quant_wide<T, 1, 4, 64, QUANT_WAVES>>(grid, bytes, g, s);
}

template <typename T>
hipError_t quant_launch(int64_t rows, int64_t outer, int64_t inner, const void* x, int64_t x_row, const void* image,
                        const float* w_scale, const float* bias, void* y, int64_t y_row, void* ws, hipStream_t s) {
  const int64_t mb = frag_blocks(rows), nb = frag_blocks(outer), steps = frag_blocks(inner);
  if (quant_in_lds(inner)) {
    QuantArgs g{};
    g.x_row = x_row;
    g.image = static_cast<const int8_t*>(image); g.w_scale = w_scale; g.bias = bias;
    g.y_row = y_row;
    g.outer = outer; g.inner = (int)inner; g.steps = (int)steps;
    // A part of the rows at a time, such that its workgroups (512 threads for 32 rows at most) are one dispatch.
    constexpr int64_t PART = OP_DISPATCH / 512 * 32;
    hipError_t e = hipSuccess;
    for (int64_t r = 0; r < rows && e == hipSuccess; r += PART) {
      g.x = static_cast<const T*>(x) + r * x_row;
      g.y = static_cast<T*>(y) + r * y_row;
      g.rows = rows - r < PART ? rows - r : PART;
      e = quant_launch_lds<T>(g, s);
    }
    return e;
  }
  int8_t* q = static_cast<int8_t*>(ws);
  float* xs = reinterpret_cast<float*>(q + mb * steps * FRAG);
  op_dispatch(op_div_up(mb * 32, 4), 256, [&](int64_t first, dim3 grid) {
    quant_rows<T, true><<<grid, 256, 0, s>>>(static_cast<const T*>(x), x_row, rows, inner, q, 0, xs, first);
  });
  op_dispatch(op_div_up(mb * nb, 4), 256, [&](int64_t first, dim3 grid) {
    quant_product<T><<<grid, 256, 0, s>>>(q, static_cast<const int8_t*>(image), xs, w_scale, bias, static_cast<T*>(y), y_row, rows,
                                          outer, steps, first);
  });
  return hipGetLastError();
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
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  op_dispatch(op_div_up(rows, 4), 256, [&](int64_t first, dim3 grid) {
    if (prec == SPZ_PREC_BF16)
      quant_rows<bf16_t, false><<<grid, 256, 0, s>>>(static_cast<const bf16_t*>(x), x_row, rows, width, q, q_row, scale, first);
    else
      quant_rows<float, false><<<grid, 256, 0, s>>>(static_cast<const float*>(x), x_row, rows, width, q, q_row, scale, first);
  });
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
  if (bytes == 0) return SPZ_OK;
  op_dispatch(op_div_up(bytes, 256), 256, [&](int64_t first, dim3 grid) {
    quant_pack<<<grid, 256, 0, static_cast<hipStream_t>(hip_stream)>>>(q, q_row, outer, inner, static_cast<int8_t*>(image), first);
  });
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
  const hipError_t e = prec == SPZ_PREC_BF16
      ? quant_launch<bf16_t>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s)
      : quant_launch<float>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s);
  return e == hipSuccess ? SPZ_OK : op_error(SPZ_EHIP, call, hipGetErrorString(e));
}

}  // extern "C"
