// The 8-bit integer product with a scale for each row of the input and each output channel
// (spz_quant_*).
//
//   y[m, n] = s[m] w_scale[n] sum_k q[m, k] w[n, k] + bias[n],   s[m] = max_k |x[m, k]| / 127
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
__device__ inline uint32_t wave_max(uint32_t x) {
  x = dpp_max<0xB1>(x);    // neighbours, pairs, the halves of 16 lanes mirrored, the 16 mirrored
  x = dpp_max<0x4E>(x);
  x = dpp_max<0x141>(x);
  x = dpp_max<0x140>(x);
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = r[0] > r[1] ? r[0] : r[1];
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return r[0] > r[1] ? r[0] : r[1];
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

// ----------------------------------------------------------------------------- rows in LDS
constexpr int64_t QUANT_LDS_INNER = 4096;
constexpr int QUANT_THREADS = 512, QUANT_WAVES = QUANT_THREADS / 64;
constexpr int QUANT_SCRATCH = QUANT_WAVES * 4096;   // bytes of LDS beside the rows

struct QuantArgs {
  const void* x; int64_t x_row;
  const int8_t* image; const float* w_scale; const float* bias;
  void* y; int64_t y_row;
  int64_t rows, outer;
  int inner, steps;         // steps of 32 inputs
  int row_tiles, parts, units;  // quant_wide: units of 64 channels, shared out over `parts` workgroups
  bool y_vec, w_vec;        // 16-byte stores of y; 16-byte loads of w_scale and bias
};

// Sixteen elements over s, rounded to integers, as bytes. The quotient that counts is the correctly
// rounded x / s; x times the reciprocal differs from it by less than NEAR, so only where some
// element lies that near to a half is the division done (8% of the waves' sixteens).
constexpr float QUANT_MAGIC = 12582912.0f;   // 1.5 * 2^23: the sum's low byte is the rounded integer
__device__ inline u32x4 quantise16(const float (&x)[16], float s, float r) {
  constexpr float NEAR = 4e-5f;   // 127 (3 * 2^-24) + 2^-18 < 3e-5
  float t[16], far = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    t[i] = fmaf(x[i], r, QUANT_MAGIC);
    far = fmaxf(far, fabsf(fmaf(x[i], r, QUANT_MAGIC - t[i])));
  }
  if (!(far < 0.5f - NEAR) || s < 1e-30f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = (float)quantised(x[i], s) + QUANT_MAGIC;
  }
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

// Rows row0 .. row0 + RT - 1 of x into LDS: units of 16 inputs, unit k of row r at k RT + (r ^ (k & 7)), so
// that 32 rows of a unit are contiguous for the products and eight units of a row fall on different
// banks here. A wave has 4 / NU rows in flight, NU units (of inputs up to 1024 NU) a lane. What lies
// past a row's inputs within its last step meets zero weights, what lies past the rows is not stored.
template <typename T, bool VEC, int RT, int NU>
__device__ inline void quantise_rows(const QuantArgs& g, int64_t row0, u32x4* a, float* scale) {
  constexpr int RU = 4 / NU, PER = RT / QUANT_WAVES;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  for (int j0 = 0; j0 < PER; j0 += RU) {
    if (row0 + wave * PER + j0 >= g.rows) break;
    uint32_t m[RU];
    if constexpr (VEC) {
      constexpr int E = OP_VEC<T>, W = 16 / E;
      u32x4 raw[RU][NU][W];
#pragma unroll
      for (int j = 0; j < RU; ++j) {
        const int64_t row = row0 + wave * PER + j0 + j;
        const T* p = static_cast<const T*>(g.x) + (row < g.rows ? row : g.rows - 1) * g.x_row;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int k = 0; k < W; ++k) {
            raw[j][u][k] = u32x4{0, 0, 0, 0};
            const uint32_t c = (u * 64 + lane) * 16;
            if (c < (uint32_t)g.inner) raw[j][u][k] = *reinterpret_cast<const u32x4*>(p + c + k * E);
          }
      }
#pragma unroll
      for (int j = 0; j < RU; ++j) {
        m[j] = 0;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int k = 0; k < W; ++k) {
            float v[E];
            unpack(raw[j][u][k], v);
#pragma unroll
            for (int i = 0; i < E; ++i) {
              const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) & 0x7FFFFFFFu;
              m[j] = b > m[j] ? b : m[j];
            }
          }
        m[j] = wave_max(m[j]);
      }
#pragma unroll
      for (int j = 0; j < RU; ++j) {
        const int r = wave * PER + j0 + j;
        bool zero;
        const float s = row_scale(m[j], zero), inv = __builtin_amdgcn_rcpf(s);
        if (lane == 0) scale[r] = s;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const int k = u * 64 + lane;
          if (k >= 2 * g.steps) continue;
          float v[16];
#pragma unroll
          for (int q = 0; q < W; ++q) {
            float t[E];
            unpack(raw[j][u][q], t);
#pragma unroll
            for (int i = 0; i < E; ++i) v[q * E + i] = t[i];
          }
          a[k * RT + (r ^ (k & 7))] = zero ? u32x4{0, 0, 0, 0} : quantise16(v, s, inv);
        }
      }
    } else {
      float v[RU][NU * 16];
#pragma unroll
      for (int j = 0; j < RU; ++j) {
        const int64_t row = row0 + wave * PER + j0 + j;
        const T* p = static_cast<const T*>(g.x) + (row < g.rows ? row : g.rows - 1) * g.x_row;
        m[j] = 0;
#pragma unroll
        for (int i = 0; i < NU * 16; ++i) {
          const int c = i * 64 + lane;
          v[j][i] = c < g.inner ? to_f<T>(p[c]) : 0.0f;
        }
      }
#pragma unroll
      for (int j = 0; j < RU; ++j) {
        const int r = wave * PER + j0 + j;
#pragma unroll
        for (int i = 0; i < NU * 16; ++i) {
          const uint32_t b = __builtin_bit_cast(uint32_t, v[j][i]) & 0x7FFFFFFFu;
          m[j] = b > m[j] ? b : m[j];
        }
        bool zero;
        const float s = row_scale(wave_max(m[j]), zero), inv = __builtin_amdgcn_rcpf(s);
        if (lane == 0) scale[r] = s;
#pragma unroll
        for (int h = 0; h < NU; ++h) {
          float t[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) t[i] = v[j][h * 16 + i];
          const u32x4 w = zero ? u32x4{0, 0, 0, 0} : quantise16(t, s, inv);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = (h * 16 + i) * 64 + lane, k = c / 16;
            if (c < g.inner)
              reinterpret_cast<uint8_t*>(a + (k * RT + (r ^ (k & 7))))[c % 16] = (uint8_t)(w[i / 4] >> (i % 4 * 8));
          }
        }
      }
    }
  }
}

// y of RBW blocks of 32 rows by 64 channels a wave: lane l holds row l % 32 and, of each 32 channels, those
// of which bit 2 is l / 32; they go through 4 KB of LDS a wave to leave as whole 128-byte pieces of rows.
template <typename T, int RBW>
__device__ inline void quant_store(const QuantArgs& g, const i32x16 (&acc)[RBW][2], const float (&xs)[RBW], int64_t row0, int64_t n0,
                                   uint8_t* scratch) {
  const int lane = threadIdx.x % 64, l = lane % 32, h = lane / 32;
  constexpr int CB = 128 / (32 * (int)sizeof(T));   // channel blocks of 32 in a 128-byte piece
#pragma unroll
  for (int cb = 0; cb < 2; cb += CB) {
    float sw[CB][4][4], bn[CB][4][4];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t n = n0 + (cb + c) * 32 + q * 8 + h * 4;
        if (g.w_vec && n + 4 <= g.outer) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(g.w_scale + n);
          f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
          if (g.bias) b = *reinterpret_cast<const f32x4*>(g.bias + n);
#pragma unroll
          for (int i = 0; i < 4; ++i) { sw[c][q][i] = w[i]; bn[c][q][i] = b[i]; }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t e = n + i < g.outer ? n + i : g.outer - 1;
            sw[c][q][i] = g.w_scale[e];
            bn[c][q][i] = g.bias ? g.bias[e] : 0.0f;
          }
        }
      }
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb) {
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = fmaf((float)acc[rb][cb + c][q * 4 + i], xs[rb] * sw[c][q][i], bn[c][q][i]);
          if constexpr (sizeof(T) == 2) {
            const int unit = (c * 4 + q) ^ (l & 7);
            *reinterpret_cast<u32x2*>(scratch + l * 128 + unit * 16 + h * 8) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
          } else {
            const int unit = (2 * q + h) ^ (l & 7);
            *reinterpret_cast<u32x4*>(scratch + l * 128 + unit * 16) = pack(v);
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      constexpr int E = OP_VEC<T>, COLS = 8 * E;
      const int64_t base = n0 + cb * 32;
      if (g.y_vec) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = i * 8 + lane / 8, unit = lane % 8;
          const u32x4 w = *reinterpret_cast<const u32x4*>(scratch + r * 128 + ((unit ^ (r & 7)) * 16));
          const int64_t row = row0 + rb * 32 + r, n = base + unit * E;
          if (row < g.rows && n < g.outer) *reinterpret_cast<u32x4*>(static_cast<T*>(g.y) + row * g.y_row + n) = w;
        }
      } else {
        for (int e = lane; e < 32 * COLS; e += 64) {
          const int r = e / COLS, c = e % COLS;
          const T w = *reinterpret_cast<const T*>(scratch + r * 128 + ((c / E ^ (r & 7)) * 16) + c % E * sizeof(T));
          const int64_t row = row0 + rb * 32 + r, n = base + c;
          if (row < g.rows && n < g.outer) static_cast<T*>(g.y)[row * g.y_row + n] = w;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
}

// A workgroup: RB blocks of 32 rows and its part of the channels; its waves take RBW blocks by 64 channels
// at a time, each on its own once the rows are in LDS. 128 rows a workgroup (RB = RBW = 4) read the
// weights from L2 at half the rate at which the vector L1 delivers; with two products a fragment
// of x or four a fragment of weights LDS is at half its rate too.
template <typename T, bool VEC, int RB, int RBW, int NU>
__global__ __launch_bounds__(QUANT_THREADS, 2) void quant_wide(QuantArgs g) {
  extern __shared__ u32x4 lds[];
  constexpr int RT = RB * 32, WM = RB / RBW, WN = QUANT_WAVES / WM;
  // Workgroups of the same rows on one XCD (workgroup b runs on XCD b % 8).
  const int tile = blockIdx.x % 8 + blockIdx.x / 8 / g.parts * 8, part = blockIdx.x / 8 % g.parts;
  if (tile >= g.row_tiles) return;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = lane % 32, h = lane / 32;
  uint8_t* scratch = reinterpret_cast<uint8_t*>(lds + 2 * g.steps * RT);
  float* scale = reinterpret_cast<float*>(scratch);
  const int64_t row0 = (int64_t)tile * RT;
  quantise_rows<T, VEC, RT, NU>(g, row0, lds, scale);
  __syncthreads();
  const int wm = wave / WN, wn = wave % WN;
  float xs[RBW];
#pragma unroll
  for (int rb = 0; rb < RBW; ++rb) xs[rb] = scale[(wm * RBW + rb) * 32 + l];
  __syncthreads();   // the scratch holds the scales until here
  scratch += wave * (QUANT_SCRATCH / QUANT_WAVES);

  const int nb = (int)((g.outer + 31) / 32);
  const int per = (g.units + g.parts - 1) / g.parts, u1 = (part + 1) * per < g.units ? (part + 1) * per : g.units;
  // x fragments of step 4 s + j: unit 8 s + 2 j + h.
  const u32x4* ax[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) ax[j] = lds + (2 * j + h) * RT + ((wm * RBW * 32 + l) ^ (2 * j + h));
  for (int unit = part * per + wn; unit < u1; unit += WN) {
    const u32x4* w[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int n = unit * 2 + c < nb ? unit * 2 + c : nb - 1;
      w[c] = reinterpret_cast<const u32x4*>(g.image) + (int64_t)n * g.steps * 64;
    }
    i32x16 acc[RBW][2] = {};
    u32x4 b[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) b[j][c] = w[c][(j < g.steps ? j : 0) * 64 + lane];
    const auto step = [&](int s, int j) {
      u32x4 x[RBW];
#pragma unroll
      for (int rb = 0; rb < RBW; ++rb) x[rb] = ax[j][s * 2 * RT + rb * 32];
      u32x4 now[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        now[c] = b[j][c];
        if (s + j + 4 < g.steps) b[j][c] = w[c][(s + j + 4) * 64 + lane];
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb)
          acc[rb][c] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, now[c]), __builtin_bit_cast(i32x4, x[rb]), acc[rb][c], 0, 0, 0);
    };
    int s = 0;
    for (; s + 4 <= g.steps; s += 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) step(s, j);
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (s + j < g.steps) step(s, j);
    quant_store<T, RBW>(g, acc, xs, row0 + wm * RBW * 32, (int64_t)unit * 64, scratch);
  }
}

// Few rows: 32 rows by 32 channels a workgroup, whose waves share the inputs out (every eighth step each) and add
// their sums in LDS: the weights' loads of a call are spread over the whole device and are in flight
// while the rows are quantised (by every workgroup for itself, from L2).
template <typename T, bool VEC, int NU>
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
  float* scale = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(lds) + (2 * g.steps * 512 > QUANT_SCRATCH ? 2 * g.steps * 512 : QUANT_SCRATCH));
  quantise_rows<T, VEC, 32, NU>(g, row0, lds, scale);
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

template <auto KERNEL> hipError_t quant_go(int64_t grid, size_t bytes, const QuantArgs& g, hipStream_t s) {
  if (bytes > 65536) {
    const hipError_t e = quant_lds_limit<KERNEL>();
    if (e != hipSuccess) return e;
  }
  KERNEL<<<dim3((unsigned)grid), QUANT_THREADS, bytes, s>>>(g);
  return hipGetLastError();
}

// Rows of up to QUANT_LDS_INNER inputs. Few row tiles: quant_few's 32 x 32 tiles. Else the largest
// tile of rows that still gives every compute unit one (and fits LDS); tiles of 32 rows share the
// channels out over workgroups where there are too few of them.
template <typename T, bool VEC> hipError_t quant_launch_lds(QuantArgs g, hipStream_t s) {
  constexpr int64_t CUS = 256;
  const int64_t t32 = op_div_up(g.rows, 32), nb = op_div_up(g.outer, 32);
  const size_t unit32 = (size_t)g.steps * 1024;   // bytes of 32 rows
  if (t32 * op_div_up(g.outer, 512) < CUS / 2) {
    const size_t bytes = (unit32 > (size_t)QUANT_SCRATCH ? unit32 : (size_t)QUANT_SCRATCH) + 128;
    if (g.inner <= 1024) return quant_go<quant_few<T, VEC, 1>>(t32 * nb, bytes, g, s);
    return quant_go<quant_few<T, VEC, 4>>(t32 * nb, bytes, g, s);
  }
  const int rb = g.inner <= 1024 && g.rows > 128 * (CUS - 1) ? 4 : g.inner <= 2048 && g.rows > 64 * (CUS - 1) ? 2 : 1;
  const int64_t tiles = op_div_up(g.rows, rb * 32);
  g.row_tiles = (int)tiles;
  g.units = (int)op_div_up(g.outer, 64);
  g.parts = 1;
  while (tiles * g.parts < CUS && g.parts * QUANT_WAVES < g.units) ++g.parts;
  const int64_t grid = op_div_up(tiles, 8) * 8 * g.parts;
  const size_t bytes = unit32 * rb + QUANT_SCRATCH;
  if (rb == 4 && g.outer > 128) return quant_go<quant_wide<T, VEC, 4, 4, 1>>(grid, bytes, g, s);
  if (rb == 4) return quant_go<quant_wide<T, VEC, 4, 1, 1>>(grid, bytes, g, s);
  if (rb == 2 && g.inner <= 1024) return quant_go<quant_wide<T, VEC, 2, 2, 1>>(grid, bytes, g, s);
  if (rb == 2) return quant_go<quant_wide<T, VEC, 2, 2, 2>>(grid, bytes, g, s);
  if (g.inner <= 1024) return quant_go<quant_wide<T, VEC, 1, 1, 1>>(grid, bytes, g, s);
  return quant_go<quant_wide<T, VEC, 1, 1, 4>>(grid, bytes, g, s);
}

template <typename T>
hipError_t quant_launch(int64_t rows, int64_t outer, int64_t inner, const void* x, int64_t x_row, const void* image,
                        const float* w_scale, const float* bias, void* y, int64_t y_row, void* ws, hipStream_t s) {
  const int64_t mb = frag_blocks(rows), nb = frag_blocks(outer), steps = frag_blocks(inner);
  if (quant_in_lds(inner)) {
    constexpr int E = OP_VEC<T>;
    QuantArgs g{};
    g.x = x; g.x_row = x_row;
    g.image = static_cast<const int8_t*>(image); g.w_scale = w_scale; g.bias = bias;
    g.y = y; g.y_row = y_row;
    g.rows = rows; g.outer = outer; g.inner = (int)inner; g.steps = (int)steps;
    g.y_vec = outer % E == 0 && op_vec_ok(y, y_row, sizeof(T));
    g.w_vec = op_aligned(w_scale, 16) && op_aligned(bias, 16);
    if (inner % 16 == 0 && op_vec_ok(x, x_row, sizeof(T))) return quant_launch_lds<T, true>(g, s);
    return quant_launch_lds<T, false>(g, s);
  }
  int8_t* q = static_cast<int8_t*>(ws);
  float* xs = reinterpret_cast<float*>(q + mb * steps * FRAG);
  quant_rows<T, true><<<dim3((unsigned)op_div_up(mb * 32, 4)), 256, 0, s>>>(static_cast<const T*>(x), x_row, rows, inner, q, 0, xs);
  quant_product<T><<<dim3((unsigned)op_div_up(mb * nb, 4)), 256, 0, s>>>(q, static_cast<const int8_t*>(image), xs, w_scale, bias,
                                                                       static_cast<T*>(y), y_row, rows, outer, steps);
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
  const hipError_t e = prec == SPZ_PREC_BF16
      ? quant_launch<bf16_t>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s)
      : quant_launch<float>(rows, outer, inner, x, x_row, image, w_scale, bias, y, y_row, workspace, s);
  return e == hipSuccess ? SPZ_OK : op_error(SPZ_EHIP, call, hipGetErrorString(e));
}

}  // extern "C"
