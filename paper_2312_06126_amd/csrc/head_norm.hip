// Norms of each head of queries and keys, and their rotation by position, in one pass.
//
// A group of lanes takes a row and walks over its heads (or some of them, where there are few rows), so that the row's
// angles are taken once. Each lane holds pairs of columns that turn together: only the two sums of a norm cross lanes.
#include "ops.h"

namespace spz {
namespace {

constexpr int HEAD_MAX_DIM = 1024, HEAD_THREADS = 256, HEAD_WAVES = HEAD_THREADS / 64;
constexpr int64_t HEAD_BLOCKS = 1024;   // most workgroups of a backward call's queries or keys: each leaves a row of partial sums
constexpr int64_t HEAD_FILL = 4096;     // waves that fill the card: with fewer rows a row's heads are divided

// Queries or keys.
struct HeadPart {
  const void* x; int64_t x_row, x_head;
  const float *w, *b;
  const void* dy; int64_t dy_row, dy_head;   // backward
  void* out; int64_t out_row, out_head;      // forward: y; backward: dx
  int64_t heads, items;                      // items: rows times shares of the heads
  int64_t first, blocks;                     // its workgroups
  int share;                                 // heads of an item
};
struct HeadArgs {
  HeadPart part[2];
  const int32_t* positions;
  const double* freqs;
  const uint8_t* valid;
  float* sums;                               // backward: [workgroups, 2, dim]
  int64_t rows;
  int dim, pairs, norm, layout;
  float eps;
  bool whole;                                // every column turns
};

// Sum over groups of L lanes that follow each other.
template <int L> __device__ inline float group_sum(float x) {
  if constexpr (L >= 16) return L == 16 ? sum16(x) : L == 32 ? sum32(x) : sum64(x);
  x = dpp_add<0x4E>(dpp_add<0xB1>(x));
  return L == 8 ? dpp_add<0x141>(x) : x;
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

// Which share of its row's heads an item is (64-bit divisions are slow).
__device__ inline int64_t share_of(const HeadPart& p, int64_t rows, int64_t it) {
  if (p.items == rows) return 0;
  return p.items < (int64_t)1 << 32 ? (int64_t)((uint32_t)it / (uint32_t)rows) : it / rows;
}

// Any columns: a wave a row, lane l holds columns l, l + 64, .. and, of columns that turn, the partner's value as well,
// which it normalises itself.
template <typename T, int K, bool BACK> __global__ __launch_bounds__(HEAD_THREADS) void head_any(HeadArgs g, int64_t first) {
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
    const int64_t share = share_of(p, g.rows, it), row = it - share * g.rows;
    const int64_t h0 = share * p.share, h1 = h0 + p.share < p.heads ? h0 + p.share : p.heads;
    T* out = static_cast<T*>(p.out) + row * p.out_row;
    if (g.valid && !g.valid[row]) {
      if (p.out)
        for (int64_t h = h0; h < h1; ++h)
          for (int c = lane; c < D; c += 64) out[h * p.out_head + c] = from_f<T>(0.0f);
      continue;
    }
    float co[K], si[K];   // si: of the column's own value of the pair, so that y = y co + partner si
#pragma unroll
    for (int i = 0; i < K; ++i) {
      co[i] = 1.0f;
      si[i] = 0.0f;
      if (pair[i] >= 0) {
        turn_of(g.positions[row], g.freqs[pair[i]], co[i], si[i]);
        if (second[i] == BACK) si[i] = -si[i];
      }
    }
    for (int64_t h = h0; h < h1; ++h) {
      const T* x = static_cast<const T*>(p.x) + row * p.x_row + h * p.x_head;
      const T* dy = BACK ? static_cast<const T*>(p.dy) + row * p.dy_row + h * p.dy_head : nullptr;
      float n[K], q[K], d[K];
      float s1 = 0.0f;
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int c = lane + 64 * i;
        n[i] = c < D ? to_f<T>(x[c]) : 0.0f;
        q[i] = pair[i] >= 0 ? to_f<T>(BACK ? dy[other[i]] : x[other[i]]) : 0.0f;
        if (BACK) d[i] = c < D ? to_f<T>(dy[c]) : 0.0f;
        s1 += n[i];
      }
      float r = 1.0f;
      if (g.norm != SPZ_NORM_NONE) {
        const float mean = g.norm == SPZ_NORM_LAYER ? group_sum<64>(s1) * inv : 0.0f;
        float s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
          n[i] -= mean;
          if (!BACK) q[i] -= mean;
          s2 += lane + 64 * i < D ? n[i] * n[i] : 0.0f;
        }
        r = 1.0f / sqrtf(group_sum<64>(s2) * inv + g.eps);
      }
      if constexpr (!BACK) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
          const int c = lane + 64 * i;
          float y = fmaf(n[i] * r, w[i], b[i]);
          if (pair[i] >= 0) y = fmaf(y, co[i], fmaf(q[i] * r, wp[i], bp[i]) * si[i]);
          if (c < D) out[h * p.out_head + c] = from_f<T>(y);
        }
      } else {
        float a1 = 0.0f, a2 = 0.0f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
          n[i] = lane + 64 * i < D ? n[i] * r : 0.0f;
          if (pair[i] >= 0) d[i] = fmaf(d[i], co[i], q[i] * si[i]);   // turned back
          dw[i] = fmaf(d[i], n[i], dw[i]);
          db[i] += d[i];
          d[i] *= w[i];
          a1 += d[i];
          a2 = fmaf(d[i], n[i], a2);
        }
        if (p.out) {
          if (g.norm != SPZ_NORM_NONE) {
            a1 = g.norm == SPZ_NORM_LAYER ? group_sum<64>(a1) * inv : 0.0f;
            a2 = group_sum<64>(a2) * inv;
          } else {
            a1 = a2 = 0.0f;
          }
#pragma unroll
          for (int i = 0; i < K; ++i) {
            const int c = lane + 64 * i;
            if (c < D) out[h * p.out_head + c] = from_f<T>(r * (d[i] - fmaf(n[i], a2, a1)));
          }
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

// N elements at any alignment of the type, as loaded and as floats.
template <typename T, int N> struct Run {
  static constexpr int WORDS = (N * (int)sizeof(T) + 3) / 4;
  uint32_t w[WORDS];
  __device__ inline void load(const T* p) {
    if constexpr (N * sizeof(T) % 4) w[0] = (uint32_t)*reinterpret_cast<const uint16_t*>(p);
    else __builtin_memcpy(w, p, sizeof(w));
  }
  __device__ inline void clear() {
#pragma unroll
    for (uint32_t& u : w) u = 0;
  }
  __device__ inline void floats(float* x) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (sizeof(T) == 4) x[i] = __builtin_bit_cast(float, w[i % WORDS]);
      else x[i] = __builtin_bit_cast(float, (i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
  }
};
template <typename T, int N> __device__ inline void store_n(T* p, const float* x) {
  if constexpr (N == 1) {
    *p = from_f<T>(x[0]);
    return;
  }
  uint32_t w[(N * sizeof(T) + 3) / 4];
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T) / 4); ++i) {
    if (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, x[i]);
    else w[i] = pack_bf16x2(x[(2 * i) % N], x[(2 * i + 1) % N]);
  }
  __builtin_memcpy(p, w, sizeof(w));
}

// Columns in vectors: a group of L lanes a row, each lane two runs of SV columns, which turn together where pairs are
// halves (columns c .. and pairs + c ..) and by themselves where they are neighbours. SV = 1 takes any number of columns:
// the last lane's second one may not exist. The next head's columns are in flight while one is worked on.
// 65536 x (16 + 4) x 64 bf16: forward 76 us, 4.4 TB/s, backward 118, 4.3 TB/s: HBM. An angle costs some 70 instructions, a
// head 100: a wave a head each, with the angles taken for each of them, took 500 and 590 us.
template <typename T, int SV, int L, bool BACK> __global__ __launch_bounds__(HEAD_THREADS) void head_vectors(HeadArgs g, int64_t first) {
  constexpr int N = 2 * SV, GROUPS = HEAD_THREADS / L;
  const int j = threadIdx.x % L;
  const int64_t blk = first + blockIdx.x;
  const HeadPart& p = g.part[blk >= g.part[1].first];
  const int D = g.dim;
  const float inv = 1.0f / (float)D;
  const bool halves = g.layout == SPZ_PAIRS_HALVES, on = j * N < D, both = on && (SV > 1 || j * N + 1 < D);
  int ca = j * N, cb = ca + SV, pair = ca / 2, turning = SV;   // turning: the lane's pairs that turn
  if (halves) {
    if (j * SV < g.pairs) { ca = pair = j * SV; cb = g.pairs + ca; }
    else { ca = 2 * g.pairs + (j - g.pairs / SV) * N; cb = ca + SV; turning = 0; }
  } else {
    turning = g.pairs - pair < 0 ? 0 : g.pairs - pair < SV ? g.pairs - pair : SV;
  }
  float w[N], b[N], dw[N], db[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = i < SV ? ca + i : cb + i - SV;
    const bool is = i < SV ? on : both;
    w[i] = is && p.w ? p.w[c] : 1.0f;
    b[i] = is && p.b ? p.b[c] : 0.0f;
    dw[i] = db[i] = 0.0f;
  }
  const auto turn = [&](float (&x)[N], const float (&co)[SV], const float (&si)[SV]) {
#pragma unroll
    for (int i = 0; i < SV; ++i) {
      const int u = 2 * i, v = 2 * i + 1;   // of neighbours
      const float a = halves ? x[i] : x[u], z = halves ? x[SV + i] : x[v];
      const float na = fmaf(a, co[i], -(z * si[i])), nz = fmaf(a, si[i], z * co[i]);
      if (halves) {
        x[i] = g.whole || i < turning ? na : a;
        x[SV + i] = g.whole || i < turning ? nz : z;
      } else {
        x[u] = g.whole || i < turning ? na : a;
        x[v] = g.whole || i < turning ? nz : z;
      }
    }
  };
  for (int64_t it = (blk - p.first) * GROUPS + threadIdx.x / L; it < (p.items + GROUPS - 1) / GROUPS * GROUPS; it += p.blocks * GROUPS) {
    const bool item = it < p.items;   // whole waves stay together for the sums
    const int64_t share = !item ? 0 : share_of(p, g.rows, it), row = item ? it - share * g.rows : 0;
    const int64_t h0 = share * p.share;
    const int count = !item ? 0 : h0 + p.share < p.heads ? p.share : (int)(p.heads - h0);
    const bool live = item && (!g.valid || g.valid[row]);
    const T* x = static_cast<const T*>(p.x) + row * p.x_row + h0 * p.x_head;
    const T* dy = BACK ? static_cast<const T*>(p.dy) + row * p.dy_row + h0 * p.dy_head : nullptr;
    T* out = static_cast<T*>(p.out) + row * p.out_row + h0 * p.out_head;
    float n[N], d[N];
    Run<T, SV> next[2], next_d[2];
    const bool reads = live && on;
    const auto fetch = [&](int h) {
      if (reads && h < count) {
        next[0].load(x + h * p.x_head + ca);
        if (both) next[1].load(x + h * p.x_head + cb);
        if (BACK) {
          next_d[0].load(dy + h * p.dy_head + ca);
          if (both) next_d[1].load(dy + h * p.dy_head + cb);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      next[i].clear();
      next_d[i].clear();
    }
    fetch(0);
    float co[SV], si[SV];
#pragma unroll
    for (int i = 0; i < SV; ++i) {
      co[i] = 1.0f;
      si[i] = 0.0f;
    }
    if (g.pairs && live && on && turning) {
      const int32_t at = g.positions[row];
#pragma unroll
      for (int i = 0; i < SV; ++i)
        if (g.whole || i < turning) {
          turn_of(at, g.freqs[pair + i], co[i], si[i]);
          if (BACK) si[i] = -si[i];
        }
    }
    for (int h = 0; h < p.share; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        next[i].floats(n + i * SV);
        if (BACK) next_d[i].floats(d + i * SV);
      }
      fetch(h + 1);
      float r = 1.0f;
      if (g.norm != SPZ_NORM_NONE) {
        if (g.norm == SPZ_NORM_LAYER) {
          float s1 = 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i) s1 += n[i];
          const float mean = group_sum<L>(s1) * inv;
#pragma unroll
          for (int i = 0; i < N; ++i) n[i] = (i < SV ? on : both) ? n[i] - mean : 0.0f;
        }
        float s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s2 = fmaf(n[i], n[i], s2);
        r = 1.0f / sqrtf(group_sum<L>(s2) * inv + g.eps);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) n[i] *= r;
      if constexpr (!BACK) {
#pragma unroll
        for (int i = 0; i < N; ++i) n[i] = fmaf(n[i], w[i], b[i]);
        if (g.pairs) turn(n, co, si);
        if (on && h < count) {
          if (!live) {
#pragma unroll
            for (int i = 0; i < N; ++i) n[i] = 0.0f;
          }
          store_n<T, SV>(out + h * p.out_head + ca, n);
          if (both) store_n<T, SV>(out + h * p.out_head + cb, n + SV);
        }
      } else {
        if (g.pairs) turn(d, co, si);
        float a1 = 0.0f, a2 = 0.0f;
        const bool counts = reads && h < count;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (!counts) d[i] = n[i] = 0.0f;
          dw[i] = fmaf(d[i], n[i], dw[i]);
          db[i] += d[i];
          d[i] *= w[i];
          a1 += d[i];
          a2 = fmaf(d[i], n[i], a2);
        }
        if (p.out) {
          if (g.norm != SPZ_NORM_NONE) {
            a1 = g.norm == SPZ_NORM_LAYER ? group_sum<L>(a1) * inv : 0.0f;
            a2 = group_sum<L>(a2) * inv;
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = r * (d[i] - fmaf(n[i], a2, a1));
          }
          if (on && h < count) {
            if (!live) {
#pragma unroll
              for (int i = 0; i < N; ++i) d[i] = 0.0f;
            }
            store_n<T, SV>(out + h * p.out_head + ca, d);
            if (both) store_n<T, SV>(out + h * p.out_head + cb, d + SV);
          }
        }
      }
    }
  }
  if constexpr (BACK) {
    // The groups of a wave, then the waves.
    __shared__ float part[HEAD_WAVES][2][L * N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int m = L; m < 64; m <<= 1) {
        dw[i] += __shfl_xor(dw[i], m);
        db[i] += __shfl_xor(db[i], m);
      }
      if (threadIdx.x % 64 < L) {
        part[threadIdx.x / 64][0][i * L + j] = dw[i];
        part[threadIdx.x / 64][1][i * L + j] = db[i];
      }
    }
    __syncthreads();
    float* to = g.sums + blk * 2 * D;
    if (threadIdx.x < L && on)
      for (int i = 0; i < (both ? N : N - 1); ++i)
        for (int v = 0; v < 2; ++v) {
          float s = 0.0f;
          for (int k = 0; k < HEAD_WAVES; ++k) s += part[k][v][i * L + j];
          to[v * D + (i < SV ? ca + i : cb + i - SV)] = s;
        }
  }
}

// The workgroups' partial sums, in a fixed order: thread (column, group) takes every 16th row.
constexpr int HSUM_COLS = 64, HSUM_GROUPS = 16;
struct HeadSums { float* out[2][2]; int64_t first[2], blocks[2]; };
__global__ __launch_bounds__(HSUM_COLS* HSUM_GROUPS) void head_sums(const float* sums, HeadSums o, int dim) {
  __shared__ float part[HSUM_GROUPS][HSUM_COLS];
  const int col = threadIdx.x % HSUM_COLS, c = blockIdx.x * HSUM_COLS + col, grp = threadIdx.x / HSUM_COLS;
  const int which = blockIdx.y >> 1, v = blockIdx.y & 1;
  float* out = o.out[which][v];
  if (!out) return;
  float s = 0.0f;
  if (c < dim) {
    const float* from = sums + (o.first[which] * 2 + v) * dim + c;
#pragma unroll 8
    for (int64_t k = grp; k < o.blocks[which]; k += HSUM_GROUPS) s += from[k * 2 * dim];
  }
  part[grp][col] = s;
  __syncthreads();
  if (grp == 0 && c < dim) {
#pragma unroll
    for (int k = 1; k < HSUM_GROUPS; ++k) s += part[k][col];
    out[c] = s;
  }
}

// How columns are held: two runs of sv in each of `lanes`, or (sv 0) any columns by whole waves. Forward 16 bytes a run;
// backward 8, whose registers leave room for twice the waves (65536 x (16 + 4) x 64 bf16: 122 us against 132). Calls that do
// not fill the card take single columns: a lane then has one angle (16 x (4 + 4) x 64 bf16: 4.0 us against 7.0).
struct HeadWay { int sv, lanes; };
HeadWay head_way(const spz_head_norm_args& a, bool back) {
  const int vec = 16 / op_size(a.prec), wide = back ? vec / 2 : vec;
  const bool few = a.dim <= 128 && a.rows * (a.heads_q + a.heads_k) * (a.dim / 2) < HEAD_FILL * 64 / 2;
  for (const int sv : {wide, back ? vec : vec / 2})
    if (!few && a.dim > 0 && a.dim % (2 * sv) == 0 && a.dim / (2 * sv) <= 64 && (a.layout == SPZ_PAIRS_NEIGHBOURS || a.pairs % sv == 0)) {
      int lanes = 4;
      while (lanes * 2 * sv < a.dim) lanes *= 2;
      return {sv, lanes};
    }
  if (a.dim > 0 && a.dim <= 128) {
    int lanes = 4;
    while (lanes * 2 < a.dim) lanes *= 2;
    return {1, lanes};
  }
  return {0, 64};
}

// Items and workgroups of the parts. A row's heads are divided where whole rows are too few waves.
void head_spread(HeadArgs& g, const HeadWay& way, bool back) {
  const int groups = HEAD_THREADS / way.lanes;
  int64_t at = 0;
  for (HeadPart& p : g.part) {
    int64_t share = p.heads;
    while (share > 1 && g.rows * op_div_up(p.heads, share) * way.lanes < HEAD_FILL * 64) share = (share + 1) / 2;
    p.share = (int)share;
    p.items = share > 0 ? g.rows * op_div_up(p.heads, share) : 0;
    p.first = at;
    p.blocks = op_div_up(p.items, groups);
    if (back && p.blocks > HEAD_BLOCKS) p.blocks = HEAD_BLOCKS;
    at += p.blocks;
  }
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

// Arrays that workgroups of one launch read and write in any order. A head is read before it is written, so an output may take the
// place of its own part's input.
const char* head_check_shares(const spz_head_norm_args& a, bool back) {
  const int e = op_size(a.prec);
  const auto part = [&](const void* p, int64_t heads, int64_t row, int64_t head) { return OpArray{p, a.dim, {a.rows, heads, 1}, {row, head, 0}}; };
  const OpArray q = part(a.q, a.heads_q, a.q_row, a.q_head), k = part(a.k, a.heads_k, a.k_row, a.k_head);
  const OpArray dy = part(back ? a.dq_out : nullptr, a.heads_q, a.dq_out_row, a.dq_out_head), dz = part(back ? a.dk_out : nullptr, a.heads_k, a.dk_out_row, a.dk_out_head);
  const OpArray to_q = back ? part(a.dq, a.heads_q, a.dq_row, a.dq_head) : part(a.q_out, a.heads_q, a.q_out_row, a.q_out_head);
  const OpArray to_k = back ? part(a.dk, a.heads_k, a.dk_row, a.dk_head) : part(a.k_out, a.heads_k, a.k_out_row, a.k_out_head);
  if (op_shares(e, to_q, to_k)) return back ? "dq and dk share elements" : "q_out and k_out share elements";
  for (const OpArray* x : {&q, &dy})
    if ((!op_same(to_q, *x) && op_shares(e, to_q, *x)) || op_shares(e, to_k, *x)) return "an output shares elements with other places of q or dq_out";
  for (const OpArray* x : {&k, &dz})
    if ((!op_same(to_k, *x) && op_shares(e, to_k, *x)) || op_shares(e, to_q, *x)) return "an output shares elements with other places of k or dk_out";
  return nullptr;
}

void head_parts(const spz_head_norm_args& a, bool back, HeadArgs& g) {
  g.rows = a.rows;
  g.part[0] = {a.q, a.q_row, a.q_head, a.w_q, a.b_q, a.dq_out, a.dq_out_row, a.dq_out_head,
               back ? a.dq : a.q_out, back ? a.dq_row : a.q_out_row, back ? a.dq_head : a.q_out_head, a.heads_q, 0, 0, 0, 0};
  g.part[1] = {a.k, a.k_row, a.k_head, a.w_k, a.b_k, a.dk_out, a.dk_out_row, a.dk_out_head,
               back ? a.dk : a.k_out, back ? a.dk_row : a.k_out_row, back ? a.dk_head : a.k_out_head, a.heads_k, 0, 0, 0, 0};
}

template <typename T> __global__ void head_zero(HeadPart p, int dim, int64_t first) {
  const int64_t i = (first + blockIdx.x) * HEAD_THREADS + threadIdx.x;
  if (i >= p.items) return;
  const int64_t it = i / dim, row = it / p.heads;
  static_cast<T*>(p.out)[row * p.out_row + (it - row * p.heads) * p.out_head + (i - it * dim)] = from_f<T>(0.0f);
}

template <typename T, bool BACK> void head_launch(const HeadArgs& g, const HeadWay& way, hipStream_t s) {
  const int64_t blocks = g.part[1].first + g.part[1].blocks;
  using std::integral_constant;
  constexpr int VEC = OP_VEC<T>;
  const auto dispatch = [&](auto kernel) {
    op_dispatch(blocks, HEAD_THREADS, [&](int64_t first, dim3 grid) { kernel<<<grid, HEAD_THREADS, 0, s>>>(g, first); });
  };
  const auto lanes = [&](auto sv) {
    constexpr int SV = decltype(sv)::value;
    switch (way.lanes) {
      case 4: return dispatch(head_vectors<T, SV, 4, BACK>);
      case 8: return dispatch(head_vectors<T, SV, 8, BACK>);
      case 16: return dispatch(head_vectors<T, SV, 16, BACK>);
      case 32: return dispatch(head_vectors<T, SV, 32, BACK>);
      default: return dispatch(head_vectors<T, SV, 64, BACK>);
    }
  };
  if (way.sv == VEC) lanes(integral_constant<int, VEC>{});
  else if (way.sv == VEC / 2) lanes(integral_constant<int, VEC / 2>{});
  else if (way.sv) lanes(integral_constant<int, 1>{});
  else if (g.dim <= 64) dispatch(head_any<T, 1, BACK>);
  else if (g.dim <= 128) dispatch(head_any<T, 2, BACK>);
  else if (g.dim <= 256) dispatch(head_any<T, 4, BACK>);
  else if (g.dim <= 512) dispatch(head_any<T, 8, BACK>);
  else dispatch(head_any<T, 16, BACK>);
}

int head_run(const char* call, const spz_head_norm_args* args, bool back, void* ws, int64_t ws_bytes, void* stream) {
  const char* bad = head_check(args);
  if (!bad) bad = head_check_arrays(*args, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  const spz_head_norm_args& a = *args;
  const int64_t need = back ? spz_head_norm_workspace(args) : 0;
  if (need > 0 && (!ws || ws_bytes < need)) return op_error(SPZ_ESIZE, call, "workspace too small");
  if (need > 0 && !op_aligned(ws, 16)) return op_error(SPZ_EINVAL, call, "workspace not aligned to 16 bytes");
  bad = head_check_shares(a, back);
  if (bad) return op_error(SPZ_EINVAL, call, bad);
  HeadArgs g{};
  head_parts(a, back, g);
  g.positions = a.positions;
  g.freqs = a.freqs;
  g.valid = a.valid;
  g.dim = (int)a.dim;
  g.pairs = (int)a.pairs;
  g.norm = a.norm;
  g.layout = a.layout;
  g.whole = 2 * a.pairs == a.dim;
  g.eps = a.eps;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (back) {
    g.sums = static_cast<float*>(ws);
    for (HeadPart& p : g.part)
      if (!p.dy && p.heads > 0 && a.rows > 0) {   // no gradient comes in: zeros, and nothing for the kernel to do
        p.items = a.rows * p.heads * a.dim;
        if (p.out && p.items > 0)
          op_dispatch(op_div_up(p.items, HEAD_THREADS), HEAD_THREADS, [&](int64_t first, dim3 grid) {
            if (a.prec == SPZ_PREC_BF16) head_zero<bf16_t><<<grid, HEAD_THREADS, 0, s>>>(p, g.dim, first);
            else head_zero<float><<<grid, HEAD_THREADS, 0, s>>>(p, g.dim, first);
          });
        p.heads = 0;
      }
  }
  const HeadWay way = head_way(a, back);
  head_spread(g, way, back);
  const int64_t blocks = g.part[1].first + g.part[1].blocks;
  if (a.dim == 0 || (!back && blocks == 0)) return SPZ_OK;
  if (blocks > 0) {
    if (a.prec == SPZ_PREC_BF16) {
      if (back) head_launch<bf16_t, true>(g, way, s);
      else head_launch<bf16_t, false>(g, way, s);
    } else {
      if (back) head_launch<float, true>(g, way, s);
      else head_launch<float, false>(g, way, s);
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
  head_spread(g, head_way(*args, true), true);
  return (g.part[1].first + g.part[1].blocks) * 2 * args->dim * 4;
}

int spz_head_norm_forward(const spz_head_norm_args* args, void* hip_stream) {
  return head_run("spz_head_norm_forward", args, false, nullptr, 0, hip_stream);
}

int spz_head_norm_backward(const spz_head_norm_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return head_run("spz_head_norm_backward", args, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
