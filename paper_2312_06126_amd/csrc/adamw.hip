// AdamW over many tensors in one launch, with moments in 32 bits or in 8 bits with a scale for each 256 of them.
//
// The tensors' addresses travel as the kernel's argument, so that a call copies nothing to the device and can be
// captured. Eight elements a thread: a block of 256 moments is half a wave, whose largest magnitude takes five exchanges.
#include "ops.h"

namespace spz {
namespace {

constexpr int ADAM_THREADS = 256, ADAM_ELEMS = 8 * ADAM_THREADS, ADAM_TENSORS = 64;
constexpr uint32_t P_MOMENT = 6;
constexpr float E4M3_MAX = 448.0f;

struct AdamTensor { void* p; const void* g; uint16_t* copy; int64_t n, at; float decay; };
struct AdamArgs {
  AdamTensor t[ADAM_TENSORS];
  int64_t first[ADAM_TENSORS];          // each tensor's first workgroup (unused ones: past the last)
  void *m, *v; float *m_scale, *v_scale;
  const float *grad_scale, *lr_at; const int64_t* step_at;
  int64_t from;                         // workgroups of earlier dispatches
  double log_beta1, log_beta2;
  float lr, b1, c1, b2, c2, eps, fix1, fix2;   // c = 1 - b; fix1 = 1 / (1 - beta1^t), fix2 = 1 / sqrt(1 - beta2^t)
  uint64_t seed; uint32_t step;
};

// Eight elements, `cnt` of them real.
template <typename T> __device__ inline void load8(const T* p, int cnt, float (&x)[8]) {
  constexpr int VW = OP_VEC<T>;
  if (cnt == 8) {
#pragma unroll
    for (int j = 0; j < 8 / VW; ++j) {
      float v[VW];
      unpack(load16(p + j * VW), v);
#pragma unroll
      for (int i = 0; i < VW; ++i) x[j * VW + i] = v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < cnt ? to_f<T>(p[i]) : 0.0f;
  }
}
template <typename T> __device__ inline void store8(T* p, int cnt, const float (&x)[8]) {
  constexpr int VW = OP_VEC<T>;
  if (cnt == 8) {
#pragma unroll
    for (int j = 0; j < 8 / VW; ++j) {
      float v[VW];
#pragma unroll
      for (int i = 0; i < VW; ++i) v[i] = x[j * VW + i];
      store16(p + j * VW, pack(v));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cnt) p[i] = from_f<T>(x[i]);
  }
}

// Eight e4m3 codes as numbers, and numbers that are values of the type as codes.
__device__ inline void from_codes(const uint8_t* p, int cnt, float (&x)[8]) {
  uint32_t w[2] = {0, 0};
  if (cnt == 8) {
    __builtin_memcpy(w, p, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cnt) w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    x[4 * k + 0] = __builtin_amdgcn_cvt_f32_fp8(w[k], 0);
    x[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8(w[k], 1);
    x[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8(w[k], 2);
    x[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8(w[k], 3);
  }
}
__device__ inline void to_codes(uint8_t* p, int cnt, const float (&x)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k], x[4 * k + 1], 0, false);
    w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k + 2], x[4 * k + 3], u, true);
  }
  if (cnt == 8) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cnt) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// x >= 0, at most 448, up or down to a value of e4m3: adding 20 random bits below its three mantissa bits and cutting
// them off carries with the probability of the distance. Below 2^-6 the type's values are 2^-9 apart, as
// they are from 2^-6 to 2^-5.
__device__ inline float round_random(float x, uint32_t word) {
  const bool low = x < 0x1p-6f;
  const float y = low ? x + 0x1p-6f : x;
  const float z = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, y) + (word << 4) + 8u) & 0xFFF00000u);
  return low ? z - 0x1p-6f : z;
}

// The square root: the hardware's (an ulp) and a step of Newton's method, whose residual is exact to some 2^-46 of x. It is the correctly
// rounded one for each of float32's mantissas at an even and at an odd exponent (all 2^24 compared; others differ by powers of
// 4, which change nothing); a third of the library's instructions.
__device__ inline float root(float x) {
  if (!(x >= 0x1p-90f && x < 0x1p120f)) return sqrtf(x);
  const float y = __builtin_amdgcn_rsqf(x), s = x * y;
  return fmaf(fmaf(-s, s, x), 0.5f * y, s);
}
// x / y within two ulp.
__device__ inline float over(float x, float y) {
  return y >= 0x1p-100f && y <= 0x1p100f ? x * __builtin_amdgcn_rcpf(y) : x / y;
}
// x / y correctly rounded from y's correctly rounded reciprocal (Markstein 1990): the residual is exact.
__device__ inline float divided(float x, float y, float by) {
  const float q = x * by;
  return fmaf(fmaf(-q, y, x), by, q);
}

// The largest of a block's magnitudes (half a wave); a NaN stays one.
__device__ inline float block_max(const float (&x)[8]) {
  uint32_t m = 0;   // magnitudes order as their bits do, NaN above infinity
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu;
    m = u > m ? u : m;
  }
  m = max32(m);
  return __builtin_bit_cast(float, m);
}

// Bound by HBM: 53 million float32 elements with bfloat16 gradients and copies and 8-bit moments 157 us, 5.4 TB/s; 7.7 million
// with moments of 32 bits 36 us, 5.9 TB/s of arrays partly in the last-level cache. (Library quotients and roots: 214 us, by
// their instructions.) With the step on the device each thread takes the corrections itself, in 64 bits: in a replayed graph 176 us and not
// 162 of the 53 million, 35.8 and not 35.3 of the 7.7 million, 5.7 and not 5.3 of 0.2 million.
template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(ADAM_THREADS) void adamw_step(AdamArgs g) {
  const int64_t blk = g.from + blockIdx.x;
  // The tensor: a lane looks at each one's first workgroup.
  const int which = __popcll(__ballot(g.first[threadIdx.x % ADAM_TENSORS] <= blk)) - 1;
  const AdamTensor t = g.t[which];
  const int64_t i0 = (blk - g.first[which]) * ADAM_ELEMS + 8 * (int64_t)threadIdx.x;
  const int64_t left = t.n - i0;
  const int cnt = left >= 8 ? 8 : left > 0 ? (int)left : 0;
  float fix1 = g.fix1, fix2 = g.fix2, lr = g.lr;
  uint32_t step = g.step;
  if (g.step_at) {
    const int64_t n = *g.step_at;
    step = (uint32_t)n;
    fix1 = (float)(-1.0 / expm1((double)n * g.log_beta1));
    fix2 = (float)(1.0 / sqrt(-expm1((double)n * g.log_beta2)));
  }
  if (g.lr_at) lr = *g.lr_at;
  const float gs = g.grad_scale ? *g.grad_scale : 1.0f;
  float p[8], d[8], m[8], v[8];
  P* const pp = static_cast<P*>(t.p) + i0;
  load8<P>(pp, cnt, p);
  load8<G>(static_cast<const G*>(t.g) + i0, cnt, d);
  const int64_t e = t.at + i0;
  const int64_t scale = e / SPZ_ADAMW_BLOCK;
  if constexpr (EIGHT) {
    from_codes(static_cast<const uint8_t*>(g.m) + e, cnt, m);
    from_codes(static_cast<const uint8_t*>(g.v) + e, cnt, v);
    const float sm = cnt ? g.m_scale[scale] : 0.0f, sv = cnt ? g.v_scale[scale] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = i < cnt ? m[i] * sm : 0.0f;
      v[i] = i < cnt ? v[i] * sv : 0.0f;
      v[i] *= v[i];
    }
  } else {
    load8<float>(static_cast<const float*>(g.m) + e, cnt, m);
    load8<float>(static_cast<const float*>(g.v) + e, cnt, v);
  }
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    {   // one rounding an operation, as the definition of the codes has it
#pragma clang fp contract(off)
      const float x = d[i] * gs;
      m[i] = g.b1 * m[i] + g.c1 * x;
      v[i] = g.b2 * v[i] + g.c2 * x * x;
    }
    r[i] = root(v[i]);
    p[i] = fmaf(-lr, fmaf(t.decay, p[i], over(m[i] * fix1, fmaf(r[i], fix2, g.eps))), p[i]);
  }
  store8<P>(pp, cnt, p);
  if (t.copy) store8<bf16_t>(reinterpret_cast<bf16_t*>(t.copy) + i0, cnt, p);
  if constexpr (EIGHT) {
    const float big_m = block_max(m), big_r = block_max(r);
    const bool fine_m = big_m < __builtin_inff(), fine_r = big_r < __builtin_inff();
    const float sm = fine_m ? big_m * (1.0f / E4M3_MAX) : __builtin_nanf(""), sr = fine_r ? big_r * (1.0f / E4M3_MAX) : __builtin_nanf("");
    if (cnt && threadIdx.x % (SPZ_ADAMW_BLOCK / 8) == 0) {
      g.m_scale[scale] = sm;
      g.v_scale[scale] = sr;
    }
    if (!cnt) return;
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint64_t b = (uint64_t)(e >> 2) + k;
      const U4 u = philox_words(U4{(uint32_t)b, step, P_MOMENT + ((uint32_t)(b >> 32) << 8), 0u}, g.seed);
      w[4 * k] = u.x; w[4 * k + 1] = u.y; w[4 * k + 2] = u.z; w[4 * k + 3] = u.w;
    }
    // Both sides of tiny scales are raised: a reciprocal below would not be a number of the type.
    const float up_m = sm < 0x1p-60f ? 0x1p60f : 1.0f, up_r = sr < 0x1p-60f ? 0x1p60f : 1.0f;
    const float high_m = sm * up_m, high_r = sr * up_r, by_m = 1.0f / high_m, by_r = 1.0f / high_r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = sm > 0.0f ? fminf(divided(__builtin_fabsf(m[i]) * up_m, high_m, by_m), E4M3_MAX) : 0.0f;
      const float y = sr > 0.0f ? fminf(divided(r[i] * up_r, high_r, by_r), E4M3_MAX) : 0.0f;
      m[i] = __builtin_copysignf(round_random(x, w[i] & 0xFFFFu), m[i]);
      const float z = round_random(y, w[i] >> 16);
      r[i] = r[i] > 0.0f && sr > 0.0f ? fmaxf(z, 0x1p-9f) : z;
    }
    to_codes(static_cast<uint8_t*>(g.m) + e, cnt, m);
    to_codes(static_cast<uint8_t*>(g.v) + e, cnt, r);
  } else {
    store8<float>(static_cast<float*>(g.m) + e, cnt, m);
    store8<float>(static_cast<float*>(g.v) + e, cnt, v);
  }
}

const char* adam_check(const spz_adamw_args* p) {
  if (!p) return "NULL arguments";
  const spz_adamw_args& a = *p;
  if (!op_prec_ok(a.p_prec) || !op_prec_ok(a.g_prec)) return "unknown precision";
  if (a.bits != 32 && a.bits != 8) return "bits are 8 or 32";
  if (a.reserved != 0) return "reserved is not 0";
  if (!op_extent_ok(a.count)) return "count out of range";
  if (a.moments < 0 || a.moments > (int64_t)1 << 40 || a.moments % SPZ_ADAMW_BLOCK) return "moments out of range or no multiple of a block";
  if (!(a.beta1 >= 0.0 && a.beta1 < 1.0) || !(a.beta2 >= 0.0 && a.beta2 < 1.0)) return "a beta outside [0, 1)";
  if (!(a.eps >= 0.0 && a.eps < 3.0e38)) return "eps out of range";
  if (!a.lr_at && !(__builtin_fabs(a.lr) < 3.0e38)) return "lr is not finite";
  if (!a.step_at && a.step < 1) return "step below 1";
  if (a.count > 0 && !a.tensors) return "NULL tensors";
  if (a.moments > 0 && (!a.m || !a.v)) return "NULL m or v";
  if (a.moments > 0 && a.bits == 8 && (!a.m_scale || !a.v_scale)) return "NULL m_scale or v_scale";
  const size_t e = a.bits == 8 ? 8 : 16;
  if (!op_aligned(a.m, e) || !op_aligned(a.v, e)) return "m or v not aligned (8 bits: 8 bytes, 32 bits: 16)";
  for (const void* q : {(const void*)a.m_scale, (const void*)a.v_scale, (const void*)a.grad_scale, (const void*)a.lr_at})
    if (!op_aligned(q, 4)) return "scale or rate not aligned to 4 bytes";
  if (!op_aligned(a.step_at, 8)) return "step_at not aligned to 8 bytes";
  for (int64_t i = 0; i < a.count; ++i) {
    const spz_adamw_tensor& t = a.tensors[i];
    if (t.n < 0 || t.at < 0 || t.at % SPZ_ADAMW_BLOCK || t.at > a.moments || t.n > a.moments - t.at) return "a tensor's elements outside the moments";
    if (t.n > 0 && (!t.p || !t.g)) return "NULL p or g";
    if (!op_aligned(t.p, op_size(a.p_prec)) || !op_aligned(t.g, op_size(a.g_prec)) || !op_aligned(t.copy, 2)) return "array not aligned to its type";
    if (!(__builtin_fabs(t.weight_decay) < 3.0e38)) return "weight_decay is not finite";
  }
  return nullptr;
}

template <typename P, typename G> void adam_launch(AdamArgs& g, bool eight, int64_t blocks, hipStream_t s) {
  op_dispatch(blocks, ADAM_THREADS, [&](int64_t first, dim3 grid) {
    g.from = first;
    if (eight) adamw_step<P, G, true><<<grid, ADAM_THREADS, 0, s>>>(g);
    else adamw_step<P, G, false><<<grid, ADAM_THREADS, 0, s>>>(g);
  });
}

}  // namespace
}  // namespace spz

using namespace spz;

extern "C" {

int spz_adamw(const spz_adamw_args* args, void* hip_stream) {
  const char* bad = adam_check(args);
  if (bad) return op_error(SPZ_EINVAL, "spz_adamw", bad);
  const spz_adamw_args& a = *args;
  AdamArgs g{};
  g.m = a.m;
  g.v = a.v;
  g.m_scale = a.m_scale;
  g.v_scale = a.v_scale;
  g.grad_scale = a.grad_scale;
  g.lr_at = a.lr_at;
  g.step_at = a.step_at;
  g.log_beta1 = log(a.beta1);
  g.log_beta2 = log(a.beta2);
  g.lr = (float)a.lr;
  g.b1 = (float)a.beta1;
  g.c1 = (float)(1.0 - a.beta1);
  g.b2 = (float)a.beta2;
  g.c2 = (float)(1.0 - a.beta2);
  g.eps = (float)a.eps;
  if (!a.step_at) {
    g.fix1 = (float)(-1.0 / expm1((double)a.step * g.log_beta1));
    g.fix2 = (float)(1.0 / sqrt(-expm1((double)a.step * g.log_beta2)));
  }
  g.seed = a.seed;
  g.step = (uint32_t)a.step;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  int64_t i = 0;
  bool some = false;
  while (i < a.count) {   // as many tensors as the argument holds
    int n = 0;
    int64_t blocks = 0;
    for (; i < a.count && n < ADAM_TENSORS; ++i) {
      const spz_adamw_tensor& t = a.tensors[i];
      if (t.n == 0) continue;
      g.t[n] = {t.p, t.g, t.copy, t.n, t.at, (float)t.weight_decay};
      g.first[n++] = blocks;
      blocks += op_div_up(t.n, ADAM_ELEMS);
    }
    for (int k = n; k < ADAM_TENSORS; ++k) g.first[k] = INT64_MAX;
    if (n == 0) break;
    some = true;
    if (a.p_prec == SPZ_PREC_BF16) {
      if (a.g_prec == SPZ_PREC_BF16) adam_launch<bf16_t, bf16_t>(g, a.bits == 8, blocks, s);
      else adam_launch<bf16_t, float>(g, a.bits == 8, blocks, s);
    } else {
      if (a.g_prec == SPZ_PREC_BF16) adam_launch<float, bf16_t>(g, a.bits == 8, blocks, s);
      else adam_launch<float, float>(g, a.bits == 8, blocks, s);
    }
  }
  return some ? op_launched("spz_adamw") : SPZ_OK;
}

}  // extern "C"
