// One AdamW step over many tensors (include/snn_ops.h), moments in 32 bits or in 8:
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// Bound by memory: 28 bytes a parameter with everything in fp32, 16.1 with 8-bit moments.  The tensors' addresses
// travel as kernel arguments, up to TENSORS in a launch, so a step needs no table on the device and no copy; a
// workgroup finds its tensor by bisection over the chunk numbers.  A thread takes four neighbouring elements: with more
// of them a thread, fewer threads hide the loads (four elements, eight, sixteen: 79 million parameters in 32 bits 403,
// 412 and 421 us, 5.5 TB/s the first; in 8 bits with bfloat16 gradients 230, 241 and 260 us, 4.8 TB/s; 7.6 million in 8
// bits 28, 30 and 34 us).
// Every operation is rounded by itself (no contraction), so that the codes of 8-bit moments do not depend on how the
// compiler joins operations.
// With 8-bit moments the arithmetic counts as well (the random bits, two roundings, the scales: 38 us for 7.6 million
// parameters, sixteen a thread, when root and quotient were the correctly rounded ones, ten operations more each; 34 so).  There the roots
// of single elements and the quotient come from the hardware's approximations, one unit of the last place off: the
// parameter feels 2^-23 of its update, and a code does not feel it, since a root taken for just below a code or just
// above goes to that code with a chance next to 1 from either side.  The root that the scale goes by is exact.
#include "seq_common.hpp"

#include <math.h>

namespace snn {
namespace {

constexpr int TENSORS = 76;
constexpr int CHUNK = 1024;          // elements of a workgroup

struct AdamP {
  float *param[TENSORS];
  const void *grad[TENSORS];
  __bf16 *copy[TENSORS];
  int64_t n[TENSORS], at[TENSORS];
  float keep[TENSORS];               // 1 - lr wd
  int first[TENSORS + 1];            // first chunk
  int count;
  void *m, *v;
  float *m_scale, *v_scale;
  float b1, c1, b2, c2, k1, k2, eps, grad_scale;   // c = 1 - b
  uint32_t salt;
};
static_assert(sizeof(AdamP) <= 4096, "kernel arguments");

// 32 bits of a counter, stirred: multiplications by the odd numbers next to 2^31 sqrt(2) and 2^31 sqrt(3), each
// followed by the high bits folded onto the low ones.
__host__ __device__ __forceinline__ uint32_t stir(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xB504F335u;
  x = (x ^ (x >> 15)) * 0xDDB3D743u;
  return x ^ (x >> 16);
}

template <int L> __device__ __forceinline__ float max_neighbours(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  if constexpr (L == 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
  }
  return v;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponent of the least power of two s with top <= 448 s = 1.75 * 2^8 s, from -60 up: the mantissa's bits above 1.75
// carry into the exponent.
__device__ __forceinline__ int scale_exponent(float top) { return max(-60, (int)((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 127 - 8); }

// The 8-bit code below or above the magnitude r >= 0 (in units of the scale): `low` steps of 2^(e-3) in the binade
// of exponent e, from -6 up; below that the steps stay, as subnormal numbers.
struct Grid {
  int e;
  float low;
};
__device__ __forceinline__ Grid grid_of(float r, float *frac) {
#pragma clang fp contract(off)
  Grid g;
  g.e = max(-6, (int)(__float_as_uint(r) >> 23) - 127);
  const float a = r * power2(3 - g.e);
  g.low = floorf(a);
  *frac = a - g.low;
  return g;
}
__device__ __forceinline__ uint32_t code_of(const Grid &g, bool up) { return (uint32_t)((g.e + 6) * 8 + (int)g.low + (up ? 1 : 0)); }

__device__ __forceinline__ uint32_t code_m(float m, float inverse, uint32_t rand) {
#pragma clang fp contract(off)
  if (!finite(m)) return 0x7Fu;
  const float y = m * inverse;
  float frac;
  const Grid g = grid_of(fabsf(y), &frac);
  const float chance = ((float)(rand & 0xFFFFu) + 0.5f) * (1.f / 65536.f);
  return code_of(g, chance < frac) | (y < 0.f ? 0x80u : 0u);
}
// The root of v is coded; up with the chance that keeps the mean of v itself, (w - lo^2) / (hi^2 - lo^2).
__device__ __forceinline__ uint32_t code_v(float v, float root, float inverse, uint32_t rand) {
#pragma clang fp contract(off)
  if (!finite(v)) return 0x7Fu;
  const float w = (v * inverse) * inverse;
  float frac;
  const Grid g = grid_of(root * inverse, &frac);
  const float step = power2(g.e - 3), lo = g.low * step, hi = (g.low + 1.f) * step;
  const float chance = ((float)(rand >> 16) + 0.5f) * (1.f / 65536.f);
  const float lo2 = lo * lo, hi2 = hi * hi;
  const bool up = chance * (hi2 - lo2) < w - lo2 || (w > 0.f && g.e == -6 && g.low == 0.f);
  return code_of(g, up);
}

// Four elements from i on, of n; zeros beyond.
template <typename T> __device__ __forceinline__ void take4(float r[4], const T *p, int64_t i, int64_t n, bool vec) {
  if (vec && i + 4 <= n) {
    const Pack<T, 4> q = *(const Pack<T, 4> *)(p + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = widen(q.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = i + j < n ? widen(p[i + j]) : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void give4(T *p, const float r[4], int64_t i, int64_t n, bool vec) {
  if (vec && i + 4 <= n) {
    Pack<T, 4> q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q.v[j] = narrow<T>(r[j]);
    *(Pack<T, 4> *)(p + i) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) p[i + j] = narrow<T>(r[j]);
  }
}

template <typename G, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamP p) {
#pragma clang fp contract(off)
  int lo = 0, hi = p.count;                                // first[lo] <= block < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int)blockIdx.x >= p.first[mid]) lo = mid; else hi = mid;
  }
  const int64_t n = p.n[lo], at = p.at[lo];
  float *param = p.param[lo];
  const G *grad = (const G *)p.grad[lo];
  __bf16 *copy = p.copy[lo];
  const float keep = p.keep[lo];
  const bool vp = ((uintptr_t)param & 15) == 0, vg = ((uintptr_t)grad & (4 * sizeof(G) - 1)) == 0, vc = ((uintptr_t)copy & 7) == 0;
  const int64_t i = (int64_t)(blockIdx.x - p.first[lo]) * CHUNK + threadIdx.x * 4;

  float w[4] = {0.f, 0.f, 0.f, 0.f}, g[4] = {0.f, 0.f, 0.f, 0.f}, m[4], v[4], root[4];
  if constexpr (BITS == 32) {
    if (i >= n) return;
    take4(w, (const float *)param, i, n, vp);
    take4(g, grad, i, n, vg);
    take4(m, (const float *)p.m + at, i, n, true);         // (at: a multiple of SNN_ADAMW_BLOCK)
    take4(v, (const float *)p.v + at, i, n, true);
  } else {
    // a lane beyond the tensor has no element of the block and only takes part in its maxima
    uint32_t cm = 0, cv = 0;
    float sm = 1.f, sv = 1.f;
    if (i < n) {
      take4(w, (const float *)param, i, n, vp);
      take4(g, grad, i, n, vg);
      cm = *(const uint32_t *)((const uint8_t *)p.m + at + i);
      cv = *(const uint32_t *)((const uint8_t *)p.v + at + i);
      sm = p.m_scale[(at + i) / SNN_ADAMW_BLOCK];
      sv = p.v_scale[(at + i) / SNN_ADAMW_BLOCK];
    }
    m[0] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 0); m[1] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 1);
    m[2] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 2); m[3] = __builtin_amdgcn_cvt_f32_fp8((int)cm, 3);
    v[0] = __builtin_amdgcn_cvt_f32_fp8((int)cv, 0); v[1] = __builtin_amdgcn_cvt_f32_fp8((int)cv, 1);
    v[2] = __builtin_amdgcn_cvt_f32_fp8((int)cv, 2); v[3] = __builtin_amdgcn_cvt_f32_fp8((int)cv, 3);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] *= sm;
      const float r = v[j] * sv;
      v[j] = r * r;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float gj = g[j] * p.grad_scale;
    m[j] = m[j] * p.b1 + gj * p.c1;
    v[j] = v[j] * p.b2 + (gj * gj) * p.c2;
    if constexpr (BITS == 8) {
      root[j] = __builtin_amdgcn_sqrtf(v[j]);
      w[j] = w[j] * keep - (m[j] * p.k1) * rcp_fast(root[j] * p.k2 + p.eps);
    } else {
      root[j] = sqrtf(v[j]);
      w[j] = w[j] * keep - (m[j] * p.k1) / (root[j] * p.k2 + p.eps);
    }
  }
  if constexpr (BITS == 8) {
    // 32 lanes hold a block: its largest finite magnitudes give the scales
    float tm = 0.f, tv = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i + j >= n) { m[j] = 0.f; v[j] = 0.f; root[j] = 0.f; }
      tm = fmaxf(tm, finite(m[j]) ? fabsf(m[j]) : 0.f);
      tv = fmaxf(tv, finite(v[j]) ? v[j] : 0.f);
    }
    const int em = scale_exponent(max_neighbours<32>(tm)), ev = scale_exponent(sqrtf(max_neighbours<32>(tv)));
    const float im = power2(-em), iv = power2(-ev);
    uint32_t qm = 0, qv = 0;
    const int64_t where = at + i;                          // (a multiple of four)
    const uint32_t first = (uint32_t)where * 0x9E3779B1u + (uint32_t)(where >> 32) * 0xC2B2AE3Du + p.salt;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t rand = stir(first + j * 0x9E3779B1u);
      qm |= code_m(m[j], im, rand) << (8 * j);
      qv |= code_v(v[j], root[j], iv, rand) << (8 * j);
    }
    if (i >= n) return;
    *(uint32_t *)((uint8_t *)p.m + where) = qm;
    *(uint32_t *)((uint8_t *)p.v + where) = qv;
    if ((threadIdx.x & 31) == 0) {
      p.m_scale[where / SNN_ADAMW_BLOCK] = power2(em);
      p.v_scale[where / SNN_ADAMW_BLOCK] = power2(ev);
    }
  } else {
    give4((float *)p.m + at, m, i, n, true);
    give4((float *)p.v + at, v, i, n, true);
  }
  give4(param, w, i, n, vp);
  if (copy) give4(copy, w, i, n, vc);
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" int32_t snn_adamw_step(const snn_adamw_args *a, const snn_adamw_tensor *tensors, int32_t count, void *stream) {
  if (!a || (count > 0 && !tensors)) return ops_fail(SNN_ERR_NULL, "AdamW: arguments are NULL");
  if (count < 0) return ops_fail(SNN_ERR_ARG, "AdamW: count must not be negative");
  if (a->bits != 32 && a->bits != 8) return ops_fail(SNN_ERR_ARG, "AdamW: bits must be 32 or 8");
  if (a->grad_type != SNN_TYPE_FP32 && a->grad_type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "AdamW: unknown type %d", a->grad_type);
  if (a->step < 1) return ops_fail(SNN_ERR_ARG, "AdamW: step must be 1 or more");
  if (!(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1)) return ops_fail(SNN_ERR_ARG, "AdamW: beta1 and beta2 must be in [0, 1)");
  if (!(a->eps >= 0) || !isfinite(a->eps) || !isfinite(a->lr) || !isfinite(a->grad_scale)) return ops_fail(SNN_ERR_ARG, "AdamW: lr, eps and grad_scale must be finite, eps not negative");
  if (!a->m || !a->v || (a->bits == 8 && (!a->m_scale || !a->v_scale))) return ops_fail(SNN_ERR_NULL, "AdamW: a moment buffer is NULL");
  if (!aligned(a->m, 16) || !aligned(a->v, 16) || !aligned(a->m_scale, 4) || !aligned(a->v_scale, 4)) return ops_fail(SNN_ERR_ARG, "AdamW: m and v must be 16-byte aligned");
  for (int i = 0; i < count; ++i) {
    const snn_adamw_tensor &t = tensors[i];
    if (t.n < 0 || t.n > (1ll << 33) || t.at < 0 || t.at % SNN_ADAMW_BLOCK) return ops_fail(SNN_ERR_ARG, "AdamW: tensor %d: n must be 0 to 2^33, at a multiple of %d", i, SNN_ADAMW_BLOCK);
    if (!t.n) continue;
    if (!t.param || !t.grad) return ops_fail(SNN_ERR_NULL, "AdamW: tensor %d: param or grad is NULL", i);
    if (!aligned(t.param, 4) || !aligned(t.grad, a->grad_type == SNN_TYPE_FP32 ? 4 : 2) || !aligned(t.copy, 2)) return ops_fail(SNN_ERR_ARG, "AdamW: tensor %d: a pointer is not aligned to its element type", i);
    if (!isfinite(t.weight_decay)) return ops_fail(SNN_ERR_ARG, "AdamW: tensor %d: weight_decay must be finite", i);
  }
  AdamP p;
  p.m = a->m; p.v = a->v; p.m_scale = a->m_scale; p.v_scale = a->v_scale;
  p.b1 = (float)a->beta1; p.c1 = (float)(1 - a->beta1);
  p.b2 = (float)a->beta2; p.c2 = (float)(1 - a->beta2);
  p.k1 = (float)(a->lr / (1 - pow(a->beta1, (double)a->step)));
  p.k2 = (float)(1 / sqrt(1 - pow(a->beta2, (double)a->step)));
  p.eps = (float)a->eps; p.grad_scale = (float)a->grad_scale;
  p.salt = stir(a->seed * 0x9E3779B1u + (uint32_t)a->step * 0x85EBCA77u);
  p.count = 0;
  p.first[0] = 0;
  for (int i = 0; i <= count; ++i) {
    const bool end = i == count;
    const int64_t chunks = end ? 0 : (tensors[i].n + CHUNK - 1) / CHUNK;
    if (!end && !chunks) continue;
    if (p.count && (end || p.count == TENSORS || p.first[p.count] + chunks > (1 << 23))) {
      const dim3 grid(p.first[p.count]), block(256);
      const hipStream_t st = (hipStream_t)stream;
      const bool wide = a->grad_type == SNN_TYPE_FP32;
      if (a->bits == 32 && wide) hipLaunchKernelGGL((adamw_kernel<float, 32>), grid, block, 0, st, p);
      else if (a->bits == 32) hipLaunchKernelGGL((adamw_kernel<__bf16, 32>), grid, block, 0, st, p);
      else if (wide) hipLaunchKernelGGL((adamw_kernel<float, 8>), grid, block, 0, st, p);
      else hipLaunchKernelGGL((adamw_kernel<__bf16, 8>), grid, block, 0, st, p);
      const int rc = ops_launched("AdamW");
      if (rc) return rc;
      p.count = 0;
    }
    if (end) break;
    const snn_adamw_tensor &t = tensors[i];
    const int k = p.count++;
    p.param[k] = t.param; p.grad[k] = t.grad; p.copy[k] = (__bf16 *)t.copy; p.n[k] = t.n; p.at[k] = t.at;
    p.keep[k] = (float)(1 - a->lr * t.weight_decay);
    p.first[k + 1] = p.first[k] + (int)chunks;
  }
  return SNN_OK;
}
