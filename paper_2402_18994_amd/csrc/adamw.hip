// One AdamW step over many tensors (include/snn_ops.h), moments in 32 bits or in 8:
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// Bound by memory: 28 bytes a parameter with everything in fp32, 16.1 with 8-bit moments.  The tensors' addresses
// travel as kernel arguments, up to TENSORS in a launch, so a step needs no table on the device and no copy; a
// workgroup finds its tensor by bisection over the chunk numbers.  A thread takes four neighbouring elements: with more
// of them a thread, fewer threads hide the loads (four elements, eight, sixteen: 79 million parameters in 32 bits 403,
// 412 and 421 us, 5.5 TB/s the first; in 8 bits with bfloat16 gradients 230, 241 and 260 us; 7.6 million in 8 bits 28, 30
// and 34 us, all in 8 bits with the arithmetic as it was before what follows).
// Every operation is rounded by itself (no contraction), so that the codes of 8-bit moments do not depend on how the
// compiler joins operations.
// With 8-bit moments the arithmetic counts as well: random bits, two roundings, the scales.  7.6 million parameters took
// 28 us with codes taken apart into exponent and steps in floating point, a branch for what is not finite and 64-bit
// places of every element; 26.3 us, 4.1 TB/s, with what stands below (a copy of 256 MiB reaches 5.4 on this card), the vector
// units issuing 97 % of the time.  A bfloat16 gradient is widened in the branch that loads it, so codes, scales and moments are
// asked for when it has come: two rounds of memory, one behind the other.  The roots of
// single elements and the quotient come from the hardware's approximations, one unit of the last place off (correctly
// rounded ones cost ten operations more each): the
// parameter feels 2^-23 of its update, and a code does not feel it, since a root taken for just below a code or just
// above goes to that code with a chance next to 1 from either side.  The scales go by exact comparisons.
#include "seq_common.hpp"

#include <float.h>
#include <math.h>
#include <stdlib.h>

#include <algorithm>

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

// Random bits: a counter of the elements, times the prime next to 2^32 / 1.618.., plus a salt of seed and step, stirred.  That prime
// and the other two (0x85EBCA77 for the step, 0xC2B2AE3D for the places' high halves) are published ones for hashing 32-bit
// words, by Y. Collet, taken as odd multipliers; nothing else of that work is used.
// 32 bits of a counter, stirred: multiplications by the odd numbers next to 2^31 sqrt(2) and 2^31 sqrt(3), each
// followed by the high bits folded onto the low ones.
__host__ __device__ __forceinline__ uint32_t stir(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xB504F335u;
  x = (x ^ (x >> 15)) * 0xDDB3D743u;
  return x ^ (x >> 16);
}

// Largest value over 32 neighbouring lanes, in all of them.  (Magnitudes are compared by their bits: integers need none of
// the care that a floating maximum takes over NaN.)
template <int CTRL> __device__ __forceinline__ uint32_t dpp_bits(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t max_of_32(uint32_t v) {
  v = max(v, dpp_bits<0xB1>(v));
  v = max(v, dpp_bits<0x4E>(v));
  v = max(v, dpp_bits<0x141>(v));
  v = max(v, dpp_bits<0x140>(v));
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max((uint32_t)r[0], (uint32_t)r[1]);
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponents of the least powers of two s with top <= 448 s = 1.75 * 2^8 s, and with sqrt(top) <= 448 s, from -60 up.  For
// the first the mantissa's bits above 1.75 carry into the exponent; for the second those above 1.75^2 = 2 * 1.53125 in the
// pair of binades that starts at an even power (the root's rounding does not reach over the next number above that).
__device__ __forceinline__ int scale_exponent(uint32_t top) { return max(-60, (int)((top + 0x1FFFFFu) >> 23) - 127 - 8); }
__device__ __forceinline__ int scale_exponent_of_root(uint32_t top) { return max(-60, ((int)(top - (127u << 23) + 0x3BFFFFu) >> 24) - 8); }

// The hardware's root, which takes what lies below the least normal number for zero: such a second moment (gradients of 1e-18,
// say) has its codes and its root like any other.
__device__ __forceinline__ float root_fast(float v) {
  const bool tiny = v < 0x1p-100f;
  const float r = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p100f : v);
  return tiny ? r * 0x1p-50f : r;
}

// Codes of magnitudes in units of the scale, up to 448: binades of eight codes from 2^-6 (code 8) on, below that the
// eight codes of the subnormal numbers, 2^-9 apart.  What lies between two codes goes up where (k + 1/2) / 65536, k being
// 16 random bits, is below a chance.  Nothing here branches: a choice of two costs less than taking turns.

// The first moment, by the share of the way to the next code.  20 bits of an fp32 mantissa lie below a code's, so the
// carry out of them is the rounding: 16 (65535 - k) + 7 on top of them carries exactly where the share exceeds the
// chance.  A subnormal magnitude gets 2^-6 added, which puts it on the codes of the first binade, eight codes up.
__device__ __forceinline__ uint32_t code_m(float m, float inverse, uint32_t rand) {
#pragma clang fp contract(off)
  const float y = fabsf(m) * inverse;
  const bool low = y < 0x1p-6f;
  const uint32_t t = __float_as_uint(low ? y + 0x1p-6f : y) + ((rand << 4 & 0xFFFF0u) ^ 0xFFFF7u);
  return ((t >> 20) - (low ? 968u : 960u)) | (__float_as_uint(m) >> 24 & 0x80u);
}
// The second moment: its root is coded, a = low + f in steps of the root's binade; up with the chance that keeps the mean
// of v itself, (a^2 - low^2) / (2 low + 1).  Scaling by powers of two is exact; a^2 comes from v, not from the root.
__device__ __forceinline__ uint32_t code_v(float v, float root, int exponent, uint32_t rand) {
#pragma clang fp contract(off)
  const int e = max(-6, (int)(__float_as_uint(root) >> 23) - 127 - exponent);
  const float steps = power2(3 - e - exponent), low = floorf(root * steps), square = (v * steps) * steps;
  const float chance = ((float)(rand >> 16) + 0.5f) * (1.f / 65536.f);
  const bool up = chance * fmaf(2.f, low, 1.f) < fmaf(-low, low, square);
  const uint32_t code = (uint32_t)((e + 6) * 8 + (int)low + (up ? 1 : 0));
  return max(code, v > 0.f ? 1u : 0u);
}

// Four elements from k on, of `left`; zeros beyond.
template <typename T> __device__ __forceinline__ void take4(float r[4], const T *p, int k, int left, bool vec) {
  if (vec && k + 4 <= left) {
    const Pack<T, 4> q = *(const Pack<T, 4> *)(p + k);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = widen(q.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = k + j < left ? widen(p[k + j]) : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void give4(T *p, const float r[4], int k, int left, bool vec) {
  if (vec && k + 4 <= left) {
    Pack<T, 4> q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q.v[j] = narrow<T>(r[j]);
    *(Pack<T, 4> *)(p + k) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (k + j < left) p[k + j] = narrow<T>(r[j]);
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
  // the workgroup's chunk of the tensor and of the moments, and this thread's place in it
  const int64_t base = (int64_t)((int)blockIdx.x - p.first[lo]) * CHUNK, at = p.at[lo] + base;
  const int left = (int)min(p.n[lo] - base, (int64_t)CHUNK), k = threadIdx.x * 4;
  float *param = p.param[lo] + base;
  const G *grad = (const G *)p.grad[lo] + base;
  __bf16 *copy = p.copy[lo];
  const float keep = p.keep[lo];
  const bool vp = ((uintptr_t)param & 15) == 0, vg = ((uintptr_t)grad & (4 * sizeof(G) - 1)) == 0, vc = ((uintptr_t)copy & 7) == 0;

  float w[4] = {0.f, 0.f, 0.f, 0.f}, g[4] = {0.f, 0.f, 0.f, 0.f}, m[4], v[4], root[4];
  if constexpr (BITS == 32) {
    if (k >= left) return;
    take4(w, (const float *)param, k, left, vp);
    take4(g, grad, k, left, vg);
    take4(m, (const float *)p.m + at, k, left, true);      // (at: a multiple of SNN_ADAMW_BLOCK)
    take4(v, (const float *)p.v + at, k, left, true);
  } else {
    // a lane beyond the tensor has no element of the block and only takes part in its maxima
    uint32_t cm = 0, cv = 0;
    float sm = 1.f, sv = 1.f;
    if (k < left) {
      take4(w, (const float *)param, k, left, vp);
      take4(g, grad, k, left, vg);
      cm = *(const uint32_t *)((const uint8_t *)p.m + at + k);
      cv = *(const uint32_t *)((const uint8_t *)p.v + at + k);
      sm = (p.m_scale + at / SNN_ADAMW_BLOCK)[k / SNN_ADAMW_BLOCK];
      sv = (p.v_scale + at / SNN_ADAMW_BLOCK)[k / SNN_ADAMW_BLOCK];
      if (k + 4 > left) {                                  // what is behind the last element counts as zero
        const uint32_t own = (1u << 8 * (left - k)) - 1;
        cm &= own;
        cv &= own;
      }
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
      root[j] = root_fast(v[j]);
      w[j] = w[j] * keep - (m[j] * p.k1) * rcp_fast(root[j] * p.k2 + p.eps);
    } else {
      root[j] = sqrtf(v[j]);
      w[j] = w[j] * keep - (m[j] * p.k1) / (root[j] * p.k2 + p.eps);
    }
  }
  if constexpr (BITS == 8) {
    // 32 lanes hold a block: its largest finite magnitudes give the scales
    uint32_t tm = 0, tv = 0, nan_m = 0, nan_v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool fm = finite(m[j]), fv = finite(v[j]);
      nan_m |= fm ? 0u : 0x7Fu << 8 * j;                   // (what is not finite is coded as zero, and then made NaN)
      nan_v |= fv ? 0u : 0x7Fu << 8 * j;
      m[j] = fm ? m[j] : 0.f;
      v[j] = fv ? v[j] : 0.f;
      root[j] = fv ? root[j] : 0.f;
      tm = max(tm, __float_as_uint(m[j]) & 0x7FFFFFFFu);
      tv = max(tv, __float_as_uint(v[j]));
    }
    const int em = scale_exponent(max_of_32(tm)), ev = scale_exponent_of_root(max_of_32(tv));
    const float im = power2(-em);
    uint32_t qm = nan_m, qv = nan_v;
    const uint32_t low = (uint32_t)at + (uint32_t)k, high = (uint32_t)(at >> 32) + (low < (uint32_t)at ? 1u : 0u);
    const uint32_t first = low * 0x9E3779B1u + high * 0xC2B2AE3Du + p.salt;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t rand = stir(first + j * 0x9E3779B1u);
      qm |= code_m(m[j], im, rand) << (8 * j);
      qv |= code_v(v[j], root[j], ev, rand) << (8 * j);
    }
    if (k >= left) return;
    *(uint32_t *)((uint8_t *)p.m + at + k) = qm;
    *(uint32_t *)((uint8_t *)p.v + at + k) = qv;
    if ((threadIdx.x & 31) == 0) {
      (p.m_scale + at / SNN_ADAMW_BLOCK)[k / SNN_ADAMW_BLOCK] = power2(em);
      (p.v_scale + at / SNN_ADAMW_BLOCK)[k / SNN_ADAMW_BLOCK] = power2(ev);
    }
  } else {
    give4((float *)p.m + at, m, k, left, true);
    give4((float *)p.v + at, v, k, left, true);
  }
  give4(param, w, k, left, vp);
  if (copy) give4(copy + base, w, k, left, vc);
}

// ---------------------------------------------------------------- host side
// Whether two of the pieces share a place.  They mostly ascend as they are, and are sorted where they do not (72 tensors: half a
// microsecond more).  Nothing here throws.
struct Piece {
  uint64_t from, to;
};
bool overlap(Piece *p, size_t n) {
  const auto before = [](const Piece &a, const Piece &b) { return a.from < b.from; };
  if (!std::is_sorted(p, p + n, before)) std::sort(p, p + n, before);
  for (size_t i = 1; i < n; ++i)
    if (p[i].from < p[i - 1].to) return true;
  return false;
}
// Workgroups of one launch update all tensors at once: what they write must lie apart.
int pieces_check(const snn_adamw_tensor *tensors, int32_t count) {
  constexpr int FEW = 256;
  Piece few[2 * FEW], *p = count <= FEW ? few : (Piece *)malloc(2 * (size_t)count * sizeof(Piece));
  if (!p) return ops_fail(SNN_ERR_ARG, "AdamW: no host memory to look at %d tensors", count);
  size_t k = 0;
  for (int i = 0; i < count; ++i) {
    const snn_adamw_tensor &t = tensors[i];
    if (!t.n) continue;
    p[k++] = {(uint64_t)(uintptr_t)t.param, (uint64_t)(uintptr_t)t.param + 4 * (uint64_t)t.n};
  }
  for (int i = 0; i < count; ++i) {
    const snn_adamw_tensor &t = tensors[i];
    if (t.n && t.copy) p[k++] = {(uint64_t)(uintptr_t)t.copy, (uint64_t)(uintptr_t)t.copy + 2 * (uint64_t)t.n};
  }
  const bool memory = overlap(p, k);
  k = 0;
  for (int i = 0; i < count; ++i) {
    const snn_adamw_tensor &t = tensors[i];
    if (t.n) p[k++] = {(uint64_t)t.at, (uint64_t)t.at + ((uint64_t)t.n + SNN_ADAMW_BLOCK - 1) / SNN_ADAMW_BLOCK * SNN_ADAMW_BLOCK};
  }
  const bool moments = overlap(p, k);
  if (p != few) free(p);
  if (memory) return ops_fail(SNN_ERR_ARG, "AdamW: two parameters or copies share memory (the same tensor twice?)");
  if (moments) return ops_fail(SNN_ERR_ARG, "AdamW: the moments of two tensors share a block");
  return SNN_OK;
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
  const int rc = pieces_check(tensors, count);
  if (rc) return rc;
  AdamP p;
  p.m = a->m; p.v = a->v; p.m_scale = a->m_scale; p.v_scale = a->v_scale;
  p.b1 = (float)a->beta1; p.c1 = (float)(1 - a->beta1);
  p.b2 = (float)a->beta2; p.c2 = (float)(1 - a->beta2);
  p.k1 = (float)(a->lr / (1 - pow(a->beta1, (double)a->step)));
  p.k2 = (float)(1 / sqrt(1 - pow(a->beta2, (double)a->step)));
  p.eps = a->eps > 0 ? fmaxf((float)a->eps, FLT_MIN) : 0.f;   // (a positive one stays positive, and has a reciprocal)
  p.grad_scale = (float)a->grad_scale;
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
      const int launched = ops_launched("AdamW");
      if (launched) return launched;
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
