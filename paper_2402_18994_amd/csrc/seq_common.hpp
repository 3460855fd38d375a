// What the kernels of the sequence operators (seq_conv.hip, seq_scan.hip, adamw.hip) share: element types,
// sums over neighbouring lanes, argument checks.  gfx950 only.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/snn_ops.h"

namespace snn {

// Keeps the text for snn_last_error(NULL) and returns `code` (snn_api.hip).
int ops_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline int ops_launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SNN_OK : ops_fail(SNN_ERR_HIP, "%s: launch failed: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline size_t rup256(size_t n) { return (n + 255) & ~(size_t)255; }

// A tensor over time in a kernel's arguments.
template <typename T> struct Rows {
  T *p;
  int64_t st, sb;
  Rows(const snn_rows &r) : p((T *)const_cast<void *>(r.p)), st(r.stride_t), sb(r.stride_b) {}
  // Of a call of `steps` steps: the stride between steps, which may be anything where there is one, is then 0.
  Rows(const snn_rows &r, int steps) : p((T *)const_cast<void *>(r.p)), st(steps > 1 ? r.stride_t : 0), sb(r.stride_b) {}
};

// ---------------------------------------------------------------- element types
// A streamed value is widened when it is loaded and rounded once (to nearest, ties to even) when it is stored.
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }
template <typename T> __device__ __forceinline__ T narrow(float x) { return (T)x; }

// VEC neighbouring elements, loaded and stored as one access.
template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// ---------------------------------------------------------------- elementary functions
// The hardware's base-2 exponential is good to about one unit of the last place; results below the least normal number are
// zero.  exp_fast rounds x log2(e) once before it, which moves the result by about |x| 2^-24 of itself: a few units of the
// last place for the step sizes that softplus makes of x = -5, up to eight at x = -10.
constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float sigmoid_fast(float x) { return rcp_fast(1.f + exp_fast(-x)); }

// log(1 + e) for 0 <= e <= 1 as 2 artanh(s), s = e / (2 + e) <= 1/3: the odd power series, whose first term left out
// is s^17 / 17 (4e-9 of the sum).  log(1 + e) by itself would lose the digits of a small e, and with them those of
// the small step sizes that long memories need.
__device__ __forceinline__ float log1p_unit(float e) {
  const float s = e * rcp_fast(2.f + e), q = s * s;
  float r = 1.f / 15.f;
  r = fmaf(r, q, 1.f / 13.f);
  r = fmaf(r, q, 1.f / 11.f);
  r = fmaf(r, q, 1.f / 9.f);
  r = fmaf(r, q, 1.f / 7.f);
  r = fmaf(r, q, 1.f / 5.f);
  r = fmaf(r, q, 1.f / 3.f);
  r = fmaf(r, q, 1.f);
  return 2.f * s * r;
}
// softplus(x) = max(x, 0) + log(1 + e^-|x|); a NaN stays one (through the second term).
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1p_unit(exp_fast(-fabsf(x))); }

// ---------------------------------------------------------------- sums over lanes
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// Sum over the L neighbouring lanes (L a power of two up to 16) that a lane belongs to, in all of them: exchanges
// with the lane whose number differs in bit 0, bit 1, then the mirror images of 8 and of 16 lanes.
template <int L> __device__ __forceinline__ float sum_neighbours(float v) {
  if constexpr (L >= 2) v += dpp<0xB1>(v);
  if constexpr (L >= 4) v += dpp<0x4E>(v);
  if constexpr (L >= 8) v += dpp<0x141>(v);
  if constexpr (L >= 16) v += dpp<0x140>(v);
  return v;
}

// Sum of column `col` of partial sums [rows][cols], for a workgroup of 16 columns (threadIdx.x % 16) by 16 runs: run r
// adds rows r, r + 16, .. with eight loads in flight, and the runs' sums are added in order.  Few columns and many rows
// leave a launch like this to the latency of its loads: 5120 columns of 256 rows took 20 us with four runs of single
// loads.  Every thread of the workgroup calls it; run 0 has the sum (of columns below `cols`).
__device__ __forceinline__ float sum_column(const float *__restrict__ part, int64_t cols, int64_t col, int rows, float *lds) {
  const int run = threadIdx.x >> 4;
  float s = 0.f;
  if (col < cols) {
    const float *p = part + col;
    int r = run;
    for (; r + 112 < rows; r += 128) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = p[(r + 16 * u) * cols];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; r < rows; r += 16) s += p[r * cols];
  }
  lds[threadIdx.x] = s;
  __syncthreads();
  if (run == 0)
#pragma unroll
    for (int k = 1; k < 16; ++k) s += lds[k * 16 + threadIdx.x];
  return s;
}

// Orders the LDS accesses of one wavefront for the compiler; the hardware keeps them in order by itself.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ int length_of(const int32_t *lengths, int b, int T) {
  return lengths ? max(0, min(T, lengths[b])) : T;
}

}  // namespace snn
