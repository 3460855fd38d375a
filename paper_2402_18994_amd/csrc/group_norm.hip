// Group norm with an optional SiLU, channels fastest (include/snn_ops.h):
//   xh = (x - mean) rstd, rstd = 1 / sqrt(variance + eps), v = xh w + b, y = v or v sigmoid(v);  q = dy y'(v), p = q w:
//   dx = rstd (p - mean(p) - xh mean(p xh)), dw = sum q xh, db = sum q.
// Means run over the channels of a group and, unless per_step, the steps of the sequence that exist.
//
// What bounds it is memory.  Where each step stands alone, and where a sequence's group fits the registers of one small workgroup, x (and
// dy) are read once: mean, squares around it, outputs.  Otherwise a sequence's rows are cut into chunks: one launch leaves every
// chunk's (mean, sum of squares around it), a second one joins them and reads the rows again, which the last-level cache still has up to
// some 200 MB.  (One workgroup of 1024 threads that holds 64 values a thread needs no second reading, but fills and empties a compute
// unit in turn: 1024 steps of 8 x 2048 channels, 32 groups, bf16: forward 24.7 us against 22.7, reverse 226, out of registers, against 40.)
// Sums over rows (dw, db) leave a row per chunk or workgroup, which a last launch adds up, or workgroups of the second one.
#include "block_rules.hpp"
#include "rows.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

enum { WHOLE = 0, STEP = 1 };                                // statistics over a unit's rows, or of each row

struct NormP {
  int T, B, D, G, C, silu;
  float eps;
  int64_t rows;                             // of a unit: T of a sequence, or T B where each row stands alone
  int units, blocks, loops;                 // workgroups of a unit and group; how many lots of rows each takes in turn
  int tpr_log2, K, R;                       // threads a row; column blocks of a row; rows of a thread
  Rows<void> x, y;
  const float *weight, *bias;
  const int32_t *lengths;
  float2 *saved;                            // [units or rows][G]: mean, rstd
  float2 *part;                             // [units][G][blocks]: a chunk's sums
  // reverse
  Rows<void> dy, dx;
  float *dpart;                             // [units * blocks][2][D]
  float *dweight, *dbias;
  unsigned main;                            // workgroups of a launch that have a part of x; behind them some are there for dweight and dbias
};

// A launch's dimension counts its threads in 32 bits: workgroups are numbered over two.
constexpr unsigned ACROSS = 1 << 20;
__device__ __forceinline__ unsigned workgroup() { return blockIdx.y * ACROSS + blockIdx.x; }
dim3 grid_of(int64_t n) { return dim3((unsigned)std::min<int64_t>(n, ACROSS), (unsigned)((n + ACROSS - 1) / ACROSS)); }

// Sum over aligned sets of 2^w lanes, in all of them.
__device__ __forceinline__ float wave_sum(float v, int w) {
  if (w >= 1) v += dpp<0xB1>(v);
  if (w >= 2) v += dpp<0x4E>(v);
  if (w >= 3) v += dpp<0x141>(v);
  if (w >= 4) v += dpp<0x140>(v);
  if (w >= 5) v = add_16_apart(v);
  if (w >= 6) v = add_32_apart(v);
  return v;
}
// Sum over the lanes whose numbers agree in their low w bits (row rotations, then the swaps).
__device__ __forceinline__ float wave_fold(float v, int w) {
  if (w <= 3) v += dpp<0x128>(v);
  if (w <= 2) v += dpp<0x124>(v);
  if (w <= 1) v += dpp<0x122>(v);
  if (w <= 0) v += dpp<0x121>(v);
  if (w <= 4) v = add_16_apart(v);
  if (w <= 5) v = add_32_apart(v);
  return v;
}
// Over a workgroup, in all threads.  `lds` takes NT / 64 floats and is free again after the next barrier.
template <int NT> __device__ __forceinline__ float block_sum(float v, float *lds) {
  v = wave_sum(v, 6);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) s += lds[w];
  return s;
}

// Vectors that a thread holds at a time, each of another row.  Rows that stand alone are taken two at a time: more of them cost registers
// and with them wavefronts.
template <typename T, int VEC, int MODE> struct Slots {
  static constexpr int N = MODE == STEP ? 2 : sizeof(T) * VEC == 16 ? 8 : 16;
};

// sum / n with `inverse` = 1 / n, brought to the nearest number by its remainder: the rounding of 1 / n alone would give equal values a mean
// that is not their value, and deviations that without much of an eps are all there is.
__device__ __forceinline__ float mean_of(float sum, float n, float inverse) {
  const float m = sum * inverse;
  return fmaf(fmaf(-m, n, sum), inverse, m);
}

// 1 / sqrt(v).  The hardware's root takes what is below the least normal number, a variance without an eps may be, for zero.
__device__ __forceinline__ float rstd_of(float v) {
  const bool small = v < 0x1p-126f;
  const float r = __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v);
  return small ? r * 0x1p32f : r;
}

__device__ __forceinline__ float silu_slope(float v) {
  const float s = sigmoid_fast(v);
  return s * fmaf(v, 1.f - s, 1.f);
}

// q and p of a value.  Rounded as they stand, so that both uses of p (its mean, and what the mean is taken from) are the same number:
// contracted into the difference, p would leave a rounding times rstd where the difference is zero.
__device__ __forceinline__ float gradient_of(float dy, float xh, float w, float b, int silu, float &p) {
#pragma clang fp contract(off)
  const float q = dy * (silu ? silu_slope(fmaf(xh, w, b)) : 1.f);
  p = q * w;
  return q;
}

// The choice of `silu`, once for a kernel in place of once a value.
template <typename F> __device__ __forceinline__ void with_silu(int silu, F f) {
  if (silu) f(std::integral_constant<int, 1>());
  else f(std::integral_constant<int, 0>());
}

// Where the vectors of a thread lie.
template <typename T, int VEC> struct Where {
  const NormP &a;
  int unit, g, len, rsub, col, rp;
  int64_t r0;
  bool step;
  __device__ __forceinline__ int channel() const { return col * VEC; }                                        // within the group
  __device__ __forceinline__ int64_t row(int s) const { return r0 + (int64_t)s * rp + rsub; }
  __device__ __forceinline__ bool there(int s) const { return row(s) < a.rows && channel() < a.C && s < a.R; }
  __device__ __forceinline__ void place(int64_t m, int &t, int &b) const {
    t = step ? (int)((uint32_t)m / (uint32_t)a.B) : (int)m;
    b = step ? (int)((uint32_t)m - (uint32_t)t * (uint32_t)a.B) : unit;
  }
  // whether the row exists: in the tensor, and in its sequence
  __device__ __forceinline__ bool live(int s) const {
    if (!there(s)) return false;
    int t, b;
    place(row(s), t, b);
    return t < (step ? length_of(a.lengths, b, a.T) : len);
  }
  template <typename R> __device__ __forceinline__ T *at(const R &r, int s) const {
    int t, b;
    place(row(s), t, b);
    return (T *)r.p + b * r.sb + t * r.st + (int64_t)g * a.C + channel();
  }
};

template <typename T, int VEC, typename W, typename R>
__device__ __forceinline__ Pack<T, VEC> fetch(const W &w, const R &r, int s, bool live) {
  const Pack<T, VEC> v = *(const Pack<T, VEC> *)(live ? w.at(r, s) : (const T *)r.p);   // (the first row's is as good as any)
  const Pack<T, VEC> zero = {};
  return live ? v : zero;
}

// The second use of packed values widens them again: left alone, the compiler keeps all the values that it formed of them for the
// first one, and has no registers for that.
template <typename P, int N> __device__ __forceinline__ void keep_packed(P (&v)[N]) {
#pragma unroll
  for (int s = 0; s < N; ++s) {
    if constexpr (sizeof(P) >= 4) {
      struct Words {
        uint32_t w[sizeof(P) / 4];
      } u = __builtin_bit_cast(Words, v[s]);
#pragma unroll
      for (int k = 0; k < (int)(sizeof(P) / 4); ++k) asm volatile("" : "+v"(u.w[k]));
      v[s] = __builtin_bit_cast(P, u);
    }
  }
}

// A vector's weights and biases, as one load each (which need no more than an element's alignment).
template <int VEC> __device__ __forceinline__ void params(const NormP &a, int d, float (&w)[VEC], float (&b)[VEC]) {
  struct alignas(4) Values {
    float v[VEC];
  } x;
#pragma unroll
  for (int v = 0; v < VEC; ++v) w[v] = 1.f, b[v] = 0.f;
  if (a.weight) {
    __builtin_memcpy(&x, a.weight + d, sizeof x);
#pragma unroll
    for (int v = 0; v < VEC; ++v) w[v] = x.v[v];
  }
  if (a.bias) {
    __builtin_memcpy(&x, a.bias + d, sizeof x);
#pragma unroll
    for (int v = 0; v < VEC; ++v) b[v] = x.v[v];
  }
}

template <typename T, int VEC>
__device__ __forceinline__ Where<T, VEC> where(const NormP &a, unsigned id, bool step, int nt) {
  const unsigned rest = id / (unsigned)a.G, turn = rest / (unsigned)a.units;
  Where<T, VEC> w{a, 0, 0, 0, 0, 0, 0, 0, step};
  w.g = (int)(id - rest * a.G);
  w.unit = (int)(rest - turn * a.units);
  w.rsub = (int)threadIdx.x >> a.tpr_log2;
  w.col = (int)threadIdx.x & ((1 << a.tpr_log2) - 1);
  w.rp = nt >> a.tpr_log2;
  w.r0 = turn * (int64_t)w.rp * a.R * a.loops;
  w.len = step ? 0 : __builtin_amdgcn_readfirstlane(length_of(a.lengths, w.unit, a.T));
  return w;
}
__device__ __forceinline__ float output_of(float x, float mean, float rstd, float w, float b, int silu) {
  const float v = fmaf((x - mean) * rstd, w, b);
  return silu ? v * sigmoid_fast(v) : v;
}

// Sums over each row (of a wavefront's lanes at most), or over all rows (in every slot).  `lds` takes NT / 64 floats.
template <int NT, int SLOTS, int MODE> __device__ __forceinline__ void sums_of(const NormP &a, float (&v)[SLOTS], float *lds) {
  if (MODE == STEP) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) v[s] = wave_sum(v[s], a.tpr_log2);
    return;
  }
#pragma unroll
  for (int s = 1; s < SLOTS; ++s) v[0] += v[s];
  v[0] = block_sum<NT>(v[0], lds);
#pragma unroll
  for (int s = 1; s < SLOTS; ++s) v[s] = v[0];
}

template <typename T, int VEC, int NT, int MODE>
__global__ __launch_bounds__(NT) void norm_forward_kernel(const NormP a) {
  constexpr int SLOTS = Slots<T, VEC, MODE>::N;
  __shared__ float lds[2][NT / 64];
  if (workgroup() >= a.main) return;
  auto w = where<T, VEC>(a, workgroup(), MODE == STEP, NT);
  float wt[VEC], bs[VEC];
  params<VEC>(a, w.channel() < a.C ? w.g * a.C + w.channel() : 0, wt, bs);
  for (int loop = 0; loop < a.loops; ++loop, w.r0 += (int64_t)w.rp * a.R) {
    Pack<T, VEC> x[SLOTS];
    bool live[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      live[s] = w.live(s);
      x[s] = fetch<T, VEC>(w, a.x, s, live[s]);
    }
    float mean[SLOTS], rstd[SLOTS];                          // (WHOLE: the same in all)
    const float count = MODE == STEP ? (float)a.C : fmaxf((float)((int64_t)w.len * a.C), 1.f), n = 1.f / count;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      mean[s] = 0.f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) mean[s] += widen(x[s].v[v]);
    }
    sums_of<NT, SLOTS, MODE>(a, mean, lds[0]);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      mean[s] = mean_of(mean[s], count, n);
      rstd[s] = 0.f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float e = live[s] ? widen(x[s].v[v]) - mean[s] : 0.f;
        rstd[s] = fmaf(e, e, rstd[s]);
      }
    }
    sums_of<NT, SLOTS, MODE>(a, rstd, lds[1]);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      rstd[s] = rstd_of(fmaf(rstd[s], n, a.eps));
      if (MODE == STEP && a.saved && w.col == 0 && w.there(s)) a.saved[w.row(s) * a.G + w.g] = {mean[s], rstd[s]};
    }
    if (MODE == WHOLE && a.saved && threadIdx.x == 0) a.saved[(int64_t)w.unit * a.G + w.g] = {mean[0], rstd[0]};
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (!w.there(s)) continue;
      Pack<T, VEC> y;
#pragma unroll
      for (int v = 0; v < VEC; ++v) y.v[v] = narrow<T>(live[s] ? output_of(widen(x[s].v[v]), mean[s], rstd[s], wt[v], bs[v], a.silu) : 0.f);
      *(Pack<T, VEC> *)w.at(a.y, s) = y;
    }
  }
}

// Adds up `acc` over the threads of a workgroup that hold the same columns; thread `tid` < columns / VEC of the first row has the sum.
template <int VEC, int NT> __device__ __forceinline__ void column_sums(const NormP &a, float (&acc)[VEC], float *lds) {
  const int tpr = 1 << a.tpr_log2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int v = 0; v < VEC; ++v) acc[v] = wave_fold(acc[v], a.tpr_log2);
  const int sets = a.tpr_log2 <= 6 ? NT / 64 : NT >> a.tpr_log2, width = tpr;
  const int set = a.tpr_log2 <= 6 ? wave : (int)threadIdx.x >> a.tpr_log2, at = a.tpr_log2 <= 6 ? lane : (int)threadIdx.x & (tpr - 1);
  __syncthreads();
  if (at < width)
#pragma unroll
    for (int v = 0; v < VEC; ++v) lds[(set * VEC + v) * width + at] = acc[v];
  __syncthreads();
  if ((int)threadIdx.x < width)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = 0.f;
      for (int k = 0; k < sets; ++k) s += lds[(k * VEC + v) * width + threadIdx.x];
      acc[v] = s;
    }
}

// SILU: 0 and 1 as the call says, or -1, which asks it for each value: where steps stand alone a kernel for each is faster (reverse of 1024
// steps of 8 x 2048 channels, 16 groups, bf16, 48 and 41 us), where a sequence's group is held at once a choice
// outside the loops is not (17.1 against 15.7 for 257 of 51 x 130, 5 groups, fp32: more registers).
template <typename T, int VEC, int NT, int MODE, int SILU>
__global__ __launch_bounds__(NT) void norm_backward_kernel(const NormP a) {
  constexpr int SLOTS = Slots<T, VEC, MODE>::N;
  __shared__ float lds[2][NT / 64];
  __shared__ float cols[NT * VEC];
  const unsigned id = workgroup();
  if (id >= a.main) return;
  auto w = where<T, VEC>(a, id, MODE == STEP, NT);
  const int chunk = (int)(id / ((unsigned)a.G * (unsigned)a.units));
  const int silu = SILU < 0 ? a.silu : SILU;
  float wt[VEC], bs[VEC], dw[VEC], db[VEC];
  params<VEC>(a, w.channel() < a.C ? w.g * a.C + w.channel() : 0, wt, bs);
#pragma unroll
  for (int v = 0; v < VEC; ++v) dw[v] = db[v] = 0.f;
  float *const out = a.dpart + ((int64_t)w.unit * a.blocks + chunk) * 2 * a.D + (int64_t)w.g * a.C;
  const float n = MODE == STEP ? 1.f / (float)a.C : 1.f / fmaxf((float)((int64_t)w.len * a.C), 1.f);
  for (int loop = 0; loop < a.loops; ++loop, w.r0 += (int64_t)w.rp * a.R) {
    Pack<T, VEC> x[SLOTS], dy[SLOTS];
    bool live[SLOTS];
    float mean[SLOTS], rstd[SLOTS], s1[SLOTS], s2[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      live[s] = w.live(s);
      x[s] = fetch<T, VEC>(w, a.x, s, live[s]);
      dy[s] = fetch<T, VEC>(w, a.dy, s, live[s]);
      const float2 m = a.saved[MODE == STEP ? (live[s] ? w.row(s) : 0) * a.G + w.g : (int64_t)w.unit * a.G + w.g];
      mean[s] = m.x;
      rstd[s] = m.y;
    }
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      s1[s] = s2[s] = 0.f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float xh = live[s] ? (widen(x[s].v[v]) - mean[s]) * rstd[s] : 0.f;
        float p;
        const float q = gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], silu, p);
        s1[s] += p;
        s2[s] = fmaf(p, xh, s2[s]);
        dw[v] = fmaf(q, xh, dw[v]);
        db[v] += q;
      }
    }
    keep_packed(x);
    keep_packed(dy);
    sums_of<NT, SLOTS, MODE>(a, s1, lds[0]);
    sums_of<NT, SLOTS, MODE>(a, s2, lds[1]);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (!w.there(s)) continue;
      Pack<T, VEC> d;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float xh = (widen(x[s].v[v]) - mean[s]) * rstd[s];
        float p;
        gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], silu, p);
        d.v[v] = narrow<T>(live[s] ? rstd[s] * (p - s1[s] * n - xh * (s2[s] * n)) : 0.f);
      }
      *(Pack<T, VEC> *)w.at(a.dx, s) = d;
    }
  }
  column_sums<VEC, NT>(a, dw, cols);
  column_sums<VEC, NT>(a, db, cols);
  if ((int)threadIdx.x < (1 << a.tpr_log2) && w.col * VEC < a.C)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      out[w.col * VEC + v] = dw[v];
      out[a.D + w.col * VEC + v] = db[v];
    }
}

// ---------------------------------------------------------------- long rows by themselves
// Rows of more vectors than a wavefront has lanes: a wavefront each, no barrier.  It holds KB vectors a lane, or (AGAIN), where the row
// is longer than they are, loads them in turn for each of its sums and for the outputs.  (A workgroup for a row waits at two or three
// barriers for every row or two: 1024 x 8 rows of 2047 channels, bf16, 81 us forward and 450 reverse, against 34 and 86; 1024 x 4 of 4096,
// 73 and 366 against 19 and 49.)
template <typename T, int VEC, int KB> struct LongRow {
  int g, t, b, base = 0;
  int64_t m;
  bool there, live;
  __device__ __forceinline__ explicit LongRow(const NormP &a) {
    const unsigned id = workgroup() * 4u + (unsigned)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = id / (unsigned)a.G;
    g = (int)(id - row * a.G);
    m = row;
    there = m < a.rows;
    t = (int)(row / (unsigned)a.B);
    b = (int)(row - (unsigned)t * a.B);
    live = there && t < length_of(a.lengths, b, a.T);
  }
  __device__ __forceinline__ int channel(int s) const { return base + (s * 64 + (int)(threadIdx.x & 63)) * VEC; }
  // Every second or fourth vector: does the row end before it?
  __device__ __forceinline__ bool ends(const NormP &a, int s) const { return s && s % (KB == 4 ? 2 : 4) == 0 && base + s * 64 * VEC >= a.C; }
  template <typename R> __device__ __forceinline__ T *at(const NormP &a, const R &r) const { return (T *)r.p + b * r.sb + t * r.st + (int64_t)g * a.C; }
  template <typename R> __device__ __forceinline__ void load(const NormP &a, const R &r, Pack<T, VEC> (&v)[KB]) const {
    const T *row = at(a, r);
#pragma unroll
    for (int s = 0; s < KB; ++s) {
      if (ends(a, s)) break;
      v[s] = *(const Pack<T, VEC> *)(row + (channel(s) < a.C ? channel(s) : 0));   // (not used behind the row)
    }
  }
  template <typename R> __device__ __forceinline__ void zeros(const NormP &a, const R &r) const {
    const Pack<T, VEC> zero = {};
    for (int c = channel(0); c < a.C; c += 64 * VEC) *(Pack<T, VEC> *)(at(a, r) + c) = zero;
  }
};
template <typename T, int VEC, int KB, bool AGAIN> __global__ __launch_bounds__(256) void norm_rows_kernel(const NormP a) {
  LongRow<T, VEC, KB> w(a);
  if (!w.there) return;
  if (!w.live) {
    w.zeros(a, a.y);
    return;
  }
  Pack<T, VEC> x[KB];
  if (!AGAIN) w.load(a, a.x, x);
  auto over_row = [&](auto f) {
    if (!AGAIN) return f();
    for (w.base = 0; w.base < a.C; w.base += KB * 64 * VEC) {
      w.load(a, a.x, x);
      f();
    }
  };
  const float n = 1.f / (float)a.C;
  float mean = 0.f, q = 0.f;
  over_row([&] {
#pragma unroll
    for (int s = 0; s < KB; ++s) {
      if (w.ends(a, s)) break;
#pragma unroll
      for (int v = 0; v < VEC; ++v) mean += w.channel(s) < a.C ? widen(x[s].v[v]) : 0.f;
    }
  });
  mean = mean_of(wave_sum(mean, 6), (float)a.C, n);
  over_row([&] {
#pragma unroll
    for (int s = 0; s < KB; ++s) {
      if (w.ends(a, s)) break;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float e = w.channel(s) < a.C ? widen(x[s].v[v]) - mean : 0.f;
        q = fmaf(e, e, q);
      }
    }
  });
  const float rstd = rstd_of(fmaf(wave_sum(q, 6), n, a.eps));
  if (a.saved && (threadIdx.x & 63) == 0) a.saved[w.m * a.G + w.g] = {mean, rstd};
  T *y = w.at(a, a.y);
  with_silu(a.silu, [&](auto silu) {
    over_row([&] {
#pragma unroll
      for (int s = 0; s < KB; ++s) {
        if (w.ends(a, s)) break;
        const int c = w.channel(s);
        float wt[VEC], bs[VEC];
        params<VEC>(a, w.g * a.C + (c < a.C ? c : 0), wt, bs);
        Pack<T, VEC> out;
#pragma unroll
        for (int v = 0; v < VEC; ++v) out.v[v] = narrow<T>(output_of(widen(x[s].v[v]), mean, rstd, wt[v], bs[v], silu.value));
        if (c < a.C) *(Pack<T, VEC> *)(y + c) = out;
        if (s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    });
  });
}
template <typename T, int VEC, int KB, bool AGAIN> __global__ __launch_bounds__(256) void norm_rows_backward_kernel(const NormP a) {
  LongRow<T, VEC, KB> w(a);
  if (!w.there) return;
  if (!w.live) {
    w.zeros(a, a.dx);
    return;
  }
  Pack<T, VEC> x[KB], dy[KB];
  auto take = [&] {
    w.load(a, a.x, x);
    w.load(a, a.dy, dy);
  };
  if (!AGAIN) take();
  auto over_row = [&](auto f) {
    if (!AGAIN) return f();
    for (w.base = 0; w.base < a.C; w.base += KB * 64 * VEC) {
      take();
      f();
    }
  };
  const float2 st = a.saved[w.m * a.G + w.g];
  const float n = 1.f / (float)a.C;
  T *dx = w.at(a, a.dx);
  with_silu(a.silu, [&](auto silu) {
    float s1 = 0.f, s2 = 0.f;
    over_row([&] {
#pragma unroll
      for (int s = 0; s < KB; ++s) {
        if (w.ends(a, s)) break;
        const int c = w.channel(s);
        float wt[VEC], bs[VEC];
        params<VEC>(a, w.g * a.C + (c < a.C ? c : 0), wt, bs);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float xh = (widen(x[s].v[v]) - st.x) * st.y;
          float p;
          gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], silu.value, p);
          p = c < a.C ? p : 0.f;                   // (behind the row x is its first value, and p xh a zero or one of the row's NaN)
          s1 += p;
          s2 = fmaf(p, xh, s2);
        }
        if (s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    });
    s1 = wave_sum(s1, 6) * n;
    s2 = wave_sum(s2, 6) * n;
    keep_packed(x);
    keep_packed(dy);
    int first = w.g * a.C;                       // (the weights are loaded again: kept, they would be most of the registers)
    asm volatile("" : "+s"(first));
    over_row([&] {
#pragma unroll
      for (int s = 0; s < KB; ++s) {
        if (w.ends(a, s)) break;
        const int c = w.channel(s);
        float wt[VEC], bs[VEC];
        params<VEC>(a, first + (c < a.C ? c : 0), wt, bs);
        Pack<T, VEC> d;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float xh = (widen(x[s].v[v]) - st.x) * st.y;
          float p;
          gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], silu.value, p);
          d.v[v] = narrow<T>(st.y * (p - s1 - xh * s2));
        }
        if (c < a.C) *(Pack<T, VEC> *)(dx + c) = d;
        if (s % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    });
  });
}
// Their dw and db: a lane has VEC columns, a wavefront every fourth row of the chunk blockIdx.y.
template <typename T, int VEC> __global__ __launch_bounds__(256) void norm_columns_kernel(const NormP a) {
  __shared__ float lds[4][2 * VEC][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = (blockIdx.x * 64 + lane) * VEC;
  const bool on = c < a.D;
  const int cc = on ? c : 0, g = cc / a.C;
  const int64_t first = (int64_t)blockIdx.y * a.R, end = min(a.rows, first + a.R);
  float wt[VEC], bs[VEC], sums[2 * VEC];
  params<VEC>(a, cc, wt, bs);
#pragma unroll
  for (int v = 0; v < 2 * VEC; ++v) sums[v] = 0.f;
  with_silu(a.silu, [&](auto silu) {
#pragma unroll 4
    for (int64_t m = first + wave; m < end; m += 4) {
      const int t = (int)((unsigned)m / (unsigned)a.B), b = (int)((unsigned)m - (unsigned)t * a.B);
      if (t >= length_of(a.lengths, b, a.T)) continue;       // (for the whole wavefront)
      const Pack<T, VEC> x = *(const Pack<T, VEC> *)((const T *)a.x.p + b * a.x.sb + t * a.x.st + cc), dy = *(const Pack<T, VEC> *)((const T *)a.dy.p + b * a.dy.sb + t * a.dy.st + cc);
      const float2 st = a.saved[m * a.G + g];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float xh = (widen(x.v[v]) - st.x) * st.y;
        float p;
        const float q = gradient_of(widen(dy.v[v]), xh, wt[v], bs[v], silu.value, p);
        sums[v] = fmaf(q, xh, sums[v]);
        sums[VEC + v] += q;
      }
    }
  });
#pragma unroll
  for (int v = 0; v < 2 * VEC; ++v) lds[wave][v][lane] = sums[v];
  __syncthreads();
  if (wave == 0 && on)
#pragma unroll
    for (int v = 0; v < 2 * VEC; ++v) {
      const float s = ((lds[0][v][lane] + lds[1][v][lane]) + lds[2][v][lane]) + lds[3][v][lane];
      a.dpart[((int64_t)blockIdx.y * 2 + v / VEC) * a.D + c + v % VEC] = s;
    }
}

// ---------------------------------------------------------------- chunks of a sequence
// A thread's column block k and its rows r0 + rsub + r rp, r < there, of which the first `live` exist in their sequence.
template <typename T, int VEC> struct Run {
  int unit, g, chunk, col, len, live, there, rp;
  int64_t first;
  __device__ __forceinline__ Run(const NormP &a, unsigned id, int nt) {
    const unsigned rest = id / (unsigned)a.G;
    g = (int)(id - rest * a.G);
    chunk = (int)(rest / (unsigned)a.units);
    unit = (int)(rest - (unsigned)chunk * a.units);
    col = ((int)threadIdx.x & ((1 << a.tpr_log2) - 1)) * VEC;
    rp = nt >> a.tpr_log2;
    len = __builtin_amdgcn_readfirstlane(length_of(a.lengths, unit, a.T));
    first = (int64_t)chunk * rp * a.R + ((int)threadIdx.x >> a.tpr_log2);
    there = rows_before(a, a.T);
    live = rows_before(a, len);
  }
  __device__ __forceinline__ int rows_before(const NormP &a, int end) const {
    const int64_t n = ((int64_t)end - first + rp - 1) >> (31 - __builtin_clz(rp));
    return n < 0 ? 0 : n < a.R ? (int)n : a.R;
  }
  template <typename R> __device__ __forceinline__ T *at(const NormP &a, const R &r, int channel) const {
    return (T *)r.p + unit * r.sb + first * r.st + (int64_t)g * a.C + channel;
  }
};
// Rows r .. r + AHEAD of those that exist; in the place of others the first row of the tensor, whose values are not used.
template <typename T, int VEC, int N>
__device__ __forceinline__ void fetch_rows(Pack<T, VEC> (&v)[N], const T *base, const void *any, int64_t step, int r, int n) {
#pragma unroll
  for (int u = 0; u < N; ++u) v[u] = *(const Pack<T, VEC> *)(r + u < n ? base + (r + u) * step : (const T *)any);
}

template <typename P, int N> __device__ __forceinline__ void take(P (&v)[N], const P (&from)[N]) {
#pragma unroll
  for (int u = 0; u < N; ++u) v[u] = from[u];
}

struct Moments {
  float n, mean, m2;
};
// What the distance d of two means adds to the squares around the joint one.  The counts come first: with none on one side d is a mean itself,
// whose square may be no fp32 number.
__device__ __forceinline__ float apart(float d, float n, float share) { return d * (d * (n * share)); }
// Both sets of values as one.
__device__ __forceinline__ Moments joined(const Moments &p, const Moments &q) {
  const float n = p.n + q.n, share = q.n > 0.f ? q.n / n : 0.f, d = q.n > 0.f ? q.mean - p.mean : 0.f;
  return {n, fmaf(d, share, p.mean), p.m2 + q.m2 + apart(d, p.n, share)};
}
template <int NT> __device__ __forceinline__ Moments block_moments(Moments m, Moments *lds) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = joined(m, Moments{__shfl_xor(m.n, o), __shfl_xor(m.mean, o), __shfl_xor(m.m2, o)});
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
  __syncthreads();
  m = lds[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) m = joined(m, lds[w]);
  return m;
}

// Forward: a chunk's mean and sum of squares around it.  A thread goes from vector to vector, each with its own mean.
template <typename T, int VEC, int NT> __global__ __launch_bounds__(NT) void norm_moments_kernel(const NormP a) {
  __shared__ Moments lds[NT / 64];
  if (workgroup() >= a.main) return;
  const Run<T, VEC> w(a, workgroup(), NT);
  Moments m = {0.f, 0.f, 0.f};
  for (int k = 0; k < a.K; ++k) {
    const int c = (k << a.tpr_log2) * VEC + w.col, n = c < a.C ? w.live : 0;
    const T *x = w.at(a, a.x, c);
    for (int r = 0; r < n; r += AHEAD) {
      Pack<T, VEC> v[AHEAD];
      fetch_rows<T, VEC>(v, x, a.x.p, w.rp * a.x.st, r, n);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) s += widen(v[u].v[i]);
        s *= 1.f / VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float e = widen(v[u].v[i]) - s;
          q = fmaf(e, e, q);
        }
        const float count = m.n + VEC, share = VEC * rcp_fast(count), d = s - m.mean;
        const bool on = r + u < n;
        m.m2 = on ? m.m2 + q + apart(d, m.n, share) : m.m2;
        m.mean = on ? fmaf(d, share, m.mean) : m.mean;
        m.n = on ? count : m.n;
      }
    }
  }
  m = block_moments<NT>(m, lds);
  if (threadIdx.x == 0) a.part[((int64_t)w.unit * a.G + w.g) * a.blocks + w.chunk] = {m.mean, m.m2};
}

// The number of values in a chunk of a unit.
__device__ __forceinline__ float chunk_count(const NormP &a, int64_t rows, int chunk, int len) {
  const int64_t n = (int64_t)len - chunk * rows;
  return (float)((n < 0 ? 0 : n < rows ? n : rows) * a.C);
}

template <typename T, int VEC, int NT> __global__ __launch_bounds__(NT) void norm_output_kernel(const NormP a) {
  __shared__ Moments lds[NT / 64];
  if (workgroup() >= a.main) return;
  const Run<T, VEC> w(a, workgroup(), NT);
  const int64_t unit = (int64_t)w.unit * a.G + w.g;
  const int c0 = min(w.col, a.C - VEC);
  Pack<T, VEC> next[AHEAD];                                  // (on their way while the chunks are joined)
  fetch_rows<T, VEC>(next, w.at(a, a.x, c0), a.x.p, w.rp * a.x.st, 0, w.live);
  Moments m = {0.f, 0.f, 0.f};
  for (int c = threadIdx.x; c < a.blocks; c += NT) {
    const float2 p = a.part[unit * a.blocks + c];
    m = joined(m, Moments{chunk_count(a, (int64_t)w.rp * a.R, c, w.len), p.x, p.y});
  }
  m = block_moments<NT>(m, lds);
  const float mean = m.mean, rstd = rstd_of(m.m2 / fmaxf(m.n, 1.f) + a.eps);
  if (a.saved && w.chunk == 0 && threadIdx.x == 0) a.saved[unit] = {mean, rstd};
  for (int k = 0; k < a.K; ++k) {
    const int c = (k << a.tpr_log2) * VEC + w.col;
    if (c >= a.C) break;
    float wt[VEC], bs[VEC];
    params<VEC>(a, w.g * a.C + c, wt, bs);
    const T *x = w.at(a, a.x, c);
    T *y = w.at(a, a.y, c);
    if (k) fetch_rows<T, VEC>(next, x, a.x.p, w.rp * a.x.st, 0, w.live);
    with_silu(a.silu, [&](auto silu) {
      for (int r = 0; r < w.there; r += AHEAD) {
        Pack<T, VEC> v[AHEAD];
        take(v, next);
        if (r + AHEAD < w.live) fetch_rows<T, VEC>(next, x, a.x.p, w.rp * a.x.st, r + AHEAD, w.live);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          Pack<T, VEC> out;
#pragma unroll
          for (int i = 0; i < VEC; ++i) out.v[i] = narrow<T>(r + u < w.live ? output_of(widen(v[u].v[i]), mean, rstd, wt[i], bs[i], silu.value) : 0.f);
          if (r + u < w.there) *(Pack<T, VEC> *)(y + (r + u) * (w.rp * a.y.st)) = out;
        }
      }
    });
  }
}

// Reverse: a chunk's sums of p and p xh, and of q xh and q over its rows.  xh is formed of the difference, as forward: x rstd - mean rstd would
// leave the rounding of mean rstd where x is the mean, and no number where that product is beyond fp32.
template <typename T, int VEC, int NT> __global__ __launch_bounds__(NT) void norm_slopes_kernel(const NormP a) {
  __shared__ float lds[2][NT / 64], cols[NT * VEC];
  if (workgroup() >= a.main) return;
  const Run<T, VEC> w(a, workgroup(), NT);
  const int64_t unit = (int64_t)w.unit * a.G + w.g;
  const float2 st = a.saved[unit];
  float *const out = a.dpart + ((int64_t)w.unit * a.blocks + w.chunk) * 2 * a.D + (int64_t)w.g * a.C;
  float s1 = 0.f, s2 = 0.f;
  for (int k = 0; k < a.K; ++k) {
    const int c = (k << a.tpr_log2) * VEC + w.col, n = c < a.C ? w.live : 0;
    float wt[VEC], bs[VEC], dw[VEC], db[VEC];
    params<VEC>(a, c < a.C ? w.g * a.C + c : 0, wt, bs);
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[i] = db[i] = 0.f;
    const T *x = w.at(a, a.x, c), *dy = w.at(a, a.dy, c);
    for (int r = 0; r < n; r += AHEAD_BWD) {
      Pack<T, VEC> v[AHEAD_BWD], d[AHEAD_BWD];
      fetch_rows<T, VEC>(v, x, a.x.p, w.rp * a.x.st, r, n);
      fetch_rows<T, VEC>(d, dy, a.dy.p, w.rp * a.dy.st, r, n);
#pragma unroll
      for (int u = 0; u < AHEAD_BWD; ++u)
        if (r + u < n)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float xh = (widen(v[u].v[i]) - st.x) * st.y;
            float p;
            const float q = gradient_of(widen(d[u].v[i]), xh, wt[i], bs[i], a.silu, p);
            dw[i] = fmaf(q, xh, dw[i]);
            db[i] += q;
          }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {                          // (p = q w: its sums are those of q, channel by channel)
      s1 = fmaf(db[i], wt[i], s1);
      s2 = fmaf(dw[i], wt[i], s2);
    }
    if (a.K == 1) {
      column_sums<VEC, NT>(a, dw, cols);
      column_sums<VEC, NT>(a, db, cols);
    }
    if ((int)threadIdx.x < (1 << a.tpr_log2) && c < a.C)    // (of several column blocks a thread has its columns to itself)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        out[c + i] = dw[i];
        out[a.D + c + i] = db[i];
      }
  }
  s1 = block_sum<NT>(s1, lds[0]);
  s2 = block_sum<NT>(s2, lds[1]);
  if (threadIdx.x == 0) a.part[unit * a.blocks + w.chunk] = {s1, s2};
}

// The gradients of weight and bias out of the chunks' sums; `block`: which 16 of their 2 D columns.
__device__ __forceinline__ void sum_parameters(const float *part, int rows, int D, float *dweight, float *dbias, int64_t block, float *lds) {
  const int64_t col = block * 16 + (threadIdx.x & 15);
  const float s = sum_column(part, 2 * (int64_t)D, col, rows, lds);
  if (threadIdx.x >= 16) return;
  if (col < D) {
    if (dweight) dweight[col] = s;
  } else if (col < 2 * (int64_t)D && dbias) dbias[col - D] = s;
}
// The workgroups behind the first `a.main` add up the parameters' gradients, which wait for nothing but the launch before.
template <typename T, int VEC, int NT> __global__ __launch_bounds__(NT) void norm_gradient_kernel(const NormP a) {
  static_assert(NT == 256, "as sum_column takes it");
  __shared__ float lds[NT];
  const unsigned id = workgroup();
  if (id >= a.main) {
    sum_parameters(a.dpart, a.units * a.blocks, a.D, a.dweight, a.dbias, id - a.main, lds);
    return;
  }
  const Run<T, VEC> w(a, id, NT);
  const int64_t unit = (int64_t)w.unit * a.G + w.g;
  const float2 st = a.saved[unit];
  const int c0 = min(w.col, a.C - VEC);
  Pack<T, VEC> next[AHEAD_BWD], dnext[AHEAD_BWD];                    // (on their way while the chunks' sums are added)
  fetch_rows<T, VEC>(next, w.at(a, a.x, c0), a.x.p, w.rp * a.x.st, 0, w.live);
  fetch_rows<T, VEC>(dnext, w.at(a, a.dy, c0), a.dy.p, w.rp * a.dy.st, 0, w.live);
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x; c < a.blocks; c += NT) {
    const float2 p = a.part[unit * a.blocks + c];
    s1 += p.x;
    s2 += p.y;
  }
  const float n = 1.f / fmaxf((float)((int64_t)w.len * a.C), 1.f);
  s1 = block_sum<NT>(s1, lds) * n;
  s2 = block_sum<NT>(s2, lds + NT / 64) * n;
  for (int k = 0; k < a.K; ++k) {
    const int c = (k << a.tpr_log2) * VEC + w.col;
    if (c >= a.C) break;
    float wt[VEC], bs[VEC];
    params<VEC>(a, w.g * a.C + c, wt, bs);
    const T *x = w.at(a, a.x, c), *dy = w.at(a, a.dy, c);
    T *dx = w.at(a, a.dx, c);
    if (k) {
      fetch_rows<T, VEC>(next, x, a.x.p, w.rp * a.x.st, 0, w.live);
      fetch_rows<T, VEC>(dnext, dy, a.dy.p, w.rp * a.dy.st, 0, w.live);
    }
    for (int r = 0; r < w.there; r += AHEAD_BWD) {
      Pack<T, VEC> v[AHEAD_BWD], d[AHEAD_BWD];
      take(v, next);
      take(d, dnext);
      if (r + AHEAD_BWD < w.live) {
        fetch_rows<T, VEC>(next, x, a.x.p, w.rp * a.x.st, r + AHEAD_BWD, w.live);
        fetch_rows<T, VEC>(dnext, dy, a.dy.p, w.rp * a.dy.st, r + AHEAD_BWD, w.live);
      }
#pragma unroll
      for (int u = 0; u < AHEAD_BWD; ++u) {
        Pack<T, VEC> out;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float xh = (widen(v[u].v[i]) - st.x) * st.y;
          float p;
          gradient_of(widen(d[u].v[i]), xh, wt[i], bs[i], a.silu, p);
          out.v[i] = narrow<T>(r + u < w.live ? st.y * (p - s1 - xh * s2) : 0.f);
        }
        if (r + u < w.there) *(Pack<T, VEC> *)(dx + (r + u) * (w.rp * a.dx.st)) = out;
      }
    }
  }
}

__global__ __launch_bounds__(256) void norm_sum_kernel(const float *__restrict__ part, int rows, int D, float *dweight, float *dbias) {
  __shared__ float lds[256];
  sum_parameters(part, rows, D, dweight, dbias, blockIdx.x, lds);
}

// ---------------------------------------------------------------- host
constexpr int MOST_CHANNELS = 16384;

int norm_sizes(const snn_norm_args *a) {
  if (!a) return ops_fail(SNN_ERR_NULL, "group norm: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0) return ops_fail(SNN_ERR_ARG, "group norm: T >= 0, B > 0 and D > 0 are required");
  if (a->groups <= 0 || a->D % a->groups) return ops_fail(SNN_ERR_ARG, "group norm: groups has to divide D");
  if (a->D > (1 << 22) || a->D / a->groups > MOST_CHANNELS) return ops_fail(SNN_ERR_ARG, "group norm: D must not exceed 2^22, a group %d channels", MOST_CHANNELS);
  const int64_t rows = (int64_t)a->T * a->B;
  if (rows >= (1ll << 31) || std::max<int64_t>(rows, a->B) * a->groups >= (1ll << 31)) return ops_fail(SNN_ERR_ARG, "group norm: T * B and T * B * groups must stay below 2^31");
  if (a->type != SNN_TYPE_FP32 && a->type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "group norm: unknown type %d", a->type);
  return SNN_OK;
}
int norm_check(const snn_norm_args *a, bool grads) {
  const int rc = norm_sizes(a);
  if (rc) return rc;
  if (!(a->eps >= 0.f) || a->eps > 3e38f) return ops_fail(SNN_ERR_ARG, "group norm: eps must not be negative and has to be finite");
  if (a->T > 0 && (!a->x.p || (!grads && !a->y.p))) return ops_fail(SNN_ERR_NULL, "group norm: x or y is NULL");
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(a->x.p, z) || !aligned(a->y.p, z) || !aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->lengths, 4))
    return ops_fail(SNN_ERR_ARG, "group norm: a pointer is not aligned to its element type");
  return SNN_OK;
}

// The workspace does not depend on the pointers, which decide how many channels a vector has.
size_t part_bytes(const snn_norm_args &a, const NormCut &c) { return c.chunks ? rup256((size_t)a.B * a.groups * c.blocks * 8) : 0; }
size_t norm_bytes(const snn_norm_args &a, bool backward) {
  size_t most = 0;
  for (int vec : {a.type == SNN_TYPE_FP32 ? 4 : 8, 2, 1}) {
    const NormCut c = norm_cut(a, vec, backward);
    most = std::max(most, part_bytes(a, c) + (backward ? rup256((size_t)(a.per_step ? 1 : a.B) * c.blocks * 2 * (size_t)a.D * 4) : 0));
  }
  return most;
}

template <typename F> int with_vector(const snn_norm_args &a, int vec, F f) {
  using std::integral_constant;
  if (a.type == SNN_TYPE_FP32)
    return vec == 4 ? f(float(), integral_constant<int, 4>()) : vec == 2 ? f(float(), integral_constant<int, 2>()) : f(float(), integral_constant<int, 1>());
  return vec == 8 ? f(__bf16(), integral_constant<int, 8>()) : vec == 2 ? f(__bf16(), integral_constant<int, 2>()) : f(__bf16(), integral_constant<int, 1>());
}

// Workgroups of the launches over x: fewer than 2^31, as T B groups is.
int64_t norm_workgroups(const snn_norm_args &a, const NormCut &c) {
  if (c.long_row) return ((int64_t)a.T * a.B * a.groups + 3) / 4;      // a wavefront a row and group
  return (int64_t)a.groups * (a.per_step ? 1 : a.B) * c.blocks;
}

NormP norm_args(const snn_norm_args &a, const NormCut &c, void *saved, void *workspace) {
  return NormP{a.T, a.B, a.D, a.groups, a.D / a.groups, a.silu, a.eps, a.per_step ? (int64_t)a.T * a.B : a.T, a.per_step ? 1 : a.B, c.blocks, c.loops,
               c.tpr_log2, c.K, c.R, Rows<void>(a.x, a.T), Rows<void>(a.y, a.T), a.weight, a.bias, a.lengths, (float2 *)saved, (float2 *)workspace,
               Rows<void>(snn_rows{}), Rows<void>(snn_rows{}), nullptr, nullptr, nullptr, (unsigned)norm_workgroups(a, c)};
}
template <typename F> void held_or_again(int kb, F f) {
  if (kb == AGAIN_ROW) f(std::integral_constant<int, 4>(), std::true_type());
  else f(std::integral_constant<int, 4>(), std::false_type());
}
template <typename T, int V> int launch_norm(const NormCut &c, bool per_step, const NormP &p, hipStream_t st) {
  const dim3 grid = grid_of(p.main);
  if (!per_step) {
    if (!c.chunks && c.nt == 512) hipLaunchKernelGGL((norm_forward_kernel<T, V, 512, WHOLE>), grid, dim3(512), 0, st, p);
    else if (!c.chunks) hipLaunchKernelGGL((norm_forward_kernel<T, V, 256, WHOLE>), grid, dim3(256), 0, st, p);
    else {
      hipLaunchKernelGGL((norm_moments_kernel<T, V, 256>), grid, dim3(256), 0, st, p);
      const int e = ops_launched("group norm, moments");
      if (e) return e;
      hipLaunchKernelGGL((norm_output_kernel<T, V, 256>), grid, dim3(256), 0, st, p);
    }
  } else if (c.long_row) {
    auto rows = [&](auto kb, auto again) { hipLaunchKernelGGL((norm_rows_kernel<T, V, kb.value, again.value>), grid, dim3(256), 0, st, p); };
    bool done = false;
    if constexpr (V <= 2)
      if (c.long_row == 64 / V) rows(std::integral_constant<int, 64 / V>(), std::false_type()), done = true;
    if (!done && c.long_row == 16) rows(std::integral_constant<int, 16>(), std::false_type()), done = true;
    if (!done) held_or_again(c.long_row, rows);
  }
  else hipLaunchKernelGGL((norm_forward_kernel<T, V, 256, STEP>), grid, dim3(256), 0, st, p);
  return ops_launched("group norm");
}
unsigned parameter_blocks(int D) { return (unsigned)((2 * (int64_t)D + 15) / 16); }
template <typename T, int V> int launch_norm_backward(const NormCut &c, bool per_step, const NormP &p, hipStream_t st) {
  const dim3 grid = grid_of(p.main);
  if (!per_step) {
    if (!c.chunks) {
      if constexpr (sizeof(T) * V < 16) {
        if (c.nt == 512) hipLaunchKernelGGL((norm_backward_kernel<T, V, 512, WHOLE, -1>), grid, dim3(512), 0, st, p);
        else hipLaunchKernelGGL((norm_backward_kernel<T, V, 256, WHOLE, -1>), grid, dim3(256), 0, st, p);
      }
    } else {
      hipLaunchKernelGGL((norm_slopes_kernel<T, V, 256>), grid, dim3(256), 0, st, p);
      const int e = ops_launched("group norm backward, sums");
      if (e) return e;
      hipLaunchKernelGGL((norm_gradient_kernel<T, V, 256>), grid_of((int64_t)p.main + (p.dweight || p.dbias ? parameter_blocks(p.D) : 0)), dim3(256), 0, st, p);
    }
  } else if (c.long_row) {
    if (p.dweight || p.dbias) {
      hipLaunchKernelGGL((norm_columns_kernel<T, V>), dim3((p.D + 64 * V - 1) / (64 * V), c.blocks), dim3(256), 0, st, p);
      const int e = ops_launched("group norm backward, parameters");
      if (e) return e;
    }
    held_or_again(c.long_row, [&](auto kb, auto again) { hipLaunchKernelGGL((norm_rows_backward_kernel<T, V, kb.value, again.value>), grid, dim3(256), 0, st, p); });
  } else if (p.silu) hipLaunchKernelGGL((norm_backward_kernel<T, V, 256, STEP, 1>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((norm_backward_kernel<T, V, 256, STEP, 0>), grid, dim3(256), 0, st, p);
  return ops_launched("group norm backward");
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" {

int32_t snn_norm_workspace_bytes(const snn_norm_args *a, int32_t backward, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  const int rc = norm_sizes(a);
  if (rc) return rc;
  *bytes = norm_bytes(*a, backward != 0);
  return SNN_OK;
}

int32_t snn_norm_saved_bytes(const snn_norm_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  const int rc = norm_sizes(a);
  if (rc) return rc;
  *bytes = (a->per_step ? std::max<size_t>(1, (size_t)a->T * a->B) : (size_t)a->B) * a->groups * 8;
  return SNN_OK;
}

int32_t snn_norm_forward(const snn_norm_args *a, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = norm_check(a, false);
  if (rc) return rc;
  if (!aligned(saved, 16)) return ops_fail(SNN_ERR_ARG, "group norm: saved has to be 16-byte aligned");
  const size_t need = norm_bytes(*a, false);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return ops_fail(SNN_ERR_WORKSPACE, "group norm: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  if (a->T == 0) return SNN_OK;
  const int vec = norm_vector(*a, nullptr);
  const NormCut c = norm_cut(*a, vec, false);
  const NormP p = norm_args(*a, c, saved, workspace);
  return with_vector(*a, vec, [&](auto t, auto v) { return launch_norm<decltype(t), v.value>(c, a->per_step, p, (hipStream_t)stream); });
}

int32_t snn_norm_backward(const snn_norm_args *a, const snn_norm_grads *g, const void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = norm_check(a, true);
  if (rc) return rc;
  if (!g || (a->T > 0 && (!g->dy.p || !g->dx.p))) return ops_fail(SNN_ERR_NULL, "group norm backward: dy or dx is NULL");
  if (!saved) return ops_fail(SNN_ERR_NULL, "group norm backward: saved is NULL");
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(saved, 16) || !aligned(g->dy.p, z) || !aligned(g->dx.p, z) || !aligned(g->dweight, 4) || !aligned(g->dbias, 4))
    return ops_fail(SNN_ERR_ARG, "group norm backward: a pointer is not aligned to its element type");
  const size_t need = norm_bytes(*a, true);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
    return ops_fail(SNN_ERR_WORKSPACE, "group norm backward: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  const int vec = norm_vector(*a, g);
  const NormCut c = norm_cut(*a, vec, true);
  NormP p = norm_args(*a, c, const_cast<void *>(saved), workspace);
  p.dy = Rows<void>(g->dy, a->T);
  p.dx = Rows<void>(g->dx, a->T);
  p.dpart = (float *)((char *)workspace + part_bytes(*a, c));
  p.dweight = g->dweight;
  p.dbias = g->dbias;
  const hipStream_t st = (hipStream_t)stream;
  if (a->T > 0 && (rc = with_vector(*a, vec, [&](auto t, auto v) { return launch_norm_backward<decltype(t), v.value>(c, a->per_step, p, st); }))) return rc;
  if ((!g->dweight && !g->dbias) || (a->T > 0 && c.chunks)) return SNN_OK;
  hipLaunchKernelGGL(norm_sum_kernel, dim3(parameter_blocks(a->D)), dim3(256), 0, st, p.dpart, a->T > 0 ? p.units * c.blocks : 0, a->D, g->dweight,
                     g->dbias);
  return ops_launched("group norm backward, gradients of the parameters");
}

}  // extern "C"
