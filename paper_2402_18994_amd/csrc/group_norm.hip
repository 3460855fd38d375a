// Group norm with an optional SiLU, channels fastest (include/snn_ops.h):
//   xh = (x - mean) rstd, rstd = 1 / sqrt(variance + eps), v = xh w + b, y = v or v sigmoid(v);  q = dy y'(v), p = q w:
//   dx = rstd (p - mean(p) - xh mean(p xh)), dw = sum q xh, db = sum q.
// Means run over the channels of a group and, unless per_step, the steps of the sequence that exist.
//
// What bounds it is memory, so x (and dy) are read once where they can be: a workgroup holds a chunk, rows by the channels of one
// group, in registers, forms the mean, then the squares around it, and writes the outputs.  Where a sequence's group is more
// than one chunk, or there are too few groups to fill the chip, one launch leaves every chunk's (mean, sum of squares around it) and
// a second one joins them and reads the rows again.  Sums over rows (dw, db) leave a row per chunk that a last launch adds up.
#include "rows.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

enum { WHOLE = 0, SUMS = 1, APPLY = 2, STEP = 3 };           // what a launch does: all; a chunk's sums; the rest; rows by themselves

struct NormP {
  int T, B, D, G, C, silu;
  float eps;
  int64_t rows;                             // of a unit: T of a sequence, or T B where each row stands alone
  int units, nchunk, loops;                 // loops: chunks that a workgroup takes in turn
  int tpr_log2, K, R;                       // threads a row; column blocks of a row; rows of a thread
  Rows<void> x, y;
  const float *weight, *bias;
  const int32_t *lengths;
  float2 *saved;                            // [units or rows][G]: mean, rstd
  float2 *part;                             // [units][G][nchunk]: a chunk's sums
  // reverse
  Rows<void> dy, dx;
  float *dpart;                             // [units * nchunk / loops][2][D]
};

__device__ __forceinline__ float wave_sum(float v, int width) {      // over aligned sets of `width` lanes, in all of them
  for (int o = 1; o < width; o <<= 1) v += __shfl_xor(v, o);
  return v;
}
// Over a workgroup, in all threads.  `lds` takes NT / 64 floats and is free again after the next barrier.
template <int NT> __device__ __forceinline__ float block_sum(float v, float *lds) {
  v = wave_sum(v, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) s += lds[w];
  return s;
}

template <typename T, int VEC> struct Slots {
  static constexpr int N = sizeof(T) * VEC == 16 ? 8 : 16;           // vectors of a thread
};

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

// Where the vectors of a thread lie.
template <typename T, int VEC, bool K1> struct Where {
  const NormP &a;
  int unit, g, len, rsub, col, rp;
  int64_t r0;
  bool step;
  __device__ __forceinline__ int k(int s) const { return K1 ? 0 : s / a.R; }
  __device__ __forceinline__ int channel(int s) const { return (k(s) << a.tpr_log2) * VEC + col * VEC; }      // within the group
  __device__ __forceinline__ int64_t row(int s) const { return r0 + (int64_t)(K1 ? s : s % a.R) * rp + rsub; }
  __device__ __forceinline__ bool there(int s) const { return row(s) < a.rows && channel(s) < a.C && (K1 ? s < a.R : s < a.K * a.R); }
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
    return (T *)r.p + b * r.sb + t * r.st + (int64_t)g * a.C + channel(s);
  }
};

template <typename T, int VEC, typename W, typename R>
__device__ __forceinline__ Pack<T, VEC> fetch(const W &w, const R &r, int s, bool live) {
  const Pack<T, VEC> v = *(const Pack<T, VEC> *)(live ? w.at(r, s) : (const T *)r.p);   // (the first row's is as good as any)
  const Pack<T, VEC> zero = {};
  return live ? v : zero;
}

template <int VEC> __device__ __forceinline__ void params(const NormP &a, int d, float (&w)[VEC], float (&b)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    w[v] = a.weight ? a.weight[d + v] : 1.f;
    b[v] = a.bias ? a.bias[d + v] : 0.f;
  }
}

template <typename T, int VEC, bool K1>
__device__ __forceinline__ Where<T, VEC, K1> where(const NormP &a, bool step, int nt) {
  const int64_t id = blockIdx.x;
  Where<T, VEC, K1> w{a, 0, 0, 0, 0, 0, 0, 0, step};
  w.g = (int)(id % a.G);
  const int64_t rest = id / a.G;
  w.unit = (int)(rest % a.units);
  w.rsub = (int)threadIdx.x >> a.tpr_log2;
  w.col = (int)threadIdx.x & ((1 << a.tpr_log2) - 1);
  w.rp = nt >> a.tpr_log2;
  w.r0 = (rest / a.units) * (int64_t)w.rp * a.R * a.loops;
  w.len = step ? 0 : __builtin_amdgcn_readfirstlane(length_of(a.lengths, w.unit, a.T));
  return w;
}
// The number of values of a unit's chunk.
__device__ __forceinline__ float chunk_count(const NormP &a, int64_t rows, int chunk, int len) {
  const int64_t n = (int64_t)len - chunk * rows;
  return (float)((n < 0 ? 0 : n < rows ? n : rows) * a.C);
}

// For each of a thread's rows (K1), or for its one row: the sum over the row.  `lds` takes SLOTS * NT / 64 floats.
template <int NT, int SLOTS, bool K1>
__device__ __forceinline__ void row_sums(const NormP &a, float (&v)[SLOTS], float *lds) {
  if (!K1) {
#pragma unroll
    for (int s = 1; s < SLOTS; ++s) v[0] += v[s];
    v[0] = block_sum<NT>(v[0], lds);
#pragma unroll
    for (int s = 1; s < SLOTS; ++s) v[s] = v[0];
    return;
  }
  const int width = min(64, 1 << a.tpr_log2);
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) v[s] = wave_sum(v[s], width);
  if (a.tpr_log2 <= 6) return;
  const int wave = threadIdx.x >> 6, each = 1 << (a.tpr_log2 - 6), first = wave & -each;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) lds[s * (NT / 64) + wave] = v[s];
  __syncthreads();
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    v[s] = 0.f;
    for (int w = 0; w < each; ++w) v[s] += lds[s * (NT / 64) + first + w];
  }
}

template <typename T, int VEC, int NT, int MODE, bool K1>
__global__ __launch_bounds__(NT) void norm_forward_kernel(const NormP a) {
  constexpr int SLOTS = Slots<T, VEC>::N;
  __shared__ float lds[2][SLOTS * (NT / 64)];
  auto w = where<T, VEC, K1>(a, MODE == STEP, NT);
  const int chunk = (int)(blockIdx.x / ((unsigned)a.G * (unsigned)a.units));
  Pack<T, VEC> x[SLOTS];
  bool live[SLOTS];
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    live[s] = w.live(s);
    x[s] = fetch<T, VEC>(w, a.x, s, live[s]);
  }
  float mean[SLOTS], rstd[SLOTS];                            // (MODE == STEP: of each row; the same in all otherwise)
  if (MODE == STEP) {
    const float n = 1.f / (float)a.C;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      mean[s] = 0.f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) mean[s] += widen(x[s].v[v]);
    }
    row_sums<NT, SLOTS, K1>(a, mean, lds[0]);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      mean[s] *= n;
      rstd[s] = 0.f;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float e = live[s] ? widen(x[s].v[v]) - mean[s] : 0.f;
        rstd[s] = fmaf(e, e, rstd[s]);
      }
    }
    row_sums<NT, SLOTS, K1>(a, rstd, lds[1]);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      rstd[s] = __builtin_amdgcn_rsqf(fmaf(rstd[s], n, a.eps));
      if (a.saved && w.col == 0 && (K1 || s == 0) && w.there(s)) a.saved[w.row(s) * a.G + w.g] = {mean[s], rstd[s]};
    }
  } else {
    const int64_t rows = (int64_t)w.rp * a.R;
    const int64_t first = ((int64_t)w.unit * a.G + w.g) * a.nchunk;
    float m, q = 0.f;
    if (MODE != APPLY) {
      const float n = MODE == WHOLE ? (float)((int64_t)w.len * a.C) : chunk_count(a, rows, chunk, w.len);
      m = 0.f;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s)
#pragma unroll
        for (int v = 0; v < VEC; ++v) m += widen(x[s].v[v]);
      m = block_sum<NT>(m, lds[0]) / fmaxf(n, 1.f);
#pragma unroll
      for (int s = 0; s < SLOTS; ++s)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float e = live[s] ? widen(x[s].v[v]) - m : 0.f;
          q = fmaf(e, e, q);
        }
      q = block_sum<NT>(q, lds[1]);
      if (MODE == SUMS) {
        if (threadIdx.x == 0) a.part[first + chunk] = {m, q};
        return;
      }
      q /= fmaxf(n, 1.f);
    } else {
      // mean of the chunks' means, each by its number; squares around it: a chunk's own, and its mean's distance
      const float n = fmaxf((float)((int64_t)w.len * a.C), 1.f);
      m = 0.f;
      for (int c = threadIdx.x; c < a.nchunk; c += NT) m += a.part[first + c].x * (chunk_count(a, rows, c, w.len) / n);
      m = block_sum<NT>(m, lds[0]);
      for (int c = threadIdx.x; c < a.nchunk; c += NT) {
        const float2 p = a.part[first + c];
        const float k = chunk_count(a, rows, c, w.len);
        q += k > 0.f ? p.y + k * (p.x - m) * (p.x - m) : 0.f;
      }
      q = block_sum<NT>(q, lds[1]) / n;
    }
    const float r = __builtin_amdgcn_rsqf(q + a.eps);
    if (a.saved && chunk == 0 && threadIdx.x == 0) a.saved[(int64_t)w.unit * a.G + w.g] = {m, r};
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      mean[s] = m;
      rstd[s] = r;
    }
  }
  float wt[VEC], bs[VEC];
  if (K1) params<VEC>(a, w.channel(0) < a.C ? w.g * a.C + w.channel(0) : 0, wt, bs);
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    if (!w.there(s)) continue;
    if (!K1) params<VEC>(a, w.g * a.C + w.channel(s), wt, bs);
    Pack<T, VEC> y;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float u = fmaf((widen(x[s].v[v]) - mean[s]) * rstd[s], wt[v], bs[v]);
      y.v[v] = narrow<T>(!live[s] ? 0.f : a.silu ? u * sigmoid_fast(u) : u);
    }
    *(Pack<T, VEC> *)w.at(a.y, s) = y;
  }
}

// Adds up `acc` over the threads of a workgroup that hold the same columns; thread `tid` < columns / VEC of the first row has the sum.
template <int VEC, int NT> __device__ __forceinline__ void column_sums(const NormP &a, float (&acc)[VEC], float *lds) {
  const int tpr = 1 << a.tpr_log2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    for (int o = tpr; o < 64; o <<= 1) acc[v] += __shfl_xor(acc[v], o);
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

template <typename T, int VEC, int NT, int MODE, bool K1>
__global__ __launch_bounds__(NT) void norm_backward_kernel(const NormP a) {
  constexpr int SLOTS = Slots<T, VEC>::N;
  __shared__ float lds[2][SLOTS * (NT / 64)];
  __shared__ float cols[MODE == APPLY ? 1 : NT * VEC];
  auto w = where<T, VEC, K1>(a, MODE == STEP, NT);
  const int chunk = (int)(blockIdx.x / ((unsigned)a.G * (unsigned)a.units));
  float wt[VEC], bs[VEC], dw[VEC], db[VEC];
  if (K1) params<VEC>(a, w.channel(0) < a.C ? w.g * a.C + w.channel(0) : 0, wt, bs);
#pragma unroll
  for (int v = 0; v < VEC; ++v) dw[v] = db[v] = 0.f;
  float *const out = a.dpart + ((int64_t)w.unit * (a.nchunk / a.loops) + chunk) * 2 * a.D + (int64_t)w.g * a.C;
  for (int loop = 0; loop < a.loops; ++loop, w.r0 += (int64_t)w.rp * a.R) {
    Pack<T, VEC> x[SLOTS], dy[SLOTS];
    bool live[SLOTS];
    float mean[SLOTS], rstd[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      live[s] = w.live(s);
      x[s] = fetch<T, VEC>(w, a.x, s, live[s]);
      dy[s] = fetch<T, VEC>(w, a.dy, s, live[s]);
      const float2 m = a.saved[MODE == STEP ? (live[s] ? w.row(s) : 0) * a.G + w.g : (int64_t)w.unit * a.G + w.g];
      mean[s] = m.x;
      rstd[s] = m.y;
    }
    float s1[SLOTS], s2[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      s1[s] = s2[s] = 0.f;
      if (!K1) params<VEC>(a, w.there(s) ? w.g * a.C + w.channel(s) : 0, wt, bs);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float xh = live[s] ? (widen(x[s].v[v]) - mean[s]) * rstd[s] : 0.f;
        float p;
        const float q = gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], a.silu, p);
        s1[s] += p;
        s2[s] = fmaf(p, xh, s2[s]);
        dw[v] = fmaf(q, xh, dw[v]);
        db[v] += q;
      }
      if (!K1 && MODE != APPLY && s % a.R == a.R - 1) {      // (a thread has these columns to itself)
        if (w.channel(s) < a.C && s < a.K * a.R)
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            float *const o = out + w.channel(s) + v;
            o[0] = loop ? o[0] + dw[v] : dw[v];
            o[a.D] = loop ? o[a.D] + db[v] : db[v];
          }
#pragma unroll
        for (int v = 0; v < VEC; ++v) dw[v] = db[v] = 0.f;
      }
    }
    if (MODE == STEP) {
      __syncthreads();                                       // (the sums of the loop before have been read)
      row_sums<NT, SLOTS, K1>(a, s1, lds[0]);
      row_sums<NT, SLOTS, K1>(a, s2, lds[1]);
      const float n = 1.f / (float)a.C;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        s1[s] *= n;
        s2[s] *= n;
      }
    } else {
      const float n = fmaxf((float)((int64_t)w.len * a.C), 1.f);
      const int64_t first = ((int64_t)w.unit * a.G + w.g) * a.nchunk;
      float p1 = 0.f, p2 = 0.f;
      if (MODE != APPLY) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
          p1 += s1[s];
          p2 += s2[s];
        }
      } else
        for (int c = threadIdx.x; c < a.nchunk; c += NT) {
          p1 += a.part[first + c].x;
          p2 += a.part[first + c].y;
        }
      p1 = block_sum<NT>(p1, lds[0]);
      p2 = block_sum<NT>(p2, lds[1]);
      if (MODE == SUMS) {
        if (threadIdx.x == 0) a.part[first + chunk] = {p1, p2};
        break;
      }
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        s1[s] = p1 / n;
        s2[s] = p2 / n;
      }
    }
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (!w.there(s)) continue;
      if (!K1) params<VEC>(a, w.g * a.C + w.channel(s), wt, bs);
      Pack<T, VEC> d;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float xh = (widen(x[s].v[v]) - mean[s]) * rstd[s];
        float p;
        gradient_of(widen(dy[s].v[v]), xh, wt[v], bs[v], a.silu, p);
        d.v[v] = narrow<T>(live[s] ? rstd[s] * (p - s1[s] - xh * s2[s]) : 0.f);
      }
      *(Pack<T, VEC> *)w.at(a.dx, s) = d;
    }
  }
  if (MODE == APPLY || !K1) return;
  column_sums<VEC, NT>(a, dw, cols);
  column_sums<VEC, NT>(a, db, cols);
  if ((int)threadIdx.x < (1 << a.tpr_log2) && w.col * VEC < a.C)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      out[w.col * VEC + v] = dw[v];
      out[a.D + w.col * VEC + v] = db[v];
    }
}

__global__ __launch_bounds__(256) void norm_sum_kernel(const float *__restrict__ part, int rows, int D, float *dweight, float *dbias) {
  __shared__ float lds[256];
  const int64_t col = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
  const float s = sum_column(part, 2 * (int64_t)D, col, rows, lds);
  if (threadIdx.x >= 16) return;
  if (col < D) {
    if (dweight) dweight[col] = s;
  } else if (col < 2 * (int64_t)D && dbias) dbias[col - D] = s;
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

// How a call is cut, for `vec` channels a vector.
struct NormCut {
  int nt, tpr_log2, K, R, loops, blocks;       // blocks: chunks a unit, by loops
  int64_t nchunk;
};
int slots_of(int vec, size_t z) { return vec * z == 16 ? 8 : 16; }
NormCut norm_cut(const snn_norm_args &a, int vec, bool backward) {
  const size_t z = a.type == SNN_TYPE_FP32 ? 4 : 2;
  const int C = a.D / a.groups, slots = slots_of(vec, z);
  const int64_t rows = a.per_step ? (int64_t)a.T * a.B : a.T, units = a.per_step ? 1 : a.B;
  NormCut c;
  auto fit = [&](int nt) {
    c.nt = nt;
    c.tpr_log2 = 0;
    while ((vec << c.tpr_log2) < C && (1 << c.tpr_log2) < nt) ++c.tpr_log2;
    c.K = (C + (vec << c.tpr_log2) - 1) / (vec << c.tpr_log2);
    c.R = c.K == 1 ? slots : a.per_step ? 1 : std::max(1, slots / c.K);
    const int64_t each = (int64_t)(nt >> c.tpr_log2) * c.R;
    c.nchunk = std::max<int64_t>(1, (rows + each - 1) / each);
  };
  fit(256);
  if (c.K > slots || (!a.per_step && c.nchunk > 1 && units * a.groups >= 128)) fit(1024);
  if (!a.per_step && c.nchunk > 1 && c.nt == 1024 && c.K <= slots) {
    const NormCut wide = c;
    fit(256);
    if (c.K > slots) c = wide;
  }
  if (a.per_step && c.K == 1)                    // (few rows: fewer a thread, more workgroups)
    while (c.R > 1 && c.nchunk * a.groups < 512) {
      c.R /= 2;
      const int64_t each = (int64_t)(c.nt >> c.tpr_log2) * c.R;
      c.nchunk = std::max<int64_t>(1, (rows + each - 1) / each);
    }
  c.loops = 1;
  if (a.per_step && backward)                    // (fewer rows of partial sums, as long as the chip is filled)
    while (c.loops < 32 && c.nchunk / (c.loops * 2) * a.groups >= 1024) c.loops *= 2;
  c.blocks = (int)((c.nchunk + c.loops - 1) / c.loops);
  c.nchunk = (int64_t)c.blocks * c.loops;
  return c;
}
int norm_vector(const snn_norm_args &a, const snn_norm_grads *g) {
  const size_t z = a.type == SNN_TYPE_FP32 ? 4 : 2;
  for (int vec : {(int)(16 / z), 2}) {
    auto take = [&](const snn_rows &r) { return rows_take(r, a.T, a.B, vec, z); };
    if (a.D / a.groups % vec == 0 && take(a.x) && (g ? take(g->dy) && take(g->dx) : take(a.y))) return vec;
  }
  return 1;
}
// The workspace does not depend on the pointers, which decide how many channels a vector has.
size_t norm_bytes(const snn_norm_args &a, bool backward) {
  size_t most = 0;
  for (int vec : {a.type == SNN_TYPE_FP32 ? 4 : 8, 2, 1}) {
    const NormCut c = norm_cut(a, vec, backward);
    const size_t units = a.per_step ? 1 : a.B;
    const size_t part = !a.per_step && c.nchunk > 1 ? rup256(units * a.groups * c.nchunk * 8) : 0;
    most = std::max(most, part + (backward ? rup256(units * c.blocks * 2 * (size_t)a.D * 4) : 0));
  }
  return most;
}

template <typename F> int with_vector(const snn_norm_args &a, int vec, const NormCut &c, F f) {
  auto deep = [&](auto t, auto v) {
    auto k = [&](auto nt) { return c.K == 1 ? f(t, v, nt, std::true_type()) : f(t, v, nt, std::false_type()); };
    return c.nt == 256 ? k(std::integral_constant<int, 256>()) : k(std::integral_constant<int, 1024>());
  };
  using std::integral_constant;
  if (a.type == SNN_TYPE_FP32)
    return vec == 4 ? deep(float(), integral_constant<int, 4>()) : vec == 2 ? deep(float(), integral_constant<int, 2>()) : deep(float(), integral_constant<int, 1>());
  return vec == 8 ? deep(__bf16(), integral_constant<int, 8>()) : vec == 2 ? deep(__bf16(), integral_constant<int, 2>()) : deep(__bf16(), integral_constant<int, 1>());
}

NormP norm_args(const snn_norm_args &a, const NormCut &c, void *saved, void *workspace) {
  NormP p{a.T, a.B, a.D, a.groups, a.D / a.groups, a.silu, a.eps, a.per_step ? (int64_t)a.T * a.B : a.T, a.per_step ? 1 : a.B, (int)c.nchunk, c.loops,
          c.tpr_log2, c.K, c.R, Rows<void>(a.x, a.T), Rows<void>(a.y, a.T), a.weight, a.bias, a.lengths, (float2 *)saved, (float2 *)workspace,
          Rows<void>(snn_rows{}), Rows<void>(snn_rows{}), nullptr};
  return p;
}
int norm_grid(const snn_norm_args &a, const NormCut &c, dim3 &grid) {
  const int64_t n = (int64_t)a.groups * (a.per_step ? 1 : a.B) * c.blocks;
  if (n * c.nt >= (1ll << 32)) return ops_fail(SNN_ERR_ARG, "group norm: too large for one launch");
  grid = dim3((unsigned)n);
  return SNN_OK;
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
  dim3 grid;
  if ((rc = norm_grid(*a, c, grid))) return rc;
  const NormP p = norm_args(*a, c, saved, workspace);
  const hipStream_t st = (hipStream_t)stream;
  return with_vector(*a, vec, c, [&](auto t, auto v, auto nt, auto k1) {
    using T = decltype(t);
    constexpr int V = v.value, N = nt.value;
    constexpr bool K1 = decltype(k1)::value;
    if (a->per_step) hipLaunchKernelGGL((norm_forward_kernel<T, V, N, STEP, K1>), grid, dim3(N), 0, st, p);
    else if (c.nchunk == 1) hipLaunchKernelGGL((norm_forward_kernel<T, V, N, WHOLE, K1>), grid, dim3(N), 0, st, p);
    else {
      hipLaunchKernelGGL((norm_forward_kernel<T, V, N, SUMS, K1>), grid, dim3(N), 0, st, p);
      const int e = ops_launched("group norm, sums");
      if (e) return e;
      hipLaunchKernelGGL((norm_forward_kernel<T, V, N, APPLY, K1>), grid, dim3(N), 0, st, p);
    }
    return ops_launched("group norm");
  });
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
  dim3 grid;
  if ((rc = norm_grid(*a, c, grid))) return rc;
  NormP p = norm_args(*a, c, const_cast<void *>(saved), workspace);
  const int units = p.units;
  p.dy = Rows<void>(g->dy, a->T);
  p.dx = Rows<void>(g->dx, a->T);
  p.dpart = (float *)((char *)workspace + (!a->per_step && c.nchunk > 1 ? rup256((size_t)units * a->groups * c.nchunk * 8) : 0));
  const hipStream_t st = (hipStream_t)stream;
  if (a->T > 0) {
    rc = with_vector(*a, vec, c, [&](auto t, auto v, auto nt, auto k1) {
      using T = decltype(t);
      constexpr int V = v.value, N = nt.value;
      constexpr bool K1 = decltype(k1)::value;
      if (a->per_step) hipLaunchKernelGGL((norm_backward_kernel<T, V, N, STEP, K1>), grid, dim3(N), 0, st, p);
      else if (c.nchunk == 1) hipLaunchKernelGGL((norm_backward_kernel<T, V, N, WHOLE, K1>), grid, dim3(N), 0, st, p);
      else {
        hipLaunchKernelGGL((norm_backward_kernel<T, V, N, SUMS, K1>), grid, dim3(N), 0, st, p);
        const int e = ops_launched("group norm backward, sums");
        if (e) return e;
        hipLaunchKernelGGL((norm_backward_kernel<T, V, N, APPLY, K1>), grid, dim3(N), 0, st, p);
      }
      return ops_launched("group norm backward");
    });
    if (rc) return rc;
  }
  if (!g->dweight && !g->dbias) return SNN_OK;
  hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((2 * (int64_t)a->D + 15) / 16)), dim3(256), 0, st, p.dpart, a->T > 0 ? units * c.blocks : 0, a->D, g->dweight,
                     g->dbias);
  return ops_launched("group norm backward, gradients of the parameters");
}

}  // extern "C"
