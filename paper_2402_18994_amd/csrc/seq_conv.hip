// Short causal convolution along time, one filter of W taps per channel (include/snn_ops.h):
//   v[t,d] = bias[d] + sum_(k<W) w[d,k] x[t-(W-1)+k, d],  y = v or v sigmoid(v).
// Every row piece is read once and written once.  Tensors are time-major with the channels fastest; a
// wavefront owns 64 lanes x VEC neighbouring channels of one sequence and walks a segment of its steps with the last
// W - 1 inputs in registers, AHEAD rows in flight.  Sequence, segment and length are the same for the whole wavefront,
// so all tests are on scalars, and a row that does not exist is a buffer access that the hardware drops.
// Measured, bfloat16, four taps: 1024 steps of 8 x 2048 channels 14.4 us a call, 67 MB at 4.7 TB/s (a copy of that size, which
// the last-level cache holds, reaches 7.8); fp32 26.4 us; forward 27 and backward 44 us for 256 steps of 128 x 1024 channels of
// uneven lengths, of which half the rows exist (0.10 and 0.13 GB); the sums of the filter's gradients 4.4 us.
// What bounds it is waiting: loads and stores of a wavefront come back in one order.  Forward, the filter is first waited for
// inside the loop, so that every round of it also waits for the stores of the round before; reverse, the row of d_state is asked
// for last and used at once, in every row, so that all that is outstanding is waited for twice in a round of two.
#include "common.hpp"
#include "seq_common.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

constexpr int AHEAD = 4;            // rows in flight per wavefront, forward (8: 2 to 7 % slower) ..
constexpr int AHEAD_BWD = 2;        // .. and of x and of dy each, reverse (4: 1 % either way, as every row waits for all of them)
constexpr int SPAN = 0x7FFF0000, NOWHERE = 0x7FFFFF00;     // see seq_scan.hip: lane offsets stay below the first

struct ConvP {
  int T, B, D, silu, seg, nseg, groups;                    // groups: of 64 * VEC channels
  Rows<void> x, y;
  const float *weight, *bias;
  const void *init;
  const int32_t *lengths;
  void *state;
  explicit ConvP(const snn_conv_args &a)
      : T(a.T), B(a.B), D(a.D), silu(a.silu), seg(1), nseg(1), groups(1), x(a.x), y(a.y), weight(a.weight), bias(a.bias), init(a.init),
        lengths(a.lengths), state(a.state) {}
};

template <typename T, int VEC, int W>
__device__ __forceinline__ void load_filter(const ConvP &a, int d, float w[W][VEC], float bias[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    bias[v] = a.bias ? a.bias[d + v] : 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k][v] = a.weight[(size_t)(d + v) * W + k];
  }
}

// VEC channels of a row; `on` (a scalar): whether the row exists, zeros if not.  `at`: the lane's byte offset.
template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> load_row(const T *row, int at, bool on) {
  using Packed = Pack<T, VEC>;
  const rsrc_t r = make_rsrc(row, SPAN);
  const int off = on ? at : NOWHERE;
  if constexpr (sizeof(T) * VEC == 16) return __builtin_bit_cast(Packed, ld_b128(r, off, 0));
  else if constexpr (sizeof(T) * VEC == 8) return __builtin_bit_cast(Packed, ld_b64(r, off, 0));
  else if constexpr (sizeof(T) * VEC == 4) return __builtin_bit_cast(Packed, ld_b32(r, off, 0));
  else return __builtin_bit_cast(Packed, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0));
}
template <typename T, int VEC> __device__ __forceinline__ void store_row(T *row, int at, Pack<T, VEC> v) {
  const rsrc_t r = make_rsrc(row, SPAN);
  if constexpr (sizeof(T) * VEC == 16) st_b128(r, at, 0, __builtin_bit_cast(u32x4, v));
  else if constexpr (sizeof(T) * VEC == 8) st_b64(r, at, 0, __builtin_bit_cast(u32x2, v));
  else if constexpr (sizeof(T) * VEC == 4) st_b32(r, at, 0, __builtin_bit_cast(uint32_t, v));
  else st_b16(r, at, 0, __builtin_bit_cast(unsigned short, v));
}
// Rows [t0, t1), which do not exist.  Segments of such rows alone, those that start behind a sequence's end, are written
// by this and cost nothing else; a first segment has the state to see to and is never one.
template <typename T, int VEC> __device__ __forceinline__ void store_zeros(T *base, int64_t st, int at, int t0, int t1) {
  const Pack<T, VEC> zero = {};
  for (int t = t0; t < t1; ++t) store_row<T, VEC>(base + t * st, at, zero);
}
// Row `t` of the input of sequence b, from -(W-1) on; zeros before the first step without `init`, and for t >= end.
template <typename T, int VEC, int W>
__device__ __forceinline__ Pack<T, VEC> input_row(const ConvP &a, int b, int at, int t, int end) {
  const T *p = t >= 0 ? (const T *)a.x.p + b * a.x.sb + t * a.x.st : (const T *)a.init + ((int64_t)(t + W - 1) * a.B + b) * a.D;
  return load_row<T, VEC>(p, at, t >= 0 ? t < end : a.init != nullptr);
}

// Forward.  A wavefront takes one (segment, sequence, channel group), in the order of the memory: wavefronts that run at
// the same time share rows of it.
template <typename T, int VEC, int W>
__global__ __launch_bounds__(256) void conv_forward_kernel(const ConvP a) {
  const int lane = threadIdx.x & 63;
  int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = (int)(id % a.groups);
  id /= a.groups;
  const int b = (int)(id % a.B), s = (int)(id / a.B);
  if (s >= a.nseg) return;
  const int len = __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T));
  const int d = (group * 64 + lane) * VEC;
  const bool live = d < a.D;
  const int at = live ? d * (int)sizeof(T) : NOWHERE;
  const int t0 = s * a.seg, t1 = min(a.T, t0 + a.seg), end = min(t1, len);
  T *y = (T *)a.y.p + b * a.y.sb;

  if (s > 0 && t0 >= len) {
    store_zeros<T, VEC>(y, a.y.st, at, t0, t1);
    return;
  }
  float w[W][VEC], bias[VEC], xs[W - 1 + AHEAD][VEC];
  load_filter<T, VEC, W>(a, live ? d : 0, w, bias);
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const Pack<T, VEC> r = input_row<T, VEC, W>(a, b, at, t0 - (W - 1) + k, len);
#pragma unroll
    for (int v = 0; v < VEC; ++v) xs[k][v] = widen(r.v[v]);
  }
  const T *x = (const T *)a.x.p + b * a.x.sb;
  Pack<T, VEC> next[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) next[u] = load_row<T, VEC>(x + (t0 + u) * a.x.st, at, t0 + u < end);
  for (int t = t0; t < t1; t += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int v = 0; v < VEC; ++v) xs[W - 1 + u][v] = widen(next[u].v[v]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) next[u] = load_row<T, VEC>(x + (t + AHEAD + u) * a.x.st, at, t + AHEAD + u < end);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      Pack<T, VEC> r;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float q = bias[v];
#pragma unroll
        for (int k = 0; k < W; ++k) q = fmaf(w[k][v], xs[u + k][v], q);
        const float g = q * sigmoid_fast(q);
        r.v[v] = narrow<T>(t + u < len ? (a.silu ? g : q) : 0.f);
      }
      store_row<T, VEC>(y + (t + u) * a.y.st, t + u < t1 ? at : NOWHERE, r);
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) xs[k][v] = xs[k + AHEAD][v];
  }
  if (a.state && s == 0) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
      store_row<T, VEC>((T *)a.state + ((int64_t)j * a.B + b) * a.D, at, input_row<T, VEC, W>(a, b, at, len - (W - 1) + j, len));
  }
}

// One step: the state [W-1][B][D] moves up a row.  64 x 2048 channels in bfloat16 4.3 us: the launch.
template <typename T, int VEC, int W>
__global__ __launch_bounds__(256) void conv_step_kernel(const ConvP a) {
  const int dv = a.D / VEC;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)a.B * dv) return;
  const int b = (int)(id / dv), d = (int)(id % dv) * VEC;
  const size_t at = (size_t)b * a.D + d, row = (size_t)a.B * a.D;
  T *state = (T *)a.state + at;
  float w[W][VEC], s[VEC];
  Pack<T, VEC> r[W];
#pragma unroll
  for (int k = 0; k < W - 1; ++k) r[k] = *(const Pack<T, VEC> *)(state + k * row);
  r[W - 1] = *(const Pack<T, VEC> *)((const T *)a.x.p + b * a.x.sb + d);
  load_filter<T, VEC, W>(a, d, w, s);
  Pack<T, VEC> out;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
#pragma unroll
    for (int k = 0; k < W; ++k) s[v] = fmaf(w[k][v], widen(r[k].v[v]), s[v]);
    if (a.silu) s[v] *= sigmoid_fast(s[v]);
    out.v[v] = narrow<T>(s[v]);
  }
  *(Pack<T, VEC> *)((T *)a.y.p + b * a.y.sb + d) = out;
#pragma unroll
  for (int k = 0; k < W - 1; ++k) *(Pack<T, VEC> *)(state + k * row) = r[k + 1];
}

// Backward.  With q[t] = dL/dv at step t, which is dy[t] times the slope of f (zero outside [0, len)):
//   dx[s] = sum_k w[k] q[s + (W-1) - k],  dw[k] = sum_(t,b) q[t] x[t-(W-1)+k],  dbias = sum_(t,b) q[t].
// A wavefront walks its segment of a sequence and W - 1 steps more (dx of the last steps needs their q; v is computed
// again from x), emitting the gradient of input row t - (W-1) at step t.  The four wavefronts of a workgroup are on the
// same channels; each takes (sequence, segment) items in turn, with dw and dbias in registers, and at the end their
// sums go through LDS into one partial sum per workgroup, added up by conv_sum_kernel in a fixed order.
struct ConvGradP {
  Rows<void> dy, dx;
  const void *d_state;
  void *dinit;
  float *partial;                    // [gridDim.y][W+1][D]
  ConvGradP(const snn_conv_grads &g, float *ws) : dy(g.dy), dx(g.dx), d_state(g.d_state), dinit(g.dinit), partial(ws) {}
};

template <typename T, int VEC, int W>
__global__ __launch_bounds__(256) void conv_backward_kernel(const ConvP a, const ConvGradP g) {
  __shared__ float part[4][64 * VEC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = (blockIdx.x * 64 + lane) * VEC;
  const bool live = d < a.D;
  const int at = live ? d * (int)sizeof(T) : NOWHERE;
  float w[W][VEC], bias[VEC], dw[W][VEC], db[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    db[v] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) dw[k][v] = 0.f;
  }
  load_filter<T, VEC, W>(a, live ? d : 0, w, bias);
  const int64_t items = (int64_t)a.B * a.nseg;
  for (int64_t item = (int64_t)blockIdx.y * 4 + wave; item < items; item += (int64_t)gridDim.y * 4) {
    const int b = (int)(item % a.B), s0 = (int)(item / a.B);
    const int len = __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T));
    const T *x = (const T *)a.x.p + b * a.x.sb;
    const T *dy = (const T *)g.dy.p + b * g.dy.sb;
    T *dx = (T *)g.dx.p + b * g.dx.sb;
    const int t0 = s0 * a.seg, t1 = min(a.T, t0 + a.seg), stop = t1 + W - 1, end = min(stop, len);
    if (s0 > 0 && t0 >= len) {
      store_zeros<T, VEC>(dx, g.dx.st, at, t0, t1);
      continue;
    }
    float xs[W - 1 + AHEAD_BWD][VEC], q[W - 1 + AHEAD_BWD][VEC];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      const Pack<T, VEC> r = input_row<T, VEC, W>(a, b, at, t0 - (W - 1) + k, len);
#pragma unroll
      for (int v = 0; v < VEC; ++v) { xs[k][v] = widen(r.v[v]); q[k][v] = 0.f; }
    }
    Pack<T, VEC> nx[AHEAD_BWD], ny[AHEAD_BWD];
    const auto fetch = [&](int t) {
#pragma unroll
      for (int u = 0; u < AHEAD_BWD; ++u) {
        nx[u] = load_row<T, VEC>(x + (t + u) * a.x.st, at, t + u < end);
        ny[u] = load_row<T, VEC>(dy + (t + u) * g.dy.st, at, t + u < end);
      }
    };
    fetch(t0);
    for (int t = t0; t < stop; t += AHEAD_BWD) {
#pragma unroll
      for (int u = 0; u < AHEAD_BWD; ++u)
#pragma unroll
        for (int v = 0; v < VEC; ++v) { xs[W - 1 + u][v] = widen(nx[u].v[v]); q[W - 1 + u][v] = widen(ny[u].v[v]); }
      fetch(t + AHEAD_BWD);
#pragma unroll
      for (int u = 0; u < AHEAD_BWD; ++u) {
        const int now = t + u, j = now - len;               // j: row of d_state that belongs to input row now - (W-1)
        const bool kept = g.d_state && j >= 0 && j < W - 1;
        const Pack<T, VEC> ds = load_row<T, VEC>((const T *)g.d_state + ((int64_t)j * a.B + b) * a.D, at, kept);
        Pack<T, VEC> out;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          float &qv = q[W - 1 + u][v];
          if (a.silu) {
            float r = bias[v];
#pragma unroll
            for (int k = 0; k < W; ++k) r = fmaf(w[k][v], xs[u + k][v], r);
            const float e = sigmoid_fast(r);
            qv *= e * (1.f + r * (1.f - e));
          }
          qv = now < len ? qv : 0.f;
          float sum = widen(ds.v[v]);
#pragma unroll
          for (int k = 0; k < W; ++k) sum = fmaf(w[k][v], q[W - 1 + u - k][v], sum);
          out.v[v] = narrow<T>(sum);
        }
        if (now < min(t1, len)) {                           // (beyond, q may be zero and the inputs infinite: 0 inf is no zero)
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            db[v] += q[W - 1 + u][v];
#pragma unroll
            for (int k = 0; k < W; ++k) dw[k][v] = fmaf(q[W - 1 + u][v], xs[u + k][v], dw[k][v]);
          }
        }
        const int r = now - (W - 1);
        if (r >= 0) store_row<T, VEC>(dx + r * g.dx.st, (r >= t0) & (now < stop) ? at : NOWHERE, out);
        else store_row<T, VEC>((T *)g.dinit + ((int64_t)now * a.B + b) * a.D, g.dinit != nullptr ? at : NOWHERE, out);
      }
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
#pragma unroll
        for (int v = 0; v < VEC; ++v) { xs[k][v] = xs[k + AHEAD_BWD][v]; q[k][v] = q[k + AHEAD_BWD][v]; }
    }
  }
#pragma unroll
  for (int k = 0; k <= W; ++k) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) part[wave][lane * VEC + v] = k < W ? dw[k < W ? k : 0][v] : db[v];
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * VEC; c += 256) {
      const int col = blockIdx.x * 64 * VEC + c;
      if (col < a.D) g.partial[((size_t)blockIdx.y * (W + 1) + k) * a.D + col] = ((part[0][c] + part[1][c]) + part[2][c]) + part[3][c];
    }
    __syncthreads();
  }
}

// dweight[d][k] and dbias[d]: sums of `rows` partial sums [W+1][D].
__global__ __launch_bounds__(256) void conv_sum_kernel(const float *__restrict__ partial, int rows, int W, int D,
                                                       float *__restrict__ dweight, float *__restrict__ dbias) {
  __shared__ float lds[256];
  const int64_t cols = (int64_t)(W + 1) * D, c = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
  const float s = sum_column(partial, cols, c, rows, lds);
  if (threadIdx.x < 16 && c < cols) {
    const int k = (int)(c / D), d = (int)(c % D);
    if (k < W) dweight[(size_t)d * W + k] = s;
    else if (dbias) dbias[d] = s;
  }
}

// ---------------------------------------------------------------- host side
int conv_check(const snn_conv_args *a, bool step, bool grads) {
  if (!a) return ops_fail(SNN_ERR_NULL, "convolution: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0) return ops_fail(SNN_ERR_ARG, "convolution: T >= 0, B > 0 and D > 0 are required");
  if ((int64_t)a->B * a->D >= (1ll << 31) || a->D > (1 << 28)) return ops_fail(SNN_ERR_ARG, "convolution: B * D must stay below 2^31, D must not exceed 2^28");
  if (a->T > (1 << 30)) return ops_fail(SNN_ERR_ARG, "convolution: T must not exceed 2^30");
  if (a->W < 1 || a->W > SNN_CONV_MAX_TAPS) return ops_fail(SNN_ERR_ARG, "convolution: W must be 1 to %d", SNN_CONV_MAX_TAPS);
  if (a->type != SNN_TYPE_FP32 && a->type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "convolution: unknown type %d", a->type);
  if (!a->weight) return ops_fail(SNN_ERR_NULL, "convolution: weight is NULL");
  if (a->T > 0 && (!a->x.p || (!grads && !a->y.p))) return ops_fail(SNN_ERR_NULL, "convolution: x or y is NULL");
  if (step) {
    if (a->T != 1) return ops_fail(SNN_ERR_ARG, "convolution step: T must be 1");
    if (a->init || a->lengths) return ops_fail(SNN_ERR_ARG, "convolution step: init and lengths must be NULL");
    if (!a->state && a->W > 1) return ops_fail(SNN_ERR_NULL, "convolution step: state is NULL");
  }
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(a->x.p, z) || !aligned(a->y.p, z) || !aligned(a->init, z) || !aligned(a->state, z) || !aligned(a->weight, 4) ||
      !aligned(a->bias, 4) || !aligned(a->lengths, 4))
    return ops_fail(SNN_ERR_ARG, "convolution: a pointer is not aligned to its element type");
  return SNN_OK;
}

bool rows_allow(const snn_rows &r, int T, int B, int vec, size_t bytes) {
  return !r.p || (aligned(r.p, bytes) && (T <= 1 || r.stride_t % vec == 0) && (B <= 1 || r.stride_b % vec == 0));
}
// Whether rows can be taken `vec` channels at a time.
bool conv_vector(const snn_conv_args &a, int vec, const snn_conv_grads *g, bool step) {
  const size_t bytes = (a.type == SNN_TYPE_FP32 ? 4 : 2) * (size_t)vec;
  const int T = step ? 1 : a.T;
  return a.D % vec == 0 && rows_allow(a.x, T, a.B, vec, bytes) && aligned(a.init, bytes) &&
         (g ? rows_allow(g->dy, T, a.B, vec, bytes) && rows_allow(g->dx, T, a.B, vec, bytes) && aligned(g->d_state, bytes) && aligned(g->dinit, bytes)
            : rows_allow(a.y, T, a.B, vec, bytes) && aligned(a.state, bytes));
}
// Four channels a lane where a row has more than one wavefront of single ones (a wavefront that is half empty with four
// is full with one).
int conv_width(const snn_conv_args &a, const snn_conv_grads *g) { return a.D > 64 && conv_vector(a, 4, g, false) ? 4 : 1; }

// How a call is cut: channel groups, steps per segment, and for the reverse pass workgroups over the items.  Segments of
// 32 steps, of 16 where that leaves fewer than 4096 wavefronts (W - 1 rows of each are read twice).  us of a call, 16 and
// 32 steps: forward, 2048 wavefronts (1024 steps of 8 x 2048 channels, bf16) 15.8 and 16.7, 16384 wavefronts 113 and
// 108; forward and reverse, 2048 wavefronts 51.2 and 53.2, 4096 wavefronts 87.8 and 79.9; 64 steps are slower by more.
struct ConvCut {
  int groups, seg, nseg, gy;
};
ConvCut conv_cut(const snn_conv_args &a, int vec) {
  ConvCut c;
  c.groups = (a.D + 64 * vec - 1) / (64 * vec);
  c.seg = (int64_t)c.groups * a.B * (a.T / 32) < 4096 ? 16 : 32;
  c.nseg = a.T > c.seg ? (a.T + c.seg - 1) / c.seg : 1;
  const int64_t all = ((int64_t)a.B * c.nseg + 3) / 4, want = std::max(1, 1024 / c.groups);
  c.gy = (int)std::min(all, want);
  return c;
}

template <typename F> int with_taps(int W, F f) {
  switch (W) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    case 7: return f(std::integral_constant<int, 7>());
    default: return f(std::integral_constant<int, 8>());
  }
}

template <typename T, int VEC> int launch_forward(const snn_conv_args &a, hipStream_t st) {
  ConvP p(a);
  const ConvCut c = conv_cut(a, VEC);
  p.seg = c.seg; p.nseg = c.nseg; p.groups = c.groups;
  const int64_t waves = (int64_t)a.B * c.nseg * c.groups;
  if (waves >= (1ll << 26)) return ops_fail(SNN_ERR_ARG, "convolution: too large for one launch");
  return with_taps(a.W, [&](auto w) {
    hipLaunchKernelGGL((conv_forward_kernel<T, VEC, w.value>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, p);
    return ops_launched("convolution");
  });
}
template <typename T, int VEC> int launch_step(const snn_conv_args &a, hipStream_t st) {
  const ConvP p(a);
  const int64_t threads = (int64_t)a.B * (a.D / VEC);
  return with_taps(a.W, [&](auto w) {
    hipLaunchKernelGGL((conv_step_kernel<T, VEC, w.value>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p);
    return ops_launched("convolution step");
  });
}
template <typename T, int VEC> int launch_backward(const snn_conv_args &a, const snn_conv_grads &g, float *ws, hipStream_t st) {
  ConvP p(a);
  const ConvGradP q(g, ws);
  const ConvCut c = conv_cut(a, VEC);
  p.seg = c.seg; p.nseg = c.nseg; p.groups = c.groups;
  return with_taps(a.W, [&](auto w) {
    hipLaunchKernelGGL((conv_backward_kernel<T, VEC, w.value>), dim3(c.groups, c.gy), dim3(256), 0, st, p, q);
    int rc = ops_launched("convolution backward");
    if (rc) return rc;
    const int64_t cols = (int64_t)(a.W + 1) * a.D;
    hipLaunchKernelGGL(conv_sum_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(256), 0, st, ws, c.gy, a.W, a.D, g.dweight, g.dbias);
    return ops_launched("convolution backward, sums");
  });
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" {

int32_t snn_conv_forward(const snn_conv_args *a, void *stream) {
  int rc = conv_check(a, false, false);
  if (rc) return rc;
  const hipStream_t st = (hipStream_t)stream;
  const bool four = conv_width(*a, nullptr) == 4;
  if (a->type == SNN_TYPE_FP32) return four ? launch_forward<float, 4>(*a, st) : launch_forward<float, 1>(*a, st);
  return four ? launch_forward<__bf16, 4>(*a, st) : launch_forward<__bf16, 1>(*a, st);
}

int32_t snn_conv_workspace_bytes(const snn_conv_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  if (!a) return ops_fail(SNN_ERR_NULL, "convolution: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0 || (int64_t)a->B * a->D >= (1ll << 31) || a->D > (1 << 28) || a->T > (1 << 30) || a->W < 1 || a->W > SNN_CONV_MAX_TAPS)
    return ops_fail(SNN_ERR_ARG, "convolution: sizes out of range");
  const int gy1 = conv_cut(*a, 1).gy, gy4 = conv_cut(*a, 4).gy;   // (which one runs depends on the pointers too)
  *bytes = rup256((size_t)(gy1 > gy4 ? gy1 : gy4) * (a->W + 1) * a->D * 4);
  return SNN_OK;
}

int32_t snn_conv_backward(const snn_conv_args *a, const snn_conv_grads *g, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = conv_check(a, false, true);
  if (rc) return rc;
  if (!g || !g->dweight || (a->T > 0 && (!g->dy.p || !g->dx.p))) return ops_fail(SNN_ERR_NULL, "convolution backward: dy, dx or dweight is NULL");
  size_t need = 0;
  if ((rc = snn_conv_workspace_bytes(a, &need))) return rc;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
    return ops_fail(SNN_ERR_WORKSPACE, "convolution backward: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(g->dy.p, z) || !aligned(g->dx.p, z) || !aligned(g->d_state, z) || !aligned(g->dinit, z) || !aligned(g->dweight, 4) || !aligned(g->dbias, 4))
    return ops_fail(SNN_ERR_ARG, "convolution backward: a pointer is not aligned to its element type");
  const hipStream_t st = (hipStream_t)stream;
  float *ws = (float *)workspace;
  const bool vec = conv_width(*a, g) == 4;
  if (a->type == SNN_TYPE_FP32) return vec ? launch_backward<float, 4>(*a, *g, ws, st) : launch_backward<float, 1>(*a, *g, ws, st);
  return vec ? launch_backward<__bf16, 4>(*a, *g, ws, st) : launch_backward<__bf16, 1>(*a, *g, ws, st);
}

int32_t snn_conv_step(const snn_conv_args *a, void *stream) {
  int rc = conv_check(a, true, false);
  if (rc) return rc;
  const hipStream_t st = (hipStream_t)stream;
  if (a->type == SNN_TYPE_FP32) return conv_vector(*a, 4, nullptr, true) ? launch_step<float, 4>(*a, st) : launch_step<float, 1>(*a, st);
  return conv_vector(*a, 8, nullptr, true) ? launch_step<__bf16, 8>(*a, st) : launch_step<__bf16, 1>(*a, st);
}

}  // extern "C"
