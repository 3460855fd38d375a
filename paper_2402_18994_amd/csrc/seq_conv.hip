// Short causal convolution along time, one filter of W taps per channel (include/snn_ops.h):
//   v[t,d] = bias[d] + sum_(k<W) w[d,k] x[t-(W-1)+k, d],  y = v or v sigmoid(v).
// Tensors are time-major with the channels fastest, so a thread owns VEC neighbouring channels of one sequence and
// walks a segment of its steps with the last W - 1 inputs in registers: every row piece is read and written once, as
// 16 bytes where the layout allows, and a wavefront's access is one contiguous kilobyte.
#include "seq_common.hpp"

#include <type_traits>

namespace snn {
namespace {

#ifndef CV
#define CV 8
#endif
#ifndef CSEG
#define CSEG 32
#endif
#ifndef CAH
#define CAH 8
#endif
#ifndef BSEG
#define BSEG 32
#endif
#ifndef BBL
#define BBL 1024
#endif
constexpr int AHEAD = CAH;            // rows in flight per thread, forward
constexpr int AHEAD_BWD = 4;

struct ConvP {
  int T, B, D, silu, seg, nseg;
  Rows<void> x, y;
  const float *weight, *bias;
  const void *init;
  const int32_t *lengths;
  void *state;
  explicit ConvP(const snn_conv_args &a)
      : T(a.T), B(a.B), D(a.D), silu(a.silu), seg(1), nseg(1), x(a.x), y(a.y), weight(a.weight), bias(a.bias), init(a.init),
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

// Row `t` of the input of sequence b, t from -(W-1) on; zeros before the first step without `init`, and for t >= end.
template <typename T, int VEC, int W>
__device__ __forceinline__ Pack<T, VEC> input_row(const ConvP &a, const T *x, int b, int d, int t, int end) {
  Pack<T, VEC> r;
#pragma unroll
  for (int v = 0; v < VEC; ++v) r.v[v] = (T)0.f;
  if (t >= 0) {
    if (t < end) r = *(const Pack<T, VEC> *)(x + (int64_t)t * a.x.st);
  } else if (a.init) {
    r = *(const Pack<T, VEC> *)((const T *)a.init + ((size_t)(t + W - 1) * a.B + b) * a.D + d);
  }
  return r;
}

// Forward: blockIdx.y is the segment.
template <typename T, int VEC, int W>
__global__ __launch_bounds__(256) void conv_forward_kernel(const ConvP a) {
  const int dv = a.D / VEC;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)a.B * dv) return;
  const int b = (int)(id / dv), d = (int)(id % dv) * VEC;
  const int len = length_of(a.lengths, b, a.T);
  const T *x = (const T *)a.x.p + b * a.x.sb + d;
  T *y = (T *)a.y.p + b * a.y.sb + d;
  const int64_t t0 = (int64_t)blockIdx.y * a.seg;
  const int t1 = (int)min((int64_t)a.T, t0 + a.seg), end = min(t1, len);

  float w[W][VEC], bias[VEC], xs[W - 1 + AHEAD][VEC];
  load_filter<T, VEC, W>(a, d, w, bias);
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const Pack<T, VEC> r = input_row<T, VEC, W>(a, x, b, d, (int)t0 - (W - 1) + k, end);
#pragma unroll
    for (int v = 0; v < VEC; ++v) xs[k][v] = widen(r.v[v]);
  }
  Pack<T, VEC> next[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) next[u] = input_row<T, VEC, W>(a, x, b, d, (int)t0 + u, end);
  for (int t = (int)t0; t < t1; t += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int v = 0; v < VEC; ++v) xs[W - 1 + u][v] = widen(next[u].v[v]);
    if (t + AHEAD < t1) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) next[u] = input_row<T, VEC, W>(a, x, b, d, t + AHEAD + u, end);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (t + u < t1) {
        Pack<T, VEC> r;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          float s = bias[v];
#pragma unroll
          for (int k = 0; k < W; ++k) s = fmaf(w[k][v], xs[u + k][v], s);
          if (a.silu) s *= sigmoid_fast(s);
          r.v[v] = narrow<T>(t + u < len ? s : 0.f);
        }
        *(Pack<T, VEC> *)(y + (int64_t)(t + u) * a.y.st) = r;
      }
    }
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) xs[k][v] = xs[k + AHEAD][v];
  }
  if (a.state && blockIdx.y == 0) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
      *(Pack<T, VEC> *)((T *)a.state + ((size_t)j * a.B + b) * a.D + d) =
          input_row<T, VEC, W>(a, x, b, d, len - (W - 1) + j, len);
  }
}

// One step: the state [W-1][B][D] moves up a row.
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

// Backward.  With q[t] = dy[t] (dv/dy at step t; zero outside [0, len)):
//   dx[s] = sum_k w[k] q[s + (W-1) - k],  dw[k] = sum_(t,b) q[t] x[t-(W-1)+k],  dbias = sum_(t,b) q[t].
// A thread walks its segment of a sequence and W - 1 steps more (dx of the last steps needs their q; v is computed
// again from x), emitting the gradient of input row t - (W-1) at step t.  A workgroup's threads stand in R rows of LX
// channel groups; every row takes (sequence, segment) items in turn, with dw and dbias in registers, and at the end
// the rows' sums go through LDS into one partial sum per workgroup, added up by sum_rows_kernel in a fixed order.
struct ConvGradP {
  Rows<void> dy, dx;
  const void *d_state;
  void *dinit;
  float *partial;                    // [gridDim.y][W+1][D]
  int lx_log2;
  ConvGradP(const snn_conv_grads &g) : dy(g.dy), dx(g.dx), d_state(g.d_state), dinit(g.dinit), partial(nullptr), lx_log2(0) {}
};

template <typename T, int VEC, int W>
__global__ __launch_bounds__(256) void conv_backward_kernel(const ConvP a, const ConvGradP g) {
  __shared__ float part[256 * VEC];
  const int lx = 1 << g.lx_log2, rows = 256 >> g.lx_log2;
  const int lane = threadIdx.x & (lx - 1), row = threadIdx.x >> g.lx_log2;
  const int dv = a.D / VEC, chunk = blockIdx.x * lx + lane;
  const bool live = chunk < dv;
  const int d = chunk * VEC;
  float w[W][VEC], bias[VEC], dw[W][VEC], db[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    db[v] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) dw[k][v] = 0.f;
  }
  if (live) {
    load_filter<T, VEC, W>(a, d, w, bias);
    const int64_t items = (int64_t)a.B * a.nseg;
    for (int64_t item = (int64_t)blockIdx.y * rows + row; item < items; item += (int64_t)gridDim.y * rows) {
      const int b = (int)(item / a.nseg), s0 = (int)(item % a.nseg);
      const int len = length_of(a.lengths, b, a.T);
      const T *x = (const T *)a.x.p + b * a.x.sb + d;
      const T *dy = (const T *)g.dy.p + b * g.dy.sb + d;
      T *dx = (T *)g.dx.p + b * g.dx.sb + d;
      const int t0 = s0 * a.seg, t1 = min(a.T, t0 + a.seg), stop = t1 + W - 1;
      float xs[W - 1 + AHEAD_BWD][VEC], q[W - 1 + AHEAD_BWD][VEC];
#pragma unroll
      for (int k = 0; k < W - 1; ++k) {
        const Pack<T, VEC> r = input_row<T, VEC, W>(a, x, b, d, t0 - (W - 1) + k, len);
#pragma unroll
        for (int v = 0; v < VEC; ++v) { xs[k][v] = widen(r.v[v]); q[k][v] = 0.f; }
      }
      Pack<T, VEC> nx[AHEAD_BWD], ny[AHEAD_BWD];
      auto fetch = [&](int t) {
#pragma unroll
        for (int u = 0; u < AHEAD_BWD; ++u) {
#pragma unroll
          for (int v = 0; v < VEC; ++v) { nx[u].v[v] = (T)0.f; ny[u].v[v] = (T)0.f; }
          if (t + u < min(stop, len)) {
            nx[u] = *(const Pack<T, VEC> *)(x + (int64_t)(t + u) * a.x.st);
            ny[u] = *(const Pack<T, VEC> *)(dy + (int64_t)(t + u) * g.dy.st);
          }
        }
      };
      fetch(t0);
      for (int t = t0; t < stop; t += AHEAD_BWD) {
#pragma unroll
        for (int u = 0; u < AHEAD_BWD; ++u)
#pragma unroll
          for (int v = 0; v < VEC; ++v) { xs[W - 1 + u][v] = widen(nx[u].v[v]); q[W - 1 + u][v] = widen(ny[u].v[v]); }
        if (t + AHEAD_BWD < stop) fetch(t + AHEAD_BWD);
#pragma unroll
        for (int u = 0; u < AHEAD_BWD; ++u) {
          const int now = t + u;
          if (now < stop) {
            Pack<T, VEC> out;
            const int j = now - len;                        // row of d_state that belongs to input row now - (W-1)
            const bool kept = g.d_state && j >= 0 && j < W - 1;
            Pack<T, VEC> ds;
            if (kept) ds = *(const Pack<T, VEC> *)((const T *)g.d_state + ((size_t)j * a.B + b) * a.D + d);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
              float &qv = q[W - 1 + u][v];
              if (a.silu) {
                float s = bias[v];
#pragma unroll
                for (int k = 0; k < W; ++k) s = fmaf(w[k][v], xs[u + k][v], s);
                const float e = sigmoid_fast(s);
                qv *= e * (1.f + s * (1.f - e));
              }
              if (now >= len) qv = 0.f;
              const float own = now < t1 ? qv : 0.f;
              db[v] += own;
              float sum = 0.f;
#pragma unroll
              for (int k = 0; k < W; ++k) {
                dw[k][v] = fmaf(own, xs[u + k][v], dw[k][v]);
                sum = fmaf(w[k][v], q[W - 1 + u - k][v], sum);
              }
              if (kept) sum += widen(ds.v[v]);
              out.v[v] = narrow<T>(sum);
            }
            const int s = now - (W - 1);
            if (s >= t0) *(Pack<T, VEC> *)(dx + (int64_t)s * g.dx.st) = out;
            else if (s < 0 && g.dinit) *(Pack<T, VEC> *)((T *)g.dinit + ((size_t)now * a.B + b) * a.D + d) = out;
          }
        }
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
#pragma unroll
          for (int v = 0; v < VEC; ++v) { xs[k][v] = xs[k + AHEAD_BWD][v]; q[k][v] = q[k + AHEAD_BWD][v]; }
      }
    }
  }
#pragma unroll
  for (int k = 0; k <= W; ++k) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) part[threadIdx.x * VEC + v] = k < W ? dw[k < W ? k : 0][v] : db[v];
    __syncthreads();
    if (row == 0 && live)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += part[(r * lx + lane) * VEC + v];
        g.partial[((size_t)blockIdx.y * (W + 1) + k) * a.D + d + v] = s;
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
  if ((int64_t)a->B * a->D >= (1ll << 31)) return ops_fail(SNN_ERR_ARG, "convolution: B * D must stay below 2^31");
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

// How a backward call is cut: channel groups per workgroup, steps per segment, workgroups over the items.
struct ConvCut {
  int lx_log2, seg, nseg, gx, gy;
};
ConvCut conv_cut(const snn_conv_args &a, int vec) {
  ConvCut c;
  const int dv = a.D / vec;
  c.lx_log2 = 0;
  while (c.lx_log2 < 6 && (1 << c.lx_log2) < dv) ++c.lx_log2;
  c.gx = (dv + (1 << c.lx_log2) - 1) >> c.lx_log2;
  c.seg = BSEG;
  while (c.seg < (1 << 20) && a.T / c.seg > 65536) c.seg *= 2;
  c.nseg = a.T > c.seg ? (a.T + c.seg - 1) / c.seg : 1;
  const int64_t rows = 256 >> c.lx_log2, items = (int64_t)a.B * c.nseg;
  const int64_t want = BBL / c.gx > 1 ? BBL / c.gx : 1;
  const int64_t all = (items + rows - 1) / rows;
  c.gy = (int)(all < want ? all : want);
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
  const int64_t threads = (int64_t)a.B * (a.D / VEC);
  p.seg = CSEG;
  while (a.T / p.seg > 32768) p.seg *= 2;              // (a grid has at most 65535 rows)
  const int gy = a.T > p.seg ? (a.T + p.seg - 1) / p.seg : 1;
  return with_taps(a.W, [&](auto w) {
    hipLaunchKernelGGL((conv_forward_kernel<T, VEC, w.value>), dim3((unsigned)((threads + 255) / 256), gy), dim3(256), 0, st, p);
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
  ConvGradP q(g);
  const ConvCut c = conv_cut(a, VEC);
  p.seg = c.seg; p.nseg = c.nseg; q.partial = ws; q.lx_log2 = c.lx_log2;
  return with_taps(a.W, [&](auto w) {
    hipLaunchKernelGGL((conv_backward_kernel<T, VEC, w.value>), dim3(c.gx, c.gy), dim3(256), 0, st, p, q);
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
  if (a->type == SNN_TYPE_FP32) return conv_vector(*a, 4, nullptr, false) ? launch_forward<float, 4>(*a, st) : launch_forward<float, 1>(*a, st);
  return conv_vector(*a, CV, nullptr, false) ? launch_forward<__bf16, CV>(*a, st) : launch_forward<__bf16, 1>(*a, st);
}

int32_t snn_conv_workspace_bytes(const snn_conv_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  if (!a) return ops_fail(SNN_ERR_NULL, "convolution: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0 || (int64_t)a->B * a->D >= (1ll << 31) || a->T > (1 << 30) || a->W < 1 || a->W > SNN_CONV_MAX_TAPS)
    return ops_fail(SNN_ERR_ARG, "convolution: sizes out of range");
  const int gy1 = conv_cut(*a, 1).gy, gy4 = a->D % 4 == 0 ? conv_cut(*a, 4).gy : 0;   // (which one runs depends on the pointers too)
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
  const bool vec = conv_vector(*a, 4, g, false);
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
