// Gated linear recurrence, one state a channel (include/snn_ops.h):
//   rho = sigmoid(r), l = -c softplus(decay) rho, a = exp(l), s = sqrt(1 - a^2), h_t = a h_(t-1) + s sigmoid(i) x, y = h.
// Reverse, g_t = dy_t + a_(t+1) g_(t+1):
//   dx = g s iota;  di = g s x iota (1 - iota);  dl = g (a h_(t-1) - a^2 / s iota x);  dr = dl l (1 - rho);
//   ddecay = sum dl l sigmoid(decay) / softplus(decay).
//
// h_t = a_t h_(t-1) + b_t is a chain of affine maps, and a run of steps is one as well: (product of a, state from zero).  A lane
// holds a run of STEPS steps of VEC channels in registers, forms its map, leaves it in LDS, joins the maps of the runs ahead of it
// in the tile onto the tile's start, and replays its steps: every stream is read once and written once, whatever the chain's
// length.  A workgroup walks the tiles of one sequence and CH channels; where there are too few of those to fill the chip, time is
// cut into segments whose maps a first launch forms (the streams are then read twice).
// Measured, bfloat16, 1024 steps of 8 x 2048 channels: forward 33 us (134 MB, 4.1 TB/s; the same accesses without arithmetic take 23), reverse 55
// (242 MB, 4.4 TB/s).  What bounds it are the vector units, 42 and 71 operations an element of which six are transcendental at half
// rate, three quarters of the time; in the rest all wavefronts of a compute unit's one workgroup load, join or store.
#include "block_rules.hpp"
#include "rows.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

constexpr float LN2 = 0.6931471805599453f;

struct RecP {
  int T, B, D, groups, tiles, nseg;          // tiles: of a segment
  float sharpness;
  Rows<void> x, i, r, y;
  const float *decay, *init;
  const int32_t *lengths;
  float *state, *saved;
  float2 *carry;                             // [nseg][B][D]: a segment's map
  explicit RecP(const snn_recurrence_args &a)
      : T(a.T), B(a.B), D(a.D), groups((a.D + CH - 1) / CH), tiles(0), nseg(1), sharpness(a.sharpness), x(a.x, a.T), i(a.i, a.T), r(a.r, a.T),
        y(a.y, a.T), decay(a.decay), init(a.init), lengths(a.lengths), state(a.state), saved(nullptr), carry(nullptr) {}
};
struct RecGradP {
  Rows<void> dy, dx, di, dr;
  const float *d_state;
  float *part, *dinit;                       // part [nseg * B][D]
  RecGradP(const snn_recurrence_grads &g, int T) : dy(g.dy, T), dx(g.dx, T), di(g.di, T), dr(g.dr, T), d_state(g.d_state), part(nullptr), dinit(g.dinit) {}
};

// sigmoid(v) and 1 - sigmoid(v), each to its own last places.  A gate below the least normal number is shut: (0, 1).  A NaN passes.
__device__ __forceinline__ float gate_of(float v, float &rest) {
  const float e = exp_fast(-v), g = rcp_fast(1.f + e);
  rest = e > 0x1p126f ? 1.f : e * g;
  return g;
}
// log2 of what a wholly open gate leaves; finite, so that a shut one (times zero) holds the state whatever `decay` is.
__device__ __forceinline__ float rate_of(float sharpness, float decay) {
  const float v = -sharpness * (LOG2E * softplus(decay));  // (sharpness LOG2E may be infinite, which times no decay is no number)
  return v < -0x1p127f ? -0x1p127f : v;
}

// 1 - a^2 for a = 2^L.  Where a^2 is near one (z = -2 ln 2 L <= 1/2), z p(z) with p the polynomial of degree 5 that is closest to
// (1 - exp(-z)) / z over [0, 1/2] (off by 1.4e-9 of it; fitted by reweighted least squares), written in L; beyond, 1 - a a, where the
// rounding of a a is 1.5 units of the result's last place.  NEAR: all channels of the wavefront leave so much at every step, since a
// wholly open gate does.
constexpr float NEAR_RATE = -0.36f;
template <bool NEAR> __device__ __forceinline__ float one_less_square(float L, float a) {
  float p = fmaf(L, -0x1.04e03ep-7f, -0x1.5768dcp-5f);
  p = fmaf(p, L, -0x1.3ae1f2p-3f);
  p = fmaf(p, L, -0x1.c6ad78p-2f);
  p = fmaf(p, L, -0x1.ebfbd4p-1f);
  p = fmaf(p, L, -0x1.62e430p+0f) * L;
  return NEAR || L > NEAR_RATE ? p : fmaf(-a, a, 1.f);
}
// (root of m, its reciprocal); a root of zero has the reciprocal 2^63, so products with what goes to zero as fast stay zero.
__device__ __forceinline__ float root_of(float m, float &inverse) {
  inverse = __builtin_amdgcn_rsqf(fmaxf(m, 0x1p-126f));
  return m * inverse;
}

// A run's raw rows of one stream; zeros behind `n`, the run's steps that exist (`all`: they do in every lane).
template <typename T, int VEC>
__device__ __forceinline__ void load_run(Pack<T, VEC> (&v)[STEPS], const T *row, int64_t st, int at, int n, bool all) {
  if (all)
#pragma unroll
    for (int s = 0; s < STEPS; ++s) v[s] = row_load<T, VEC>(row + s * st, at);
  else
#pragma unroll
    for (int s = 0; s < STEPS; ++s) v[s] = row_load<T, VEC>(row + s * st, s < n ? at : ROW_NOWHERE);
}

// WAVES wavefronts, of which each holds 64 / LANES runs of LANES lanes by VEC channels.
template <typename T, int VEC, int WAVES> struct Shape {
  static constexpr int LANES = CH / VEC, HALVES = 64 / LANES, RUNS = WAVES * HALVES, TILE = RUNS * STEPS;
  // byte offset of a lane in a stream: its channel, and its half's steps
  template <typename R> static __device__ __forceinline__ int offset(const R &r, int lane, int d, bool live) {
    return live ? (int)((lane / LANES) * STEPS * r.st * (int64_t)sizeof(T)) + d * (int)sizeof(T) : ROW_NOWHERE;
  }
};
struct alignas(8) Link {
  float a, h;
};

// The runs of a wavefront's two halves as one map, in both halves; `first` is that of the half that comes first.
template <int HALVES, bool REVERSE> __device__ __forceinline__ Link whole_wave(Link m, Link &first) {
  first = m;
  if constexpr (HALVES == 2) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(m.a), __float_as_uint(m.a), false, false);
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(m.h), __float_as_uint(m.h), false, false);
    const Link low = {__uint_as_float(a[0]), __uint_as_float(h[0])}, high = {__uint_as_float(a[1]), __uint_as_float(h[1])};
    first = REVERSE ? high : low;
    const Link then = REVERSE ? low : high;
    return {first.a * then.a, fmaf(then.a, first.h, then.h)};
  }
  return m;
}
// The maps of a tile's wavefronts stand in `link`; joins them onto `h` in order (reverse: from the last one on) and returns what a
// lane's own run starts from; `h` and `p` become state and product behind the tile.
template <int VEC, int WAVES, int HALVES, bool REVERSE, bool PRODUCT>
__device__ __forceinline__ void join(const Link (*link)[CH], int c, int wave, bool second, const Link (&first)[VEC], float (&h)[VEC], float (&p)[VEC],
                                     float (&start)[VEC]) {
  const int own = REVERSE ? WAVES - 1 - wave : wave;
  auto add = [&](int k) {
    const int q = REVERSE ? WAVES - 1 - k : k;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const Link m = link[q][c + v];
      h[v] = fmaf(m.a, h[v], m.h);
      if (PRODUCT) p[v] *= m.a;
    }
  };
#pragma unroll 4
  for (int k = 0; k < own; ++k) add(k);
#pragma unroll
  for (int v = 0; v < VEC; ++v) start[v] = HALVES == 2 && second ? fmaf(first[v].a, h[v], first[v].h) : h[v];
#pragma unroll 4
  for (int k = own; k < WAVES; ++k) add(k);
}

// OUT: outputs.  Otherwise the map of the segment alone.
template <typename T, int VEC, int WAVES, bool OUT>
__global__ __launch_bounds__(WAVES * 64) void recurrence_forward_kernel(const RecP a) {
  using S = Shape<T, VEC, WAVES>;
  __shared__ Link link[2][WAVES][CH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned id = blockIdx.x;
  const int group = (int)(id % (unsigned)a.groups);
  id /= (unsigned)a.groups;
  const int b = (int)(id % (unsigned)a.B), seg = (int)(id / (unsigned)a.B);
  const int c = (lane % S::LANES) * VEC, d = group * CH + c;
  const bool live = d < a.D, second = lane >= S::LANES;
  const int dd = live ? d : 0;
  const int len = __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T));
  const int at_x = S::offset(a.x, lane, d, live), at_i = S::offset(a.i, lane, d, live), at_r = S::offset(a.r, lane, d, live);
  const int at_y = OUT ? S::offset(a.y, lane, d, live) : 0;
  const T *x = (const T *)a.x.p + b * a.x.sb, *i = (const T *)a.i.p + b * a.i.sb, *r = (const T *)a.r.p + b * a.r.sb;
  T *y = (T *)a.y.p + b * a.y.sb;
  const int64_t cell = (int64_t)b * a.D + dd;
  const int t_end = min(a.T, (seg + 1) * a.tiles * S::TILE);

  const int wave_t = wave * S::HALVES * STEPS, half_t = lane / S::LANES * STEPS;
  Pack<T, VEC> rx[STEPS], ri[STEPS], rr[STEPS];
  int t0 = seg * a.tiles * S::TILE;
  auto fetch = [&](int t) {
    const int tw = t + wave_t, n = len - (tw + half_t);
    const bool all = tw + S::HALVES * STEPS <= len;
    load_run<T, VEC>(rr, r + tw * a.r.st, a.r.st, at_r, n, all);
    load_run<T, VEC>(ri, i + tw * a.i.st, a.i.st, at_i, n, all);
    load_run<T, VEC>(rx, x + tw * a.x.st, a.x.st, at_x, n, all);
  };
  fetch(t0);
  float rate[VEC], h[VEC], p[VEC];
  bool far = false;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    rate[v] = rate_of(a.sharpness, a.decay[dd + v]);
    far = far || !(rate[v] >= NEAR_RATE);
    h[v] = OUT && a.init ? a.init[cell + v] : 0.f;
    p[v] = 1.f;
  }
  const bool near = __ballot(far) == 0;
  if (OUT)
#pragma unroll 4
    for (int k = 0; k < seg; ++k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float2 m = a.carry[(int64_t)k * a.B * a.D + cell + v];
        h[v] = fmaf(m.x, h[v], m.y);
      }

  for (int buf = 0; t0 < t_end; t0 += S::TILE, buf ^= 1) {
    const int tw = t0 + wave_t, t_run = tw + half_t, n = len - t_run;
    if (t0 >= len) {                                       // (for the whole workgroup)
      if (!OUT) break;
      const Pack<T, VEC> zero = {};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) row_store<T, VEC>(y + (tw + s) * a.y.st, t_run + s < a.T ? at_y : ROW_NOWHERE, zero);
      continue;
    }
    float fa[STEPS][VEC], fb[STEPS][VEC], start[VEC];
    Link first[VEC];
    // FAST: every step of the wavefront exists, and NEAR; otherwise those that do not exist have a = 1 and b = 0
    auto maps = [&](auto fast) {
      constexpr bool FAST = decltype(fast)::value;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        Link m = {1.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const bool on = FAST || s < n;
          float rest;
          const float rho = gate_of(widen(rr[s].v[v]), rest), iota = gate_of(widen(ri[s].v[v]), rest);
          const float L = on ? rate[v] * rho : 0.f, e = __builtin_amdgcn_exp2f(L);
          fa[s][v] = e;
          fb[s][v] = on ? __builtin_amdgcn_sqrtf(one_less_square<FAST>(L, e)) * iota * widen(rx[s].v[v]) : 0.f;
          m.h = fmaf(e, m.h, fb[s][v]);
          m.a *= e;
        }
        m = whole_wave<S::HALVES, false>(m, first[v]);
        if (!second) link[buf][wave][c + v] = m;
      }
    };
    const bool all = tw + S::HALVES * STEPS <= len;
    if (all && near) maps(std::true_type());
    else maps(std::false_type());
    if (t0 + S::TILE < t_end) fetch(t0 + S::TILE);
    lds_barrier();                                         // (two buffers: one barrier a tile)
    join<VEC, WAVES, S::HALVES, false, !OUT>(link[buf], c, wave, second, first, h, p, start);
    if (OUT) {
      if (a.saved && live && t_run < a.T)
#pragma unroll
        for (int v = 0; v < VEC; ++v) a.saved[(int64_t)(t_run / STEPS) * a.B * a.D + cell + v] = start[v];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        Pack<T, VEC> out;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          start[v] = fmaf(fa[s][v], start[v], fb[s][v]);
          out.v[v] = narrow<T>(start[v]);
        }
        if (!all) {
          const Pack<T, VEC> zero = {};
          if (s >= n) out = zero;
        }
        row_store<T, VEC>(y + (tw + s) * a.y.st, all || t_run + s < a.T ? at_y : ROW_NOWHERE, out);
      }
    }
  }
  if (live && wave == 0 && !second)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (!OUT) a.carry[(int64_t)seg * a.B * a.D + cell + v] = {p[v], h[v]};
      else if (a.state && seg == a.nseg - 1) a.state[cell + v] = h[v];
    }
}

// Reverse.  What travels from step to step is q = a g; a run's map is (product of a, q from zero).
template <typename T, int VEC, int WAVES, bool OUT>
__global__ __launch_bounds__(WAVES * 64) void recurrence_backward_kernel(const RecP a, const RecGradP g) {
  using S = Shape<T, VEC, WAVES>;
  __shared__ Link link[2][WAVES][CH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned id = blockIdx.x;
  const int group = (int)(id % (unsigned)a.groups);
  id /= (unsigned)a.groups;
  const int b = (int)(id % (unsigned)a.B), seg = (int)(id / (unsigned)a.B) + (OUT ? 0 : 1);     // (no segment comes before the first)
  const int c = (lane % S::LANES) * VEC, d = group * CH + c;
  const bool live = d < a.D, second = lane < 64 - S::LANES;                                     // (the upper half's steps come first)
  const int dd = live ? d : 0;
  const int len = __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T));
  const int at_x = S::offset(a.x, lane, d, live), at_i = S::offset(a.i, lane, d, live), at_r = S::offset(a.r, lane, d, live);
  const int at_dy = S::offset(g.dy, lane, d, live);
  const int at_dx = OUT ? S::offset(g.dx, lane, d, live) : 0, at_di = OUT ? S::offset(g.di, lane, d, live) : 0, at_dr = OUT ? S::offset(g.dr, lane, d, live) : 0;
  const T *x = (const T *)a.x.p + b * a.x.sb, *i = (const T *)a.i.p + b * a.i.sb, *r = (const T *)a.r.p + b * a.r.sb, *dy = (const T *)g.dy.p + b * g.dy.sb;
  T *dx = (T *)g.dx.p + b * g.dx.sb, *di = (T *)g.di.p + b * g.di.sb, *dr = (T *)g.dr.p + b * g.dr.sb;
  const int64_t cell = (int64_t)b * a.D + dd;
  const int t_begin = seg * a.tiles * S::TILE, t_end = min(a.T, t_begin + a.tiles * S::TILE);

  float rate[VEC], q[VEC], p[VEC], sum[VEC];
  bool far = false;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    rate[v] = rate_of(a.sharpness, a.decay[dd + v]);
    far = far || !(rate[v] >= NEAR_RATE);
    q[v] = OUT && g.d_state ? g.d_state[cell + v] : 0.f;
    p[v] = 1.f;
    sum[v] = 0.f;
  }
  const bool near = __ballot(far) == 0;
  if (OUT)
#pragma unroll 4
    for (int k = a.nseg - 1; k > seg; --k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float2 m = a.carry[(int64_t)k * a.B * a.D + cell + v];
        q[v] = fmaf(m.x, q[v], m.y);
      }

  const int wave_t = wave * S::HALVES * STEPS, half_t = lane / S::LANES * STEPS;
  Pack<T, VEC> nx[STEPS], ni[STEPS], nr[STEPS], ng[STEPS];
  float nbefore[VEC];
  auto fetch = [&](int t) {
    const int tw = t + wave_t, n = len - (tw + half_t);
    const bool all = tw + S::HALVES * STEPS <= len;
    load_run<T, VEC>(nr, r + tw * a.r.st, a.r.st, at_r, n, all);
    if (OUT) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) nbefore[v] = a.saved[(int64_t)(n > 0 ? (tw + half_t) / STEPS : 0) * a.B * a.D + cell + v];
      load_run<T, VEC>(ni, i + tw * a.i.st, a.i.st, at_i, n, all);
      load_run<T, VEC>(nx, x + tw * a.x.st, a.x.st, at_x, n, all);
    }
    load_run<T, VEC>(ng, dy + tw * g.dy.st, g.dy.st, at_dy, n, all);
  };
  int t0 = t_begin + (t_end - 1 - t_begin) / S::TILE * S::TILE;
  for (; t0 >= t_begin && t0 >= len; t0 -= S::TILE) {      // tiles behind the sequence's end
    if (!OUT) continue;
    const int tw = t0 + wave_t, t_run = tw + half_t;
    const Pack<T, VEC> zero = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bool there = t_run + s < a.T;
      row_store<T, VEC>(dx + (tw + s) * g.dx.st, there ? at_dx : ROW_NOWHERE, zero);
      row_store<T, VEC>(di + (tw + s) * g.di.st, there ? at_di : ROW_NOWHERE, zero);
      row_store<T, VEC>(dr + (tw + s) * g.dr.st, there ? at_dr : ROW_NOWHERE, zero);
    }
  }
  if (t0 >= t_begin) fetch(t0);
  for (int buf = 0; t0 >= t_begin; t0 -= S::TILE, buf ^= 1) {
    const int tw = t0 + wave_t, t_run = tw + half_t, n = len - t_run;
    const bool all = tw + S::HALVES * STEPS <= len;
    Pack<T, VEC> rx[STEPS], ri[STEPS], rr[STEPS], rg[STEPS];
    float before[VEC];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      rr[s] = nr[s];
      rg[s] = ng[s];
      if (OUT) {
        rx[s] = nx[s];
        ri[s] = ni[s];
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) before[v] = OUT ? nbefore[v] : 0.f;
    if (t0 - S::TILE >= t_begin) fetch(t0 - S::TILE);
    // What each step multiplies g by: dx = g to_x, di = dx to_i, dr = g to_l closed (and g to_l is what sums up to ddecay).
    float fa[STEPS][VEC], to_x[STEPS][VEC], to_i[STEPS][VEC], to_l[STEPS][VEC], closed[STEPS][VEC], start[VEC];
    Link first[VEC];
    auto maps = [&](auto fast) {
      constexpr bool FAST = decltype(fast)::value;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        Link m = {1.f, 0.f};
        float h = OUT ? (FAST || n > 0 ? before[v] : 0.f) : 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const bool on = FAST || s < n;
          const float rho = gate_of(widen(rr[s].v[v]), closed[s][v]);
          const float L = on ? rate[v] * rho : 0.f, e = __builtin_amdgcn_exp2f(L);
          fa[s][v] = e;
          if (!OUT) continue;
          float rest, inverse;
          const float iota = gate_of(widen(ri[s].v[v]), rest), gain = root_of(one_less_square<FAST>(L, e), inverse), xv = widen(rx[s].v[v]);
          const float gi = gain * iota, le = L * LN2 * e;  // (l a; its limit is zero, also where l is as large as it gets)
          to_x[s][v] = gi;
          to_i[s][v] = rest * xv;
          to_l[s][v] = le * h - e * (le * inverse) * (iota * xv);
          h = fmaf(e, h, on ? gi * xv : 0.f);
        }
#pragma unroll
        for (int s = STEPS - 1; s >= 0; --s) {
          m.h = fa[s][v] * (widen(rg[s].v[v]) + m.h);
          m.a *= fa[s][v];
        }
        m = whole_wave<S::HALVES, true>(m, first[v]);
        if (!second) link[buf][wave][c + v] = m;
      }
    };
    if (all && near) maps(std::true_type());
    else maps(std::false_type());
    lds_barrier();
    join<VEC, WAVES, S::HALVES, true, !OUT>(link[buf], c, wave, second, first, q, p, start);
    if (!OUT) continue;
    auto give = [&](auto exist) {
      constexpr bool ALL = decltype(exist)::value;
#pragma unroll
      for (int s = STEPS - 1; s >= 0; --s) {
        const bool on = ALL || s < n;
        Pack<T, VEC> ox, oi, ol;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float gt = widen(rg[s].v[v]) + start[v];
          const float vx = on ? gt * to_x[s][v] : 0.f, pull = on ? gt * to_l[s][v] : 0.f;
          ox.v[v] = narrow<T>(vx);
          oi.v[v] = narrow<T>(on ? vx * to_i[s][v] : 0.f);
          ol.v[v] = narrow<T>(on ? pull * closed[s][v] : 0.f);
          sum[v] += pull;
          start[v] = fa[s][v] * gt;
        }
        const bool there = ALL || t_run + s < a.T;
        row_store<T, VEC>(dx + (tw + s) * g.dx.st, there ? at_dx : ROW_NOWHERE, ox);
        row_store<T, VEC>(di + (tw + s) * g.di.st, there ? at_di : ROW_NOWHERE, oi);
        row_store<T, VEC>(dr + (tw + s) * g.dr.st, there ? at_dr : ROW_NOWHERE, ol);
      }
    };
    if (all) give(std::true_type());
    else give(std::false_type());
  }
  if (!OUT) {
    if (live && wave == 0 && !second)
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.carry[(int64_t)seg * a.B * a.D + cell + v] = {p[v], q[v]};
    return;
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    float s = sum[v];
    if (S::HALVES == 2) {
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
      s = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    if (!second) link[0][wave][c + v].a = s;
  }
  __syncthreads();
  if (live && wave == 0 && !second)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = 0.f;
      for (int k = 0; k < WAVES; ++k) s += link[0][k][c + v].a;
      g.part[((int64_t)seg * a.B + b) * a.D + d + v] = s;
      if (g.dinit && seg == 0) g.dinit[cell + v] = q[v];
    }
}

// ddecay: the partial sums' sum times sigmoid(decay) / softplus(decay), which goes to 1 as decay goes to -inf.
__global__ __launch_bounds__(256) void recurrence_sum_kernel(const float *__restrict__ part, int rows, int D, const float *__restrict__ decay, float *__restrict__ out) {
  __shared__ float lds[256];
  const int64_t col = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
  const float s = sum_column(part, D, col, rows, lds);
  if (threadIdx.x < 16 && col < D) {
    const float v = decay[col], rate = softplus(v);
    out[col] = s * (rate > 0.f ? sigmoid_fast(v) * rcp_fast(rate) : v != v ? v : 1.f);
  }
}

template <typename T, int VEC> __global__ __launch_bounds__(256) void recurrence_step_kernel(const RecP a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int cols = a.D / VEC;
  if (id >= (int64_t)a.B * cols) return;
  const int b = (int)(id / cols), d = (int)(id % cols) * VEC;
  using P = Pack<T, VEC>;
  using F = Pack<float, VEC>;
  const P x = *(const P *)((const T *)a.x.p + b * a.x.sb + d), i = *(const P *)((const T *)a.i.p + b * a.i.sb + d),
          r = *(const P *)((const T *)a.r.p + b * a.r.sb + d);
  F h = *(const F *)(a.state + (int64_t)b * a.D + d);
  const F w = *(const F *)(a.decay + d);
  P y;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    float rest, inverse;
    const float L = rate_of(a.sharpness, w.v[v]) * gate_of(widen(r.v[v]), rest), e = __builtin_amdgcn_exp2f(L);
    h.v[v] = fmaf(e, h.v[v], root_of(one_less_square<false>(L, e), inverse) * gate_of(widen(i.v[v]), rest) * widen(x.v[v]));
    y.v[v] = narrow<T>(h.v[v]);
  }
  *(F *)(a.state + (int64_t)b * a.D + d) = h;
  *(P *)((T *)a.y.p + b * a.y.sb + d) = y;
}

// ---------------------------------------------------------------- host
int recurrence_check(const snn_recurrence_args *a, bool step, bool grads) {
  if (!a) return ops_fail(SNN_ERR_NULL, "recurrence: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0) return ops_fail(SNN_ERR_ARG, "recurrence: T >= 0, B > 0 and D > 0 are required");
  if (a->D > (1 << 22) || (int64_t)a->B * ((a->D + CH - 1) / CH) >= (1 << 22) || a->T > (1 << 30))
    return ops_fail(SNN_ERR_ARG, "recurrence: D must not exceed 2^22, B * (D / %d, rounded up) must stay below 2^22, T must not exceed 2^30", CH);
  if (a->type != SNN_TYPE_FP32 && a->type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "recurrence: unknown type %d", a->type);
  if (!(a->sharpness > 0.f) || a->sharpness > 3e38f) return ops_fail(SNN_ERR_ARG, "recurrence: sharpness has to be positive and finite");
  if (!a->decay) return ops_fail(SNN_ERR_NULL, "recurrence: decay is NULL");
  if (a->T > 0 && (!a->x.p || !a->i.p || !a->r.p || (!grads && !a->y.p))) return ops_fail(SNN_ERR_NULL, "recurrence: x, i, r or y is NULL");
  if (step) {
    if (a->T != 1) return ops_fail(SNN_ERR_ARG, "recurrence step: T must be 1");
    if (a->init || a->lengths) return ops_fail(SNN_ERR_ARG, "recurrence step: init and lengths must be NULL");
    if (!a->state) return ops_fail(SNN_ERR_NULL, "recurrence step: state is NULL");
  }
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(a->x.p, z) || !aligned(a->i.p, z) || !aligned(a->r.p, z) || !aligned(a->y.p, z) || !aligned(a->decay, 4) || !aligned(a->init, 4) ||
      !aligned(a->lengths, 4) || !aligned(a->state, 4))
    return ops_fail(SNN_ERR_ARG, "recurrence: a pointer is not aligned to its element type");
  return SNN_OK;
}
bool strides_fit(const snn_rows &r, int T, size_t z) { return T <= 1 || !r.p || (r.stride_t >= 0 && r.stride_t < (int64_t)((1 << 30) / (STEPS * z))); }

// The workspace does not depend on the pointers, which decide between one channel a lane and two.
int most_segments(const snn_recurrence_args &a, bool backward) { return std::max(recurrence_cut(a, 1, backward).nseg, recurrence_cut(a, 2, backward).nseg); }

template <typename T, int VEC, int WAVES> int launch_forward(RecP p, hipStream_t st) {
  const int64_t each = (int64_t)p.groups * p.B;
  if constexpr (WAVES == 4)                                // (wider workgroups are not cut)
    if (p.nseg > 1) {
      hipLaunchKernelGGL((recurrence_forward_kernel<T, VEC, WAVES, false>), dim3((unsigned)(each * (p.nseg - 1))), dim3(WAVES * 64), 0, st, p);
      const int rc = ops_launched("recurrence, segments");
      if (rc) return rc;
    }
  hipLaunchKernelGGL((recurrence_forward_kernel<T, VEC, WAVES, true>), dim3((unsigned)(each * p.nseg)), dim3(WAVES * 64), 0, st, p);
  return ops_launched("recurrence");
}
template <typename T, int VEC, int WAVES> int launch_backward(RecP p, RecGradP g, float *ddecay, hipStream_t st) {
  const int64_t each = (int64_t)p.groups * p.B;
  if constexpr (WAVES == 4)
    if (p.nseg > 1) {
      hipLaunchKernelGGL((recurrence_backward_kernel<T, VEC, WAVES, false>), dim3((unsigned)(each * (p.nseg - 1))), dim3(WAVES * 64), 0, st, p, g);
      const int rc = ops_launched("recurrence backward, segments");
      if (rc) return rc;
    }
  hipLaunchKernelGGL((recurrence_backward_kernel<T, VEC, WAVES, true>), dim3((unsigned)(each * p.nseg)), dim3(WAVES * 64), 0, st, p, g);
  const int rc = ops_launched("recurrence backward");
  if (rc) return rc;
  hipLaunchKernelGGL(recurrence_sum_kernel, dim3((p.D + 15) / 16), dim3(256), 0, st, g.part, p.nseg * p.B, p.D, p.decay, ddecay);
  return ops_launched("recurrence backward, sums");
}

template <int WIDE, typename F> int with_shape(const snn_recurrence_args &a, bool two, int waves, F f) {
  auto go = [&](auto t, auto v) {
    return waves == WIDE ? f(t, v, std::integral_constant<int, WIDE>()) : f(t, v, std::integral_constant<int, 4>());
  };
  if (a.type == SNN_TYPE_FP32) return go(float(), std::integral_constant<int, 1>());
  return two ? go(__bf16(), std::integral_constant<int, 2>()) : go(__bf16(), std::integral_constant<int, 1>());
}

int recurrence_sizes(const snn_recurrence_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  if (!a) return ops_fail(SNN_ERR_NULL, "recurrence: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0 || a->D > (1 << 22) || (int64_t)a->B * ((a->D + CH - 1) / CH) >= (1 << 22) || a->T > (1 << 30))
    return ops_fail(SNN_ERR_ARG, "recurrence: sizes out of range");
  return SNN_OK;
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" {

int32_t snn_recurrence_workspace_bytes(const snn_recurrence_args *a, int32_t backward, size_t *bytes) {
  const int rc = recurrence_sizes(a, bytes);
  if (rc) return rc;
  const int n = most_segments(*a, backward != 0);
  const size_t row = (size_t)a->B * a->D * 4;
  *bytes = (n > 1 ? rup256(2 * n * row) : 0) + (backward ? rup256(n * row) : 0);
  return SNN_OK;
}

int32_t snn_recurrence_saved_bytes(const snn_recurrence_args *a, size_t *bytes) {
  const int rc = recurrence_sizes(a, bytes);
  if (rc) return rc;
  *bytes = (size_t)std::max(1, (a->T + STEPS - 1) / STEPS) * a->B * a->D * 4;
  return SNN_OK;
}

int32_t snn_recurrence_forward(const snn_recurrence_args *a, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = recurrence_check(a, false, false);
  if (rc) return rc;
  const size_t z = type_bytes(a->type);
  if (!strides_fit(a->x, a->T, z) || !strides_fit(a->i, a->T, z) || !strides_fit(a->r, a->T, z) || !strides_fit(a->y, a->T, z))
    return ops_fail(SNN_ERR_ARG, "recurrence: strides between steps must not be negative or put eight steps 1 GiB apart");
  if (!aligned(saved, 16)) return ops_fail(SNN_ERR_ARG, "recurrence: saved has to be 16-byte aligned");
  size_t need = 0;
  if ((rc = snn_recurrence_workspace_bytes(a, 0, &need))) return rc;
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return ops_fail(SNN_ERR_WORKSPACE, "recurrence: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  const bool two = two_channels(*a, nullptr);
  const RecCut c = recurrence_cut(*a, two ? 2 : 1, false);
  RecP p(*a);
  p.tiles = c.tiles;
  p.nseg = c.nseg;
  p.saved = (float *)saved;
  p.carry = (float2 *)workspace;
  return with_shape<16>(*a, two, c.waves, [&](auto t, auto v, auto w) { return launch_forward<decltype(t), v.value, w.value>(p, (hipStream_t)stream); });
}

int32_t snn_recurrence_backward(const snn_recurrence_args *a, const snn_recurrence_grads *g, const void *saved, void *workspace, size_t workspace_bytes,
                                void *stream) {
  int rc = recurrence_check(a, false, true);
  if (rc) return rc;
  if (!g || !g->ddecay || (a->T > 0 && (!g->dy.p || !g->dx.p || !g->di.p || !g->dr.p)))
    return ops_fail(SNN_ERR_NULL, "recurrence backward: dy, dx, di, dr or ddecay is NULL");
  if (!saved) return ops_fail(SNN_ERR_NULL, "recurrence backward: saved is NULL");
  const size_t z = type_bytes(a->type);
  if (!aligned(saved, 16) || !aligned(g->dy.p, z) || !aligned(g->dx.p, z) || !aligned(g->di.p, z) || !aligned(g->dr.p, z) || !aligned(g->d_state, 4) ||
      !aligned(g->ddecay, 4) || !aligned(g->dinit, 4))
    return ops_fail(SNN_ERR_ARG, "recurrence backward: a pointer is not aligned to its element type");
  for (const snn_rows *r : {&a->x, &a->i, &a->r, &g->dy, &g->dx, &g->di, &g->dr})
    if (!strides_fit(*r, a->T, z)) return ops_fail(SNN_ERR_ARG, "recurrence backward: strides between steps must not be negative or put eight steps 1 GiB apart");
  size_t need = 0;
  if ((rc = snn_recurrence_workspace_bytes(a, 1, &need))) return rc;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
    return ops_fail(SNN_ERR_WORKSPACE, "recurrence backward: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  const bool two = two_channels(*a, g);
  const RecCut c = recurrence_cut(*a, two ? 2 : 1, true);
  RecP p(*a);
  p.tiles = c.tiles;
  p.nseg = c.nseg;
  p.saved = (float *)const_cast<void *>(saved);
  p.carry = (float2 *)workspace;
  RecGradP q(*g, a->T);
  const int n = most_segments(*a, true);
  q.part = (float *)((char *)workspace + (n > 1 ? rup256((size_t)2 * n * a->B * a->D * 4) : 0));
  return with_shape<8>(*a, two, c.waves,
                    [&](auto t, auto v, auto w) { return launch_backward<decltype(t), v.value, w.value>(p, q, g->ddecay, (hipStream_t)stream); });
}

int32_t snn_recurrence_step(const snn_recurrence_args *a, void *stream) {
  const int rc = recurrence_check(a, true, false);
  if (rc) return rc;
  const RecP p(*a);
  const size_t z = type_bytes(a->type);
  auto take = [&](const snn_rows &r) { return rows_take(r, 1, a->B, 4, z); };
  const bool four = a->D % 4 == 0 && take(a->x) && take(a->i) && take(a->r) && take(a->y) && aligned(a->state, 16) && aligned(a->decay, 16);
  const int64_t threads = (int64_t)a->B * (four ? a->D / 4 : a->D);
  const dim3 grid((unsigned)((threads + 255) / 256));
  const hipStream_t st = (hipStream_t)stream;
  if (a->type == SNN_TYPE_FP32) {
    if (four) hipLaunchKernelGGL((recurrence_step_kernel<float, 4>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((recurrence_step_kernel<float, 1>), grid, dim3(256), 0, st, p);
  } else if (four) hipLaunchKernelGGL((recurrence_step_kernel<__bf16, 4>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((recurrence_step_kernel<__bf16, 1>), grid, dim3(256), 0, st, p);
  return ops_launched("recurrence step");
}

}  // extern "C"
