// Selective scan (include/snn_ops.h): N leaky states per channel, whose decay and input gain follow the data,
//   delta = softplus(dt + dt_bias),  h[t,n] = a[t,n] h[t-1,n] + delta x Bv[n],  a[t,n] = exp(delta A[n]),
//   y = (sum_n Cv[n] h[t,n] + skip x) z sigmoid(z).
//
// What bounds it.  An element of x costs N exponentials and about 4 N other vector operations (reverse: three times
// that) for 8 bytes of bfloat16 streams (reverse: 14 and 4 N / 16 of saved states): at N = 16 the vector units, 41 us for
// 1024 steps of 8 x 2048 channels by the formula's operations against 27 us for its bytes.
//
// Layout of the work.  A lane holds NS = 2 or 4 states of a channel; L = 4, 8 or 16 neighbouring lanes hold all of
// them (N <= NP = NS L, states beyond N are zero), so a wavefront carries 64 / L channels, and the state never leaves the
// registers.  Time goes in tiles of 16 steps: for a tile the 64 lanes first do what is once per (step, channel) -
// loads, softplus, the products delta and delta x - spread evenly, and put it into LDS; then every lane steps through
// the tile, reading its channel's (delta, delta x) and its own values of Bv and Cv as broadcasts; outputs go back
// through LDS and leave in the first mapping.  Holding only a few states a lane costs LDS reads, but gives four to eight
// times the wavefronts at N = 16 without computing anything twice.
//
// Where sequences and channels are too few to fill the chip, time is cut into chunks as well: the state after a chunk
// is exp(A sum(delta)) times the state before it plus the chunk's own (that factor may be out of range where no step is: grown_sum),
// so a first launch runs every chunk from zero
// (scan_forward_kernel, LOCAL), a second joins them in order (scan_join_kernel), and the third scans with the right
// states.  The reverse pass is cut the same way, from the other end.
//
// Measured (us): forward, 1024 steps of 8 x 2048 channels of 16 states, bfloat16, gated: 102 (2048 wavefronts of two
// states a lane, vector units issuing 82 % of the time), 8192 steps of 1024 channels: 30 + 8 + 43 for the three launches.
// Forward and backward at the first size: 407, of it 113 forward with its states saved, 50 reverse from zero (98 %
// issuing), 5 the join, 264 the reverse pass (88 %, 0.24 GB of traffic), 7 and 4 the sums.  101 ragged steps of
// 51 x 130 channels of 11 states, fp32, forward and backward: 60.
#include "common.hpp"
#include "seq_common.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

constexpr int TILE = 16;
constexpr int GROUP = 2;

struct ScanP {
  int T, B, D, N, G, softplus;
  int chunk, nchunks;                // steps per chunk (a multiple of TILE), chunks
  int blocks;                        // workgroups per (chunk, sequence, group)
  Rows<void> x, dt, z, bv, cv, y;
  const float *A, *skip, *dt_bias, *init;
  const int32_t *lengths;
  float *state;
  float *saved;                      // [tile][B][D][NP]: the state before every tile, or NULL
  float *local;                      // [chunk][B][D][NP]: of the chunks from zero, then (joined) the states before them
  float *sums;                       // [chunk][B][D]: sum of delta
  explicit ScanP(const snn_scan_args &a)
      : T(a.T), B(a.B), D(a.D), N(a.N), G(a.groups), softplus(a.softplus), chunk(TILE), nchunks(1), blocks(1), x(a.x, a.T), dt(a.dt, a.T),
        z(a.z, a.T), bv(a.bv, a.T), cv(a.cv, a.T), y(a.y, a.T), A(a.A), skip(a.skip), dt_bias(a.dt_bias), init(a.init), lengths(a.lengths),
        state(a.state), saved(nullptr), local(nullptr), sums(nullptr) {}
};

struct ScanGradP {
  Rows<void> dy, dx, ddt, dz;
  const float *d_state;
  float *dinit;
  float *dA;                         // [chunk * B][D][NP] partial sums
  float *dsum;                       // [chunk * B][2][D]: of dskip and ddt_bias
  float *dbc;                        // [blocks][T][B][G][2][NP] partial sums of dBv and dCv
  ScanGradP(const snn_scan_grads &g, int T)
      : dy(g.dy, T), dx(g.dx, T), ddt(g.ddt, T), dz(g.dz, T), d_state(g.d_state), dinit(g.dinit), dA(nullptr), dsum(nullptr), dbc(nullptr) {}
};

// Where a wavefront's work lies.
template <int L, int WAVES> struct Place {
  static constexpr int CH = 64 / L, E = CH * TILE / 64;
  int blk, g, b, s, lane, wave, ch, part, ec, et;
  int d, ed;                         // channel of the scan and of the elementwise mapping
  bool live, elive;
  __device__ Place(const ScanP &p) {
    unsigned id = blockIdx.x;
    blk = id % p.blocks; id /= p.blocks;
    g = id % p.G; id /= p.G;
    b = id % p.B; s = id / p.B;
    lane = threadIdx.x & 63; wave = threadIdx.x >> 6;
    ch = lane / L; part = lane % L;
    ec = lane % CH; et = lane / CH;
    const int dg = p.D / p.G, c0 = (blk * WAVES + wave) * CH;
    live = c0 + ch < dg; elive = c0 + ec < dg;
    d = g * dg + (live ? c0 + ch : 0);
    ed = g * dg + (elive ? c0 + ec : 0);
  }
};

// The loads and address computations below are the same for all lanes: a lane without a channel, a state or a step of
// its own takes another one's, and the value is replaced by zero afterwards.  Where lanes took turns instead, under high
// register pressure, the compiler put copies of values that all lanes need later into the region where only some run.

// The length of a sequence, in a scalar register: tiles are whole or not for all lanes alike.
__device__ __forceinline__ int wave_length(const ScanP &p, int b) { return __builtin_amdgcn_readfirstlane(length_of(p.lengths, b, p.T)); }

// A lane's states out of [D][N] or [B][D][N] rows, zero beyond N.
template <int NS> __device__ __forceinline__ void load_states(float r[NS], const float *row, int part, int N, bool live) {
#pragma unroll
  for (int j = 0; j < NS; ++j) r[j] = 0.f;
  if (row)
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      const float v = row[min(part * NS + j, N - 1)];
      r[j] = live & (part * NS + j < N) ? v : 0.f;
    }
}
template <int NS> __device__ __forceinline__ void store_states(float *row, const float r[NS], int part, int N) {
#pragma unroll
  for (int j = 0; j < NS; ++j)
    if (part * NS + j < N) row[part * NS + j] = r[j];
}
// The decay of a state, in base 2.  That of a state which forgets at once, A = -inf, becomes the lowest finite number, so
// that it stays what it is over steps that do not exist: their delta is 0.
__device__ __forceinline__ float decay_rate(float A) {
  const float r = A * LOG2E;
  return r < -3.4028234663852886e38f ? -3.4028234663852886e38f : r;
}
// The rate itself where the reverse pass multiplies by it: what a state that forgets at once hands back through its decay is zero, and
// zero times the lowest finite number still is.
__device__ __forceinline__ float finite_rate(float A) { return A < -3.4028234663852886e38f ? -3.4028234663852886e38f : A; }
// A lane's states out of rows of the library's own, which are padded and aligned.
template <int NS> using States = Pack<float, NS>;
template <int NS> __device__ __forceinline__ States<NS> pick(const float *p) { return *(const States<NS> *)p; }
template <int NS> __device__ __forceinline__ void put_states(float *p, const float r[NS]) {
  States<NS> v;
#pragma unroll
  for (int j = 0; j < NS; ++j) v.v[j] = r[j];
  *(States<NS> *)p = v;
}

// Streamed tensors go through buffer instructions: a base that the whole wavefront shares (tensor, sequence, tile), the
// byte offset of the lane in it (channel, step within the tile: one register, computed once) and a scalar offset for
// the steps of a round.  The host keeps the sum below SPAN (scan_strides); at NOWHERE a load gives zero and a store is
// dropped, so steps that do not exist need no branch.
constexpr int SPAN = 0x7FFF0000, NOWHERE = 0x7FFFFF00;
__device__ __forceinline__ float take(rsrc_t r, int voff, int soff, float) { return __uint_as_float(ld_b32(r, voff, soff)); }
__device__ __forceinline__ __bf16 take(rsrc_t r, int voff, int soff, __bf16) {
  return __builtin_bit_cast(__bf16, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(r, voff, soff, 0));
}
__device__ __forceinline__ void give(rsrc_t r, int voff, int soff, float v) { st_b32(r, voff, soff, __float_as_uint(v)); }
__device__ __forceinline__ void give(rsrc_t r, int voff, int soff, __bf16 v) { st_b16(r, voff, soff, __builtin_bit_cast(unsigned short, v)); }

// What a lane loads of the rows of Bv (or Cv), THREADS threads sharing a tile of TILE x NP values: value n of step
// et + i COUNT / NP; threads beyond one for every value repeat what others do.  In LDS they stand as fp32 [TILE][NP],
// zero beyond N and for steps that do not exist.
template <typename T, int NP, int THREADS> struct Vectors {
  static constexpr int COUNT = THREADS < TILE * NP ? THREADS : TILE * NP, STEP = COUNT / NP, EACH = TILE / STEP;
  static_assert(STEP * EACH == TILE, "a tile is a whole number of rounds");
  const T *p;
  int64_t st;
  int et, n, at, row;                // `at`: the lane's offset; `row`: bytes between steps
  T r[EACH];
  __device__ Vectors(const Rows<void> &src, int b, int g, int N, int me)
      : p((const T *)src.p + b * src.sb + (int64_t)g * N), st(src.st), et(me % COUNT / NP), n(me % NP), row((int)(src.st * sizeof(T))) {
    at = n < N ? n * (int)sizeof(T) + et * row : NOWHERE;
  }
  __device__ __forceinline__ void fetch(int t0, int end) {
    const rsrc_t q = make_rsrc(p + t0 * st, SPAN);
#pragma unroll
    for (int i = 0; i < EACH; ++i) r[i] = take(q, t0 + et + i * STEP < end ? at : NOWHERE, i * STEP * row, (T)0.f);
  }
  __device__ __forceinline__ void put(float *lds) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) lds[(et + i * STEP) * NP + n] = widen(r[i]);
  }
};

// What a lane loads or stores of a streamed tensor in the elementwise mapping: channel ed, steps et + i TILE / E.
template <typename T, int E> struct Stream {
  static constexpr int STEP = TILE / E;
  T *p;
  int64_t st;
  int et, at, row;
  T r[E];
  __device__ Stream(const Rows<void> &src, int b, int d, int et_) : p((T *)src.p + b * src.sb), st(src.st), et(et_), row((int)(src.st * sizeof(T))) {
    at = d * (int)sizeof(T) + et * row;
  }
  __device__ __forceinline__ void fetch(int t0, int end) {
    const rsrc_t q = make_rsrc(p + t0 * st, SPAN);
#pragma unroll
    for (int i = 0; i < E; ++i) r[i] = take(q, t0 + et + i * STEP < end ? at : NOWHERE, i * STEP * row, (T)0.f);
  }
  __device__ __forceinline__ void put(const float v[E], int t0, int end, bool live) const {
    const rsrc_t q = make_rsrc(p + t0 * st, SPAN);
#pragma unroll
    for (int i = 0; i < E; ++i) give(q, live & (t0 + et + i * STEP < end) ? at : NOWHERE, i * STEP * row, narrow<T>(v[i]));
  }
};

// ---------------------------------------------------------------- forward
// LOCAL: the chunk from zero, for its end state and its sum of delta alone; no outputs.
template <typename T, int NS, int L, int WAVES, bool GATE, bool LOCAL>
__global__ __launch_bounds__(64 * WAVES) void scan_forward_kernel(const ScanP p) {
  using P = Place<L, WAVES>;
  constexpr int CH = P::CH, E = P::E, NP = NS * L, KEEP = TILE / L;
  __shared__ float2 s_d[WAVES][TILE * CH];
  __shared__ __attribute__((aligned(16))) float s_b[WAVES][TILE * NP], s_c[WAVES][LOCAL ? 4 : TILE * NP];
  __shared__ float s_y[WAVES][LOCAL ? 4 : TILE * CH];
  const P me(p);
  float2 *sd = s_d[me.wave];
  float *sb = s_b[me.wave], *sc = s_c[me.wave], *sy = s_y[me.wave];
  const int c0 = me.s * p.chunk, c1 = min(p.T, c0 + p.chunk), end = min(c1, wave_length(p, me.b));
  const size_t seq = (size_t)me.b * p.D + me.d;

  float A[NS], h[NS], sum = 0.f;
  load_states<NS>(A, p.A + (size_t)me.d * p.N, me.part, p.N, me.live);
#pragma unroll
  for (int j = 0; j < NS; ++j) { A[j] = decay_rate(A[j]); h[j] = 0.f; }
  if constexpr (!LOCAL) {
    if (p.nchunks > 1) {
      const States<NS> v = pick<NS>(p.local + ((size_t)me.s * p.B * p.D + seq) * NP + me.part * NS);
#pragma unroll
      for (int j = 0; j < NS; ++j) h[j] = me.live ? v.v[j] : 0.f;
    } else {
      load_states<NS>(h, p.init ? p.init + seq * p.N : nullptr, me.part, p.N, me.live);
    }
  }
  const float dt_bias = p.dt_bias ? p.dt_bias[me.ed] : 0.f, skip = p.skip ? p.skip[me.ed] : 0.f;

  Stream<T, E> gx(p.x, me.b, me.ed, me.et), gd(p.dt, me.b, me.ed, me.et), gz(p.z, me.b, me.ed, me.et), gy(p.y, me.b, me.ed, me.et);
  Vectors<T, NP, 64> gb(p.bv, me.b, me.g, p.N, me.lane), gc(p.cv, me.b, me.g, p.N, me.lane);
  auto load = [&](int t0) {
    gx.fetch(t0, end);
    gd.fetch(t0, end);
    gb.fetch(t0, end);
    if constexpr (!LOCAL) {
      if constexpr (GATE) gz.fetch(t0, end);
      gc.fetch(t0, end);
    }
  };
  load(c0);
  int t0 = c0;
  for (; t0 < end; t0 += TILE) {
    float x[E], z[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = me.et + i * (TILE / E);
      const bool on = (t0 + t < end) & me.elive;
      const float raw = widen(gd.r[i]) + dt_bias;
      x[i] = on ? widen(gx.r[i]) : 0.f;
      z[i] = !LOCAL && GATE ? widen(gz.r[i]) : 0.f;
      const float soft = softplus(raw), delta = on ? (p.softplus ? soft : raw) : 0.f;
      sd[t * CH + me.ec] = make_float2(delta, delta * x[i]);
    }
    gb.put(sb);
    if constexpr (!LOCAL) gc.put(sc);
    load(t0 + TILE);                                        // (what does not exist is not read)
    wave_lds_order();
    if constexpr (!LOCAL) {
      const rsrc_t to = make_rsrc(p.saved + ((size_t)(t0 / TILE) * p.B + me.b) * p.D * NP, SPAN);
      const int at = (p.saved != nullptr) & me.live ? (me.d * NP + me.part * NS) * 4 : NOWHERE;
      if constexpr (NS == 4) st_b128(to, at, 0, (u32x4){__float_as_uint(h[0]), __float_as_uint(h[1]), __float_as_uint(h[2]), __float_as_uint(h[3])});
      else st_b64(to, at, 0, (u32x2){__float_as_uint(h[0]), __float_as_uint(h[1])});
    }
    float keep[KEEP];                                       // outputs of the steps whose number mod L is this lane's part
    // what GROUP steps read of LDS, loaded while the GROUP before them is computed
    float2 u[2][GROUP];
    States<NS> bs[2][GROUP], cs[2][GROUP];
    const auto read = [&](int t) {
#pragma unroll
      for (int k = 0; k < GROUP; ++k) {
        const int i = t / GROUP % 2;
        u[i][k] = sd[(t + k) * CH + me.ch];
        bs[i][k] = pick<NS>(sb + (t + k) * NP + me.part * NS);
        if constexpr (!LOCAL) cs[i][k] = pick<NS>(sc + (t + k) * NP + me.part * NS);
      }
    };
    read(0);
#pragma unroll
    for (int t = 0; t < TILE; ++t) {
      const int i = t / GROUP % 2, k = t % GROUP;
      if (k == 0) {
        if (t + GROUP < TILE) read(t + GROUP);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < NS; ++j) h[j] = fmaf(__builtin_amdgcn_exp2f(u[i][k].x * A[j]), h[j], u[i][k].y * bs[i][k].v[j]);
      if constexpr (LOCAL) {
        sum += u[i][k].x;
      } else {
        float v = cs[i][k].v[0] * h[0];
#pragma unroll
        for (int j = 1; j < NS; ++j) v = fmaf(cs[i][k].v[j], h[j], v);
        v = sum_neighbours<L>(v);
        keep[t / L] = t % L == 0 || me.part == t % L ? v : keep[t / L];
      }
    }
    if constexpr (!LOCAL) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) sy[(i * L + me.part) * CH + me.ch] = keep[i];
      wave_lds_order();
      float out[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int t = me.et + i * (TILE / E);
        const float inner = sy[t * CH + me.ec], with = fmaf(skip, x[i], inner);
        float v = p.skip ? with : inner;                    // (a skip that is absent is no zero: 0 inf)
        if constexpr (GATE) v *= z[i] * sigmoid_fast(z[i]);
        out[i] = t0 + t < end ? v : 0.f;
      }
      gy.put(out, t0, c1, me.elive);
    }
    wave_lds_order();
  }
  if constexpr (!LOCAL) {
    float zero[E];
#pragma unroll
    for (int i = 0; i < E; ++i) zero[i] = 0.f;
    for (; t0 < c1; t0 += TILE) gy.put(zero, t0, c1, me.elive);          // steps that do not exist
  }
  if (!me.live) return;
  if constexpr (LOCAL) {
    put_states<NS>(p.local + ((size_t)me.s * p.B * p.D + seq) * NP + me.part * NS, h);
    if (me.part == 0) p.sums[(size_t)me.s * p.B * p.D + seq] = sum;
  } else if (p.state && me.s == p.nchunks - 1) {
    store_states<NS>(p.state + seq * p.N, h, me.part, p.N);
  }
}

// h 2^e + v for an e that may be far above the exponents of fp32, while h is zero or the product in range: a state that grows
// (A > 0 or delta < 0) over a chunk, each of whose steps is in range.  So 2^e is applied in three parts of at most 126,
// 378 in all, which takes the least number above the greatest.  A NaN stays one.
__device__ __forceinline__ float grown_sum(float e, float h, float v) {
  const float e0 = e > 126.f ? 126.f : e, rest = e > 126.f ? e - 126.f : 0.f;
  const float e1 = fminf(rest, 126.f), e2 = fminf(rest - e1, 126.f);
  return fmaf(__builtin_amdgcn_exp2f(e0), h * __builtin_amdgcn_exp2f(e1) * __builtin_amdgcn_exp2f(e2), v);
}

// Joins the chunks: local[s] (of the chunk from zero) becomes the state before chunk s, in order; with REVERSE the
// gradient behind it, from the last one.  A thread per (sequence, channel, state); the loads of eight chunks are in
// flight at a time.
template <int NP, bool REVERSE> __global__ __launch_bounds__(256) void scan_join_kernel(const ScanP p, const float *first) {
  constexpr int AHEAD = 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, seqs = (int64_t)p.B * p.D, all = seqs * NP;
  if (id >= all) return;
  const int n = (int)(id % NP);
  const int64_t seq = id / NP;
  const bool live = n < p.N;
  const float A = live ? decay_rate(p.A[(seq % p.D) * p.N + n]) : 0.f;
  float h = first && live ? first[seq * p.N + n] : 0.f;
  const int last = p.nchunks - 1;                          // (the chunk that nobody follows was not run from zero)
  for (int i0 = 0; i0 <= last; i0 += AHEAD) {
    float v[AHEAD], e[AHEAD];
    bool grows = false;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + k, s = REVERSE ? last - i : i;
      v[k] = i < last ? p.local[s * all + id] : 0.f;
      e[k] = (i < last ? p.sums[s * seqs + seq] : 0.f) * A;
      grows |= e[k] > 126.f;
    }
    const auto join = [&](auto sum) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int i = i0 + k, s = REVERSE ? last - i : i;
        if (i <= last) p.local[s * all + id] = h;
        h = sum(e[k], h, v[k]);
      }
    };
    // (a branch of the whole wavefront: the long form throughout made 8192 steps of 1024 channels 3 us longer)
    if (__any(grows)) join(grown_sum);
    else join([](float e, float h, float v) { return fmaf(__builtin_amdgcn_exp2f(e), h, v); });
  }
}

// ---------------------------------------------------------------- reverse
// The chunk from a zero gradient behind it: the gradient of the state before it and the sum of delta.
template <typename T, int NS, int L, int WAVES, bool GATE>
__global__ __launch_bounds__(64 * WAVES) void scan_reverse_local_kernel(const ScanP p, const ScanGradP g) {
  using P = Place<L, WAVES>;
  constexpr int CH = P::CH, E = P::E, NP = NS * L;
  __shared__ float2 s_d[WAVES][TILE * CH];
  __shared__ __attribute__((aligned(16))) float s_c[WAVES][TILE * NP];
  P me(p);
  me.s += 1;                                               // (nothing is in front of chunk 0)
  float2 *sd = s_d[me.wave];
  float *sc = s_c[me.wave];
  const int c0 = me.s * p.chunk, c1 = min(p.T, c0 + p.chunk), end = min(c1, wave_length(p, me.b));
  const size_t seq = (size_t)me.b * p.D + me.d;
  float A[NS], q[NS], sum = 0.f;
  load_states<NS>(A, p.A + (size_t)me.d * p.N, me.part, p.N, me.live);
#pragma unroll
  for (int j = 0; j < NS; ++j) { A[j] = decay_rate(A[j]); q[j] = 0.f; }
  const float dt_bias = p.dt_bias ? p.dt_bias[me.ed] : 0.f;
  Stream<T, E> gy(g.dy, me.b, me.ed, me.et), gd(p.dt, me.b, me.ed, me.et), gz(p.z, me.b, me.ed, me.et);
  Vectors<T, NP, 64> gc(p.cv, me.b, me.g, p.N, me.lane);
  auto load = [&](int t0) {
    gy.fetch(t0, end);
    gd.fetch(t0, end);
    if constexpr (GATE) gz.fetch(t0, end);
    gc.fetch(t0, end);
  };
  const int tiles = end > c0 ? (end - c0 + TILE - 1) / TILE : 0;
  if (tiles) load(c0 + (tiles - 1) * TILE);
  for (int i0 = tiles - 1; i0 >= 0; --i0) {
    const int t0 = c0 + i0 * TILE;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = me.et + i * (TILE / E);
      const float raw = widen(gd.r[i]) + dt_bias;
      float dy = widen(gy.r[i]);
      if constexpr (GATE) { const float z = widen(gz.r[i]); dy *= z * sigmoid_fast(z); }
      const bool on = (t0 + t < end) & me.elive;
      const float soft = softplus(raw);
      sd[t * CH + me.ec] = make_float2(on ? (p.softplus ? soft : raw) : 0.f, on ? dy : 0.f);
    }
    gc.put(sc);
    load(max(t0 - TILE, c0));
    wave_lds_order();
#pragma unroll
    for (int t = TILE - 1; t >= 0; --t) {
      const float2 u = sd[t * CH + me.ch];
      const States<NS> c = pick<NS>(sc + t * NP + me.part * NS);
#pragma unroll
      for (int j = 0; j < NS; ++j) q[j] = fmaf(u.y, c.v[j], q[j]) * __builtin_amdgcn_exp2f(u.x * A[j]);
      sum += u.x;
    }
    wave_lds_order();
  }
  if (!me.live) return;
  put_states<NS>(p.local + ((size_t)me.s * p.B * p.D + seq) * NP + me.part * NS, q);
  if (me.part == 0) p.sums[(size_t)me.s * p.B * p.D + seq] = sum;
}

// Sums v (NS of dBv, NS of dCv) over the wavefront's channels, lane bits log2(L) to 5.  While there are values enough,
// the halves of the wavefront trade: each keeps half the values, summed; then the rows of 16 likewise; what is left of
// the bits goes by rotations.  This lane gets NS / 2 sums: of dBv in lanes 0-31, of dCv in 32-63, the first ones where
// lane bit 4 is 0, the others where it is 1.
template <int NS, int L> __device__ __forceinline__ void sum_channels(const float v[2 * NS], float c[NS / 2]) {
  float a[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v[j]), __builtin_bit_cast(unsigned, v[j + NS]), false, false);
    a[j] = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
#pragma unroll
  for (int j = 0; j < NS / 2; ++j) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a[j]), __builtin_bit_cast(unsigned, a[j + NS / 2]), false, false);
    c[j] = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    if constexpr (L <= 8) c[j] += dpp<0x128>(c[j]);
    if constexpr (L <= 4) c[j] += dpp<0x124>(c[j]);
  }
}

// The reverse pass proper.  Per tile, from the last: the states of the tile once more from the one that the forward
// pass saved in front of it, kept with their decays (registers; the first half's states in LDS), then back through the steps:
//   g = q + dy0 C,   dC += dy0 h,  dB += g delta x  (over the channels),   u = g a h[t-1]
//   d(delta) = sum_n u A + x sum_n g B,   dx = delta sum_n g B + dy0 skip,   dA += u delta,   q = g a.
// The workgroup's wavefronts share the rows of Bv and Cv, and add their channel sums of dBv and dCv through LDS in a
// fixed order; sums over workgroups are left to scan_sum_rows_kernel.
template <typename T, int NS, int L, int WAVES, bool GATE>
__global__ __launch_bounds__(64 * WAVES, 2) void scan_reverse_kernel(const ScanP p, const ScanGradP g) {
  using P = Place<L, WAVES>;
  constexpr int CH = P::CH, E = P::E, NP = NS * L, THREADS = 64 * WAVES, KEEP = TILE / L, TWINS = 16 / L, HALF = TILE / 2;
  __shared__ float4 s_d[WAVES][TILE * CH];                  // delta, delta x, dy0, d(delta) / d(dt)
  __shared__ float s_y[WAVES][TILE * CH];                   // sum C h
  __shared__ float2 s_g[WAVES][TILE * CH];                  // sum g B, sum u A
  __shared__ States<NS> s_h[WAVES][(HALF - 1) * 64];        // states of the first half of a tile
  __shared__ __attribute__((aligned(16))) float s_b[TILE * NP], s_c[TILE * NP];
  __shared__ __attribute__((aligned(16))) float s_s[WAVES][2][TILE * NP];
  const P me(p);
  float4 *sd = s_d[me.wave];
  float *sy = s_y[me.wave];
  float2 *sg = s_g[me.wave];
  States<NS> *sh = s_h[me.wave] + me.lane;
  const int c0 = me.s * p.chunk, c1 = min(p.T, c0 + p.chunk), end = min(c1, wave_length(p, me.b));
  const size_t seq = (size_t)me.b * p.D + me.d;
  float A[NS], A2[NS], q[NS], dA[NS];
  load_states<NS>(A, p.A + (size_t)me.d * p.N, me.part, p.N, me.live);
#pragma unroll
  for (int j = 0; j < NS; ++j) { A2[j] = decay_rate(A[j]); A[j] = finite_rate(A[j]); dA[j] = 0.f; }
  if (p.nchunks > 1) {
    const States<NS> v = pick<NS>(p.local + ((size_t)me.s * p.B * p.D + seq) * NP + me.part * NS);
#pragma unroll
    for (int j = 0; j < NS; ++j) q[j] = me.live ? v.v[j] : 0.f;
  } else {
    load_states<NS>(q, g.d_state ? g.d_state + seq * p.N : nullptr, me.part, p.N, me.live);
  }
  const float dt_bias = p.dt_bias ? p.dt_bias[me.ed] : 0.f, skip = p.skip ? p.skip[me.ed] : 0.f;
  int has = p.skip != nullptr;                             // (in a vector register: scalar ones are short here, 404 us against 406)
  asm("" : "+v"(has));
  float dskip = 0.f, ddtb = 0.f;

  Stream<T, E> gx(p.x, me.b, me.ed, me.et), gd(p.dt, me.b, me.ed, me.et), gy(g.dy, me.b, me.ed, me.et), gz(p.z, me.b, me.ed, me.et);
  const Stream<T, E> wx(g.dx, me.b, me.ed, me.et), wd(g.ddt, me.b, me.ed, me.et), wz(g.dz, me.b, me.ed, me.et);
  Vectors<T, NP, THREADS> gb(p.bv, me.b, me.g, p.N, threadIdx.x), gc(p.cv, me.b, me.g, p.N, threadIdx.x);
  States<NS> rh;
  auto load = [&](int t0) {
    gx.fetch(t0, end);
    gd.fetch(t0, end);
    gy.fetch(t0, end);
    if constexpr (GATE) gz.fetch(t0, end);
    gb.fetch(t0, end);
    gc.fetch(t0, end);
    rh = pick<NS>(p.saved + ((size_t)(t0 / TILE) * p.B * p.D + seq) * NP + me.part * NS);
  };
  const int tiles = end > c0 ? (end - c0 + TILE - 1) / TILE : 0;
  {
    float zero[E];
#pragma unroll
    for (int i = 0; i < E; ++i) zero[i] = 0.f;
    for (int t0 = c0 + tiles * TILE; t0 < c1; t0 += TILE) {                // steps that do not exist
      wx.put(zero, t0, c1, me.elive);
      wd.put(zero, t0, c1, me.elive);
      if constexpr (GATE) wz.put(zero, t0, c1, me.elive);
    }
  }
  if (tiles) load(c0 + (tiles - 1) * TILE);
  for (int i0 = tiles - 1; i0 >= 0; --i0) {
    const int t0 = c0 + i0 * TILE;
    float x[E], z[E], dy[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = me.et + i * (TILE / E);
      const bool on = (t0 + t < end) & me.elive;
      const float raw = widen(gd.r[i]) + dt_bias;
      x[i] = on ? widen(gx.r[i]) : 0.f;
      dy[i] = on ? widen(gy.r[i]) : 0.f;
      z[i] = GATE && on ? widen(gz.r[i]) : 0.f;
      const float e = exp_fast(-fabsf(raw)), r = rcp_fast(1.f + e);
      const float soft = softplus(raw), delta = on ? (p.softplus ? soft : raw) : 0.f;
      const float slope = p.softplus ? (raw >= 0.f ? r : e * r) : 1.f;
      const float dy0 = GATE ? dy[i] * z[i] * sigmoid_fast(z[i]) : dy[i];
      sd[t * CH + me.ec] = make_float4(delta, delta * x[i], dy0, slope);
    }
    gb.put(s_b);
    gc.put(s_c);
    float h0[NS], hn[NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) hn[j] = h0[j] = me.live ? rh.v[j] : 0.f;
    float h[HALF + 1][NS], a[TILE][NS];                     // h: of the steps from HALF - 1 on
    __syncthreads();
    float k0[KEEP], k1[KEEP];                               // of the steps whose number mod L is this lane's part
    {
      float2 u[2];                                          // what a step reads of LDS, loaded a step ahead
      States<NS> bs[2], cs[2];
      const auto read = [&](int t) {
        u[t % 2] = *(const float2 *)(sd + t * CH + me.ch);
        bs[t % 2] = pick<NS>(s_b + t * NP + me.part * NS);
        if constexpr (GATE) cs[t % 2] = pick<NS>(s_c + t * NP + me.part * NS);
      };
      read(0);
#pragma unroll
      for (int t = 0; t < TILE; ++t) {
        if (t + 1 < TILE) read(t + 1);
        __builtin_amdgcn_sched_barrier(0);
        const float2 un = u[t % 2];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          a[t][j] = __builtin_amdgcn_exp2f(un.x * A2[j]);
          hn[j] = fmaf(a[t][j], hn[j], un.y * bs[t % 2].v[j]);
          if (t >= HALF - 1) h[t - HALF + 1][j] = hn[j];
        }
        if (t < HALF - 1) put_states<NS>((float *)(sh + t * 64), hn);
        if constexpr (GATE) {                               // dz needs the output before the gate
          float v = cs[t % 2].v[0] * hn[0];
#pragma unroll
          for (int j = 1; j < NS; ++j) v = fmaf(cs[t % 2].v[j], hn[j], v);
          v = sum_neighbours<L>(v);
          k0[t / L] = t % L == 0 || me.part == t % L ? v : k0[t / L];
        }
      }
      if constexpr (GATE)
#pragma unroll
        for (int i = 0; i < KEEP; ++i) sy[(i * L + me.part) * CH + me.ch] = k0[i];
    }
    asm volatile("" ::: "memory");                          // (the rows of Bv, Cv and sd are read again, not kept in registers)
    float hc[NS];                                           // the state after step t
    float kv[TILE / TWINS][NS / 2];                         // of the steps whose number mod TWINS is this lane's among its twins
    float4 ur[2];                                           // what a step reads of LDS, loaded a step ahead
    States<NS> br[2], cr[2], hr[2];
    const auto read = [&](int t) {
      ur[t % 2] = sd[t * CH + me.ch];
      br[t % 2] = pick<NS>(s_b + t * NP + me.part * NS);
      cr[t % 2] = pick<NS>(s_c + t * NP + me.part * NS);
      if (t > 0 && t < HALF) hr[t % 2] = sh[(t - 1) * 64];
    };
    read(TILE - 1);
#pragma unroll
    for (int t = TILE - 1; t >= 0; --t) {
      if (t > 0) read(t - 1);
      __builtin_amdgcn_sched_barrier(0);
      if (t == HALF - 1) {
        // The tile in front, for which half of the registers of h and a are free by now.  No branch for the first tile,
        // which has none (no step of it exists then): sums that only a later block needs would be put off to there, and
        // what they are sums of would be kept in registers until then.
        const int next = max(t0 - TILE, c0), stop = i0 > 0 ? end : 0;
        gx.fetch(next, stop);
        gd.fetch(next, stop);
        gy.fetch(next, stop);
        if constexpr (GATE) gz.fetch(next, stop);
        gb.fetch(next, stop);
        gc.fetch(next, stop);
        rh = pick<NS>(p.saved + ((size_t)(next / TILE) * p.B * p.D + seq) * NP + me.part * NS);
      }
      const float4 u = ur[t % 2];
      float v[2 * NS], gsum = 0.f, usum = 0.f, hp[NS];
      const bool exists = t0 + t < end;                     // (else delta is 0, but the state may be infinite: dA would be NaN)
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        if (t == TILE - 1) hc[j] = h[HALF][j];
        if (t >= HALF) hp[j] = h[t - HALF][j];
        else if (t > 0) hp[j] = hr[t % 2].v[j];
        else hp[j] = h0[j];
        const float gh = fmaf(u.z, cr[t % 2].v[j], q[j]);
        v[j] = gh * u.y;
        v[NS + j] = u.z * hc[j];
        gsum = fmaf(gh, br[t % 2].v[j], gsum);
        q[j] = gh * a[t][j];
        const float w = q[j] * hp[j];
        hc[j] = hp[j];
        usum = fmaf(w, A[j], usum);
        dA[j] = fmaf(exists ? w : 0.f, u.x, dA[j]);
      }
      gsum = sum_neighbours<L>(gsum);
      usum = sum_neighbours<L>(usum);
      const bool mine = t % L == L - 1 || me.part == t % L;
      k0[t / L] = mine ? gsum : k0[t / L];
      k1[t / L] = mine ? usum : k1[t / L];
      float s[NS / 2];
      sum_channels<NS, L>(v, s);
      const bool twin = t % TWINS == TWINS - 1 || (me.lane & 15) / L == t % TWINS;
#pragma unroll
      for (int j = 0; j < NS / 2; ++j) kv[t / TWINS][j] = twin ? s[j] : kv[t / TWINS][j];
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) sg[(i * L + me.part) * CH + me.ch] = make_float2(k0[i], k1[i]);
#pragma unroll
    for (int i = 0; i < TILE / TWINS; ++i)
      put_states<NS / 2>(&s_s[me.wave][me.lane >> 5][(i * TWINS + (me.lane & 15) / L) * NP + me.part * NS + ((me.lane >> 4) & 1) * (NS / 2)], kv[i]);
    wave_lds_order();
    float ox[E], od[E], oz[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = me.et + i * (TILE / E);
      const bool on = (t0 + t < end) & me.elive;
      const float4 u = sd[t * CH + me.ec];
      const float2 r = sg[t * CH + me.ec];
      if constexpr (GATE) {
        const float inner = sy[t * CH + me.ec], with = inner + skip * x[i];
        const float e = sigmoid_fast(z[i]), v = dy[i] * (has ? with : inner) * e * (1.f + z[i] * (1.f - e));
        oz[i] = on ? v : 0.f;
      }
      const float own = u.z * skip, vx = fmaf(u.x, r.x, has ? own : 0.f), vd = fmaf(x[i], r.x, r.y) * u.w;
      ox[i] = on ? vx : 0.f;
      od[i] = on ? vd : 0.f;
      ddtb += od[i];
      dskip = fmaf(u.z, x[i], dskip);
    }
    wx.put(ox, t0, c1, me.elive);
    wd.put(od, t0, c1, me.elive);
    if constexpr (GATE) wz.put(oz, t0, c1, me.elive);
    __syncthreads();
    const int pitch = p.B * p.G * 2 * NP * 4;               // bytes between steps (scan_sizes: 16 of them stay below SPAN)
    const rsrc_t out = make_rsrc(g.dbc + ((((size_t)me.blk * p.T + t0) * p.B + me.b) * p.G + me.g) * (2 * NP), SPAN);
#pragma unroll
    for (int i = 0; i < (2 * TILE * NP + THREADS - 1) / THREADS; ++i) {
      const int at = i * THREADS + threadIdx.x, t = at / (2 * NP), kn = at % (2 * NP);
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += s_s[w][kn / NP][t % TILE * NP + kn % NP];
      st_b32(out, (t0 + t < end) & (at < 2 * TILE * NP) ? t * pitch + kn * 4 : NOWHERE, 0, __float_as_uint(s));
    }
  }
  // sums over the lanes that share a channel of the elementwise mapping: lane bits log2(CH) to 5
  wave_lds_order();
  sd[me.lane].x = dskip;
  sd[me.lane].y = ddtb;
  wave_lds_order();
  if (me.lane < CH && me.elive) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < L; ++i) { s0 += sd[i * CH + me.lane].x; s1 += sd[i * CH + me.lane].y; }
    float *to = g.dsum + ((size_t)me.s * p.B + me.b) * 2 * p.D + me.ed;
    to[0] = s0;
    to[p.D] = s1;
  }
  if (!me.live) return;
  put_states<NS>(g.dA + (((size_t)me.s * p.B + me.b) * p.D + me.d) * NP + me.part * NS, dA);
  if (g.dinit && me.s == 0) store_states<NS>(g.dinit + seq * p.N, q, me.part, p.N);
}

// dBv and dCv: sums of the workgroups' partial sums, zero where the step does not exist.  A thread per value.
template <typename T, int NP>
__global__ __launch_bounds__(256) void scan_sum_rows_kernel(const ScanP p, const float *__restrict__ dbc, Rows<void> dbv, Rows<void> dcv) {
  const int64_t all = (int64_t)p.T * p.B * p.G * 2 * NP;
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
    const int n = (int)(id % NP), kind = (int)(id / NP % 2);
    const int64_t row = id / (2 * NP);
    const int gr = (int)(row % p.G), b = (int)(row / p.G % p.B), t = (int)(row / p.G / p.B);
    if (n >= p.N) continue;
    float s = 0.f;
    if (t < length_of(p.lengths, b, p.T)) {
      int k = 0;
      for (; k + 8 <= p.blocks; k += 8) {                   // (eight loads in flight)
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = dbc[(k + u) * all + id];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += v[u];
      }
      for (; k < p.blocks; ++k) s += dbc[k * all + id];
    }
    const Rows<void> &to = kind ? dcv : dbv;
    ((T *)to.p)[t * to.st + b * to.sb + (int64_t)gr * p.N + n] = narrow<T>(s);
  }
}

// dA, dskip, ddt_bias: sums over chunks and sequences.
template <int NP>
__global__ __launch_bounds__(256) void scan_sum_params_kernel(const ScanP p, const float *__restrict__ dA_part, const float *__restrict__ dsum,
                                                              float *__restrict__ dA, float *__restrict__ dskip, float *__restrict__ ddt_bias) {
  __shared__ float lds[256];
  const int rows = p.nchunks * p.B;
  const int64_t na = (int64_t)p.D * NP, blocks = (na + 15) / 16;
  const bool first = blockIdx.x < blocks;                   // workgroups of dA, then those of the other two
  const int64_t cols = first ? na : 2 * (int64_t)p.D, c = (blockIdx.x - (first ? 0 : blocks)) * 16 + (threadIdx.x & 15);
  const float s = sum_column(first ? dA_part : dsum, cols, c, rows, lds);
  if (threadIdx.x >= 16 || c >= cols) return;
  if (first) {
    const int n = (int)(c % NP);
    if (n < p.N) dA[c / NP * p.N + n] = s;
  } else if (c < p.D) {
    if (dskip) dskip[c] = s;
  } else if (ddt_bias) {
    ddt_bias[c - p.D] = s;
  }
}

// ---------------------------------------------------------------- one step
// A lane holds four states of a (sequence, channel); the state [B][D][N] is read and written once, 16 bytes a lane where
// N is a multiple of four and the rows are aligned (FOUR).  64 x 2048 channels of 16 states take 7.8 us, 17 MB at 2.2 TB/s:
// waiting, one access after another - the eight values of B and C are loaded each for itself where they exist, skip and z behind
// the store of the state, some ten rounds in all.  Where there is little it is the launch (128 channels 2.7 us).
template <typename T, int L, bool FOUR> __global__ __launch_bounds__(256) void scan_step_kernel(const ScanP p) {
  constexpr int NS = 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)p.B * p.D * L) return;                 // (the L lanes of a channel leave together)
  const int part = (int)(id % L);
  const int64_t seq = id / L;
  const int b = (int)(seq / p.D), d = (int)(seq % p.D), gr = d / (p.D / p.G);
  const bool some = part * NS < p.N;
  const T *bv = (const T *)p.bv.p + b * p.bv.sb + (int64_t)gr * p.N, *cv = (const T *)p.cv.p + b * p.cv.sb + (int64_t)gr * p.N;
  float A[NS], h[NS], bq[NS], cq[NS];
  float *state = p.state + seq * p.N;
  if constexpr (FOUR) {                                     // (N is 4, 8, .. : lanes beyond it read the last four)
    const int at = min(part * NS, p.N - NS);
    const States<NS> av = pick<NS>(p.A + (int64_t)d * p.N + at), hv = pick<NS>(state + at);
#pragma unroll
    for (int j = 0; j < NS; ++j) { A[j] = some ? av.v[j] : 0.f; h[j] = some ? hv.v[j] : 0.f; }
  } else {
    load_states<NS>(A, p.A + (int64_t)d * p.N, part, p.N, true);
    load_states<NS>(h, state, part, p.N, true);
  }
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int n = part * NS + j;
    bq[j] = n < p.N ? widen(bv[n]) : 0.f;
    cq[j] = n < p.N ? widen(cv[n]) : 0.f;
  }
  const float x = widen(((const T *)p.x.p)[b * p.x.sb + d]);
  const float raw = widen(((const T *)p.dt.p)[b * p.dt.sb + d]) + (p.dt_bias ? p.dt_bias[d] : 0.f);
  const float delta = p.softplus ? softplus(raw) : raw, u = delta * x;
  float v = 0.f;
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    h[j] = fmaf(__builtin_amdgcn_exp2f(delta * decay_rate(A[j])), h[j], u * bq[j]);
    v = fmaf(cq[j], h[j], v);
  }
  v = sum_neighbours<L>(v);
  if constexpr (FOUR) {
    if (some) put_states<NS>(state + part * NS, h);
  } else {
    store_states<NS>(state, h, part, p.N);
  }
  if (part == 0) {
    if (p.skip) v = fmaf(p.skip[d], x, v);
    if (p.z.p) { const float z = widen(((const T *)p.z.p)[b * p.z.sb + d]); v *= z * sigmoid_fast(z); }
    ((T *)p.y.p)[b * p.y.sb + d] = narrow<T>(v);
  }
}

// ---------------------------------------------------------------- host side
// How a call's states lie in lanes: NS of a channel in each of L lanes, NP = NS L of them with those that are zero, and
// wavefronts of a workgroup (64 channels to a workgroup where that is eight wavefronts or less).
struct Shape {
  int NS, L, waves;
  int channels() const { return 64 / L * waves; }
};
template <int NS_, int L_, int W_> struct FixedShape {
  static constexpr int NS = NS_, L = L_, W = W_, NP = NS_ * L_;
};
int padded(int N) { return N <= 8 ? 8 : N <= 16 ? 16 : N <= 32 ? 32 : 64; }
// Wavefronts of a call with four states a lane, time uncut.
int64_t waves_of_four(const snn_scan_args &a) {
  const int64_t dg = a.D / a.groups, per = 256 / padded(a.N);
  return (int64_t)a.B * a.groups * ((dg + per - 1) / per);
}
// Workgroups per (chunk, sequence, group).
int blocks_of(const snn_scan_args &a, const Shape &k) {
  const int dg = a.D / a.groups;
  return (dg + k.channels() - 1) / k.channels();
}

// Four states a lane.  Two, with twice the wavefronts and more to do around each state, where a forward pass of nine to
// sixteen states has more than 768 wavefronts of four and its workgroups of eight wavefronts of two are at most one for each
// of the 256 CUs: one more, and a CU that has two takes twice as long.  1024 steps of B x 2048 channels of 16 states, us with
// two and with four (cut in chunks of time below 1024 wavefronts): 768 wavefronts of four 98 and 94, 896 100 and 115, 1024 101
// and 117, 1152 184 and 160, 1536 197 and 163; at 4096 wavefronts 93 and 79.  32 states, 1024 wavefronts: 112 and 109.
// (Up to eight states: always two in each of four lanes.)
Shape shape_of(const snn_scan_args &a, bool backward) {
  const int np = padded(a.N);
  if (np == 8) return {2, 4, 4};
  const Shape two = {2, np / 2, 8};
  if (!backward && np == 16 && waves_of_four(a) > 768 && (int64_t)a.B * a.groups * blocks_of(a, two) <= 256) return two;
  return {4, np / 4, 4};
}

int scan_sizes(const snn_scan_args *a) {
  if (!a) return ops_fail(SNN_ERR_NULL, "scan: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0) return ops_fail(SNN_ERR_ARG, "scan: T >= 0, B > 0 and D > 0 are required");
  if (a->N < 1 || a->N > SNN_SCAN_MAX_STATES) return ops_fail(SNN_ERR_ARG, "scan: N must be 1 to %d", SNN_SCAN_MAX_STATES);
  if (a->groups < 1 || a->D % a->groups) return ops_fail(SNN_ERR_ARG, "scan: groups must divide D");
  if (a->D > (1 << 22)) return ops_fail(SNN_ERR_ARG, "scan: D must not exceed 2^22");
  if ((int64_t)a->B * a->D >= (1ll << 31) / 64) return ops_fail(SNN_ERR_ARG, "scan: B * D must stay below 2^25");
  if (a->T > (1 << 30)) return ops_fail(SNN_ERR_ARG, "scan: T must not exceed 2^30");
  if ((int64_t)a->B * a->groups >= (1 << 18)) return ops_fail(SNN_ERR_ARG, "scan: B * groups must stay below 2^18");
  if ((int64_t)a->T * a->B * a->groups >= (1ll << 32)) return ops_fail(SNN_ERR_ARG, "scan: T * B * groups must stay below 2^32");
  return SNN_OK;
}

int scan_check(const snn_scan_args *a, bool step, bool grads) {
  int rc = scan_sizes(a);
  if (rc) return rc;
  if (a->type != SNN_TYPE_FP32 && a->type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "scan: unknown type %d", a->type);
  if (!a->A) return ops_fail(SNN_ERR_NULL, "scan: A is NULL");
  if (a->T > 0 && (!a->x.p || !a->dt.p || !a->bv.p || !a->cv.p || (!grads && !a->y.p)))
    return ops_fail(SNN_ERR_NULL, "scan: x, dt, bv, cv or y is NULL");
  if (step) {
    if (a->T != 1) return ops_fail(SNN_ERR_ARG, "scan step: T must be 1");
    if (a->init || a->lengths) return ops_fail(SNN_ERR_ARG, "scan step: init and lengths must be NULL");
    if (!a->state) return ops_fail(SNN_ERR_NULL, "scan step: state is NULL");
  }
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  for (const void *q : {a->x.p, a->dt.p, a->z.p, a->bv.p, a->cv.p, a->y.p})
    if (!aligned(q, z)) return ops_fail(SNN_ERR_ARG, "scan: a pointer is not aligned to its element type");
  for (const void *q : {(const void *)a->A, (const void *)a->skip, (const void *)a->dt_bias, (const void *)a->init, (const void *)a->lengths, (const void *)a->state})
    if (!aligned(q, 4)) return ops_fail(SNN_ERR_ARG, "scan: a pointer is not aligned to its element type");
  return SNN_OK;
}

// Strides of the streamed tensors: a lane's offset within a tile (15 steps and its channel) stays below SPAN.
int scan_strides(const snn_scan_args *a, const snn_rows *rows, int count) {
  const int64_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  for (int i = 0; i < count; ++i) {
    if (!rows[i].p || a->T <= 1) continue;
    if (rows[i].stride_t < 0 || rows[i].stride_t > (1 << 28) || (15 * rows[i].stride_t + a->D + a->groups * (int64_t)a->N) * z >= SPAN)
      return ops_fail(SNN_ERR_ARG, "scan: a stride between steps is negative or too large: 15 steps have to stay below 2 GiB");
  }
  return SNN_OK;
}

// How time is cut: into chunks of at least 48 steps for 4096 wavefronts, four to a SIMD, where there are few; not at
// all below 128 steps, or where there are 1024 wavefronts (forward, which does a chunk twice but for the outputs) or 1536
// (reverse, which does half of the work twice).  16 states, one cut for 4096 wavefronts against none, us: forward, 512 wavefronts (1024 steps of
// 4 x 2048 channels) 70 and 100; 1024 wavefronts 119 and 116; forward and reverse, 512 wavefronts 240 and 324, 1024
// wavefronts 417 and 445, 1536 wavefronts 331 and 332.  Cut for 2048 wavefronts, the case of 512 takes 75 and 253.  Chunks of at
// least 32, 48 and 64 steps, forward and reverse: 500 steps of 2 x 512 channels 69, 65 and 73; 200 steps of 4 x 1024 67,
// 66 and 74; 100 steps of 8 x 512 67, 64 and 61, the last of which is not cut.
void scan_cut(const snn_scan_args &a, const Shape &k, bool backward, int *chunk, int *nchunks) {
  const int64_t waves = (int64_t)a.B * a.groups * blocks_of(a, k) * k.waves, enough = backward ? 1536 : 1024;
  int64_t n = waves < enough ? 4096 / waves : 1;
  if (n > a.T / 48) n = a.T / 48;
  if (n < 1 || a.T < 128) n = 1;
  const int64_t tiles = ((int64_t)a.T + TILE - 1) / TILE;
  const int64_t each = tiles ? (tiles + n - 1) / n : 1;
  *chunk = (int)(each * TILE);
  *nchunks = (int)(tiles ? (tiles + each - 1) / each : 1);
}

// The pieces of a workspace: chunk states, sums of delta, and for the reverse pass the partial sums.
struct ScanSpace {
  size_t local, sums, dA, dsum, dbc, all;
};
ScanSpace scan_space(const snn_scan_args &a, bool backward) {
  const Shape k = shape_of(a, backward);
  int chunk, n;
  scan_cut(a, k, backward, &chunk, &n);
  const size_t seqs = (size_t)a.B * a.D, np = padded(a.N);
  ScanSpace s;
  s.local = 0;
  s.sums = s.local + (n > 1 ? rup256(n * seqs * np * 4) : 0);
  s.dA = s.sums + (n > 1 ? rup256(n * seqs * 4) : 0);
  s.dsum = s.dA + (backward ? rup256(n * seqs * np * 4) : 0);
  s.dbc = s.dsum + (backward ? rup256(n * seqs * 8) : 0);
  s.all = s.dbc + (backward ? rup256((size_t)blocks_of(a, k) * a.T * a.B * a.groups * 2 * np * 4) : 0);
  return s;
}

// f(a value of the streamed type, a FixedShape)
template <bool BACKWARD, typename F> int with_kind(const snn_scan_args &a, const Shape &k, F f) {
  const auto shapes = [&](auto zero) {
    if (k.NS == 4) return k.L == 4 ? f(zero, FixedShape<4, 4, 4>()) : k.L == 8 ? f(zero, FixedShape<4, 8, 4>()) : f(zero, FixedShape<4, 16, 4>());
    if constexpr (!BACKWARD)
      if (k.L == 8) return f(zero, FixedShape<2, 8, 8>());
    return f(zero, FixedShape<2, 4, 4>());
  };
  return a.type == SNN_TYPE_FP32 ? shapes(0.f) : shapes((__bf16)0.f);
}

ScanP plan(const snn_scan_args &a, const Shape &k, bool backward, const void *saved, char *ws, const ScanSpace &s) {
  ScanP p(a);
  scan_cut(a, k, backward, &p.chunk, &p.nchunks);
  p.blocks = blocks_of(a, k);
  p.saved = (float *)const_cast<void *>(saved);
  if (p.nchunks > 1) { p.local = (float *)(ws + s.local); p.sums = (float *)(ws + s.sums); }
  return p;
}

template <typename T, typename K, bool GATE> int forward(const snn_scan_args &a, const Shape &k, void *saved, char *ws, hipStream_t st) {
  const ScanP p = plan(a, k, false, saved, ws, scan_space(a, false));
  const unsigned per = (unsigned)((size_t)p.blocks * p.G * p.B);
  int rc = SNN_OK;
  if (p.nchunks > 1) {
    hipLaunchKernelGGL((scan_forward_kernel<T, K::NS, K::L, K::W, false, true>), dim3(per * (p.nchunks - 1)), dim3(64 * K::W), 0, st, p);
    if ((rc = ops_launched("scan, chunks"))) return rc;
    hipLaunchKernelGGL((scan_join_kernel<K::NP, false>), dim3((unsigned)(((int64_t)p.B * p.D * K::NP + 255) / 256)), dim3(256), 0, st, p, a.init);
    if ((rc = ops_launched("scan, join"))) return rc;
  }
  hipLaunchKernelGGL((scan_forward_kernel<T, K::NS, K::L, K::W, GATE, false>), dim3(per * p.nchunks), dim3(64 * K::W), 0, st, p);
  return ops_launched("scan");
}

template <typename T, typename K, bool GATE>
int backward(const snn_scan_args &a, const Shape &k, const snn_scan_grads &gr, const void *saved, char *ws, hipStream_t st) {
  const ScanSpace s = scan_space(a, true);
  const ScanP p = plan(a, k, true, saved, ws, s);
  ScanGradP g(gr, a.T);
  g.dA = (float *)(ws + s.dA);
  g.dsum = (float *)(ws + s.dsum);
  g.dbc = (float *)(ws + s.dbc);
  const unsigned per = (unsigned)((size_t)p.blocks * p.G * p.B);
  int rc = SNN_OK;
  if (p.nchunks > 1) {
    hipLaunchKernelGGL((scan_reverse_local_kernel<T, K::NS, K::L, K::W, GATE>), dim3(per * (p.nchunks - 1)), dim3(64 * K::W), 0, st, p, g);
    if ((rc = ops_launched("scan reverse, chunks"))) return rc;
    hipLaunchKernelGGL((scan_join_kernel<K::NP, true>), dim3((unsigned)(((int64_t)p.B * p.D * K::NP + 255) / 256)), dim3(256), 0, st, p, gr.d_state);
    if ((rc = ops_launched("scan reverse, join"))) return rc;
  }
  hipLaunchKernelGGL((scan_reverse_kernel<T, K::NS, K::L, K::W, GATE>), dim3(per * p.nchunks), dim3(64 * K::W), 0, st, p, g);
  if ((rc = ops_launched("scan reverse"))) return rc;
  const int64_t values = (int64_t)a.T * a.B * a.groups * 2 * K::NP;
  if (values) {
    hipLaunchKernelGGL((scan_sum_rows_kernel<T, K::NP>), dim3((unsigned)std::min<int64_t>((values + 255) / 256, 1 << 16)), dim3(256), 0, st, p, g.dbc, Rows<void>(gr.dbv, a.T), Rows<void>(gr.dcv, a.T));
    if ((rc = ops_launched("scan reverse, rows"))) return rc;
  }
  const int64_t groups = ((int64_t)a.D * K::NP + 15) / 16 + (2 * (int64_t)a.D + 15) / 16;
  hipLaunchKernelGGL((scan_sum_params_kernel<K::NP>), dim3((unsigned)groups), dim3(256), 0, st, p, g.dA, g.dsum, gr.dA, gr.dskip, gr.ddt_bias);
  return ops_launched("scan reverse, parameters");
}

template <typename T, int L> int step(const snn_scan_args &a, hipStream_t st) {
  const ScanP p(a);
  const dim3 grid((unsigned)(((int64_t)a.B * a.D * L + 255) / 256));
  if (a.N % 4 == 0 && aligned(a.A, 16) && aligned(a.state, 16)) hipLaunchKernelGGL((scan_step_kernel<T, L, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((scan_step_kernel<T, L, false>), grid, dim3(256), 0, st, p);
  return ops_launched("scan step");
}
template <typename T> int step_of(const snn_scan_args &a, hipStream_t st) {
  return a.N <= 4 ? step<T, 1>(a, st) : a.N <= 8 ? step<T, 2>(a, st) : a.N <= 16 ? step<T, 4>(a, st) : a.N <= 32 ? step<T, 8>(a, st) : step<T, 16>(a, st);
}

int check_workspace(size_t need, const void *ws, size_t have) {
  if (need && (!ws || !aligned(ws, 16) || have < need))
    return ops_fail(SNN_ERR_WORKSPACE, "scan: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, ws ? have : (size_t)0);
  return SNN_OK;
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" {

int32_t snn_scan_workspace_bytes(const snn_scan_args *a, int32_t backward, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  int rc = scan_sizes(a);
  if (rc) return rc;
  *bytes = scan_space(*a, backward != 0).all;
  return SNN_OK;
}

int32_t snn_scan_saved_bytes(const snn_scan_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  int rc = scan_sizes(a);
  if (rc) return rc;
  *bytes = ((size_t)a->T + TILE - 1) / TILE * a->B * a->D * padded(a->N) * 4;
  return SNN_OK;
}

int32_t snn_scan_forward(const snn_scan_args *a, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = scan_check(a, false, false);
  if (rc) return rc;
  const snn_rows rows[] = {a->x, a->dt, a->z, a->bv, a->cv, a->y};
  if ((rc = scan_strides(a, rows, 6))) return rc;
  if (!aligned(saved, 16)) return ops_fail(SNN_ERR_ARG, "scan: saved must be 16-byte aligned");
  if ((rc = check_workspace(scan_space(*a, false).all, workspace, workspace_bytes))) return rc;
  const Shape k = shape_of(*a, false);
  return with_kind<false>(*a, k, [&](auto zero, auto fixed) {
    using T = decltype(zero);
    using K = decltype(fixed);
    return a->z.p ? forward<T, K, true>(*a, k, saved, (char *)workspace, (hipStream_t)stream)
                  : forward<T, K, false>(*a, k, saved, (char *)workspace, (hipStream_t)stream);
  });
}

int32_t snn_scan_backward(const snn_scan_args *a, const snn_scan_grads *g, const void *saved, void *workspace,
                          size_t workspace_bytes, void *stream) {
  int rc = scan_check(a, false, true);
  if (rc) return rc;
  if (!g || !g->dA || (a->T > 0 && (!saved || !g->dy.p || !g->dx.p || !g->ddt.p || !g->dbv.p || !g->dcv.p || (a->z.p && !g->dz.p))))
    return ops_fail(SNN_ERR_NULL, "scan backward: saved, dy, dx, ddt, dz, dbv, dcv or dA is NULL");
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  for (const void *q : {g->dy.p, g->dx.p, g->ddt.p, g->dz.p, g->dbv.p, g->dcv.p})
    if (!aligned(q, z)) return ops_fail(SNN_ERR_ARG, "scan backward: a pointer is not aligned to its element type");
  for (const void *q : {(const void *)g->d_state, (const void *)g->dA, (const void *)g->dskip, (const void *)g->ddt_bias, (const void *)g->dinit})
    if (!aligned(q, 4)) return ops_fail(SNN_ERR_ARG, "scan backward: a pointer is not aligned to its element type");
  const snn_rows rows[] = {a->x, a->dt, a->z, a->bv, a->cv, g->dy, g->dx, g->ddt, g->dz};
  if ((rc = scan_strides(a, rows, 9))) return rc;
  if (!aligned(saved, 16)) return ops_fail(SNN_ERR_ARG, "scan backward: saved must be 16-byte aligned");
  if ((rc = check_workspace(scan_space(*a, true).all, workspace, workspace_bytes))) return rc;
  const Shape k = shape_of(*a, true);
  return with_kind<true>(*a, k, [&](auto zero, auto fixed) {
    using T = decltype(zero);
    using K = decltype(fixed);
    return a->z.p ? backward<T, K, true>(*a, k, *g, saved, (char *)workspace, (hipStream_t)stream)
                  : backward<T, K, false>(*a, k, *g, saved, (char *)workspace, (hipStream_t)stream);
  });
}

int32_t snn_scan_step(const snn_scan_args *a, void *stream) {
  int rc = scan_check(a, true, false);
  if (rc) return rc;
  return a->type == SNN_TYPE_FP32 ? step_of<float>(*a, (hipStream_t)stream) : step_of<__bf16>(*a, (hipStream_t)stream);
}

}  // extern "C"
