// Gated units (include/snn_ops.h): y = act(G) U, G = x gate^T, U = x up^T.  Reverse: dG = dy U act'(G), dU = dy act(G);
//   dx = dG gate + dU up;  dgate = dG^T x, dup = dU^T x.
//
// Every product here is C[m][n] = sum_k A(m,k) B(n,k) with k fastest on both sides, by one kernel on the matrix units: tiles of both
// sides travel from memory straight into LDS, 64 k a stage, and the wavefronts multiply 32 x 32 blocks out of it.  The forward
// product takes gate and up rows in turns of 32, so that a wavefront holds both of a unit's sums and forms act(G) U itself.
// Operands that do not lie that way (reverse: both sides of the weights' gradients, the weights of dx; any whose rows are not
// multiples of 64 elements; fp32) are laid out first, as panels [k / 64][row][64]: a stage of a tile is one piece of memory.
//
// Measured: 4096 rows, 2048 -> 8192, bf16, 235 to 250 us (1100 to 1170 TFLOP/s; a library's plain product of that size 1435); both reverse
// products of 8192 rows, 2048 -> 4096 440 (1250).  What bounds it: loads into LDS alone take 118 of the first, products alone 124, a tile's
// outputs 25, and one barrier a stage does not let them overlap wholly.
//
// fp32 enters as three bfloat16 pieces, x = hi + mid + lo exactly (8 bits each).  Six of the nine products of pieces are summed, the
// small ones first; those left out are 2^-25 of the product.  That costs 6 of the 16 times that bfloat16 is faster.
#include "gemm_stream.hpp"
#include "block_rules.hpp"
#include "rows.hpp"

#include <algorithm>
#include <type_traits>

namespace snn {
namespace {

constexpr int WIDE_WM = 2, WIDE_WN = 4;      // wavefronts of a wide tile

// One side of a product: stage `kp` of plane `plane`, row r at p + r row + kp stage + plane plane (bytes).
struct Side {
  const char *p, *p2;                        // p2: up, where rows of two matrices take turns
  int64_t row, stage, plane;
  int rows;
};
// Rows in memory: what (t, b) a row m = t B + b is, and whether it exists.
struct Steps {
  int T, B;
  const int32_t *lengths;
  __device__ __forceinline__ bool live(int m, int &t, int &b) const {
    t = (int)((unsigned)m / (unsigned)B);
    b = m - t * B;
    return !lengths || t < lengths[b];
  }
};
struct GemmP {
  Side a, b;
  int panels, segs;                          // stages of a plane; products of planes
  int mt, nt, splits;                        // tiles, parts of the contraction
  // what becomes of it
  Steps steps;
  Rows<void> out = Rows<void>(snn_rows{});   // y or dx
  void *w0, *w1;                             // dgate, dup
  float *part;                               // [splits][rows of a][pitch]: sums of a part; UNITS: G and U (of a part), or NULL
  int what, pitch, act;
  int64_t part_size;                         // UNITS: of a part's G and U
  int M, N;                                  // rows of a; columns (units)
};
enum { UNITS, GRADS };                       // what a product is; of GRADS each job is one of
enum { DX, DW };
struct Jobs {                                // products of one launch: the workgroups before `first` are the first one's
  GemmP job[2];
  int first;
};

// Which pieces meet in product `seg` of six, the smallest first: mid mid, hi lo, lo hi, hi mid, mid hi, hi hi (hi = 0).
__device__ __forceinline__ int segment_a(int seg, int segs) { return segs == 1 ? 0 : (0x102010 >> (20 - 4 * seg)) & 0xF; }
__device__ __forceinline__ int segment_b(int seg, int segs) { return segs == 1 ? 0 : (0x120100 >> (20 - 4 * seg)) & 0xF; }

// act(g) and its slope.  The normal distribution's function as erfc(-g / sqrt(2)) / 2, which keeps its last places where it is small:
// 1 + erf(g / sqrt(2)) is a multiple of 2^-24, 5 % off at g = -5 and zero below -5.6.  (It costs 4 to 6 us more: 4096 rows, 2048 -> 8192, bf16,
// 261 and 267 us, reverse 621 and 625; 8192 rows, 512 -> 2048, 54 and 58, 142 and 146.)
__device__ __forceinline__ float normal_below(float g) { return 0.5f * erfcf(g * -0.70710678118654752f); }
__device__ __forceinline__ float act_of(int act, float g) { return act == SNN_ACT_SILU ? g * sigmoid_fast(g) : g * normal_below(g); }
__device__ __forceinline__ float act_slope(int act, float g) {
  if (act == SNN_ACT_SILU) {
    const float s = sigmoid_fast(g);
    return s * fmaf(g, 1.f - s, 1.f);
  }
  return normal_below(g) + g * 0.3989422804014327f * exp_fast(-0.5f * g * g);
}

// G and U of 32 rows by 32 units as the accumulators hold them, which is how they are kept for the reverse pass: [G, U][g][lane][4],
// row lane % 32, unit 8 g + 4 (lane / 32) + 0..3.  (Every store of a wavefront is one KiB; row by row it would be 32 pieces of 32
// bytes, and the forward pass with them took 180 us longer where memory needs 50: 8192 rows, 4096 units.)
__host__ __device__ inline int64_t kept_block(int mb, int fb, int F) { return ((int64_t)mb * ((F + 31) / 32) + fb) * KEPT; }

// Four neighbouring values of a row from column n on.
template <typename T> __device__ __forceinline__ void give4(T *row, int n, int N, bool wide, const float (&v)[4]) {
  if (wide && n + 4 <= N) {
    Pack<T, 4> q;
#pragma unroll
    for (int k = 0; k < 4; ++k) q.v[k] = narrow<T>(v[k]);
    *(Pack<T, 4> *)(row + n) = q;
  } else
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) row[n + k] = narrow<T>(v[k]);
}

// WM x WN wavefronts, each TM x TN blocks of 32 x 32 (m x n).  T: the type of what comes out.
template <typename T, int WHAT, int WM, int WN, int TM, int TN, int SK, int NS>
__global__ __launch_bounds__(WM * WN * 64) void gemm_kernel(const Jobs jobs) {
  // SK: k of a stage; a row of it is RB bytes, RC chunks of 16, and a load of a wavefront brings RPL rows.  NS: stages in LDS
  constexpr int RB = 2 * SK, RC = RB / 16, RPL = 64 / RC, QS = SK / 16, PER = KS / SK;
  constexpr int NW = WM * WN, BM = WM * TM * 32, BN = WN * TN * 32, AI = BM / RPL / NW, BI = BN / RPL / NW;
  constexpr int STAGE = (BM + BN) * RB;
  // chunk c of row r lies at place c ^ turn(r): 16 rows that are read together touch every bank once
  auto turn = [](int r) { return SK == 64 ? (r >> 1) & 7 : (r >> 2) & 3; };
  static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0 && (WHAT != UNITS || TN % 2 == 0), "whole loads; gate and up in one wavefront");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const bool later = WHAT == GRADS && (int)blockIdx.x >= jobs.first;
  const GemmP &a = jobs.job[later];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // Tiles: neighbours in time share an XCD's L2, so every XCD (workgroups go around them in turn) takes a run of tiles, and runs
  // walk eight rows of tiles before the next column.
  int id = (int)blockIdx.x - (later ? jobs.first : 0);
  const int all = a.mt * a.nt, split = id / all;
  id -= split * all;
  {
    const int each = all / 8, more = all % 8, x = id % 8;
    id = (x < more ? x * (each + 1) : more * (each + 1) + (x - more) * each) + id / 8;
  }
  const int band = id / (8 * a.nt), in = id - band * 8 * a.nt, high = min(8, a.mt - band * 8);
  const int tm = band * 8 + in % high, tn = in / high;
  const int m0 = tm * BM, n0 = tn * (WHAT == UNITS ? BN / 2 : BN);

  // what a lane loads: 16 bytes of row lane / RC of a load's rows, the chunk that belongs at this place of the LDS
  int av[AI], bv[BI];
#pragma unroll
  for (int q = 0; q < AI; ++q) {
    const int r = RPL * (wave + NW * q) + lane / RC, c = (lane % RC) ^ turn(r);
    av[q] = m0 + r < a.a.rows ? (int)(r * a.a.row) + c * 16 : ROW_NOWHERE;
  }
#pragma unroll
  for (int q = 0; q < BI; ++q) {
    const int r = RPL * (wave + NW * q) + lane / RC, c = (lane % RC) ^ turn(r);
    const int rr = WHAT == UNITS ? (r >> 6) * 32 + (r & 31) : r;
    bv[q] = n0 + rr < a.b.rows ? (int)(rr * a.b.row) + c * 16 : ROW_NOWHERE;
  }
  const int panels = a.panels * PER, stages = panels * a.segs, first = (int)((int64_t)stages * split / a.splits), last = (int)((int64_t)stages * (split + 1) / a.splits);
  const char *const pa = a.a.p + (int64_t)m0 * a.a.row, *const pb = a.b.p + (int64_t)n0 * a.b.row,
             *const pu = WHAT == UNITS ? a.b.p2 + (int64_t)n0 * a.b.row : nullptr;
  const unsigned lds0 = (unsigned)(uintptr_t)(lds_ptr_t)lds;
  int seg = first / panels, kp = first - seg * panels, asked_to = first;
  struct Asked {                             // scalar operands of a stage's loads
    u32x4 a, b, up;
    unsigned dst;
  } asked;
  auto prepare = [&](int buf) {              // (behind the last stage: buffers of no size, so that the number of loads stays the same)
    const int64_t at = kp / PER, in_row = (kp % PER) * RB;
    const int64_t at_a = segment_a(seg, a.segs) * a.a.plane + at * a.a.stage + in_row, at_b = segment_b(seg, a.segs) * a.b.plane + at * a.b.stage + in_row;
    const unsigned size = asked_to < last ? ROW_SPAN : 0;
    asked.a = raw_rsrc(pa + at_a, size);
    asked.b = raw_rsrc(pb + at_b, size);
    asked.up = WHAT == UNITS ? raw_rsrc(pu + at_b, size) : asked.b;
    asked.dst = __builtin_amdgcn_readfirstlane(lds0 + buf * STAGE + wave * 1024);
    ++asked_to;
    if (++kp == panels) {
      kp = 0;
      ++seg;
    }
  };
  auto load = [&](int q) {                   // load q of AI + BI
    if (q < AI) load_to_lds_b128(asked.a, asked.dst + q * NW * 1024, av[q < AI ? q : 0], 0);
    else {
      const int p = q - AI;
      const bool up = WHAT == UNITS && ((RPL * (wave + NW * p)) & 32);
      load_to_lds_b128(up ? asked.up : asked.b, asked.dst + BM * RB + p * NW * 1024, bv[p], 0);
    }
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const int h = lane >> 5, ra = wm * TM * 32 + (lane & 31), rb = wn * TN * 32 + (lane & 31);
  int fa[QS], fb[QS];
#pragma unroll
  for (int s = 0; s < QS; ++s) {
    fa[s] = ra * RB + (((2 * s + h) ^ turn(ra)) << 4);
    fb[s] = BM * RB + rb * RB + (((2 * s + h) ^ turn(rb)) << 4);
  }
  // Stage by stage, a step (16 k) at a time.  The last step is multiplied behind the next stage's barrier, out of registers, so that
  // the matrix units have work while that stage's first fragments arrive; every other step's fragments are read under the
  // step before, and the loads of a later stage go out from the first step on.  An MFMA keeps the matrix unit for 32 cycles, in which
  // a wavefront can issue about one of these: the order is fixed by hand, one behind each MFMA.
  constexpr int Q = TM * TN, LOADS = AI + BI, EVERY = QS * Q / 2 / LOADS < 1 ? 1 : QS * Q / 2 / LOADS;
  static_assert(LOADS <= QS * Q && TM + TN <= Q, "a place for every load and read");
  bf16x8 xa[2][TM], xb[2][TN];
  auto read = [&](const char *st, int s, int f) {            // fragment f of step s
    if (f < TN) xb[s & 1][f < TN ? f : 0] = *(const bf16x8 *)(st + fb[s] + f * 32 * RB);
    else xa[s & 1][f - TN < TM ? f - TN : 0] = *(const bf16x8 *)(st + fa[s] + (f - TN) * 32 * RB);
  };
  const bf16x8 none = {};
#pragma unroll
  for (int i = 0; i < TM; ++i) xa[1][i] = none;
#pragma unroll
  for (int j = 0; j < TN; ++j) xb[1][j] = none;
#pragma unroll
  for (int n = 0; n < NS - 1; ++n) {
    prepare(n);
#pragma unroll
    for (int q = 0; q < LOADS; ++q) load(q);
  }
  for (int kt = first, buf = 0; kt < last; ++kt) {
    // this wavefront's loads of the stage have landed, and behind the barrier everyone's; everyone has left the stage before
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * LOADS) : "memory");
    lds_barrier();
    const char *st = lds + buf * STAGE;
    prepare(buf ? buf - 1 : NS - 1);
    buf = buf + 1 < NS ? buf + 1 : 0;
    __builtin_amdgcn_s_setprio(1);                           // (3 % of the forward product: the wavefront ahead stays ahead)
    static_for<QS * Q>([&](auto X) {
      constexpr int x = decltype(X)::value, g = x / Q, y = x % Q, s = (g + QS - 1) % QS, i = y / TN, j = y % TN;
      __builtin_amdgcn_sched_barrier(0);
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[s & 1][j], xa[s & 1][i], acc[i][j], 0, 0, 0);
      if constexpr (2 * y < TM + TN) read(st, g, 2 * y);
      if constexpr (2 * y + 1 < TM + TN) read(st, g, 2 * y + 1);
      if constexpr (x % EVERY == EVERY - 1 && x / EVERY < LOADS) load(x / EVERY);
    });
    __builtin_amdgcn_s_setprio(0);
  }
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (no load outlives the workgroup's LDS)
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[1][j], xa[1][i], acc[i][j], 0, 0, 0);

  // A lane holds, of block (i, j), row m = lane % 32 and columns 8 g + 4 h + 0..3 in element 4 g + 0..3.
  if (WHAT == UNITS && a.part)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN / 2; ++j) {
        const int mb = m0 / 32 + wm * TM + i, fb = n0 / 32 + wn * TN / 2 + j;
        if (mb * 32 >= a.M || fb * 32 >= a.N) continue;
        float *const at = a.part + split * a.part_size + kept_block(mb, fb, a.N) + lane * 4;
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const f32x16 &v = acc[i][2 * j + w];
            *(Pack<float, 4> *)(at + (w * 4 + g) * 256) = {{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]}};
          }
      }
  if constexpr (WHAT == UNITS) {
    if (a.splits > 1) return;                                // (units_sum_kernel goes on)
    constexpr int U = BN / 2, PITCH = U * (int)sizeof(T) + 16;
    if constexpr (sizeof(T) == 2) {
      // Through LDS, so that a row's outputs leave together.  (From the accumulators, which have four units of 32 rows, 4096 rows, 2048 -> 8192
      // took 258 us against 246.  fp32 rows leave in 16-byte pieces as it is, and wide tiles of them do not fit.)
      static_assert(BM * PITCH <= NS * STAGE, "the tile's outputs fit");
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN / 2; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            Pack<T, 4> y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y.v[k] = narrow<T>(act_of(a.act, acc[i][2 * j][4 * g + k]) * acc[i][2 * j + 1][4 * g + k]);
            *(Pack<T, 4> *)(lds + ((wm * TM + i) * 32 + (lane & 31)) * PITCH + ((wn * TN / 2 + j) * 32 + 8 * g + 4 * h) * (int)sizeof(T)) = y;
          }
      __syncthreads();
      const uintptr_t all = (uintptr_t)a.out.p | (uintptr_t)(a.out.st * (int64_t)sizeof(T)) | (uintptr_t)(a.out.sb * (int64_t)sizeof(T)) | (uintptr_t)((int64_t)a.N * sizeof(T));
      auto pieces = [&](auto piece) {                        // rows in pieces of this type
        typedef decltype(piece) Piece;
        constexpr int E = (int)(sizeof(Piece) / sizeof(T));
        for (int q = threadIdx.x; q < BM * (U / E); q += NW * 64) {
          const int r = q / (U / E), c = q % (U / E) * E, m = m0 + r;
          if (m >= a.M || n0 + c >= a.N) continue;
          int t, b;
          const bool live = a.steps.live(m, t, b);
          const Piece v = *(const Piece *)(lds + r * PITCH + c * (int)sizeof(T));
          *(Piece *)((T *)a.out.p + t * a.out.st + b * a.out.sb + n0 + c) = live ? v : Piece{};
        }
      };
      if (all % 16 == 0) pieces(u32x4{});
      else if (all % 8 == 0) pieces(u32x2{});
      else pieces((unsigned short)0);
    } else {
      const bool wide = ((uintptr_t)a.out.p | (uintptr_t)(a.out.st * (int64_t)sizeof(T)) | (uintptr_t)(a.out.sb * (int64_t)sizeof(T))) % (4 * sizeof(T)) == 0;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = m0 + (wm * TM + i) * 32 + (lane & 31);
        if (m >= a.M) continue;
        int t, b;
        const bool live = a.steps.live(m, t, b);
        T *row = (T *)a.out.p + t * a.out.st + b * a.out.sb;
#pragma unroll
        for (int j = 0; j < TN / 2; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int n = n0 + (wn * TN / 2 + j) * 32 + 8 * g + 4 * h;
            if (n >= a.N) continue;
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = live ? act_of(a.act, acc[i][2 * j][4 * g + k]) * acc[i][2 * j + 1][4 * g + k] : 0.f;
            give4<T>(row, n, a.N, wide, y);
          }
      }
    }
  } else {
    const bool rows_out = a.what == DX, in_parts = a.splits > 1;
    const bool wide = rows_out ? ((uintptr_t)a.out.p | (uintptr_t)(a.out.st * (int64_t)sizeof(T)) | (uintptr_t)(a.out.sb * (int64_t)sizeof(T))) % (4 * sizeof(T)) == 0
                               : ((uintptr_t)a.w0 | (uintptr_t)a.w1 | (uintptr_t)((int64_t)a.N * sizeof(T))) % (4 * sizeof(T)) == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + (wm * TM + i) * 32 + (lane & 31);
      if (m >= a.M) continue;
      int t = 0, b = 0;
      const bool live = in_parts || !rows_out || a.steps.live(m, t, b);
      T *row = in_parts ? nullptr : rows_out ? (T *)a.out.p + t * a.out.st + b * a.out.sb : m < a.M / 2 ? (T *)a.w0 + (int64_t)m * a.N : (T *)a.w1 + (int64_t)(m - a.M / 2) * a.N;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int n = n0 + (wn * TN + j) * 32 + 8 * g + 4 * h;
          if (n >= a.N) continue;
          float v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = live ? acc[i][j][4 * g + k] : 0.f;
          if (in_parts) *(Pack<float, 4> *)(a.part + ((int64_t)split * a.M + m) * a.pitch + n) = {{v[0], v[1], v[2], v[3]}};
          else give4<T>(row, n, a.N, wide, v);
        }
    }
  }
}

// The parts' sums, rounded, to where a product without parts writes them.  A thread has four columns of a row; `first`: workgroups of
// the first job.
template <typename T> __global__ __launch_bounds__(256) void gemm_sum_kernel(const Jobs jobs) {
  const bool later = (int)blockIdx.x >= jobs.first;
  const GemmP &a = jobs.job[later];
  const int quads = a.pitch / 4;
  const int64_t id = ((int64_t)blockIdx.x - (later ? jobs.first : 0)) * 256 + threadIdx.x;
  const int64_t m = id / quads;
  const int n = (int)(id - m * quads) * 4;
  if (m >= a.M || n >= a.N) return;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    const Pack<float, 4> p = *(const Pack<float, 4> *)(a.part + ((int64_t)s * a.M + m) * a.pitch + n);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += p.v[k];
  }
  int t = 0, b = 0;
  if (a.what == DX && !a.steps.live((int)m, t, b)) v[0] = v[1] = v[2] = v[3] = 0.f;
  T *row = a.what == DX ? (T *)a.out.p + t * a.out.st + b * a.out.sb : m < a.M / 2 ? (T *)a.w0 + m * a.N : (T *)a.w1 + (m - a.M / 2) * a.N;
  give4<T>(row, n, a.N, ((uintptr_t)row & (4 * sizeof(T) - 1)) == 0, v);
}

// G and U out of parts, and what becomes of them.  A wavefront has 32 rows by 32 units as they are kept.
template <typename T> __global__ __launch_bounds__(256) void units_sum_kernel(const GemmP a, float *kept) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fbs = (a.N + 31) / 32;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int mb = (int)(id / fbs), fb = (int)(id - (int64_t)mb * fbs), m = mb * 32 + (lane & 31), n = fb * 32 + 4 * (lane >> 5);
  if (mb * 32 >= a.M) return;
  const int64_t at = kept_block(mb, fb, a.N) + lane * 4;
  int t = 0, b = 0;
  const bool live = m < a.M && a.steps.live(m, t, b);
  T *row = (T *)a.out.p + t * a.out.st + b * a.out.sb;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    Pack<float, 4> vg = *(const Pack<float, 4> *)(a.part + at + g * 256), vu = *(const Pack<float, 4> *)(a.part + at + (4 + g) * 256);
    for (int s = 1; s < a.splits; ++s) {
      const Pack<float, 4> pg = *(const Pack<float, 4> *)(a.part + s * a.part_size + at + g * 256), pu = *(const Pack<float, 4> *)(a.part + s * a.part_size + at + (4 + g) * 256);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        vg.v[k] += pg.v[k];
        vu.v[k] += pu.v[k];
      }
    }
    if (kept) {
      *(Pack<float, 4> *)(kept + at + g * 256) = vg;
      *(Pack<float, 4> *)(kept + at + (4 + g) * 256) = vu;
    }
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = live ? act_of(a.act, vg.v[k]) * vu.v[k] : 0.f;
    if (m < a.M && n + 8 * g < a.N) give4<T>(row, n + 8 * g, a.N, ((uintptr_t)row & (4 * sizeof(T) - 1)) == 0, y);
  }
}

// ---------------------------------------------------------------- few rows
// Up to 64 rows (a token of every stream): the matrices pass through once and bound it.  A workgroup has 16 units, gate and up, and
// each of its wavefronts every WAVES-th piece of 128 bytes of the rows; their sums meet in LDS.  A wavefront brings its pieces into
// LDS by itself, NB - 1 of them ahead (no barrier), and takes the operands of the matrix instructions from there: loaded straight
// into operand registers, where neighbouring lanes have different rows, every 16 lanes touch 16 cache lines, and a compute unit
// gets 16 bytes a cycle (64 rows, 2048 -> 4096, bf16: 14.4 us against 9.3).  fp32 stays fp32 here: the fp32 matrix instructions
// keep up, and the matrices need no pass before.
constexpr int FEW_UNITS = 16;

struct FewP {
  const void *gate, *up;
  Rows<void> x, y;
  Steps steps;
  float *kept;                               // as the tiles keep it, or NULL
  int M, D, F, act;
};
typedef __attribute__((ext_vector_type(4))) float f4;

// The sums of the wavefronts, [wavefront][gate, up][16 rows][unit][row], to outputs.
template <typename T, int MB, int WAVES> __device__ __forceinline__ void few_finish(const FewP &a, const f4 (&acc)[2][MB], float *lds, int f0, int m0) {
  constexpr int SET = 2 * MB * 16 * 17;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[wave * SET + ((w * MB + i) * 16 + 4 * (lane >> 4) + e) * 17 + (lane & 15)] = acc[w][i][e];
  __syncthreads();
  for (int o = threadIdx.x; o < MB * 256; o += WAVES * 64) {
    const int n = o & 15, in = o >> 4, m = m0 + in;
    if (m >= a.M || f0 + n >= a.F) continue;
    float vg = 0.f, vu = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      vg += lds[w * SET + ((in >> 4) * 16 + n) * 17 + (in & 15)];
      vu += lds[w * SET + ((MB + (in >> 4)) * 16 + n) * 17 + (in & 15)];
    }
    if (a.kept) {
      const int u = (f0 + n) & 31;
      float *const at = a.kept + kept_block(m >> 5, (f0 + n) >> 5, a.F) + (u >> 3) * 256 + ((m & 31) + (u & 4) * 8) * 4 + (u & 3);
      at[0] = vg;
      at[1024] = vu;
    }
    int t, b;
    const bool live = a.steps.live(m, t, b);
    ((T *)a.y.p)[t * a.y.st + b * a.y.sb + f0 + n] = narrow<T>(live ? act_of(a.act, vg) * vu : 0.f);
  }
}
// 16 units by 16 rows: 16 bytes of a row a lane, the four sets of 16 lanes one after another along k.
template <typename T> __device__ __forceinline__ void few_multiply(f4 &acc, const u32x4 &w, const u32x4 &x) {
  if constexpr (sizeof(T) == 2) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(x[e]), acc, 0, 0, 0);
}

// Rows in 16-byte pieces, those of x within 2^30 bytes of the first.
template <typename T, int MB, int WAVES, int NB> __global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(const FewP a) {
  constexpr int E = 16 / (int)sizeof(T), PIECE = 8 * E, ROWS = 32 + 16 * MB, LOADS = ROWS / 8, SIZE = ROWS * 128;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), f0 = blockIdx.x * FEW_UNITS,
            m0 = blockIdx.y * MB * 16;
  // rows of a piece: 16 of gate, 16 of up, those of x; chunk c of row r at place c ^ (r / 2 % 8), as in the tiles
  int at[LOADS];
#pragma unroll
  for (int q = 0; q < LOADS; ++q) {
    const int r = 8 * q + lane / 8, c = (lane & 7) ^ ((r >> 1) & 7);
    int64_t row = 0;
    bool there;
    if (q < 4) {
      there = f0 + (r & 15) < a.F;
      row = (int64_t)(r & 15) * a.D;
    } else {
      int t, b;
      there = m0 + r - 32 < a.M;
      a.steps.live(there ? m0 + r - 32 : 0, t, b);
      row = t * a.x.st + b * a.x.sb;
    }
    at[q] = there ? (int)(row * (int64_t)sizeof(T)) + c * 16 : ROW_NOWHERE;
  }
  const int chunk = ((lane & 7) ^ (lane / 16 & 7)) * E, chunk_odd = ((lane & 7) ^ ((lane / 16 + 4) & 7)) * E;   // (rows 8 q + lane / 8, q even and odd)
  const T *const gate = (const T *)a.gate + (int64_t)f0 * a.D, *const up = (const T *)a.up + (int64_t)f0 * a.D;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_ptr_t)lds + wave * NB * SIZE);
  auto ask = [&](int n, int k) {             // the piece from k on into buffer n; behind D nothing (zeros)
    const unsigned size = k < a.D ? ROW_SPAN : 0;
    const u32x4 rg = raw_rsrc(gate + k, size), ru = raw_rsrc(up + k, size), rx = raw_rsrc((const T *)a.x.p + k, size);
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const bool in = k + ((q & 1) ? chunk_odd : chunk) < a.D;
      load_to_lds_b128(q < 2 ? rg : q < 4 ? ru : rx, lds0 + n * SIZE + q * 1024, in ? at[q] : ROW_NOWHERE, 0);
    }
  };
  f4 acc[2][MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[0][i] = acc[1][i] = f4{0.f, 0.f, 0.f, 0.f};
  const char *const mine = lds + wave * NB * SIZE;
  const int r = lane & 15;
  int from[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) from[s] = r * 128 + (((4 * s + (lane >> 4)) ^ ((r >> 1) & 7)) << 4);
#pragma unroll
  for (int n = 0; n < NB - 1; ++n) ask(n, (wave + n * WAVES) * PIECE);
  int buf = 0;
  for (int k = wave * PIECE; k < a.D; k += WAVES * PIECE) {
    ask(buf ? buf - 1 : NB - 1, k + (NB - 1) * WAVES * PIECE);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 1) * LOADS) : "memory");     // the oldest piece is there
    const char *p = mine + buf * SIZE;
    buf = buf + 1 < NB ? buf + 1 : 0;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32x4 g = *(const u32x4 *)(p + from[s]), u = *(const u32x4 *)(p + 2048 + from[s]);
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const u32x4 x = *(const u32x4 *)(p + 4096 + i * 2048 + from[s]);
        few_multiply<T>(acc[0][i], g, x);
        few_multiply<T>(acc[1][i], u, x);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the buffer has been read before it is asked for again)
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  few_finish<T, MB, WAVES>(a, acc, (float *)lds, f0, m0);
}

// The same for rows that lie otherwise: element by element into the operand registers.
template <typename T, int MB> __global__ __launch_bounds__(256) void few_rows_any_kernel(const FewP a) {
  constexpr int WAVES = 4, E = 16 / (int)sizeof(T);
  __shared__ float lds[WAVES * 2 * MB * 16 * 17];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), f0 = blockIdx.x * FEW_UNITS,
            m0 = blockIdx.y * MB * 16;
  const int f = f0 + (lane & 15);
  const bool unit = f < a.F;
  const T *gate = (const T *)a.gate + (int64_t)(unit ? f : 0) * a.D, *up = (const T *)a.up + (int64_t)(unit ? f : 0) * a.D;
  const T *x[MB];
  bool row[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int m = m0 + i * 16 + (lane & 15);
    int t, b;
    row[i] = m < a.M;
    a.steps.live(row[i] ? m : 0, t, b);
    x[i] = (const T *)a.x.p + t * a.x.st + b * a.x.sb;
  }
  f4 acc[2][MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[0][i] = acc[1][i] = f4{0.f, 0.f, 0.f, 0.f};
  auto load = [&](const T *p, bool on, int k) {
    Pack<T, E> v;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool there = on && k + e < a.D;
      const T q = p[there ? k + e : 0];
      v.v[e] = there ? q : narrow<T>(0.f);
    }
    return __builtin_bit_cast(u32x4, v);
  };
  for (int k = wave * 4 * E; k < a.D; k += WAVES * 4 * E) {
    const int at = k + (lane >> 4) * E;
    const u32x4 g = load(gate, unit, at), u = load(up, unit, at);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const u32x4 v = load(x[i], row[i], at);
      few_multiply<T>(acc[0][i], g, v);
      few_multiply<T>(acc[1][i], u, v);
    }
  }
  few_finish<T, MB, WAVES>(a, acc, lds, f0, m0);
}

// ---------------------------------------------------------------- layouts
// Piece `plane` of a value that enters the products.
template <typename T> struct Pieces;
template <> struct Pieces<__bf16> {
  static constexpr int N = 1;
  static __device__ __forceinline__ void split(__bf16 x, __bf16 (&p)[1]) { p[0] = x; }
};
template <> struct Pieces<float> {
  static constexpr int N = 3;
  // hi + mid + lo = x; where x would round to infinity its upper half is cut off instead; infinities and NaN are hi alone
  static __device__ __forceinline__ void split(float x, __bf16 (&p)[3]) {
    float hi = (float)(__bf16)x;
    if (fabsf(x) < __builtin_huge_valf() && fabsf(hi) == __builtin_huge_valf()) hi = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    const float r = fabsf(x) < __builtin_huge_valf() ? x - hi : 0.f, mid = (float)(__bf16)r;
    p[0] = (__bf16)hi;
    p[1] = (__bf16)mid;
    p[2] = (__bf16)(r - mid);
  }
};
typedef Pack<__bf16, 8> Chunk;

struct LayP {
  const void *src;                           // rows of `cols` elements
  int64_t st, sb;                            // row m = t B + b at t st + b sb
  Steps steps;
  int rows, cols;
  char *dst;                                 // panels
  int64_t stage, plane;                      // bytes
  int wide;                                  // eight elements at a time
};
struct LayJobs {                             // x, gate, up: one launch
  LayP job[3];
};

// Eight elements of a row from column c on, zeros in the place of those that do not exist.
template <typename T> __device__ __forceinline__ Pack<T, 8> eight_of(const T *row, int c, int cols, bool live, bool wide) {
  Pack<T, 8> v = {};
  if (live && wide && c + 8 <= cols) v = *(const Pack<T, 8> *)(row + c);
  else if (live)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k < cols) v.v[k] = row[c + k];
  return v;
}

// Rows as they are: panel c / 64, row m, 64 columns.  A thread makes one chunk of every piece.
template <typename T> __global__ __launch_bounds__(256) void lay_rows_kernel(const LayJobs jobs) {
  const LayP &a = jobs.job[blockIdx.z];
  const int m = blockIdx.x * 32 + threadIdx.x / 8, c = blockIdx.y * KS + (threadIdx.x & 7) * 8;
  if (m >= a.rows || (int)blockIdx.y * KS >= a.cols) return;
  int t, b;
  const bool live = a.steps.live(m, t, b);
  const Pack<T, 8> v = eight_of((const T *)a.src + t * a.st + b * a.sb, c, a.cols, live, a.wide);
  constexpr int P = Pieces<T>::N;
  Chunk out[P];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    __bf16 p[P];
    Pieces<T>::split(v.v[k], p);
#pragma unroll
    for (int q = 0; q < P; ++q) out[q].v[k] = p[q];
  }
#pragma unroll
  for (int q = 0; q < P; ++q) *(Chunk *)(a.dst + q * a.plane + blockIdx.y * a.stage + (int64_t)m * 128 + (threadIdx.x & 7) * 16) = out[q];
}

// Columns as rows: panel m / 64, row c, 64 of the source's rows.
template <typename T> __device__ __forceinline__ void put_transposed(const T (&tile)[KS][KS + 1], char *dst, int64_t plane, int64_t first_row, int cols_left) {
  constexpr int P = Pieces<T>::N;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int c = (threadIdx.x + 256 * u) / 8, k0 = (threadIdx.x & 7) * 8;
    Chunk out[P];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      __bf16 p[P];
      Pieces<T>::split(tile[k0 + k][c], p);
#pragma unroll
      for (int q = 0; q < P; ++q) out[q].v[k] = p[q];
    }
    if (c < cols_left)
#pragma unroll
      for (int q = 0; q < P; ++q) *(Chunk *)(dst + q * plane + (first_row + c) * 128 + (threadIdx.x & 7) * 16) = out[q];
  }
}
template <typename T> __device__ __forceinline__ void lay_transposed(const LayP &a, T (&tile)[KS][KS + 1], int bx, int by) {
  const int m0 = bx * KS, c0 = by * KS;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = (threadIdx.x + 256 * u) / 8, c = (threadIdx.x & 7) * 8, m = m0 + r;
    int t = 0, b = 0;
    const bool live = m < a.rows && a.steps.live(m, t, b);
    const Pack<T, 8> v = eight_of((const T *)a.src + t * a.st + b * a.sb, c0 + c, a.cols, live, a.wide);
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[r][c + k] = v.v[k];
  }
  __syncthreads();
  put_transposed<T>(tile, a.dst + bx * a.stage, a.plane, c0, a.cols - c0);
}

// dG and dU from dy and the sums of the forward pass, both ways round: [f / 64][m][64] (dU behind dG along f) and [m / 64][f][64].
// They are rounded to the streamed type here, since both products take operands of that type: half a step a term, at random, so that the
// gradients are 2.3e-3 of their norm off in bfloat16 where rounding their sums alone is 1.7e-3.  In two pieces, which would spare
// that, both products (450 us of 8192 rows, 2048 -> 4096) would take twice as long.
struct SlopeP {
  Steps steps;
  Rows<void> dy;
  const float *kept;
  int act, M, F, panels, wide;               // panels: of F; wide: dy eight at a time
  char *rows, *cols;
  int64_t rows_stage, rows_plane, cols_stage, cols_plane;
};
template <typename T> __device__ __forceinline__ void slopes(const SlopeP &a, T (&tile)[2][KS][KS + 1], int bx, int by) {
  const int m0 = bx * KS, f0 = by * KS, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mb = m0 / 32 + (wave & 1), fb = f0 / 32 + (wave >> 1), h = lane >> 5, r = (wave & 1) * 32 + (lane & 31), c = (wave >> 1) * 32 + 4 * h;
  const bool there = mb * 32 < a.M && fb * 32 < a.F;
  Pack<float, 4> g[4], u[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float *at = a.kept + (there ? kept_block(mb, fb, a.F) : 0) + q * 256 + lane * 4;
    g[q] = *(const Pack<float, 4> *)at;
    u[q] = *(const Pack<float, 4> *)(at + 1024);
  }
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int row = (threadIdx.x + 256 * v) / 8, k0 = (threadIdx.x & 7) * 8, m = m0 + row;
    int t = 0, b = 0;
    const bool live = m < a.M && a.steps.live(m, t, b);
    const Pack<T, 8> d = eight_of((const T *)a.dy.p + t * a.dy.st + b * a.dy.sb, f0 + k0, a.F, live, a.wide);
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[0][row][k0 + k] = d.v[k];
  }
  __syncthreads();
  bool live = false;
  if (m0 + r < a.M) {
    int t, b;
    live = a.steps.live(m0 + r, t, b);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k) {            // (every place is its own lane's)
      const bool on = live && f0 + c + 8 * q + k < a.F;
      T &at = tile[0][r][c + 8 * q + k];
      const float d = widen(at), gv = g[q].v[k];
      at = narrow<T>(on ? d * u[q].v[k] * act_slope(a.act, gv) : 0.f);
      tile[1][r][c + 8 * q + k] = narrow<T>(on ? d * act_of(a.act, gv) : 0.f);
    }
  __syncthreads();
  constexpr int P = Pieces<T>::N;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int row = (threadIdx.x + 256 * v) / 8, k0 = (threadIdx.x & 7) * 8;
      Chunk out[P];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        __bf16 p[P];
        Pieces<T>::split(tile[w][row][k0 + k], p);
#pragma unroll
        for (int q = 0; q < P; ++q) out[q].v[k] = p[q];
      }
      if (m0 + row < a.M)
#pragma unroll
        for (int q = 0; q < P; ++q)
          *(Chunk *)(a.rows + q * a.rows_plane + (w * a.panels + by) * a.rows_stage + (int64_t)(m0 + row) * 128 + (threadIdx.x & 7) * 16) = out[q];
    }
    put_transposed<T>(tile[w], a.cols + bx * a.cols_stage, a.cols_plane, (int64_t)w * a.F + f0, a.F - f0);
  }
}

// What the reverse products read, in one launch: the slopes' tiles, then those of x, gate and up (first[i]: the first workgroup of job i;
// tiles along the rows first).
struct ReadyP {
  SlopeP slope;
  LayJobs lays;
  int first[3], along[4];                    // along: tiles along the rows, of the slopes and of each job
};
template <typename T> __global__ __launch_bounds__(256) void ready_kernel(const ReadyP a) {
  __shared__ T tile[2][KS][KS + 1];          // (slopes: dy stands in the first one at the start)
  const int id = blockIdx.x;
  if (id < a.first[0]) {
    slopes<T>(a.slope, tile, id % a.along[0], id / a.along[0]);
    return;
  }
  const int job = id < a.first[1] ? 0 : id < a.first[2] ? 1 : 2, at = id - a.first[job];
  lay_transposed<T>(a.lays.job[job], tile[0], at % a.along[job + 1], at / a.along[job + 1]);
}

// ---------------------------------------------------------------- host
int units_sizes(const snn_units_args *a) {
  if (!a) return ops_fail(SNN_ERR_NULL, "gated units: arguments are NULL");
  if (a->T < 0 || a->B <= 0 || a->D <= 0 || a->F <= 0) return ops_fail(SNN_ERR_ARG, "gated units: T >= 0, B > 0, D > 0 and F > 0 are required");
  if (a->D > (1 << 18) || a->F > (1 << 18) || (int64_t)a->T * a->B > (1ll << 28))
    return ops_fail(SNN_ERR_ARG, "gated units: D and F must not exceed 2^18, T * B 2^28");
  if (a->type != SNN_TYPE_FP32 && a->type != SNN_TYPE_BF16) return ops_fail(SNN_ERR_ARG, "gated units: unknown type %d", a->type);
  if (a->act != SNN_ACT_SILU && a->act != SNN_ACT_GELU) return ops_fail(SNN_ERR_ARG, "gated units: unknown activation %d", a->act);
  return SNN_OK;
}
int units_check(const snn_units_args *a, bool grads) {
  const int rc = units_sizes(a);
  if (rc) return rc;
  if (!a->gate || !a->up) return ops_fail(SNN_ERR_NULL, "gated units: gate or up is NULL");
  if (a->T > 0 && (!a->x.p || (!grads && !a->y.p))) return ops_fail(SNN_ERR_NULL, "gated units: x or y is NULL");
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(a->x.p, z) || !aligned(a->y.p, z) || !aligned(a->gate, z) || !aligned(a->up, z) || !aligned(a->lengths, 4))
    return ops_fail(SNN_ERR_ARG, "gated units: a pointer is not aligned to its element type");
  return SNN_OK;
}

// Workgroups of a product.
int64_t blocks_of(const GemmP &p) { return (int64_t)p.mt * p.nt * p.splits; }
template <typename T, int WHAT> int launch_gemm(const Jobs &jobs, int64_t n, bool wide, hipStream_t st) {
  if (n * 512 >= (1ll << 32)) return ops_fail(SNN_ERR_ARG, "gated units: too large for one launch");
  const int stages = gemm_stages(n, wide);
  auto k = wide ? gemm_kernel<T, WHAT, WIDE_WM, WIDE_WN, 8 / WIDE_WM, 8 / WIDE_WN, 64, 2>
           : stages == 4 ? gemm_kernel<T, WHAT, 2, 2, 2, 2, 64, 4> : gemm_kernel<T, WHAT, 2, 2, 2, 2, 64, 2>;
  const int bytes = stages * (wide ? 256 + 256 : 128 + 128) * 128;
  const hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return ops_fail(SNN_ERR_HIP, "gated units: %s", hipGetErrorString(e));
  hipLaunchKernelGGL(k, dim3((unsigned)n), dim3(wide ? 64 * WIDE_WM * WIDE_WN : 256), bytes, st, jobs);
  return ops_launched("gated units, product");
}

// A launch for `n` jobs.
template <typename T> int lay(const LayJobs &jobs, int n, hipStream_t st) {
  int rows = 0, cols = 0;
  for (int i = 0; i < n; ++i) rows = std::max(rows, jobs.job[i].rows), cols = std::max(cols, jobs.job[i].cols);
  hipLaunchKernelGGL(lay_rows_kernel<T>, dim3((rows + 31) / 32, panels_of(cols), n), dim3(256), 0, st, jobs);
  return ops_launched("gated units, layout");
}
// x or a matrix as a job.
template <typename T> LayP lay_x(const snn_units_args &a, char *dst, int64_t stage, int64_t plane) {
  return LayP{a.x.p, a.T > 1 ? a.x.stride_t : 0, a.x.stride_b, Steps{a.T, a.B, a.lengths}, a.T * a.B, a.D, dst, stage, plane, rows_take(a.x, a.T, a.B, 8, sizeof(T))};
}
template <typename T> LayP lay_matrix(const snn_units_args &a, const void *w, char *dst, int64_t stage, int64_t plane) {
  return LayP{w, 0, a.D, Steps{1, 1 << 30, nullptr}, a.F, a.D, dst, stage, plane, a.D % 8 == 0 && aligned(w, 8 * sizeof(T))};
}

template <typename T, int MB, int WAVES, int NB> int launch_few(const FewP &p, bool wide, hipStream_t st) {
  const dim3 grid((p.F + FEW_UNITS - 1) / FEW_UNITS, (p.M + 16 * MB - 1) / (16 * MB));
  if (!wide) hipLaunchKernelGGL((few_rows_any_kernel<T, MB>), grid, dim3(256), 0, st, p);
  else {
    auto k = few_rows_kernel<T, MB, WAVES, NB>;
    const int bytes = WAVES * NB * (32 + 16 * MB) * 128;
    const hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return ops_fail(SNN_ERR_HIP, "gated units: %s", hipGetErrorString(e));
    hipLaunchKernelGGL(k, grid, dim3(WAVES * 64), bytes, st, p);
  }
  return ops_launched("gated units, few rows");
}
template <typename T> int units_few(const snn_units_args &a, void *saved, hipStream_t st) {
  const FewP p{a.gate, a.up, Rows<void>(a.x, a.T), Rows<void>(a.y, a.T), Steps{a.T, a.B, a.lengths}, (float *)saved, a.T * a.B, a.D, a.F, a.act};
  const bool wide = few_in_pieces(a);
  const int blocks = few_blocks(p.M);
  // (wavefronts by buffers: what 160 KiB of LDS hold)
  return blocks == 1 ? launch_few<T, 1, 8, 3>(p, wide, st) : blocks == 2 ? launch_few<T, 2, 8, 2>(p, wide, st) : launch_few<T, 4, 4, 3>(p, wide, st);
}

template <typename T> int units_forward(const snn_units_args &a, void *saved, char *ws, hipStream_t st) {
  const int M = a.T * a.B, planes = Pieces<T>::N;
  const Steps steps{a.T, a.B, a.lengths};
  GemmP p{};
  p.panels = panels_of(a.D);
  p.segs = planes == 3 ? 6 : 1;
  int64_t row;
  int jobs = 0, rc;
  LayJobs lays;
  if (x_direct(a, row)) p.a = Side{(const char *)a.x.p, nullptr, row, 128, 0, M};
  else {
    p.a = Side{ws, nullptr, 128, (int64_t)M * 128, (int64_t)M * 128 * p.panels, M};
    lays.job[jobs++] = lay_x<T>(a, ws, p.a.stage, p.a.plane);
    ws += rup256(panel_bytes(M, a.D, planes));
  }
  if (weights_direct(a)) p.b = Side{(const char *)a.gate, (const char *)a.up, (int64_t)a.D * 2, 128, 0, a.F};
  else {
    char *const up = ws + rup256(panel_bytes(a.F, a.D, planes));
    p.b = Side{ws, up, 128, (int64_t)a.F * 128, (int64_t)a.F * 128 * p.panels, a.F};
    lays.job[jobs++] = lay_matrix<T>(a, a.gate, ws, p.b.stage, p.b.plane);
    lays.job[jobs++] = lay_matrix<T>(a, a.up, up, p.b.stage, p.b.plane);
  }
  if (jobs && (rc = lay<T>(lays, jobs, st))) return rc;
  const Product how = units_product(a);
  p.mt = how.mt;
  p.nt = how.nt;
  p.splits = how.splits;
  p.steps = steps;
  p.out = Rows<void>(a.y, a.T);
  p.part = (float *)saved;
  p.part_size = kept_size(a);
  p.act = a.act;
  p.M = M;
  p.N = a.F;
  if (p.splits == 1) return launch_gemm<T, UNITS>(Jobs{{p, p}, 0}, blocks_of(p), how.tile.wide, st);
  p.part = (float *)(weights_direct(a) ? ws : ws + 2 * rup256(panel_bytes(a.F, a.D, planes)));
  if ((rc = launch_gemm<T, UNITS>(Jobs{{p, p}, 0}, blocks_of(p), how.tile.wide, st))) return rc;
  const int64_t blocks = (int64_t)((M + 31) / 32) * ((a.F + 31) / 32);
  hipLaunchKernelGGL(units_sum_kernel<T>, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, st, p, (float *)saved);
  return ops_launched("gated units, sums");
}

template <typename T> __global__ __launch_bounds__(256) void clear_kernel(T *p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = narrow<T>(0.f);
}

template <typename T> int units_backward(const snn_units_args &a, const snn_units_grads &g, const float *saved, char *ws, hipStream_t st) {
  const UnitsPlan u = units_plan(a);
  const int M = (int)u.M, pf = panels_of(a.F), pm = panels_of(M);
  int rc;
  if (M == 0) {
    const int64_t n = (int64_t)a.F * a.D;
    for (void *w : {g.dgate, g.dup}) {
      hipLaunchKernelGGL(clear_kernel<T>, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16)), dim3(256), 0, st, (T *)w, n);   // (up to 2^36 elements)
      if ((rc = ops_launched("gated units backward, no steps"))) return rc;
    }
    return SNN_OK;
  }
  const Steps steps{a.T, a.B, a.lengths};
  char *const rows = ws, *const cols = rows + u.rows, *const xt = cols + u.cols, *const wt = xt + u.xt, *const part = wt + u.wt;
  const int64_t st_r = (int64_t)M * 128, st_c = (int64_t)2 * a.F * 128, st_x = (int64_t)a.D * 128, pl_w = st_x * 2 * pf;
  ReadyP r{{steps, Rows<void>(g.dy, a.T), saved, a.act, M, a.F, pf, rows_take(g.dy, a.T, a.B, 8, sizeof(T)), rows, cols, st_r, st_r * 2 * pf, st_c, st_c * pm},
           {{lay_x<T>(a, xt, st_x, st_x * pm), lay_matrix<T>(a, a.gate, wt, st_x, pl_w), lay_matrix<T>(a, a.up, wt + st_x * pf, st_x, pl_w)}},
           {},
           {pm, pm, pf, pf}};
  const int64_t pd = panels_of(a.D), n0 = (int64_t)pm * pf, n1 = n0 + pm * pd, n2 = n1 + pf * pd, n3 = n2 + pf * pd;
  if (n3 * 256 >= (1ll << 32)) return ops_fail(SNN_ERR_ARG, "gated units backward: too large for one launch");
  r.first[0] = (int)n0; r.first[1] = (int)n1; r.first[2] = (int)n2;
  hipLaunchKernelGGL(ready_kernel<T>, dim3((unsigned)n3), dim3(256), 0, st, r);
  if ((rc = ops_launched("gated units backward, slopes"))) return rc;

  Jobs jobs{};
  GemmP &x = jobs.job[0], &w = jobs.job[1];
  x.what = DX;
  x.a = Side{rows, nullptr, 128, st_r, st_r * 2 * pf, M};
  x.b = Side{wt, nullptr, 128, st_x, pl_w, a.D};
  x.panels = 2 * pf;
  x.M = M;
  x.part = (float *)part;
  w.what = DW;
  w.a = Side{cols, nullptr, 128, st_c, st_c * pm, 2 * a.F};
  w.b = Side{xt, nullptr, 128, st_x, st_x * pm, a.D};
  w.panels = pm;
  w.M = 2 * a.F;
  w.part = (float *)(part + u.part_dx);
  for (GemmP *p : {&x, &w}) {
    const Product &how = p == &x ? u.dx : u.dw;
    p->mt = how.mt; p->nt = how.nt; p->splits = how.splits;
    p->segs = u.segs;
    p->steps = steps;
    p->N = a.D;
    p->pitch = pitch_of(a.D);
    p->out = Rows<void>(g.dx, a.T);
    p->w0 = g.dgate;
    p->w1 = g.dup;
  }
  jobs.first = (int)blocks_of(x);
  if ((rc = launch_gemm<T, GRADS>(jobs, blocks_of(x) + blocks_of(w), u.dx.tile.wide, st))) return rc;
  // (a product without parts has no sums)
  auto sums = [](const GemmP &p) { return p.splits > 1 ? ((int64_t)p.M * (p.pitch / 4) + 255) / 256 : 0; };
  const int64_t n = sums(x) + sums(w);
  if (!n) return SNN_OK;
  if (n * 256 >= (1ll << 32)) return ops_fail(SNN_ERR_ARG, "gated units backward: too large for one launch");
  jobs.first = (int)sums(x);
  hipLaunchKernelGGL(gemm_sum_kernel<T>, dim3((unsigned)n), dim3(256), 0, st, jobs);
  return ops_launched("gated units backward, sums");
}

}  // namespace
}  // namespace snn

using namespace snn;

extern "C" {

int32_t snn_units_workspace_bytes(const snn_units_args *a, int32_t backward, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  const int rc = units_sizes(a);
  if (rc) return rc;
  const int planes = a->type == SNN_TYPE_FP32 ? 3 : 1;
  if (backward) {
    const UnitsPlan u = units_plan(*a);
    *bytes = u.rows + u.cols + u.xt + u.wt + u.part_dx + u.part_dw;
    return SNN_OK;
  }
  int64_t row;
  *bytes = few_rows(*a) ? 0 : (x_direct(*a, row) ? 0 : rup256(panel_bytes((int64_t)a->T * a->B, a->D, planes))) + (weights_direct(*a) ? 0 : 2 * rup256(panel_bytes(a->F, a->D, planes))) +
                                (units_product(*a).splits > 1 ? rup256(units_product(*a).splits * kept_size(*a) * 4) : 0);
  return SNN_OK;
}

int32_t snn_units_saved_bytes(const snn_units_args *a, size_t *bytes) {
  if (!bytes) return ops_fail(SNN_ERR_NULL, "bytes is NULL");
  const int rc = units_sizes(a);
  if (rc) return rc;
  *bytes = (size_t)std::max<int64_t>(1, ((int64_t)a->T * a->B + 31) / 32) * ((a->F + 31) / 32) * KEPT * 4;
  return SNN_OK;
}

int32_t snn_units_forward(const snn_units_args *a, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = units_check(a, false);
  if (rc) return rc;
  if (!aligned(saved, 16)) return ops_fail(SNN_ERR_ARG, "gated units: saved has to be 16-byte aligned");
  size_t need = 0;
  if ((rc = snn_units_workspace_bytes(a, 0, &need))) return rc;
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return ops_fail(SNN_ERR_WORKSPACE, "gated units: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  if (a->T == 0) return SNN_OK;
  if (few_rows(*a)) return a->type == SNN_TYPE_FP32 ? units_few<float>(*a, saved, (hipStream_t)stream) : units_few<__bf16>(*a, saved, (hipStream_t)stream);
  return a->type == SNN_TYPE_FP32 ? units_forward<float>(*a, saved, (char *)workspace, (hipStream_t)stream)
                                  : units_forward<__bf16>(*a, saved, (char *)workspace, (hipStream_t)stream);
}

int32_t snn_units_backward(const snn_units_args *a, const snn_units_grads *g, const void *saved, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = units_check(a, true);
  if (rc) return rc;
  if (!g || !g->dgate || !g->dup || (a->T > 0 && (!g->dy.p || !g->dx.p))) return ops_fail(SNN_ERR_NULL, "gated units backward: dy, dx, dgate or dup is NULL");
  if (!saved) return ops_fail(SNN_ERR_NULL, "gated units backward: saved is NULL");
  const size_t z = a->type == SNN_TYPE_FP32 ? 4 : 2;
  if (!aligned(saved, 16) || !aligned(g->dy.p, z) || !aligned(g->dx.p, z) || !aligned(g->dgate, z) || !aligned(g->dup, z))
    return ops_fail(SNN_ERR_ARG, "gated units backward: a pointer is not aligned to its element type");
  size_t need = 0;
  if ((rc = snn_units_workspace_bytes(a, 1, &need))) return rc;
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return ops_fail(SNN_ERR_WORKSPACE, "gated units backward: %zu bytes of 16-byte aligned workspace are needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
  return a->type == SNN_TYPE_FP32 ? units_backward<float>(*a, *g, (const float *)saved, (char *)workspace, (hipStream_t)stream)
                                  : units_backward<__bf16>(*a, *g, (const float *)saved, (char *)workspace, (hipStream_t)stream);
}

}  // extern "C"
