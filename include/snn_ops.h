/*
 * snn_ops.h - C ABI of the sequence operators and the AdamW step of the MI355X (gfx950) library.
 *
 * Beside the spiking layers of snn.h (leaky integrators whose leak is a constant of the neuron) stand here a
 * leaky integrator whose leak and input gain follow the data, the short convolution along time that feeds it,
 * and the optimiser step that trains both:
 *
 *   convolution      v[t,d] = bias[d] + sum_(k<W) weight[d,k] x[t-(W-1)+k, d];  y = v, or v sigmoid(v) (SiLU)
 *   selective scan   delta = softplus(dt + dt_bias);  h[t,d,n] = exp(delta A[d,n]) h[t-1,d,n] + delta x[t,d] Bv[t,n]
 *                    y[t,d] = (sum_n Cv[t,n] h[t,d,n] + skip[d] x[t,d]) z sigmoid(z)
 *   AdamW            m, v: running means of the gradient and its square;
 *                    p <- p (1 - lr wd) - lr m' / (sqrt(v') + eps), m', v' corrected for their start at zero
 *
 * Conventions (those of snn.h: plain pointers and sizes, an snn_status from every call, the text of an error from
 * snn_last_error(NULL), no device memory allocated, everything enqueued on the stream given and nothing waited for,
 * nothing read from the environment, no state kept between calls; every call can be captured into a graph)
 *   - Tensors with a time axis are time-major, channels fastest.  An snn_rows names one: element (t, b, d) is
 *     p[t * stride_t + b * stride_b + d], strides in elements, of the call's `type`.  Strides may be anything that
 *     fits the memory (parts of wider rows, batch-major memory); outputs must not overlap what the call reads.
 *     Offsets are 64 bits wide.
 *   - `type` is that of the streamed tensors.  Arithmetic, states, parameters and their gradients are fp32; a
 *     streamed output is rounded once, when it is stored.
 *   - `lengths` (device, int32 [B], may be NULL): steps t >= lengths[b] of sequence b do not exist.  Inputs there
 *     are not used (they may hold anything), outputs and gradients there are zero, states are those after the last
 *     step that exists.  Values outside [0, T] count as the nearer end.
 *   - T = 0 is a call without steps: states pass through, gradients of parameters are zero.
 *   - Sizes that are refused (SNN_ERR_ARG): convolution, B * D from 2^31 or D above 2^28 on, or more than 2^26 wavefronts
 *     (64 channels, or 256 where rows are aligned to four, by 32 steps of a sequence); scan, D above 2^22, B * D from 2^25,
 *     B * groups from 2^18, T * B * groups from 2^32, strides between steps that are negative or put 16 steps of a tensor
 *     2 GiB apart; AdamW, tensors of more than 2^33 elements.
 *   - Sums have a fixed order: the same call gives the same bits.
 *   - The scan's A may be any number.  -inf is a state that forgets at once; its gradients are the limits (zero for A).  States
 *     may grow (A > 0, or negative steps without softplus) as far as fp32 goes, however time is cut.  Infinities and NaN in
 *     steps that exist stay in their sequence and channel and in the sums over them; where the definition makes an
 *     infinity, that or NaN comes out (the states that fill N up to what lanes hold multiply an infinite input by zero).
 */
#ifndef SNN_OPS_H_
#define SNN_OPS_H_

#include "snn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SNN_TYPE_FP32 = 0, SNN_TYPE_BF16 = 1 } snn_type;

typedef struct {
  const void *p;             /* device; written where the field that holds it is an output */
  int64_t stride_t, stride_b;
} snn_rows;

/* ------------------------------------------------------------------ convolution along time */
#define SNN_CONV_MAX_TAPS 8

typedef struct {
  int32_t T, B, D, W;        /* W taps: 1..SNN_CONV_MAX_TAPS */
  int32_t type;              /* snn_type of x, y, init, state and their gradients */
  int32_t silu;              /* 1: y = v sigmoid(v); 0: y = v */
  snn_rows x, y;             /* y is written */
  const float *weight;       /* [D][W] */
  const float *bias;         /* [D], or NULL */
  const void *init;          /* [W-1][B][D]: the inputs before the first step, oldest first; NULL: zeros */
  const int32_t *lengths;
  void *state;               /* [W-1][B][D]: the last W-1 inputs, written (snn_conv_step: read and written); NULL: not wanted */
} snn_conv_args;

typedef struct {
  snn_rows dy, dx;           /* dx is written */
  const void *d_state;       /* gradient of `state`, or NULL */
  float *dweight, *dbias;    /* written; dbias may be NULL */
  void *dinit;               /* written, or NULL */
} snn_conv_grads;

int32_t snn_conv_forward(const snn_conv_args *a, void *hip_stream);

/* Gradients of a forward call: `a` as it was given to it (y, state and bias' presence aside, which are not used; the
 * bias itself is).  `workspace`: 16-byte aligned device memory of at least snn_conv_workspace_bytes. */
int32_t snn_conv_workspace_bytes(const snn_conv_args *a, size_t *bytes);
int32_t snn_conv_backward(const snn_conv_args *a, const snn_conv_grads *g, void *workspace, size_t workspace_bytes,
                          void *hip_stream);

/* One step of every sequence: x and y hold B rows (stride_t is not used), `state` is moved on in place.  T must be 1;
 * init and lengths must be NULL. */
int32_t snn_conv_step(const snn_conv_args *a, void *hip_stream);

/* ------------------------------------------------------------------ selective scan */
#define SNN_SCAN_MAX_STATES 64

typedef struct {
  int32_t T, B, D, N;        /* N states per channel: 1..SNN_SCAN_MAX_STATES */
  int32_t groups;            /* channels d with the same d / (D / groups) share Bv and Cv; groups divides D */
  int32_t type;
  int32_t softplus;          /* 1: delta = softplus(dt + dt_bias); 0: delta = dt + dt_bias */
  snn_rows x, dt;            /* [T][B][D] */
  snn_rows z;                /* [T][B][D], or p = NULL: no gate */
  snn_rows bv, cv;           /* [T][B][groups][N], the last two dense */
  snn_rows y;                /* written */
  const float *A;            /* [D][N] */
  const float *skip;         /* [D], or NULL */
  const float *dt_bias;      /* [D], or NULL */
  const float *init;         /* [B][D][N], or NULL: zeros */
  const int32_t *lengths;
  float *state;              /* [B][D][N], written (snn_scan_step: read and written), or NULL */
} snn_scan_args;

typedef struct {
  snn_rows dy;
  const float *d_state;      /* [B][D][N], gradient of `state`, or NULL */
  snn_rows dx, ddt, dz;      /* written; dz.p = NULL where there is no gate */
  snn_rows dbv, dcv;         /* written */
  float *dA;                 /* [D][N], written */
  float *dskip, *ddt_bias;   /* [D], written, or NULL */
  float *dinit;              /* [B][D][N], written, or NULL */
} snn_scan_grads;

/* Device bytes a forward (backward != 0: a backward) call needs as workspace, 16-byte aligned; and what a forward
 * call that will be followed by a backward one leaves in `saved` (16-byte aligned): the state before every 16th step. */
int32_t snn_scan_workspace_bytes(const snn_scan_args *a, int32_t backward, size_t *bytes);
int32_t snn_scan_saved_bytes(const snn_scan_args *a, size_t *bytes);

/* `saved` may be NULL: nothing is kept. */
int32_t snn_scan_forward(const snn_scan_args *a, void *saved, void *workspace, size_t workspace_bytes, void *hip_stream);
/* `a` as it was given to the forward call (y and state are not used), `saved` as it left it. */
int32_t snn_scan_backward(const snn_scan_args *a, const snn_scan_grads *g, const void *saved, void *workspace,
                          size_t workspace_bytes, void *hip_stream);
/* One step of every sequence, `state` moved on in place.  T must be 1; init and lengths must be NULL. */
int32_t snn_scan_step(const snn_scan_args *a, void *hip_stream);

/* ------------------------------------------------------------------ AdamW */
#define SNN_ADAMW_BLOCK 128        /* elements of an 8-bit moment that share a scale */

/* One tensor.  Its moments are elements [at, at + n) of the call's moment buffers; `at` is a multiple of
 * SNN_ADAMW_BLOCK.  The blocks of two tensors do not overlap, nor does the memory of the parameters and copies: a call where
 * they do (a tensor given twice, say) is refused with SNN_ERR_ARG. */
typedef struct {
  float *param;              /* device, fp32, updated */
  const void *grad;          /* device, of the call's grad_type */
  void *copy;                /* device, bfloat16, receives the updated parameter rounded; or NULL */
  int64_t n, at;
  double weight_decay;
} snn_adamw_tensor;

/* Moments in 32 bits: m and v fp32, scales NULL.  In 8 bits: m and v bytes in the OCP e4m3 format, m_scale and
 * v_scale one fp32 power of two per block (the least that brings the block's largest magnitude to 448 or below, 2^-60
 * at least): the first moment is m m_scale, the second moment is (v v_scale)^2.  A value between two codes goes up or
 * down with the probability that keeps the mean (of the moment, also for the second): where the moments move by
 * less than half a code a step, as they do at beta2 = 0.999, rounding to the nearest would not let them move at all.
 * A second moment above zero never rounds to zero.  The random numbers are a fixed function of `seed`, `step` and the
 * element's place, so a run repeats.  A moment that is not finite is kept as NaN and leaves its block's scale alone. */
typedef struct {
  int32_t bits;              /* 32 or 8 */
  int32_t grad_type;         /* snn_type */
  void *m, *v;               /* 16-byte aligned */
  float *m_scale, *v_scale;
  int64_t step;              /* 1 for the first step */
  uint32_t seed;
  double lr, beta1, beta2, eps;
  double grad_scale;         /* gradients are multiplied by it first */
} snn_adamw_args;

/* `tensors`: host array; read before the call returns.  A tensor with n = 0 is passed over.  A call captured into a graph
 * is replayed with the step number and the rates that it was captured with. */
int32_t snn_adamw_step(const snn_adamw_args *a, const snn_adamw_tensor *tensors, int32_t count, void *hip_stream);

/* The same for a network of snn.h, in the place of snn_sgd_step: every W and R, and the decays where they are trained
 * (these without weight decay, and kept in [0, 1] as snn_sgd_step keeps them), then the refresh of the operand copies.
 * `a` as above, with grad_type SNN_TYPE_FP32 and moment buffers of snn_adamw_network_elements elements (a multiple of
 * SNN_ADAMW_BLOCK; layer by layer W, R, decays), zeroed before the first step.  Needs a preceding snn_backward (else
 * SNN_ERR_STATE).  Currents and spike gradients that the pass's launches kept to themselves cannot be read after it
 * (snn_get_tensor gives SNN_ERR_STATE): they would have to be formed again on weights that are gone. */
int32_t snn_adamw_network_elements(const snn_ctx *ctx, int64_t *elements);
int32_t snn_adamw_network_step(snn_ctx *ctx, const snn_adamw_args *a, double weight_decay);

#ifdef __cplusplus
}
#endif
#endif /* SNN_OPS_H_ */
