/*
 * libthemis, forecasting operators: what an arrival-rate forecaster consists of, so that the
 * predicted rates which the solvers of themis.h take can be made (and the forecaster trained)
 * on the device, on the solver's stream.  The paper's optimizer predicts the rate of the next
 * seconds from the rates seen (Section "Optimizer"); these are the operators of such a sequence
 * model:
 *
 *   themis_ssm_*     a selective state space scan with its short causal convolution and its
 *                    gate: over whole histories (forward, backward) and for one tick of many
 *                    pipelines (step);
 *   themis_linear_*  a matrix product with bias, activation and residual, and its gradients.
 *
 * The conventions of themis.h hold: return codes, no exceptions, device pointers owned by the
 * caller, nothing allocated on the device, a caller-provided workspace (256-byte aligned; may
 * be NULL when its size is 0), work enqueued on the given stream without synchronising, scalar
 * arguments validated on the host before anything is launched.  Results do not depend on the
 * order in which blocks run: there are no floating-point atomics.  Every output element is
 * written by every call that succeeds.
 */
#ifndef THEMIS_FORECAST_H_
#define THEMIS_FORECAST_H_

#include <stddef.h>
#include <stdint.h>

#include "themis.h"

#ifdef __cplusplus
extern "C" {
#endif

/* type of the sequence data ("T" below) */
#define THEMIS_DTYPE_F32 0
#define THEMIS_DTYPE_BF16 1
#define THEMIS_DTYPE_F16 2

/* ------------------------------------------------------------------------------------------
 * Selective state space scan.  For row b (a pipeline), time t, channel d in group g, state n:
 *     c_t = conv_bias[d] + sum_k conv_weight[d][k] x[t-W+1+k]      (W = conv_width)
 *     u_t = silu(c_t),   s_t = softplus(dt_t + dt_bias[d])
 *     h_t[n] = exp(s_t A[d][n]) h_{t-1}[n] + s_t u_t B_t[g][n]
 *     v_t = sum_n C_t[g][n] h_t[n] + skip[d] u_t
 *     y_t = v_t silu(z_t)                                          (no z: y_t = v_t)
 * All of it is computed in 32 bits; y is rounded once.  x before the first time is taken from
 * conv_state, h before it from ssm_state (zeros where these are NULL).  A row's times from
 * lengths[b] on do not exist: y (and every gradient) is 0 there, the states end at lengths[b],
 * and what the inputs hold there is not used (it may be NaN).  lengths below 0 count as 0,
 * above `length` as `length`.
 */
#define THEMIS_SSM_MAX_STATE 64
#define THEMIS_SSM_MIN_CONV 2
#define THEMIS_SSM_MAX_CONV 4
/* times between two saved states (checkpoints) */
#define THEMIS_SSM_CHUNK 16

typedef struct {
    int32_t batch;      /* rows, >= 0 */
    int32_t length;     /* times, in 0..2^30 (step: not used, one) */
    int32_t channels;   /* D in 1..65535 */
    int32_t state;      /* N in 1..THEMIS_SSM_MAX_STATE */
    int32_t groups;     /* G >= 1, divides channels: channel d uses group d / (D / G) */
    int32_t conv_width; /* W in 2..4 */
    int32_t dtype;      /* THEMIS_DTYPE_*: x, dt, z, B, C, y, conv_state and their gradients */
    uint32_t flags;     /* 0 */
    /* strides in elements (>= 0) of the inputs; the last axis (channels, states) is contiguous.
     * A step ignores the time strides. */
    int64_t x_row, x_time, dt_row, dt_time, z_row, z_time;
    int64_t b_row, b_time, b_group, c_row, c_time, c_group;
} themis_ssm_problem_t;

typedef struct {
    const void *x, *dt;         /* T [batch][length][D] */
    const void *z;              /* T [batch][length][D], or NULL */
    const void *b, *c;          /* T [batch][length][G][N] */
    const float *a;             /* [D][N] */
    const float *conv_weight;   /* [D][W] */
    const float *conv_bias;     /* [D], or NULL */
    const float *skip;          /* [D], or NULL */
    const float *dt_bias;       /* [D], or NULL */
    const void *conv_state;     /* T [batch][W-1][D]: the last W-1 x, oldest first; or NULL */
    const float *ssm_state;     /* [batch][D][N], or NULL */
    const int32_t *lengths;     /* [batch], or NULL: every row has `length` times.  A step uses
                                   it as a mask: rows with lengths[b] < 1 stay as they are */
} themis_ssm_inputs_t;

typedef struct {
    void *y;            /* T [batch][length][D] (step: [batch][D]), contiguous */
    void *conv_state;   /* T [batch][W-1][D], or NULL (not wanted) */
    float *ssm_state;   /* [batch][D][N], or NULL */
    float *checkpoints; /* forward: the states before times 0, 16, 32, ...,
                           [batch][themis_ssm_checkpoints][D][N], for the backward call; or NULL */
} themis_ssm_outputs_t;

/* Gradients, all contiguous; a NULL one is not wanted. */
typedef struct {
    void *x, *dt, *z, *b, *c;                                  /* T */
    float *a, *conv_weight, *conv_bias, *skip, *dt_bias;       /* sums over rows and times */
} themis_ssm_grads_t;

/* number of saved states of a row: ceil(length / THEMIS_SSM_CHUNK) */
int themis_ssm_checkpoints(const themis_ssm_problem_t *problem, int32_t *out_count);
/* workspace of themis_ssm_forward (backward == 0) or themis_ssm_backward (backward != 0) */
int themis_ssm_workspace_bytes(const themis_ssm_problem_t *problem, int backward, size_t *out_bytes);

/* Whole histories.  The state outputs must not be the state inputs' memory. */
int themis_ssm_forward(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in,
                       const themis_ssm_outputs_t *out, void *d_workspace, size_t workspace_bytes,
                       void *cuda_stream);

/*
 * Gradients of sum(dy * y) for the inputs of a forward call and the checkpoints that it left.
 * dy is T [batch][length][D], contiguous.  Initial states are constants: they get no gradient,
 * and the final states' gradient is taken as 0 (truncated back-propagation through time).
 */
int themis_ssm_backward(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in,
                        const float *checkpoints, const void *dy, const themis_ssm_grads_t *grads,
                        void *d_workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * One time of every row: x, dt, z are [batch][D], b and c [batch][G][N]; conv_state and
 * ssm_state are required on both sides and may be the same memory (updated in place).  No
 * workspace.
 */
int themis_ssm_step(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in,
                    const themis_ssm_outputs_t *out, void *cuda_stream);

/* ------------------------------------------------------------------------------------------
 * Matrix product with an epilogue.
 *     pre = x weight^T + bias,   y = act(pre) + residual
 * accumulated in 32 bits; y (and pre, where it is wanted) are rounded once.
 */
#define THEMIS_ACT_NONE 0
#define THEMIS_ACT_RELU 1
#define THEMIS_ACT_SILU 2
#define THEMIS_ACT_GELU 3   /* 0.5 v (1 + erf(v / sqrt 2)) */

typedef struct {
    int32_t rows;         /* M >= 0 */
    int32_t out_features; /* N >= 1 */
    int32_t in_features;  /* K >= 1 */
    int32_t dtype;        /* THEMIS_DTYPE_BF16 or THEMIS_DTYPE_F16 */
    int32_t activation;   /* THEMIS_ACT_* */
    uint32_t flags;       /* 0 */
    /* elements from one row to the next (>= the row's length): x, weight, residual, and dy of
     * the backward call; every other matrix is contiguous */
    int64_t x_row, weight_row, residual_row, dy_row;
} themis_linear_problem_t;

/* workspace of the forward (backward == 0) or backward call for this problem; `unaligned` != 0
 * if a pointer of x, weight or dy is not 16-byte aligned (those operands are then copied) */
int themis_linear_workspace_bytes(const themis_linear_problem_t *problem, int backward, int unaligned,
                                  size_t *out_bytes);

/*
 *   d_x         T [M][K]         d_weight  T [N][K]
 *   d_bias      float [N], or NULL
 *   d_residual  T [M][N], or NULL
 *   d_y         T [M][N] out, contiguous
 *   d_pre       T [M][N] out, contiguous, or NULL: what the backward call of an activation needs
 *   d_status    int32 or NULL: THEMIS_STATUS_TIMEOUT is written to it if a bounded on-device wait
 *               expired (the result is then void); never written otherwise.  Any memory that the
 *               device can write; in pinned host memory the host can poll it.  With NULL an
 *               expired wait is not reported
 */
int themis_linear_forward(const themis_linear_problem_t *problem, const void *d_x, const void *d_weight,
                          const float *d_bias, const void *d_residual, void *d_y, void *d_pre,
                          int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * With q = dy act'(pre) (q = dy without an activation; d_pre is then ignored):
 *   d_dx = q weight  T [M][K],   d_dweight = q^T x  T [N][K],   d_dbias = column sums of q  float [N];
 * a NULL output is not computed.  q is rounded to T before the two products (they take 16-bit
 * operands); the bias gradient sums the unrounded q.  The residual's gradient is dy itself.
 */
int themis_linear_backward(const themis_linear_problem_t *problem, const void *d_dy, const void *d_x,
                           const void *d_weight, const void *d_pre, void *d_dx, void *d_dweight,
                           float *d_dbias, int32_t *d_status, void *d_workspace, size_t workspace_bytes,
                           void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* THEMIS_FORECAST_H_ */
