/*
 * snn_seq.h -- C ABI of the sequence operators that join the LIF layer of snn_lif.h along
 * the same time axis: a short causal convolution, a selective state space scan, and a
 * block's gate, norm and scaled residual with the next block's norm.
 *
 * They keep the conventions of snn_lif.h (device pointers owned by the caller; the library
 * never allocates, never synchronizes, keeps no state; arguments are checked before anything
 * is launched; statuses are snn_status) with these differences:
 *   - A [T][B][X] tensor is given as an snn_seq: its first element and the elements between
 *     consecutive steps and between consecutive sequences; the last axis is contiguous.  So
 *     time-major tensors, batch-major ones and slices of wider rows are all read in place.
 *     Inputs may repeat rows (a step of 0); outputs must not overlap themselves or any input.
 *   - Pointers need only their element's alignment (SNN_E_ALIGN otherwise).
 *   - Parameters and their gradients, states of the scan, saved data and workspaces are
 *     float32 (the convolution's state holds inputs, in the I/O dtype).  Everything is
 *     computed in float32 and rounded once (to nearest even) where it is stored as bfloat16.
 *   - lengths: NULLABLE int32 [B], device memory: sequence b has min(max(lengths[b], 0), T)
 *     steps.  Rows behind them are padding: inputs there are not read (whatever they hold),
 *     outputs and gradients there are written as 0, states stay as they were at the end.
 *   - T == 0, B == 0 or F == 0 is an empty problem: SNN_OK, nothing is launched or written.
 *   - Limits: T <= 2^30, B <= 2^24, F <= 2^24, T * B <= 2^30, B * F <= 2^31 and
 *     T * B * groups < 2^31 in the scan, and every tensor spans less than 2^44 elements.
 *   - A workspace is scratch: it holds nothing between calls, and calls that may run at the
 *     same time need one each.
 * Results do not change from run to run: sums over steps, sequences and features are formed
 * in a fixed order.
 */
#ifndef SNN_SEQ_H
#define SNN_SEQ_H

#include "snn_lif.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    const void *data; /* first element; written through where the tensor is an output */
    int64_t t;        /* elements from one step to the next */
    int64_t b;        /* elements from one sequence to the next */
} snn_seq;

/* ---------------------------------------------------------------------------------------
 * Short causal convolution, one filter per feature:
 *   u[t][b][f] = bias[f] + sum_j weight[f][j] x[t - (W-1) + j][b][f],   y = act(u)
 * with the W-1 inputs before step 0 taken from state_in, or 0. */
typedef enum { SNN_ACT_NONE = 0, SNN_ACT_SILU = 1 /* u / (1 + e^-u) */ } snn_act;

typedef struct {
    int32_t io;    /* snn_io */
    int32_t width; /* W, 1 to 8 taps */
    int32_t act;   /* snn_act */
} snn_conv_cfg;

/*   weight [F][W], bias [F] (NULLABLE) float32; state_in [W-1][B][F] io dtype, oldest first,
 *   NULLABLE; state_out [W-1][B][F] NULLABLE: the last W-1 inputs of each sequence (those of
 *   state_in among them where it is shorter).  state_out may be state_in (in place). */
snn_status snn_conv_forward(const snn_conv_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *x,
                            const float *weight, const float *bias, const void *state_in,
                            const int32_t *lengths, const snn_seq *y, void *state_out, void *stream);

/* Bytes of the backward's workspace.  Host-only. */
snn_status snn_conv_workspace_bytes(const snn_conv_cfg *cfg, int64_t T, int64_t B, int64_t F, size_t *bytes);

/*   x .. lengths as in the forward; grad_y [T][B][F]; grad_state_out [W-1][B][F] NULLABLE;
 *   out: grad_x [T][B][F], grad_weight [F][W], grad_bias [F] (NULLABLE), grad_state_in
 *   [W-1][B][F] (NULLABLE; not grad_state_out). */
snn_status snn_conv_backward(const snn_conv_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *x,
                             const float *weight, const float *bias, const void *state_in,
                             const int32_t *lengths, const snn_seq *grad_y, const void *grad_state_out,
                             const snn_seq *grad_x, float *grad_weight, float *grad_bias,
                             void *grad_state_in, void *workspace, void *stream);

/* ---------------------------------------------------------------------------------------
 * Selective state space scan: S states per feature, B and C shared by the F / G features of
 * a group,
 *   d[t][b][f]    = softplus(dt[t][b][f] + dt_bias[f])      (or the sum itself)
 *   h[t][b][f][n] = e^{d A[f][n]} h[t-1][b][f][n] + d Bm[t][b][g][n] x[t][b][f]
 *   y[t][b][f]    = sum_n Cm[t][b][g][n] h[t][b][f][n] + D[f] x[t][b][f],   g = f / (F/G).
 * States may grow (d A > 0): each step's e^{d A} has to fit float32, their product need not. */
typedef struct {
    int32_t io;       /* snn_io: x, dt, Bm, Cm, y and their gradients */
    int32_t states;   /* S, 1 to 64 */
    int32_t groups;   /* G >= 1, divides F */
    int32_t softplus; /* 1: as above; 0: d = dt + dt_bias */
} snn_scan_cfg;

/* Bytes that the forward keeps for the backward (states at fixed intervals of steps), and of
 * the forward's and the backward's workspaces.  Host-only. */
snn_status snn_scan_saved_bytes(const snn_scan_cfg *cfg, int64_t T, int64_t B, int64_t F, size_t *bytes);
snn_status snn_scan_workspace_bytes(const snn_scan_cfg *cfg, int64_t T, int64_t B, int64_t F,
                                    size_t *forward_bytes, size_t *backward_bytes);

/*   x, dt [T][B][F], Bm, Cm [T][B][G*S] io dtype; A [F][S], D [F] (NULLABLE: 0), dt_bias [F]
 *   (NULLABLE: 0) float32; h_in [B][F][S] float32 NULLABLE (0);
 *   out: y [T][B][F]; h_out [B][F][S] NULLABLE, the state after each sequence's last step,
 *   may be h_in (in place); saved NULLABLE: given where a backward follows (it may be NULL
 *   when its size is 0 too).
 *   workspace may be NULL when its size is 0. */
snn_status snn_scan_forward(const snn_scan_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *x,
                            const snn_seq *dt, const float *A, const snn_seq *Bm, const snn_seq *Cm,
                            const float *D, const float *dt_bias, const float *h_in,
                            const int32_t *lengths, const snn_seq *y, float *h_out, void *saved,
                            void *workspace, void *stream);

/*   x .. lengths, saved as in the forward (h_in unchanged since); grad_y [T][B][F];
 *   grad_h_out [B][F][S] float32 NULLABLE;
 *   out: grad_x, grad_dt [T][B][F], grad_Bm, grad_Cm [T][B][G*S], grad_A [F][S], grad_D,
 *   grad_dt_bias [F] (NULLABLE), grad_h_in [B][F][S] (NULLABLE; not grad_h_out). */
snn_status snn_scan_backward(const snn_scan_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *x,
                             const snn_seq *dt, const float *A, const snn_seq *Bm, const snn_seq *Cm,
                             const float *D, const float *dt_bias, const float *h_in,
                             const int32_t *lengths, const void *saved, const snn_seq *grad_y,
                             const float *grad_h_out, const snn_seq *grad_x, const snn_seq *grad_dt,
                             float *grad_A, const snn_seq *grad_Bm, const snn_seq *grad_Cm, float *grad_D,
                             float *grad_dt_bias, float *grad_h_in, void *workspace, void *stream);

/* ---------------------------------------------------------------------------------------
 * The end of a block and the start of the next, per row (t, b) over its F features:
 *   g  = y * z / (1 + e^-z)                               (z NULL: g = y)
 *   n  = g / sqrt(mean(g^2) + eps) * w_post               (w_post NULL: n = g)
 *   r' = r + scale * n                                    (r NULL: 0; scale NULL: 1)
 *   u  = r' / sqrt(mean(r'^2) + eps) * w_pre              (w_pre NULL: no u)
 * u is formed from r' before it is rounded to the I/O dtype. */
typedef struct {
    int32_t io; /* snn_io */
    float eps;  /* > 0 and finite */
} snn_norm_cfg;

/*   y, z, r [T][B][F] io dtype; w_post, scale, w_pre [F] float32;
 *   out: r_new [T][B][F]; u [T][B][F] (with w_pre); rstd NULLABLE float32 [2][T][B]: the two
 *   reciprocal roots, for the backward. */
snn_status snn_norm_forward(const snn_norm_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *y,
                            const snn_seq *z, const snn_seq *r, const float *w_post, const float *scale,
                            const float *w_pre, const int32_t *lengths, const snn_seq *r_new,
                            const snn_seq *u, float *rstd, void *stream);

/* Bytes of the backward's workspace.  Host-only. */
snn_status snn_norm_workspace_bytes(const snn_norm_cfg *cfg, int64_t T, int64_t B, int64_t F, size_t *bytes);

/*   y .. lengths, rstd as in the forward; grad_r_new, grad_u [T][B][F], each NULLABLE (0);
 *   out, each with its input only: grad_y, grad_z, grad_r [T][B][F], grad_w_post, grad_scale,
 *   grad_w_pre [F] float32. */
snn_status snn_norm_backward(const snn_norm_cfg *cfg, int64_t T, int64_t B, int64_t F, const snn_seq *y,
                             const snn_seq *z, const snn_seq *r, const float *w_post, const float *scale,
                             const float *w_pre, const int32_t *lengths, const float *rstd,
                             const snn_seq *grad_r_new, const snn_seq *grad_u, const snn_seq *grad_y, const snn_seq *grad_z,
                             const snn_seq *grad_r, float *grad_w_post, float *grad_scale, float *grad_w_pre,
                             void *workspace, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SNN_SEQ_H */
