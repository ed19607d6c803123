/*
 * seq_ops.h -- C ABI of the sequence operators: what a state-space layer runs
 * between its pointwise convolutions (conv_fwd.h with R = S = 1), on the same
 * channels-first tensors.  In libconvfwd.so.
 *
 *   causal convolution   one short filter per channel along the length
 *   selective scan       the recurrence h(t) = exp(dt(t) A) h(t-1) + dt(t) u(t) B(t)
 *   norms                root-mean-square norms over the channels, before and
 *                        after a block, with its gate, scale and residual
 *
 * each forward, backward, and (the first two) for single tokens.
 *
 * Layouts: sequences are [N, D, L] with the length innermost and of stride 1;
 * batch and channel strides (in elements) are the caller's, so a tensor may be
 * a slice of channels of a larger one.  Outputs, parameters, states and
 * gradients are dense.  T is the call's element type (CONV_DTYPE_F32 or
 * CONV_DTYPE_BF16); sums, states, statistics and parameter gradients are fp32,
 * and what is stored as T is rounded once, to nearest even.  Only element
 * alignment is required.
 *
 * Lengths: `lengths` (device, [N], may be null) gives each sequence's valid
 * steps, taken as min(max(length, 0), L).  Steps behind it are not read (their
 * values may be anything, NaN included); outputs and gradients there are zero.
 * A sequence of length 0 leaves its state as it was.
 *
 * Ownership: all pointers are DEVICE memory of the caller, scratch included:
 * a call that needs scratch takes `workspace`, of at least the bytes that the
 * call's _workspace function returns (0: none needed, the pointer is ignored),
 * 16-byte aligned.  Its contents need not survive the call, and mean nothing
 * before it.  The library allocates and keeps nothing here, so calls on
 * different streams, captured calls and replayed graphs do not meet as long as
 * their workspaces do not.  Outputs must overlap no input of the call, except
 * where stated.  The calling thread's current device must own the stream.
 *
 * Extents: N D < 2^31, L <= 2^30; the scan's and the norms' D <= 2^30.
 *
 * Asynchrony, errors and thread safety are those of conv_fwd.h: the calls
 * enqueue kernels on `stream` and return; CONV_EINVAL (an extent, option or
 * combination), CONV_ENULL (a required pointer), CONV_ERANGE (more work than
 * one launch holds) and CONV_ESCRATCH (a workspace too small) are reported
 * before anything is launched.  Results do not change from run to run: every
 * sum has a fixed order.
 */
#ifndef SEQ_OPS_H
#define SEQ_OPS_H

#include "conv_fwd.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SEQ_ACT_NONE = 0, SEQ_ACT_SILU = 1 };

#define SEQ_CONV_MAX_TAPS 8
#define SEQ_SCAN_MAX_STATE 64
#define SEQ_SCAN_CHUNK 128 /* steps between two checkpoints of a scan */

/*
 * Causal convolution of each channel with R taps, 1 <= R <= 8:
 *
 *   out[n][d][t] = act(bias[d] + sum_{r<R} weight[d][r] x[n][d][t - (R-1) + r])
 *
 * x before t = 0 is initial_state[n][d][0..R-2] (oldest first; zero without
 * one).  final_state is the last R-1 entries of (initial_state, x[0..len-1]):
 * the initial_state of the call that continues the sequence.
 */
typedef struct {
  int32_t N, D, L, R;
  int32_t dtype;      /* of x, states, out and their gradients            */
  int32_t activation; /* SEQ_ACT_*                                        */
  int64_t x_n, x_d;   /* strides of x                                     */
  int64_t dout_n, dout_d;
  const void* x;
  const float* weight;       /* [D, R]                                    */
  const float* bias;         /* [D] or null                               */
  const void* initial_state; /* [N, D, R-1] or null                       */
  const int32_t* lengths;    /* [N] or null                               */
  void* out;                 /* [N, D, L]                      (fwd, step) */
  void* final_state;         /* [N, D, R-1] or null            (fwd, step) */
  const void* dout;          /* [N, D, L]                           (bwd) */
  const void* dfinal_state;  /* [N, D, R-1] or null                 (bwd) */
  void* dx;                  /* [N, D, L]                           (bwd) */
  float* dweight;            /* [D, R]                              (bwd) */
  float* dbias;              /* [D] or null                         (bwd) */
  void* dinitial_state;      /* [N, D, R-1] or null                 (bwd) */
  void* workspace;
  int64_t workspace_bytes;
} seq_conv_t;

int seq_causal_conv_fwd(const seq_conv_t* p, void* stream);
/* The gradients, from x as the forward call had it. */
int seq_causal_conv_bwd(const seq_conv_t* p, void* stream);
/* Bytes of workspace that seq_causal_conv_bwd needs, or a negative status. */
int64_t seq_causal_conv_bwd_workspace(const seq_conv_t* p);
/*
 * One token: L = 1, x [N, D] of strides x_n and x_d, out [N, D].
 * initial_state and final_state are required if R > 1 and may be the same
 * memory.  No lengths.
 */
int seq_causal_conv_step(const seq_conv_t* p, void* stream);

/*
 * Selective scan with S states a channel, 1 <= S <= 64.  Channels are in G
 * groups of D / G consecutive ones, which share B and C (D % G == 0).
 *
 *   dt = delta + delta_bias, through softplus if delta_softplus
 *   h[s](t) = exp(dt(t) A[d][s]) h[s](t-1) + dt(t) u(t) B[g][s](t)
 *   y(t) = sum_s C[g][s](t) h[s](t) + Dskip[d] u(t)
 *   out(t) = y(t) z(t) sigmoid(z(t)), or y(t) without z
 *
 * h(-1) is initial_state (zero without one), final_state is h(len - 1).  The
 * steps are composed in parallel, so decays have to stay in fp32's range over
 * SEQ_SCAN_CHUNK steps: exp(A sum dt) may underflow (a state that has died
 * away), but where it overflows (A dt positive and large) states may be NaN.
 */
typedef struct {
  int32_t N, D, L, S, G;
  int32_t dtype; /* of u, delta, z, B, C, out and their gradients         */
  int32_t delta_softplus;
  int32_t reserved; /* 0 */
  int64_t u_n, u_d, delta_n, delta_d, z_n, z_d, dout_n, dout_d;
  int64_t B_n, B_g, B_s, C_n, C_g, C_s;
  const void *u, *delta, *z; /* [N, D, L]; z may be null                  */
  const float* A;            /* [D, S]; -infinity: no memory, but over dt = 0 */
  const void *B, *C;         /* [N, G, S, L]                              */
  const float* Dskip;        /* [D] or null                               */
  const float* delta_bias;   /* [D] or null                               */
  const float* initial_state; /* [N, D, S] or null                        */
  const int32_t* lengths;     /* [N] or null                              */
  void* out;                  /* [N, D, L]                    (fwd, step) */
  float* final_state;         /* [N, D, S] or null            (fwd, step) */
  /* States before every SEQ_SCAN_CHUNK-th step, for the backward call:
   * [N, ceil(L / SEQ_SCAN_CHUNK), D, S], written by fwd if not null,
   * required by bwd.  Those behind a sequence's end are not written. */
  float* checkpoints;
  const void* dout;           /* [N, D, L]                          (bwd) */
  const float* dfinal_state;  /* [N, D, S] or null                  (bwd) */
  void *du, *ddelta, *dz;     /* [N, D, L]; dz iff z                (bwd) */
  float* dA;                  /* [D, S]                             (bwd) */
  void *dB, *dC;              /* [N, G, S, L]                       (bwd) */
  float* dDskip;              /* [D], required iff Dskip            (bwd) */
  float* ddelta_bias;         /* [D], required iff delta_bias       (bwd) */
  float* dinitial_state;      /* [N, D, S] or null                  (bwd) */
  void* workspace;
  int64_t workspace_bytes;
} seq_scan_t;

int seq_selective_scan_fwd(const seq_scan_t* p, void* stream);
int64_t seq_selective_scan_fwd_workspace(const seq_scan_t* p);
int seq_selective_scan_bwd(const seq_scan_t* p, void* stream);
int64_t seq_selective_scan_bwd_workspace(const seq_scan_t* p);
/*
 * One token: L = 1; u, delta, z and out are [N, D], B and C [N, G, S] with
 * their state strides B_s and C_s.  initial_state and final_state are required
 * and may be the same memory.  No lengths, no checkpoints.
 */
int seq_selective_scan_step(const seq_scan_t* p, void* stream);

/*
 * Root-mean-square norms over the channels of each position [n, :, l];
 * rstd(v) = 1 / sqrt(mean_d v[d]^2 + eps).
 *
 *   before a block:  sum = residual + scale[d] x;  out = weight[d] sum rstd(sum)
 *   after a block:   v = x gate sigmoid(gate);
 *                    out = residual + scale[d] weight[d] v rstd(v)
 *
 * scale, residual and gate may each be null (one, zero, v = x).  The type of
 * residual, sum and their gradients (after a block: of out and dout, too) is
 * res_dtype: T or fp32.
 */
typedef struct {
  int32_t N, D, L;
  int32_t dtype, res_dtype;
  float eps;
  int64_t x_n, x_d, gate_n, gate_d, res_n, res_d, dout_n, dout_d, dsum_n, dsum_d;
  const void* x;
  const float* weight;  /* [D]                                            */
  const float* scale;   /* [D] or null                                    */
  const void* gate;     /* post: [N, D, L] or null                        */
  const void* residual; /* fwd: [N, D, L] or null                         */
  void* out;            /* fwd: [N, D, L], T (pre) or res_dtype (post)    */
  void* sum;            /* pre fwd: [N, D, L] res_dtype, may be null;
                           pre bwd: input, strides res_n and res_d        */
  const void* dout;     /* bwd: as out                                    */
  const void* dsum;     /* pre bwd: what came to sum from elsewhere, or null */
  void* dx;             /* bwd: [N, D, L]                                 */
  void* dgate;          /* post bwd: [N, D, L], iff gate                  */
  void* dresidual;      /* pre bwd: [N, D, L] res_dtype, or null (post: the
                           residual's gradient is dout itself)            */
  float* dweight;       /* bwd: [D]                                       */
  float* dscale;        /* bwd: [D], iff scale                            */
  void* workspace;
  int64_t workspace_bytes;
} seq_norm_t;

int seq_norm_pre_fwd(const seq_norm_t* p, void* stream);
/* From sum as the forward call stored it; x only where scale is given. */
int seq_norm_pre_bwd(const seq_norm_t* p, void* stream);
int seq_norm_post_fwd(const seq_norm_t* p, void* stream);
int seq_norm_post_bwd(const seq_norm_t* p, void* stream);
/* Bytes of workspace that either forward (backward) call needs, or a negative
 * status; they depend on the extents and types alone. */
int64_t seq_norm_fwd_workspace(const seq_norm_t* p);
int64_t seq_norm_bwd_workspace(const seq_norm_t* p);

#ifdef __cplusplus
}
#endif

#endif /* SEQ_OPS_H */
