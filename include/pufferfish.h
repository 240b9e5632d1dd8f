/*
 * pufferfish.h -- C ABI of the MI355X (gfx950) library for Pufferfish's
 * pre-factorized low-rank layers: forward and backward of a dense weight W
 * replaced by rank-r factors U V^T.
 *
 * General rules
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The layer
 *     entry points never allocate, free or synchronise; work is enqueued on
 *     `stream` (a hipStream_t passed as void*, NULL = the default stream).
 *     The one exception is the benchmark-only pf_timing_* group at the end of
 *     this file, which creates HIP events while enabled and waits for them in
 *     pf_timing_collect(); with timing disabled (the default) nothing of the
 *     kind happens.
 *   - Descriptors are small HOST structs passed by pointer.
 *   - Arrays are dense row-major, last index fastest.
 *   - `dtype` PF_F32: all tensors float.  PF_BF16: activations and factors are
 *     bfloat16, products accumulate in float, activation outputs (Y, dX, T_save)
 *     are rounded to bfloat16.  Parameter gradients (dU, dV, dbias, ...) are
 *     ALWAYS float: descriptors that carry a `wgrad_dtype` accept PF_F32 only.
 *   - Activations, factors, biases and saved tensors must be 16-byte aligned
 *     (any device allocation is); parameter-gradient outputs need only 4-byte
 *     alignment, so they may be slices of ONE flat float buffer laid out back
 *     to back -- the single all-reduce payload of the paper's Section 4
 *     ("implementation details").  Otherwise PF_ERR_UNSUPPORTED.
 *   - `accumulate` != 0 adds parameter gradients to what the buffers hold
 *     (gradient accumulation, back-propagation through time); 0 overwrites.
 *   - Scratch memory comes from the caller: ask pf_*_workspace_bytes(desc),
 *     pass at least that many bytes, 256-byte aligned (PF_ERR_UNSUPPORTED
 *     otherwise).  A NULL workspace is accepted when the query returns 0.
 *     The queries return 0 also for a descriptor the entry point would
 *     reject; the entry point then reports why.
 *   - Every call returns a pf_status.  Arguments are validated on the host
 *     before anything is launched: PF_ERR_NULL (a required pointer is NULL),
 *     PF_ERR_SHAPE (a dimension is not positive, or a convolution has no
 *     output pixel), PF_ERR_UNSUPPORTED (dtype/layout/groups value not built),
 *     PF_ERR_WORKSPACE (workspace too small or NULL), PF_ERR_LAUNCH (HIP
 *     reported an error; see pf_last_hip_error()).  A batch of zero rows
 *     (M, N or B equal to 0) is legal: activation outputs are empty and
 *     non-accumulated parameter gradients are set to zero.
 */
#ifndef PUFFERFISH_H
#define PUFFERFISH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PF_OK = 0,
    PF_ERR_NULL = 1,
    PF_ERR_SHAPE = 2,
    PF_ERR_UNSUPPORTED = 3,
    PF_ERR_WORKSPACE = 4,
    PF_ERR_LAUNCH = 5
} pf_status;

typedef enum { PF_F32 = 0, PF_BF16 = 1 } pf_dtype;
/* Activation layouts of the convolution entry points (only NCHW is built). */
typedef enum { PF_NCHW = 0, PF_NHWC = 1 } pf_layout;

const char *pf_status_string(int status);
/* hipError_t of the last failed launch on the calling thread (0 = none). */
int pf_last_hip_error(void);
/* Library version, major * 100 + minor. */
int pf_version(void);

/* ------------------------------------------------------------------ */
/* Fully connected layer (paper Section 2.1; Appendix B "FC layer";     */
/* Transformer projections and FFN matrices of Section 2.4 are this     */
/* layer with M = number of tokens).                                   */
/*   X[M x in], V[in x r] input-side factor, U[out x r] output-side     */
/*   factor, W = U V^T (out x in), T = X V (M x r), Y = T U^T + bias.   */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t M, in, out, r;
    int dtype;       /* pf_dtype */
    int wgrad_dtype; /* pf_dtype of dU, dV, dbias: PF_F32 (anything else: PF_ERR_UNSUPPORTED) */
    int has_bias;    /* bias[out] is read (fwd) / dbias[out] is written (bwd) */
} pf_linear_desc;

size_t pf_lowrank_linear_fwd_workspace_bytes(const pf_linear_desc *d);
size_t pf_lowrank_linear_bwd_workspace_bytes(const pf_linear_desc *d);

/* Y = (X V) U^T + bias.  T_save (nullable, [M x r], dtype) receives T for
 * the backward pass; when NULL, T never leaves the chip. */
int pf_lowrank_linear_fwd(const pf_linear_desc *d, const void *X, const void *V,
                          const void *U, const void *bias /* nullable */,
                          void *Y, void *T_save /* nullable */,
                          void *workspace, size_t workspace_bytes, void *stream);

/* Given dY[M x out]:  dT = dY U,  dX = dT V^T,  dU = dY^T T,  dV = X^T dT,
 * dbias = column sums of dY.  T_saved (nullable) is the forward pass's
 * T_save; when NULL, T is recomputed from X and V.  dX, dU, dV, dbias are
 * each nullable (skipped); dU, dV, dbias are float. */
int pf_lowrank_linear_bwd(const pf_linear_desc *d, const void *X, const void *V,
                          const void *U, const void *dY,
                          const void *T_saved /* nullable */,
                          void *dX, void *dU, void *dV, void *dbias,
                          int accumulate, void *workspace,
                          size_t workspace_bytes, void *stream);

/* For callers that cannot allocate device memory or hand over a         */
/* workspace (code running under HIP graph capture, tight serving        */
/* loops, harnesses that forbid hipMalloc): pf_lowrank_linear_bwd with   */
/* its scratch memory in a device array that is part of the library,     */
/* PF_STATIC_SCRATCH_BYTES per GPU, held until the process ends.  Same   */
/* arguments, results and errors as pf_lowrank_linear_bwd minus the      */
/* workspace; a descriptor whose pf_lowrank_linear_bwd_workspace_bytes   */
/* exceeds PF_STATIC_SCRATCH_BYTES gets PF_ERR_WORKSPACE.  The call      */
/* allocates and frees nothing.  All calls on one GPU share that GPU's   */
/* array: calls enqueued on one stream are ordered and safe, calls that  */
/* can overlap on one GPU (different streams, different threads) race.   */
#define PF_STATIC_SCRATCH_BYTES (40u << 20)
size_t pf_static_scratch_bytes(void);
int pf_lowrank_linear_bwd_static(const pf_linear_desc *d, const void *X,
                                 const void *V, const void *U, const void *dY,
                                 const void *T_saved /* nullable */, void *dX,
                                 void *dU, void *dV, void *dbias,
                                 int accumulate, void *stream);

/* ------------------------------------------------------------------ */
/* Several factorized projections of the same shape that read the SAME */
/* input, e.g. the query, key and value matrices of an attention block  */
/* (paper Section 2.4; each is the layer of Section 2.1):              */
/*   Y_g = (X V_g) U_g^T + bias_g,  g = 0 .. groups-1.                  */
/*   V[groups, in, r], U[groups, out, r], bias[groups, out],            */
/*   Y[groups, M, out], T_save[groups, M, r] (nullable).                */
/* Backward: dY[groups, M, out] gives dX = sum_g dY_g U_g V_g^T (ONE    */
/* tensor [M, in]: the input is shared) and dU, dV, dbias per group in  */
/* the layouts of U, V, bias (float; each nullable).  Results equal     */
/* those of `groups` calls of pf_lowrank_linear_fwd/bwd with the input   */
/* gradients added up; X and the running sum dX are read and written    */
/* once instead of once per projection.                                 */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t M, n_in, n_out, r;
    int groups; /* 1 .. 64 */
    int dtype;  /* pf_dtype */
    int has_bias;
} pf_linear_shared_desc;

size_t pf_lowrank_linear_shared_fwd_workspace_bytes(const pf_linear_shared_desc *d);
size_t pf_lowrank_linear_shared_bwd_workspace_bytes(const pf_linear_shared_desc *d);

int pf_lowrank_linear_shared_fwd(const pf_linear_shared_desc *d, const void *X,
                                 const void *V, const void *U,
                                 const void *bias /* nullable */, void *Y,
                                 void *T_save /* nullable */, void *workspace,
                                 size_t workspace_bytes, void *stream);

int pf_lowrank_linear_shared_bwd(const pf_linear_shared_desc *d, const void *X,
                                 const void *V, const void *U, const void *dY,
                                 const void *T_saved /* nullable */, void *dX,
                                 void *dU, void *dV, void *dbias, int accumulate,
                                 void *workspace, size_t workspace_bytes,
                                 void *stream);

/* ------------------------------------------------------------------ */
/* Convolution layer (paper Section 2.2 "Factorizing a convolution      */
/* layer"; Appendix B "Convolution layer").                            */
/*   X[N,Cin,H,W] (NCHW); Uk[r,Cin,k,k] = the r thin k x k basis        */
/*   filters (conv_u; stride and zero padding of the original layer);   */
/*   Vp[Cout,r] = the 1x1 convolution (conv_v; stride 1, no padding);   */
/*   T[N,r,Ho,Wo]; Y[N,Cout,Ho,Wo]; Ho = (H + 2 pad - k) / stride + 1.   */
/*   Cross-correlation (no kernel flip); nothing between the stages.    */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t N, Cin, H, W, Cout, r;
    int k, stride, pad;
    int layout;      /* pf_layout of X, T, Y and their gradients: PF_NCHW (anything else: PF_ERR_UNSUPPORTED) */
    int dtype;       /* pf_dtype */
    int wgrad_dtype; /* pf_dtype of dUk, dVp: PF_F32 (anything else: PF_ERR_UNSUPPORTED) */
} pf_conv_desc;

size_t pf_lowrank_conv_fwd_workspace_bytes(const pf_conv_desc *d);
size_t pf_lowrank_conv_bwd_workspace_bytes(const pf_conv_desc *d);

/* Bytes of the optional W_save buffer, in either dtype: the factors that the
 * backward pass's kernels read re-ordered (0 when they read them in place). */
size_t pf_lowrank_conv_saved_weights_bytes(const pf_conv_desc *d);

/* T = Uk * X (k x k, stride, pad), Y = Vp * T (1x1).  T_save nullable.
 * W_save (nullable, pf_lowrank_conv_saved_weights_bytes(d) bytes): like T_save a
 * tensor kept for the backward pass -- the forward call's weight re-ordering
 * launch fills it, and a backward call that is handed it (with Uk, Vp
 * unchanged in between) skips its own re-ordering launch. */
int pf_lowrank_conv_fwd(const pf_conv_desc *d, const void *X, const void *Uk,
                        const void *Vp, void *Y, void *T_save /* nullable */,
                        void *W_save /* nullable */,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Given dY[N,Cout,Ho,Wo]:  dT = Vp^T dY (1x1),  dVp[o,q] = sum dY T,
 * dX = transposed k x k convolution of dT with Uk,
 * dUk[q,c,i,j] = sum dT[n,q,y,x] Xpad[n,c,y s+i-p,x s+j-p].
 * T_saved nullable (recomputed); W_saved nullable (the forward call's W_save).
 * dX, dUk, dVp each nullable; dUk, dVp float. */
int pf_lowrank_conv_bwd(const pf_conv_desc *d, const void *X, const void *Uk,
                        const void *Vp, const void *dY,
                        const void *T_saved /* nullable */,
                        const void *W_saved /* nullable */, void *dX,
                        void *dUk, void *dVp, int accumulate, void *workspace,
                        size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* Layer epilogues: what the paper's models put directly after a        */
/* factorized layer, applied where the layer's output is formed, and    */
/* the matching step of the backward pass.                              */
/*                                                                      */
/* Linear (Section 2.4: FFN(x) = max(0, x W1 + b1) W2 + b2; each        */
/* sub-layer of a Transformer block sits inside a residual connection): */
/*   Z = (X V) U^T + bias + residual,   Y = act(Z)                      */
/*   residual: nullable, [M x out] in dtype.  act: pf_activation.       */
/* Backward takes dZ = dL/dZ where pf_lowrank_linear_bwd takes dY (for  */
/* PF_ACT_NONE they are the same tensor; a residual input receives dZ   */
/* as it is) and forms the gradient the layer BELOW needs:              */
/*   dX = (dZ U V^T + dX_add) * [X > 0]                                 */
/*   dX_add: nullable [M x in] (the gradient arriving over a skip       */
/*   connection that branches off X); the mask only when x_is_relu != 0 */
/*   (X is the output of a ReLU: dX is then dL/dZ of the layer below).  */
/*   dU, dV, dbias as in pf_lowrank_linear_bwd with dY = dZ.            */
/*                                                                      */
/* Convolution (Appendix D: a batch-norm layer after every convolution, */
/* ReLU after it, the shortcut of a ResNet block added before the last  */
/* ReLU), with the statistics fixed (running mean and variance): the    */
/* normalisation is then a per-channel scale and shift,                 */
/*   scale = gamma / sqrt(var + eps), shift = beta - mean * scale:      */
/*   Z[n,o,y,x] = scale[o] (Vp * (Uk * X))[n,o,y,x] + shift[o] + R,     */
/*   Y = act(Z);  scale, shift: float[Cout], each nullable (1 and 0).   */
/* Backward from dZ:  dP = scale dZ, dT = Vp^T dP, dVp = dP T^T,        */
/*   dshift[o] = sum over n,y,x of dZ (float[Cout], nullable),          */
/*   dX = (transposed convolution of dT + dX_add) * [X > 0].            */
/* The scale is a constant here and has no gradient.  A W_saved handed */
/* to the backward call must come from pf_lowrank_conv_fwd_ep called   */
/* with the same scale (the saved copy of the 1x1 filters carries it). */
/*                                                                      */
/* Workspace: the *_fwd_ep calls and pf_lowrank_linear_bwd_ep need what */
/* the plain calls need; pf_lowrank_conv_bwd_ep has its own query.      */
/* Errors as for the plain calls; an unknown act: PF_ERR_UNSUPPORTED.   */
/* ------------------------------------------------------------------ */
typedef enum { PF_ACT_NONE = 0, PF_ACT_RELU = 1 } pf_activation;

int pf_lowrank_linear_fwd_ep(const pf_linear_desc *d, const void *X, const void *V,
                             const void *U, const void *bias /* nullable */,
                             const void *residual /* nullable */, int act,
                             void *Y, void *T_save /* nullable */,
                             void *workspace, size_t workspace_bytes,
                             void *stream);
int pf_lowrank_linear_bwd_ep(const pf_linear_desc *d, const void *X, const void *V,
                             const void *U, const void *dZ,
                             const void *T_saved /* nullable */,
                             const void *dX_add /* nullable */, int x_is_relu,
                             void *dX, void *dU, void *dV, void *dbias,
                             int accumulate, void *workspace,
                             size_t workspace_bytes, void *stream);

size_t pf_lowrank_conv_bwd_ep_workspace_bytes(const pf_conv_desc *d);
int pf_lowrank_conv_fwd_ep(const pf_conv_desc *d, const void *X, const void *Uk,
                           const void *Vp, const void *scale /* nullable */,
                           const void *shift /* nullable */,
                           const void *residual /* nullable */, int act,
                           void *Y, void *T_save /* nullable */,
                           void *W_save /* nullable */, void *workspace,
                           size_t workspace_bytes, void *stream);
int pf_lowrank_conv_bwd_ep(const pf_conv_desc *d, const void *X, const void *Uk,
                           const void *Vp, const void *scale /* nullable */,
                           const void *dZ, const void *T_saved /* nullable */,
                           const void *W_saved /* nullable */,
                           const void *dX_add /* nullable */, int x_is_relu,
                           void *dX, void *dUk, void *dVp,
                           void *dshift /* nullable */, int accumulate,
                           void *workspace, size_t workspace_bytes,
                           void *stream);

/* ------------------------------------------------------------------ */
/* LSTM cell (paper Section 2.3, eq. (2); architecture table of the     */
/* low-rank LSTM in Appendix D).  One time step for a batch of B rows:  */
/*   Tx = x Vx, Th = h_prev Vh,                                        */
/*   z = Tx Ux^T + Th Uh^T + bias   (z[B x 4h], gate blocks i|f|g|o),   */
/*   i,f,o = sigmoid(z), g = tanh(z), c = f c_prev + i g, h = o tanh(c).*/
/*   groups == 4: one factor pair per gate, as eq. (2) has it:          */
/*     Vx[d_in x 4r], gate g reads columns g r..(g+1) r-1 of Tx;        */
/*   groups == 1: the stacked 4h x d_in matrix is one rank-r product:   */
/*     Vx[d_in x r] shared by the gates.                                */
/*   Ux, Uh are [4h x r] in both cases; bias[4h] is the sum of the      */
/*   equation's two bias vectors.  dtype must be PF_F32.                */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t B, d_in, h, r;
    int groups;   /* 1 or 4 */
    int dtype;    /* PF_F32 */
    int has_bias;
} pf_lstm_desc;

size_t pf_lowrank_lstm_cell_fwd_workspace_bytes(const pf_lstm_desc *d);
size_t pf_lowrank_lstm_cell_bwd_workspace_bytes(const pf_lstm_desc *d);

/* Outputs h_out[B x h], c_out[B x h]; saved for backward: gates_save[B x 4h]
 * (activated i|f|g|o), Tx_save, Th_save [B x groups r] -- all three required. */
int pf_lowrank_lstm_cell_fwd(const pf_lstm_desc *d, const void *x,
                             const void *h_prev, const void *c_prev,
                             const void *Vx, const void *Ux, const void *Vh,
                             const void *Uh, const void *bias /* nullable */,
                             void *h_out, void *c_out, void *gates_save,
                             void *Tx_save, void *Th_save, void *workspace,
                             size_t workspace_bytes, void *stream);

/* One step of back-propagation through time.  dh = dL/dh_t (from the layer
 * above plus from step t+1), dc_next = dL/dc_t from step t+1 (NULL = 0).
 * Outputs dx (nullable), dh_prev, dc_prev and the float parameter gradients
 * dVx, dUx, dVh, dUh, dbias (dbias nullable), overwritten or accumulated. */
int pf_lowrank_lstm_cell_bwd(const pf_lstm_desc *d, const void *x,
                             const void *h_prev, const void *c_prev,
                             const void *c_out, const void *gates_saved,
                             const void *Tx_saved, const void *Th_saved,
                             const void *Vx, const void *Ux, const void *Vh,
                             const void *Uh, const void *dh,
                             const void *dc_next /* nullable */,
                             void *dx /* nullable */, void *dh_prev,
                             void *dc_prev, void *dVx, void *dUx, void *dVh,
                             void *dUh, void *dbias /* nullable */,
                             int accumulate, void *workspace,
                             size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* Factorized LSTM layer over a whole sequence (Section 2.3, eq. (2)     */
/* applied for t = 0 .. T-1 with h_t, c_t fed to step t+1), fp32.       */
/* Same arithmetic as T calls of the cell; the input path x_t Vx Ux^T   */
/* does not depend on the recurrence and is computed for all time steps */
/* at once, and the parameter gradients are formed once over all steps. */
/*   x[T,B,d_in]; h0, c0 [B,h]; factors and bias as for the cell.       */
/* These run on the small-batch schedule of the stack entry points      */
/* below (a sequence is a stack of one layer) and share its limits:     */
/* B <= 32 and d_in, h, r >= 4, otherwise PF_ERR_UNSUPPORTED -- larger   */
/* batches go step by step through the cell entry points, which take    */
/* any B.                                                               */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t T, B, d_in, h, r;
    int groups;   /* 1 or 4 */
    int dtype;    /* PF_F32 */
    int has_bias;
} pf_lstm_seq_desc;

size_t pf_lowrank_lstm_seq_fwd_workspace_bytes(const pf_lstm_seq_desc *d);
size_t pf_lowrank_lstm_seq_bwd_workspace_bytes(const pf_lstm_seq_desc *d);

/* Outputs h_all, c_all [T,B,h] (h_all[t] = h_t); saved for backward:
 * gates_all[T,B,4h] (activated i|f|g|o), Tx_all, Th_all [T,B,groups r].  All
 * device pointers, all required (bias nullable); T == 0 or B == 0: nothing is
 * done.  Errors as for the cell, plus the limits stated above. */
int pf_lowrank_lstm_seq_fwd(const pf_lstm_seq_desc *d, const void *x,
                            const void *h0, const void *c0, const void *Vx,
                            const void *Ux, const void *Vh, const void *Uh,
                            const void *bias /* nullable */, void *h_all,
                            void *c_all, void *gates_all, void *Tx_all,
                            void *Th_all, void *workspace,
                            size_t workspace_bytes, void *stream);

/* Back-propagation through time.  dh_all[T,B,h] = dL/dh_t arriving from
 * above at every step; dhT, dcT [B,h] = gradients arriving at the final state
 * (NULL = 0).  Outputs dx_all[T,B,d_in] (nullable), dh0, dc0 [B,h] and the
 * float parameter gradients (dbias nullable), overwritten or accumulated. */
int pf_lowrank_lstm_seq_bwd(const pf_lstm_seq_desc *d, const void *x,
                            const void *h0, const void *c0, const void *h_all,
                            const void *c_all, const void *gates_all,
                            const void *Tx_all, const void *Th_all,
                            const void *Vx, const void *Ux, const void *Vh,
                            const void *Uh, const void *dh_all,
                            const void *dhT /* nullable */,
                            const void *dcT /* nullable */,
                            void *dx_all /* nullable */, void *dh0, void *dc0,
                            void *dVx, void *dUx, void *dVh, void *dUh,
                            void *dbias /* nullable */, int accumulate,
                            void *workspace, size_t workspace_bytes,
                            void *stream);

/* ------------------------------------------------------------------ */
/* A stack of `layers` factorized LSTM layers over a sequence (the      */
/* 2-layer language model of Appendix D; eq. (2) per layer, layer l > 0 */
/* reading h_all of layer l - 1).  The result is that of running        */
/* pf_lowrank_lstm_seq_* layer after layer; the steps are scheduled     */
/* along the diagonals l + t = const, which shortens the chain of       */
/* dependent launches from T * layers steps to T + layers - 1.          */
/* Layer 0 has d_in inputs, the others h; every layer has the same h, r */
/* and groups.  fp32, B <= 32, 1 <= layers <= 4, every extent >= 4.     */
/* Per-layer tensors are passed as HOST arrays of `layers` DEVICE       */
/* pointers (the arrays are read during the call only); shapes per      */
/* layer as for the sequence entry points.                              */
/* Where the factors fit the chip's registers the workgroups of one     */
/* cooperative launch run all steps and wait for one another.  The waits */
/* are bounded; should one ever run out (the call has returned by then, */
/* so no status can say so), every output not yet written is NaN.       */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t T, B, d_in, h, r;
    int groups;   /* 1 or 4 */
    int layers;   /* 1..4 */
    int dtype;    /* PF_F32 */
    int has_bias;
} pf_lstm_stack_desc;

size_t pf_lowrank_lstm_stack_fwd_workspace_bytes(const pf_lstm_stack_desc *d);
size_t pf_lowrank_lstm_stack_bwd_workspace_bytes(const pf_lstm_stack_desc *d);

/* x[T,B,d_in] device.  h0, c0, Vx, Ux, Vh, Uh, bias (array nullable when
 * has_bias == 0): inputs per layer; h_all, c_all, gates_all, Tx_all, Th_all:
 * outputs per layer (h_all[layers-1] is the output of the stack).  T == 0 or
 * B == 0: nothing is done.  Errors as for the cell. */
int pf_lowrank_lstm_stack_fwd(const pf_lstm_stack_desc *d, const void *x,
                              const void *const *h0, const void *const *c0,
                              const void *const *Vx, const void *const *Ux,
                              const void *const *Vh, const void *const *Uh,
                              const void *const *bias /* nullable */,
                              void *const *h_all, void *const *c_all,
                              void *const *gates_all, void *const *Tx_all,
                              void *const *Th_all, void *workspace,
                              size_t workspace_bytes, void *stream);

/* dh_top[T,B,h] = dL/dh_t of the LAST layer arriving from above at every
 * step; dhT, dcT (arrays and entries nullable = 0): gradients arriving at each
 * layer's final state.  Outputs: dx_all[T,B,d_in] (nullable), dh0, dc0 per
 * layer, and the float parameter gradients per layer (dbias array nullable),
 * overwritten or accumulated. */
int pf_lowrank_lstm_stack_bwd(const pf_lstm_stack_desc *d, const void *x,
                              const void *const *h0, const void *const *c0,
                              const void *const *h_all,
                              const void *const *c_all,
                              const void *const *gates_all,
                              const void *const *Tx_all,
                              const void *const *Th_all,
                              const void *const *Vx, const void *const *Ux,
                              const void *const *Vh, const void *const *Uh,
                              const void *dh_top,
                              const void *const *dhT /* nullable */,
                              const void *const *dcT /* nullable */,
                              void *dx_all /* nullable */, void *const *dh0,
                              void *const *dc0, void *const *dVx,
                              void *const *dUx, void *const *dVh,
                              void *const *dUh,
                              void *const *dbias /* nullable */,
                              int accumulate, void *workspace,
                              size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* What a Transformer layer has between its factorized projections      */
/* (paper Section 2.4): Y[groups, M, out] of pf_lowrank_linear_shared_*  */
/* holds queries, keys and values as [B, L, heads, head_dim] with        */
/* M = B L and out = heads head_dim; the calls below take them there,    */
/* and their backward calls write where pf_lowrank_linear_shared_bwd     */
/* reads dY.                                                            */
/*   Strides: these calls alone take tensors that are not dense.  A      */
/* stride triple holds the elements from one sequence, one token and one */
/* head to the next; the values of a head are adjacent.  Three zeros:    */
/* dense [B, L, heads, head_dim].  Otherwise every stride has to be a    */
/* multiple of 16 bytes and not negative (PF_ERR_UNSUPPORTED); the       */
/* strides of a tensor that is written must not make elements meet.      */
/* ------------------------------------------------------------------ */

/* ------------------------------------------------------------------ */
/* Norms of queries and keys for each head, with the position rotation  */
/* in the same pass.  For each head x of head_dim values:               */
/*   PF_NORM_RMS:  u = gamma x / sqrt(mean(x^2) + eps)                  */
/*   PF_NORM_NONE: u = x                                                */
/* then the first rot_dim values of u are turned in pairs: pair i of    */
/* rot_dim / 2 by the angle position * theta^(-2 i / rot_dim),           */
/*   y1 = u1 cos - u2 sin,  y2 = u1 sin + u2 cos;                       */
/* PF_ROT_HALVES pairs value i with i + rot_dim / 2, PF_ROT_PAIRS value  */
/* 2 i with 2 i + 1.  Angles are formed and reduced in double, so that   */
/* far positions are as exact as near ones.                             */
/*   Q[B, L, heads_q, head_dim], K[B, L, heads_k, head_dim] in dtype;    */
/*   gamma_q, gamma_k: float[head_dim], nullable (1);                    */
/*   positions: int32[B, L], nullable (token l of a sequence stands at l)*/
/* heads_k == 0: no keys, K and all that belongs to it are not touched.  */
/* head_dim: a multiple of 8, 8 .. 256; rot_dim: a multiple of 4,        */
/* 0 .. head_dim; B L heads < 2^30 (PF_ERR_UNSUPPORTED otherwise).       */
/* An output may be the input it belongs to (Qo: Q, dQ: Q or dQo, ..), at */
/* the same strides; other overlaps of outputs with inputs or each other  */
/* are refused (PF_ERR_UNSUPPORTED).                                      */
/* ------------------------------------------------------------------ */
typedef enum { PF_NORM_NONE = 0, PF_NORM_RMS = 1 } pf_norm;
typedef enum { PF_ROT_HALVES = 0, PF_ROT_PAIRS = 1 } pf_rotation;

typedef struct {
    int64_t B, L;
    int heads_q, heads_k, head_dim, rot_dim;
    int norm;     /* pf_norm */
    int rotation; /* pf_rotation */
    int dtype;    /* pf_dtype */
    float eps;
    double theta;
    int64_t q_stride[3], k_stride[3];   /* Q, K: sequence, token, head */
    int64_t qo_stride[3], ko_stride[3]; /* Qo, Ko (backward: dQo, dKo) */
    int64_t dq_stride[3], dk_stride[3]; /* dQ, dK */
} pf_qk_norm_desc;

/* Qo, Ko: the queries and keys that the attention reads. */
int pf_qk_norm_rotate_fwd(const pf_qk_norm_desc *d, const void *Q, const void *K,
                          const void *gamma_q /* nullable */,
                          const void *gamma_k /* nullable */,
                          const void *positions /* nullable */, void *Qo, void *Ko,
                          void *stream);

/* From dQo = dL/dQo, dKo = dL/dKo and the forward call's inputs: dQ, dK, and
 * dgamma_q, dgamma_k (float[head_dim], each nullable; overwritten or
 * accumulated; untouched with PF_NORM_NONE; at one address for both, for a
 * gamma that queries and keys share: their sum).  The same call gives the same
 * bits each time.  With PF_NORM_NONE Q and K are not read (nullable). */
size_t pf_qk_norm_rotate_bwd_workspace_bytes(const pf_qk_norm_desc *d);
int pf_qk_norm_rotate_bwd(const pf_qk_norm_desc *d, const void *Q, const void *K,
                          const void *gamma_q, const void *gamma_k,
                          const void *positions, const void *dQo, const void *dKo,
                          void *dQ, void *dK, void *dgamma_q, void *dgamma_k,
                          int accumulate, void *workspace, size_t workspace_bytes,
                          void *stream);

/* ------------------------------------------------------------------ */
/* Attention with a learned relative position bias by buckets.          */
/*   Q[B, Lq, heads_q, head_dim], K, V[B, Lk, heads_kv, head_dim];       */
/*   heads_q is a multiple of heads_kv, query head h reads key head      */
/*   h / (heads_q / heads_kv).  Query i of sequence b stands at position */
/*   p = q_start[b] + i, key j at position j.                            */
/*   S = scale q . k_j + table[bucket(j - p), h]                         */
/*   A query sees the keys j < kv_len[b], with `causal` those of them    */
/*   with j <= p.  O = softmax(S) V over what it sees,                   */
/*   lse[B, heads_q, Lq] (float, nullable) = log sum exp S.              */
/*   A query that sees nothing, and a query i >= q_len[b], has O = 0 and */
/*   lse = -infinity and takes no part in any gradient; what K and V hold */
/*   from kv_len[b] on, and Q and dO from q_len[b] on or of queries that */
/*   stand before the first key (causal), does not matter (not even NaN). */
/*   A key that a causal mask hides from some queries of a sequence and  */
/*   not from all has to be finite.                                      */
/*   q_start, q_len, kv_len: int32[B] on the device, each nullable       */
/*   (0, Lq, Lk); lengths are taken as within 0 .. Lq and 0 .. Lk,       */
/*   q_start as within -2^30 .. 2^30.                                    */
/* Buckets: table[buckets, heads_q] float; buckets == 0: no bias, table  */
/* unused.  With `bidirectional` keys after the query use the upper half */
/* of the buckets, else all of them bucket 0.  A side of nb buckets has  */
/* e = nb / 2 for the distances 0 .. e - 1 and the others spaced          */
/* logarithmically up to max_distance:                                   */
/*   bucket(n) = min(nb - 1, e + floor((nb - e) log(n/e) / log(max_distance/e))) */
/* for n >= e, with the borders where exact arithmetic has them.         */
/* Entries of the table may have any size, the type's lowest value and    */
/* -infinity among them: what all keys that a query sees have in common   */
/* costs its scores no digits (finite ones beyond 2.3e38 count as that).  */
/* Limits (PF_ERR_UNSUPPORTED): head_dim a multiple of 8, 8 .. 128;       */
/* buckets 0 or 2 .. 256, with bidirectional a multiple of 2 and >= 4;    */
/* max_distance > e and <= 1024; Lq, Lk < 2^29; launches of fewer than    */
/* 2^32 threads (about 2^24 tiles of 128 queries of a head, or of 64 keys  */
/* of a key head); less than 2^22 elements from one token to the next.    */
/* Lq == 0 or Lk == 0 is legal.  Outputs that overlap Q, K, V, O, dO, lse, */
/* the table or each other are refused (PF_ERR_UNSUPPORTED).              */
/* Sums are the same bits in every call of the same sizes.                */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t B, Lq, Lk;
    int heads_q, heads_kv, head_dim;
    int causal;
    int buckets, max_distance, bidirectional;
    int dtype; /* pf_dtype */
    float scale;
    int64_t q_stride[3], k_stride[3], v_stride[3]; /* Q, K, V: sequence, token, head */
} pf_attention_desc;

size_t pf_attention_fwd_workspace_bytes(const pf_attention_desc *d);
int pf_attention_fwd(const pf_attention_desc *d, const void *Q, const void *K,
                     const void *V, const void *table /* nullable */,
                     const void *q_start /* nullable */,
                     const void *q_len /* nullable */,
                     const void *kv_len /* nullable */, void *O,
                     void *lse /* nullable */, void *workspace,
                     size_t workspace_bytes, void *stream);

/* O, lse: the forward call's.  dQ, dK, dV in dtype, dense [B, L, heads,
 * head_dim] (gradients of a key head are summed over the query heads that
 * read it); dtable[buckets, heads_q] float, nullable, overwritten or
 * accumulated.  O and dO are dense. */
size_t pf_attention_bwd_workspace_bytes(const pf_attention_desc *d);
int pf_attention_bwd(const pf_attention_desc *d, const void *Q, const void *K,
                     const void *V, const void *table, const void *q_start,
                     const void *q_len, const void *kv_len, const void *O,
                     const void *lse, const void *dO, void *dQ, void *dK, void *dV,
                     void *dtable /* nullable */, int accumulate, void *workspace,
                     size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* One AdamW step over many tensors in one launch.  For each value:      */
/*   g = grad_scale grad                                                 */
/*   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2          */
/*   p = p (1 - lr weight_decay)                                         */
/*       - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)     */
/* t = steps + 1; the call stores t in `steps` (device int64).  lr and   */
/* grad_scale are device floats, so that a captured step follows a       */
/* schedule.                                                             */
/*   param, grad: float.  copy (nullable): the parameters rounded to     */
/*   bfloat16, as the layers above read them.                            */
/*   state_bits 32: m, v float.                                          */
/*   state_bits 8: every 256 consecutive values of a tensor (the last     */
/*   ones: fewer) share a scale; m holds e4m3 codes of m / m_scale, v     */
/*   those of sqrt(v) / v_scale (the root halves the range that a code    */
/*   has to span); m_scale, v_scale float[ceil(count / 256)] are powers   */
/*   of two, the smallest (from 2^-126) that keep the codes within 448.   */
/*   A root that is not zero is not held as zero.  The step itself uses   */
/*   m and v before they are rounded.  Values that are not finite are     */
/*   held as NaN and do not change the scale of the others.               */
/* Alignment: 4 bytes everywhere (copy: 2 bytes): slices of flat buffers  */
/* will do.  The tensors of a call must not overlap.                      */
/*                                                                       */
/* The addresses live in a plan: ask its size, let pf_adamw_plan_fill     */
/* write it to HOST memory, copy it to the device once (256-byte aligned),*/
/* and hand it to every step, with the size that was asked and the same   */
/* descriptor (a plan for states of other bits is refused).  A plan holds */
/* a counter of the launch that runs: steps of one plan must not overlap. */
/* ------------------------------------------------------------------ */
typedef struct {
    void *param;
    const void *grad;
    void *m, *v;
    void *m_scale, *v_scale; /* state_bits 8 */
    void *copy;              /* nullable */
    int64_t count;
    float weight_decay;
} pf_adamw_tensor;

typedef struct {
    int64_t tensors;
    int state_bits; /* 32 or 8 */
    double beta1, beta2, eps;
} pf_adamw_desc;

size_t pf_adamw_plan_bytes(const pf_adamw_desc *d, const pf_adamw_tensor *tensors);
int pf_adamw_plan_fill(const pf_adamw_desc *d, const pf_adamw_tensor *tensors,
                       void *plan_host, size_t plan_bytes);
int pf_adamw_step(const pf_adamw_desc *d, void *plan, size_t plan_bytes,
                  const void *lr, const void *grad_scale /* nullable: 1 */,
                  void *steps, void *stream);

/* ------------------------------------------------------------------ */
/* Truncated-SVD factor initialisation (Algorithm 1, the step before    */
/* the factorized layers are trained): W[m x n] (fp32, row-major) ->    */
/*   U[m x r] = Ut_r S_r^(1/2),  V[n x r] = Vt_r S_r^(1/2)  (fp32),     */
/* so that U V^T is the best rank-r approximation of W; sigma (nullable)*/
/* receives all min(m, n) singular values in descending order.          */
/* One-sided Jacobi in double precision; factors are unique only up to  */
/* the sign of each column pair.  r <= min(m, n) <= 8192 (else          */
/* PF_ERR_SHAPE / PF_ERR_UNSUPPORTED).  For a convolution unroll        */
/* W[c_out, c_in, k, k] to [c_in k^2, c_out] first (Section 2.2).       */
/* Sweeps stop once a whole sweep found every column pair orthogonal to */
/* max(m,n) * 2^-52 relative (the rounding level of the inner products; */
/* at least 1e-15); at most 40 sweeps run.                              */
/* The call is asynchronous, so convergence cannot                      */
/* come back in the status: info (nullable, DEVICE int[2]) receives     */
/* info[0] = sweeps over the columns of W that ran (they start from a   */
/* preconditioned basis, whose own sweeps are not counted; checking it  */
/* is the first), info[1] = rotations applied in the last               */
/* of them -- 0 means converged; anything else means the 40 sweeps did  */
/* not suffice and the factors are approximate, or that W holds NaN or  */
/* infinity, which then show in the outputs.  (The workgroups wait      */
/* for one another in bounded waits; should one ever run out, all       */
/* outputs are NaN and info[1] is not 0.)                               */
/* ------------------------------------------------------------------ */
typedef struct {
    int64_t m, n, r;
} pf_svd_desc;

size_t pf_svd_split_workspace_bytes(const pf_svd_desc *d);
int pf_svd_split(const pf_svd_desc *d, const void *W, void *U, void *V,
                 void *sigma /* nullable */, void *info /* nullable */,
                 void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* Dense (un-factorized) comparators, for benchmarks only: the layers   */
/* of Section 2.1 / 2.2 before factorization, on the same tiling code.  */
/*   linear: W[out x in];  conv: Wd[Cout,Cin,k,k].                      */
/* ------------------------------------------------------------------ */
size_t pf_dense_linear_workspace_bytes(const pf_linear_desc *d);
int pf_dense_linear_fwd(const pf_linear_desc *d, const void *X, const void *W,
                        const void *bias, void *Y, void *workspace,
                        size_t workspace_bytes, void *stream);
int pf_dense_linear_bwd(const pf_linear_desc *d, const void *X, const void *W,
                        const void *dY, void *dX, void *dW, void *dbias,
                        int accumulate, void *workspace, size_t workspace_bytes,
                        void *stream);
size_t pf_dense_conv_workspace_bytes(const pf_conv_desc *d);
int pf_dense_conv_fwd(const pf_conv_desc *d, const void *X, const void *Wd,
                      void *Y, void *workspace, size_t workspace_bytes,
                      void *stream);
int pf_dense_conv_bwd(const pf_conv_desc *d, const void *X, const void *Wd,
                      const void *dY, void *dX, void *dWd, int accumulate,
                      void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------ */
/* Per-kernel timing (HIP events recorded around every kernel launch on */
/* the launch stream while enabled).  Not thread-safe; for benchmarks.  */
/* While enabled every launch creates two hipEvents (host objects), so  */
/* do not enable it under stream capture; pf_timing_collect() blocks    */
/* the calling thread until the recorded events have completed.         */
/* ------------------------------------------------------------------ */
void pf_timing_enable(int on);
/* Synchronises the recorded events, adds them to the totals and returns the
 * number of distinct kernels seen so far. */
int pf_timing_collect(void);
/* Entry i of the totals: name (static string), launches, total milliseconds. */
int pf_timing_entry(int i, const char **name, int64_t *launches, double *total_ms);
void pf_timing_reset(void);

#ifdef __cplusplus
}
#endif
#endif /* PUFFERFISH_H */
