/*
 * mxc.h -- C ABI of the MI355X (gfx950) conv2d library.
 *
 * The three compute calls are the convolution layer of the MXNet paper: the
 * hand-optimised "big" operator of Section 3.1 (Graph Optimization), whose
 * forward and backward evaluation Section 2.1 describes and whose kernels
 * Section 4 ("Raw performance") reports as taking most of the run time of the
 * CNN benchmarks.  The paper prints no formula; the definitions below are the
 * ones this library implements.
 *
 * Notation.  x[N,C,H,W] input, w[K,C,R,S] filter, y/dy[N,K,P,Q] output and its
 * gradient, with
 *     P = floor((H + 2*pad - R)/stride) + 1,  Q = floor((W + 2*pad - S)/stride) + 1.
 * One stride and one pad serve both axes; dilation 1, groups 1, no bias in the three plain calls;
 * cross-correlation (no filter flip); x outside the image reads as 0.
 * Infinities and NaN: in fp32, and in the gradients of bf16 layers whose K is no multiple of 8, a tap outside the image
 * is left out of the sum whatever the other operand holds.  Every other bf16 call may multiply padding, and the places
 * that the packings of first layers (C <= 4) leave empty, as zeros: there an infinite or NaN element of one operand
 * makes NaN of the results in whose window, or packed block, it meets such a place.  Whether it does depends on the
 * kernel that runs the layer, and so on its sizes (backward-data of first layers at stride 1 has one of either kind).
 * A ReLU makes 0 of a NaN in fp32; in bf16 it makes 0 or, where the NaN has no sign, leaves it, by kernel again.
 * Finite inputs are not affected.
 *
 * Common rules for every call.
 *   - All data pointers are DEVICE pointers on the current HIP device, 16-byte
 *     aligned, owned by the caller; the library allocates no device memory,
 *     never synchronises and never changes the current device.
 *   - Work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  Calls return as soon as the launches are queued.
 *   - `dtype` is the element type of x, w, y, dy, dx: MXC_F32, or MXC_BF16
 *     (bf16 storage, fp32 accumulation, results rounded to nearest-even).
 *     dw is fp32 for both dtypes (mxc_conv2d_bwd_weight_bf16 and the prepared-input
 *     form with dw_dtype MXC_BF16 round that fp32 sum once to bf16).
 *   - `layout` says how the caller's tensors are stored:
 *       MXC_NCHW: x[N][C][H][W], w/dw[K][C][R][S], y/dy[N][K][P][Q]
 *       MXC_NHWC: x[N][H][W][C], w/dw[K][R][S][C], y/dy[N][P][Q][K]
 *     all dense.  Kernels work in NHWC/KRSC; NCHW tensors are converted through
 *     the workspace.
 *   - Outputs are fully overwritten (no accumulation into them).
 *   - `workspace` is scratch memory of at least the size reported by
 *     mxc_conv2d_workspace_bytes for the same arguments (may be NULL when that
 *     size is 0).  Its contents are undefined afterwards.  Two calls that share
 *     a workspace must be ordered on one stream.
 *   - Return value: MXC_OK or an error code.  Argument errors (every code but
 *     MXC_ERR_LAUNCH) are found before anything is launched; after MXC_ERR_LAUNCH
 *     some of the call's kernels may already be queued and the output is undefined.
 *     No call throws, aborts or exits.  Shapes are checked before pointers.
 */
#ifndef MXC_H
#define MXC_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MXC_OK = 0,
    MXC_ERR_NULL = 1,        /* a required pointer is NULL                         */
    MXC_ERR_SHAPE = 2,       /* non-positive dim/stride, negative pad, empty output */
    MXC_ERR_UNSUPPORTED = 3, /* unknown dtype / layout / pass                       */
    MXC_ERR_WORKSPACE = 4,   /* workspace missing or smaller than required          */
    MXC_ERR_ALIGN = 5,       /* a pointer is not 16-byte aligned                    */
    MXC_ERR_LAUNCH = 6       /* the HIP runtime rejected a kernel launch            */
};

enum { MXC_F32 = 0, MXC_BF16 = 1 };
enum { MXC_NCHW = 0, MXC_NHWC = 1 };
enum { MXC_FWD = 0, MXC_BWD_DATA = 1, MXC_BWD_WEIGHT = 2,
       /* the following: mxc_conv2d_workspace_bytes only */
       MXC_BWD_DATA_RELU = 3, MXC_BIAS_GRAD = 4,
       MXC_BWD_DATA_FILTER = 5,          /* bytes of the prepared filter of mxc_conv2d_bwd_data_prepare_filter */
       MXC_BWD_DATA_PREPARED = 6,        /* workspace of mxc_conv2d_bwd_data_prepared without x_mask           */
       MXC_BWD_DATA_PREPARED_RELU = 7,   /* ... with x_mask                                                     */
       MXC_BWD_WEIGHT_BF16 = 8,          /* workspace of mxc_conv2d_bwd_weight_bf16                             */
       MXC_INPUT_PREPARED = 9,           /* bytes of the prepared input of mxc_conv2d_prepare_input (0: none)   */
       MXC_FWD_PREPARED_INPUT = 10,      /* workspace of mxc_conv2d_fwd_prepared_input                          */
       MXC_BWD_WEIGHT_PREPARED_INPUT = 11,       /* workspace of mxc_conv2d_bwd_weight_prepared_input, fp32 dw  */
       MXC_BWD_WEIGHT_PREPARED_INPUT_BF16 = 12,  /* ... bf16 dw                                                 */
       MXC_FWD_TRANSFORM = 13 };         /* workspace of mxc_conv2d_fwd_transform                               */

/*
 * Forward (the layer's "forward" evaluation, paper Section 2.1):
 *   y[n,k,p,q] = sum_{c,r,s} x[n,c,p*stride-pad+r,q*stride-pad+s] * w[k,c,r,s]
 * x, w: inputs; y: output (N*K*P*Q elements of `dtype`).
 */
int mxc_conv2d_fwd(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                   int dtype, int layout,
                   const void *x, const void *w, void *y,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward w.r.t. the input (derivative of forward in x; paper Section 2.1,
 * "backward"):
 *   dx[n,c,h,v] = sum over (k,r,s) such that p=(h+pad-r)/stride and
 *                 q=(v+pad-s)/stride are integers inside the output,
 *                 of dy[n,k,p,q] * w[k,c,r,s].
 * Every element of dx is written; positions no filter tap reaches get 0.
 * dy, w: inputs; dx: output (N*C*H*W elements of `dtype`).
 */
int mxc_conv2d_bwd_data(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                        int dtype, int layout,
                        const void *dy, const void *w, void *dx,
                        void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward w.r.t. the filter (derivative of forward in w; the gradient that the
 * paper's update step w -= eta*g of Section 2.2 consumes):
 *   dw[k,c,r,s] = sum_{n,p,q} dy[n,k,p,q] * x[n,c,p*stride-pad+r,q*stride-pad+s]
 * x, dy: inputs of `dtype`; dw: output, K*C*R*S fp32 values in the filter order
 * of `layout`.  The reduction is split across workgroups and summed in a fixed
 * order: results are bit-identical from run to run.
 */
int mxc_conv2d_bwd_weight(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                          int dtype, int layout,
                          const void *x, const void *dy, void *dw,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward w.r.t. the filter with the gradient delivered in bf16: the same sums as mxc_conv2d_bwd_weight
 * (fp32 accumulation, fp32 split partial sums added in a fixed order), rounded ONCE to bf16 (nearest even) by
 * the kernel that forms the final sum - for a gradient exchange or an optimizer that takes bf16 (half the bytes
 * of the push of paper Section 2.3).  dtype must be MXC_BF16 (else MXC_ERR_UNSUPPORTED); dw: K*C*R*S bf16
 * values in the filter order of `layout`.  Workspace: query MXC_BWD_WEIGHT_BF16.  Otherwise as
 * mxc_conv2d_bwd_weight.
 */
int mxc_conv2d_bwd_weight_bf16(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                               int dtype, int layout,
                               const void *x, const void *dy, void *dw,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * mxc_conv2d_bwd_weight for callers that cannot allocate device memory or hand over a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * computation, kernels and results as mxc_conv2d_bwd_weight, with the split-reduction partial sums
 * (and, for MXC_NCHW, the converted operands) held in a 64 MiB array that is part of the library's
 * device code - one copy per GPU, kept until the process ends.  The call allocates nothing.  x, dy,
 * dw as in mxc_conv2d_bwd_weight, still caller-owned.
 *   - Problems whose scratch need (what mxc_conv2d_workspace_bytes reports for MXC_BWD_WEIGHT)
 *     exceeds 64 MiB are rejected with MXC_ERR_WORKSPACE before anything is launched.
 *   - All calls on one GPU share that GPU's array: calls that may overlap on one GPU (different
 *     streams, or several host threads) race on it; order them on one stream.  The array keeps the
 *     last call's contents; no call depends on them.
 *   - The first call on a device looks up the array's device address (hipGetSymbolAddress): make
 *     that call outside any stream capture.  If the lookup fails: MXC_ERR_LAUNCH, nothing launched.
 * Other errors as mxc_conv2d_bwd_weight.
 */
int mxc_conv2d_bwd_weight_static(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                                 int dtype, int layout,
                                 const void *x, const void *dy, void *dw, void *hip_stream);

/*
 * Convolution grouped with the operations that follow it (the paper groups operators into a
 * single call where it can, Section 3.1 "Graph Optimization", and chains layers as
 * layer => Activation(relu) => layer, Section 2.1):
 *   y[n,k,p,q] = act( forward(x, w)[n,k,p,q] + bias[k] ),   act(t) = max(0, t) if relu == 1, t if relu == 0.
 * bias: K fp32 values in device memory (4-byte aligned), or NULL for no bias.  The sum is formed
 * in fp32 and rounded once to `dtype`.  Everything else (layouts, workspace = that of MXC_FWD,
 * ownership, errors) as mxc_conv2d_fwd; relu outside {0,1}: MXC_ERR_UNSUPPORTED.
 */
int mxc_conv2d_fwd_bias_act(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                            int dtype, int layout,
                            const void *x, const void *w, const float *bias, int relu, void *y,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward w.r.t. the input, grouped with the derivative of the ReLU that produced the input:
 * with x = max(0, z) the output of the layer below,
 *   dz[n,c,h,v] = backward_data(dy, w)[n,c,h,v]  if x[n,c,h,v] > 0,  else 0
 * (the derivative of max(0, .) at 0 is taken as 0).  x: N*C*H*W elements of `dtype` in `layout`
 * (read only); dz is written to dx.  Workspace: query with pass MXC_BWD_DATA_RELU.  Otherwise as
 * mxc_conv2d_bwd_data.
 */
int mxc_conv2d_bwd_data_relu(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                             int dtype, int layout,
                             const void *dy, const void *w, const void *x, void *dx,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward w.r.t. the input with the filter prepared ahead of time.  Every backward-data path first brings
 * the filter into the form its kernels read (re-packed per stride residue class, transposed, ...): work that
 * depends on w alone.  A training loop changes w once per step (the update of Section 2.2), serving never:
 *   mxc_conv2d_bwd_data_prepare_filter  writes that form of w into w_prepared (device memory of the caller, at
 *       least mxc_conv2d_workspace_bytes(MXC_BWD_DATA_FILTER, ...) bytes, 16-byte aligned; opaque contents, valid
 *       for exactly these N..pad, dtype and layout until w changes);
 *   mxc_conv2d_bwd_data_prepared        is mxc_conv2d_bwd_data (x_mask == NULL) or mxc_conv2d_bwd_data_relu
 *       (x_mask = the layer's input) reading w_prepared instead of w; same results bit for bit.  Workspace:
 *       query MXC_BWD_DATA_PREPARED / MXC_BWD_DATA_PREPARED_RELU.
 * prepared_bytes: size of the w_prepared buffer (checked against the required size: MXC_ERR_WORKSPACE).
 * Everything else as mxc_conv2d_bwd_data.
 */
int mxc_conv2d_bwd_data_prepare_filter(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                                       int dtype, int layout,
                                       const void *w, void *w_prepared, size_t prepared_bytes, void *hip_stream);
int mxc_conv2d_bwd_data_prepared(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                                 int dtype, int layout,
                                 const void *dy, const void *w_prepared, size_t prepared_bytes, const void *x_mask, void *dx,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Forward and backward-weight on an input prepared once.  Layers whose channel count is not a multiple of 8
 * (the first layer of every network of Section 4: C = 3) first bring x into the form their kernels read -
 * space-to-depth packed for strided filters, zero-bordered with 4 channels per pixel, or channel-padded -
 * and both passes of a training step (Section 2.1: forward, then the gradient of the weights) read the same
 * form of the same x:
 *   mxc_conv2d_prepare_input             writes that form into x_prepared (device memory of the caller, at least
 *       mxc_conv2d_workspace_bytes(MXC_INPUT_PREPARED, ...) bytes, 16-byte aligned; opaque contents, valid for
 *       exactly these N..pad, dtype and layout until x changes).  A layer that reads x as it is has 0 bytes:
 *       the call does nothing (x_prepared may be NULL) and the two calls below take x itself as x_prepared;
 *   mxc_conv2d_fwd_prepared_input        is mxc_conv2d_fwd_bias_act (bias may be NULL, relu 0 or 1) reading
 *       x_prepared; same results bit for bit.  Workspace: query MXC_FWD_PREPARED_INPUT;
 *   mxc_conv2d_bwd_weight_prepared_input is mxc_conv2d_bwd_weight (dw_dtype MXC_F32) or mxc_conv2d_bwd_weight_bf16
 *       (dw_dtype MXC_BF16) reading x_prepared; same results bit for bit.  Workspace: query
 *       MXC_BWD_WEIGHT_PREPARED_INPUT / MXC_BWD_WEIGHT_PREPARED_INPUT_BF16.
 * layout must be MXC_NHWC (MXC_ERR_UNSUPPORTED otherwise: the NCHW boundary converts every operand per call).
 * prepared_bytes: size of the x_prepared buffer (checked: MXC_ERR_WORKSPACE).  Everything else as the calls named.
 */
int mxc_conv2d_prepare_input(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                             int dtype, int layout,
                             const void *x, void *x_prepared, size_t prepared_bytes, void *hip_stream);
int mxc_conv2d_fwd_prepared_input(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                                  int dtype, int layout,
                                  const void *x_prepared, size_t prepared_bytes, const void *w, const float *bias, int relu,
                                  void *y, void *workspace, size_t workspace_bytes, void *hip_stream);
int mxc_conv2d_bwd_weight_prepared_input(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                                         int dtype, int layout,
                                         const void *x_prepared, size_t prepared_bytes, const void *dy, void *dw, int dw_dtype,
                                         void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Forward by another algorithm: the 3x3 stride-1 convolution evaluated in a transform domain (minimal filtering,
 * 2x2 output blocks from 4x4 input patches: 16 multiplications per channel and block instead of 36), the same
 * y = act(conv(x, w) + bias) as mxc_conv2d_fwd_bias_act (Section 2.1; one of the hand-optimised "big" operators
 * of Section 3.1).  Filter and input are transformed, rounded once to bf16 and multiplied on the matrix cores as
 * 16 independent GEMMs with fp32 sums; the result is transformed back and rounded once.  Its error is therefore
 * not that of the direct form: |y - exact| <= 2^-8 * W + 2^-8 * |exact|, W = the sum, over the transform-domain
 * entries a result combines, of sum_c |U||V| (U, V the transformed filter and input); for the layers of the
 * benchmark stacks that is well inside 1e-2 of sum |x||w|.
 * Only R = S = 3, stride = 1, dtype MXC_BF16, layout MXC_NHWC, C % 8 == 0 and K % 8 == 0 (MXC_ERR_UNSUPPORTED
 * otherwise; callers fall back to mxc_conv2d_fwd_bias_act).  bias may be NULL, relu is 0 or 1.  Workspace: query
 * MXC_FWD_TRANSFORM (16 transformed copies of the tiled input in bf16 and of the output in fp32: large).
 * Everything else as mxc_conv2d_fwd.
 */
int mxc_conv2d_fwd_transform(int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                             int dtype, int layout,
                             const void *x, const void *w, const float *bias, int relu, void *y,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Gradient of the bias of mxc_conv2d_fwd_bias_act (derivative of forward + bias[k] in bias):
 *   db[k] = sum_{n,p,q} dy[n,k,p,q]
 * dy: N*K*P*Q elements of `dtype` in `layout` (NCHW: [N][K][P][Q]; NHWC: [N][P][Q][K]); db: K fp32
 * values.  Summed in a fixed order (bit-identical from run to run).  Workspace: query
 * mxc_conv2d_workspace_bytes with pass MXC_BIAS_GRAD (only N, K, P, Q matter: pass the layer's
 * shape).  Errors: MXC_ERR_SHAPE, MXC_ERR_UNSUPPORTED, MXC_ERR_NULL, MXC_ERR_ALIGN,
 * MXC_ERR_WORKSPACE, MXC_ERR_LAUNCH.
 */
int mxc_bias_grad(int N, int K, int P, int Q, int dtype, int layout,
                  const void *dy, float *db,
                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * FullyConnected (the layer of the paper's running example, Section 2.1), run through the same
 * matrix-core GEMM as the convolutions: it is the convolution with H = W = R = S = 1, for which NCHW
 * and NHWC coincide.  x: [N][C], w: [K][C], y / dy: [N][K], all of `dtype`; dw: [K][C] fp32.
 *   forward:         y[n,k]  = act( sum_c x[n,c] * w[k,c] + bias[k] )     (bias may be NULL; relu 0 or 1)
 *   backward-data:   dx[n,c] = sum_k dy[n,k] * w[k,c],  set to 0 where x_mask[n,c] <= 0 if x_mask != NULL
 *                    (x_mask: the layer's input when that is a ReLU output)
 *   backward-weight: dw[k,c] = sum_n dy[n,k] * x[n,c]
 * Problems of a few hundred rows split their long reduction over workgroups (fp32 partial sums added
 * in a fixed order: deterministic).  Workspace: mxc_conv2d_workspace_bytes(pass, N, C, 1, 1, K, 1, 1,
 * 1, 0, dtype, MXC_NHWC, ...) with pass MXC_FWD, MXC_BWD_DATA_RELU (with or without mask) or
 * MXC_BWD_WEIGHT.  Ownership, stream and error behaviour as the convolution entry points.
 */
int mxc_fc_fwd(int N, int C, int K, int dtype, const void *x, const void *w, const float *bias, int relu, void *y,
               void *workspace, size_t workspace_bytes, void *hip_stream);
int mxc_fc_bwd_data(int N, int C, int K, int dtype, const void *dy, const void *w, const void *x_mask, void *dx,
                    void *workspace, size_t workspace_bytes, void *hip_stream);
int mxc_fc_bwd_weight(int N, int C, int K, int dtype, const void *x, const void *dy, void *dw,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Softmax output layer (the last layer of the paper's running example, Section 2.1).
 *   forward:   p[n,k] = exp(z[n,k] - max_j z[n,j]) / sum_j exp(z[n,j] - max_j z[n,j])      z, p: [N][K] of `dtype`
 *   backward:  dz[n,k] = (p[n,k] - (k == labels[n])) * scale        the gradient of the cross-entropy against integer
 *              labels (device int32, values in [0, K); a value outside selects no class), times `scale` (e.g. 1/N)
 * Arithmetic in fp32, one rounding to `dtype`.  No workspace.  Errors: MXC_ERR_SHAPE, MXC_ERR_UNSUPPORTED,
 * MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes for tensors, 4 for labels), MXC_ERR_LAUNCH.
 */
int mxc_softmax_fwd(int N, int K, int dtype, const void *z, void *p, void *hip_stream);
int mxc_softmax_xent_bwd(int N, int K, int dtype, const void *p, const int *labels, float scale, void *dz, void *hip_stream);

/*
 * The weight update that consumes dw (the paper's  w = w - eta*g  of Section 2.2, with the
 * momentum and weight decay of its Section 4 experiment; the paper does not print the momentum
 * form, the classic one is used):
 *   v'[i] = momentum*v[i] - lr*(g[i] + wd*w[i]),   w'[i] = w[i] + v'[i],   i < n
 * w: fp32 master weights, updated in place; g: fp32 gradient (mxc_conv2d_bwd_weight's dw, same
 * element order as w); v: fp32 velocity, updated in place, or NULL when momentum == 0 (then
 * v = 0 is used and nothing is stored); w_bf16: if not NULL, receives w' rounded to bf16 (nearest
 * even) for the next forward pass.  All device pointers, 16-byte aligned, caller-owned; n > 0.
 * Errors: MXC_ERR_SHAPE (n == 0 or too large for one launch), MXC_ERR_NULL (w or g NULL, or v NULL
 * with momentum != 0), MXC_ERR_ALIGN, MXC_ERR_LAUNCH.
 */
int mxc_sgd_update(size_t n, float *w, const float *g, float *v, void *w_bf16,
                   float lr, float momentum, float wd, void *hip_stream);

/*
 * Log probabilities of given tokens (or classes) under softmax(scale * z), with the entropy of every row, its most
 * probable tokens, and the gradient of a weighted sum of the log probabilities and entropies.  z: [N] rows of K
 * logits of `dtype`, `ld` elements from one row to the next (ld >= K; the ld - K between two rows are neither read
 * nor written).  With d[k] = scale*(z[n,k] - max_j z[n,j]), S = sum_k exp(d[k]), T = sum_k exp(d[k])*d[k], p = exp(d)/S:
 *   logp[n]    = d[labels[n]] - log S          entropy[n] = -sum_k p[k]*log p[k] = log S - T/S
 *   stats[n]   = (max_j z[n,j], log S): two numbers from which any log p[k] = scale*(z[n,k] - stats[0]) - stats[1]
 *   top_logp[n,i], top_index[n,i], i < top: log probability and index of the i-th most probable token; of equal ones the
 *                lowest index first; past the K-th token minus infinity and index -1
 *   dz[n,k]    = scale*( dlogp[n]*((k == labels[n]) - p[k]) - dentropy[n]*p[k]*(log p[k] + entropy[n]) )
 * labels: device int32; a label outside [0, K) has logp 0 and no gradient of logp.  A logit of minus infinity has
 * probability 0; a row of nothing else has log probabilities of minus infinity, entropy 0, stats (-inf, 0) and a zero
 * gradient.  A row that holds a NaN or plus infinity has NaN results; its top_index names tokens of the row in the order of the logits, where a NaN
 * comes before plus infinity, one whose sign bit is set after minus infinity, and top_logp is NaN beside each.  Arithmetic, logp, entropy, stats and
 * top_logp are fp32; dz is rounded once to `dtype` and has z's ld.
 *   mxc_logprob_fwd      any of logp (and with it labels), entropy, stats may be NULL; top in 0..MXC_LOGPROB_MAX_TOP,
 *                        with top == 0 top_logp and top_index may be NULL
 *   mxc_logprob_bwd      the gradient from stats and entropy of mxc_logprob_fwd; dlogp or dentropy may be NULL (zeros);
 *                        labels may be NULL without dlogp, entropy without dentropy
 *   mxc_logprob_fwd_bwd  both at once, which reads z once: logp or entropy may be NULL
 * dz may be z itself.  scale must be positive, and finite times log2(e) (2.358e38 at most).  Workspace: mxc_logprob_workspace_bytes (top 0 for
 * mxc_logprob_fwd_bwd, none for mxc_logprob_bwd).  Results are bit-identical from run to run.  Errors: MXC_ERR_SHAPE (non-positive N
 * or K, K above MXC_LOGPROB_MAX_K, ld < K, top out of range, more rows than one launch holds), MXC_ERR_UNSUPPORTED (dtype, scale), MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes for z and dz,
 * 4 for the others), MXC_ERR_WORKSPACE, MXC_ERR_LAUNCH.
 */
enum { MXC_LOGPROB_MAX_TOP = 64, MXC_LOGPROB_MAX_K = 1 << 30 };
int mxc_logprob_workspace_bytes(int N, int K, int dtype, int top, size_t *out_bytes);
int mxc_logprob_fwd(int N, int K, int ld, int dtype, const void *z, const int *labels, float scale, int top,
                    float *logp, float *entropy, float *stats, float *top_logp, int *top_index,
                    void *workspace, size_t workspace_bytes, void *hip_stream);
int mxc_logprob_bwd(int N, int K, int ld, int dtype, const void *z, const int *labels, float scale, const float *stats,
                    const float *entropy, const float *dlogp, const float *dentropy, void *dz, void *hip_stream);
int mxc_logprob_fwd_bwd(int N, int K, int ld, int dtype, const void *z, const int *labels, float scale,
                        const float *dlogp, const float *dentropy, float *logp, float *entropy, void *dz,
                        void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Microscaled 4-bit floating point (the MXFP4 format of the OCP Microscaling Formats specification 1.0).  A row of C values is cut
 * into blocks of 32; a block has one scale 2^(b - 127), b a byte, and a value is sign * {0, .5, 1, 1.5, 2, 3, 4, 6} times
 * that.  For N rows of C values:
 *   codes:  [N][ceil(C/32)*16] bytes; value 2j of a row is the low half of byte j, value 2j+1 the high half; the places past
 *           column C hold 0
 *   scales: [N][ceil(C/512)*16] bytes, one for each block; the bytes past the last block hold 0
 *   mxc_mxfp4_quantize    b = floor(log2(largest |x| of the block)) - 2 + 127, at least 0; values are rounded to the nearest
 *       representable one, ties to the even code, larger ones than 6 to 6.  A block that holds an infinity or a NaN has b = 255
 *       and codes 0: all of it reads as NaN.
 *   mxc_mxfp4_dequantize  the numbers the codes stand for, rounded once to `dtype`
 * x, y: [N][C] of `dtype`, dense.  No workspace.  Errors: MXC_ERR_SHAPE (also for more values than one launch holds: about 2^35 in a call, 2^27 filter rows), MXC_ERR_UNSUPPORTED (dtype),
 * MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes), MXC_ERR_LAUNCH.
 *
 * FullyConnected on a filter in this form: y[n,k] = act( sum_c q(x)[n,c] * w[k,c] + bias[k] ), x: [N][C] and y: [N][K]
 * of `dtype`, w_codes and w_scales as above for K rows of C values, q(x) the values of mxc_mxfp4_quantize (the
 * input is brought into 4 bits within the call), products exact, sums in fp32 (their order depends on the sizes alone), one rounding to `dtype`.  bias
 * (fp32) may be NULL, relu is 0 or 1 (a NaN stays).  A NaN in q(x) or w makes NaN of the results of its row or column.  Places of w_codes past column C must hold 0
 * (their scales are read as they are: no infinity arises from them).  Workspace: mxc_mxfp4_fc_workspace_bytes.  Errors as above (MXC_ERR_SHAPE also for C above
 * MXC_MXFP4_FC_MAX_C), and MXC_ERR_WORKSPACE.
 */
enum { MXC_MXFP4_FC_MAX_C = 1 << 23 };
int mxc_mxfp4_quantize(int N, int C, int dtype, const void *x, void *codes, void *scales, void *hip_stream);
int mxc_mxfp4_dequantize(int N, int C, int dtype, const void *codes, const void *scales, void *y, void *hip_stream);
int mxc_mxfp4_fc_workspace_bytes(int N, int C, int K, int dtype, size_t *out_bytes);
int mxc_mxfp4_fc_fwd(int N, int C, int K, int dtype, const void *x, const void *w_codes, const void *w_scales,
                     const float *bias, int relu, void *y, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * AdamW step over many tensors in one call (a launch for every MXC_ADAMW_GROUP tensors, or MXC_ADAMW8_GROUP,
 * and 2^34 values).  For each value, with
 * gs = grad_scale*g and t = step (1 for the first):
 *   m' = beta1*m + (1 - beta1)*gs,   v' = beta2*v + (1 - beta2)*gs*gs
 *   w' = w*(1 - lr*wd) - lr/(1 - beta1^t) * m' / ( sqrt(v')/sqrt(1 - beta2^t) + eps )
 * count tensors; sizes, w, g, m, v, w_bf16, state: HOST arrays of `count` element counts and device pointers (read before the
 * call returns).  w: fp32 master weights, in place; g: gradients of grad_dtype (MXC_F32 or MXC_BF16); m, v: fp32, in place;
 * w_bf16: NULL, or for each tensor where w' goes rounded to bf16.  A tensor of size 0 is passed over, whatever its pointers.
 * The factors are computed from the double arguments in 64 bits and used in 32.
 * mxc_adamw8_update keeps m and r = sqrt(v) in 8 bits: state: mxc_adamw8_state_bytes(n) bytes a tensor, zeros at the start.
 * 256 values have 528 bytes: 256 codes of m, 256 of r (each sign, 4 bits of exponent, 3 of mantissa, largest 448: e4m3), 8 scales of
 * m, 8 of r (bytes b for 2^(b - 127), one for every 32 values: the smallest with which the block's largest value is 448 or less;
 * 0 for a block of zeros).  A value goes to one of its two neighbours at random, so that its mean is the value: up where its place
 * between them plus u >= 1, u a multiple of 2^-16 taken from a hash of the value's index, the tensor's number and `seed` (16 bits of it for m, 16 for r; the
 * same call gives the same codes).  An r that is not 0 does not become code 0: a weight's step never divides by eps alone
 * because of a rounding.  A block of m or r that holds an infinity or a NaN gets scale 255 and reads as NaN.
 * Errors, found before anything is launched: MXC_ERR_SHAPE (count <= 0, step < 1, a tensor of more than 2^33 values), MXC_ERR_UNSUPPORTED (grad_dtype;
 * beta1 or beta2 outside [0, 1); negative eps; a factor that is not finite), MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes), MXC_ERR_LAUNCH.
 */
enum { MXC_ADAMW_GROUP = 72, MXC_ADAMW8_GROUP = 88 };
int mxc_adamw_update(int count, const size_t *sizes, void *const *w, const void *const *g, int grad_dtype, void *const *m,
                     void *const *v, void *const *w_bf16, double lr, double beta1, double beta2, double eps, double wd,
                     double grad_scale, long long step, void *hip_stream);
int mxc_adamw8_state_bytes(size_t n, size_t *out_bytes);
int mxc_adamw8_update(int count, const size_t *sizes, void *const *w, const void *const *g, int grad_dtype, void *const *state,
                      void *const *w_bf16, double lr, double beta1, double beta2, double eps, double wd,
                      double grad_scale, long long step, unsigned seed, void *hip_stream);

/*
 * Embedding: rows of a table for given tokens, and the table's gradient.  tokens: [N] device int32; w: [V][C] and y, dy: [N][C] of `dtype`; dw: [V][C]
 * fp32 for both dtypes.  A token outside [0, V) (padding) has a row of zeros and no gradient.
 *   mxc_embedding_fwd:  y[n,c] = scale * w[tokens[n],c], rounded once to `dtype`
 *   mxc_embedding_bwd:  dw[v,c] = scale * sum over n with tokens[n] == v of dy[n,c], zeros for a token that stands nowhere; with accumulate == 1 this
 *                       is added to the dw that is there, and rows of tokens that stand nowhere are neither read nor written (a table whose product
 *                       with the last layer's input has left its gradient there)
 * Sums in fp32 in an order that depends on N, V, C and the tokens alone (bit-identical from run to run).  Workspace: mxc_embedding_workspace_bytes, for the
 * gradient.  Errors: MXC_ERR_SHAPE (non-positive sizes, N, V or C above the limits below), MXC_ERR_UNSUPPORTED (dtype, scale that is not finite,
 * accumulate), MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes, 4 for tokens), MXC_ERR_WORKSPACE, MXC_ERR_LAUNCH.
 */
enum { MXC_EMBEDDING_MAX_N = 1 << 23, MXC_EMBEDDING_MAX_V = 1 << 23, MXC_EMBEDDING_MAX_C = 1 << 20 };
int mxc_embedding_fwd(int N, int V, int C, int dtype, const int *tokens, const void *w, float scale, void *y, void *hip_stream);
int mxc_embedding_workspace_bytes(int N, int V, int C, int dtype, size_t *out_bytes);
int mxc_embedding_bwd(int N, int V, int C, int dtype, const int *tokens, const void *dy, float scale, int accumulate, float *dw,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Layer norm over the rows of x: [N][C] of `dtype`, dense; gamma, beta: C fp32 values.
 *   mxc_layernorm_fwd:  mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps),  z = (x - mean) * rstd
 *                       y = z * gamma + beta,  stats[n] = (mean, rstd);  gamma (ones), beta (zeros) and stats may each be NULL; y may be x
 *   mxc_layernorm_bwd:  from x and the stats of the forward call, with g = dy * gamma:
 *                       dx = rstd * (g - sum_c g / C - z * sum_c g * z / C),  dgamma[c] = sum_n dy * z,  dbeta[c] = sum_n dy
 *                       gamma (ones), dgamma and dbeta may each be NULL; dx may be dy or x
 * Arithmetic, stats, dgamma and dbeta are fp32 (the squares are those of the differences from the mean, and where the mean is more than 16 deviations, sqrt(var + eps), from zero
 * its rounding is taken out of z and the variance too: a large mean costs no digits; the gradient's z has the mean as stats hold it), y and dx are rounded
 * once to `dtype`.  An infinity or a NaN in x makes NaN of its row's y and dx and of all of dgamma, and its row's stats are not finite; one in dy makes values that are not
 * finite of its row's dx and of its column's dgamma and dbeta.  Other rows and columns are left alone.  A row whose sum passes the
 * largest fp32 number has NaN for y; one whose sum of squared differences does has rstd 0 and beta for y.  dgamma and dbeta are added in a fixed order.
 * Workspace: mxc_layernorm_workspace_bytes, for the gradient.  Errors: MXC_ERR_SHAPE (non-positive sizes, C above MXC_LAYERNORM_MAX_C), MXC_ERR_UNSUPPORTED
 * (dtype; eps that is not a normal positive number), MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes, 4 for stats), MXC_ERR_WORKSPACE, MXC_ERR_LAUNCH.
 */
enum { MXC_LAYERNORM_MAX_C = 1 << 20 };
int mxc_layernorm_fwd(int N, int C, int dtype, const void *x, const float *gamma, const float *beta, float eps, void *y, float *stats, void *hip_stream);
int mxc_layernorm_workspace_bytes(int N, int C, int dtype, size_t *out_bytes);
int mxc_layernorm_bwd(int N, int C, int dtype, const void *x, const float *gamma, const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Orthogonal update directions by Newton-Schulz steps, and the optimiser's step that uses them (Muon).  count matrices of rows[i] x cols[i] values,
 * dense; rows, cols and the lists of device pointers are HOST arrays, read before the call returns.
 *   mxc_orthogonalize:  X = x / |x|, |x| the root of the sum of squares;  `steps` times  X <- a X + (b A + c A A) X,  A = X X^T,  with a = 3.4445,
 *                       b = -4.7750, c = 2.0315 and X turned so that its rows are not longer than its columns;  y = X, bf16.  x is of `dtype`.  Singular values of x
 *                       above 0.0025 |x| come out between 0.68 and 1.21 after 5 steps; their directions stay.  A matrix of
 *                       zeros gives zeros; an infinity or a NaN in x makes NaN of the whole of y.
 *   mxc_muon_update:    with gs = grad_scale*g:  m' = momentum*m + gs,  u = gs + momentum*m' (nesterov == 1) or m' (0),
 *                       w' = w*(1 - lr*wd) - lr*f*O,  O = u made orthogonal as above, not rounded between;  f = rms*sqrt(max(rows, cols)), with which
 *                       the step's values have a root mean square of about lr*rms (0.2 is usual beside AdamW's learning rates), or with rms == 0
 *                       f = sqrt(max(1, rows/cols)).  w: fp32 master weights, in place; m: fp32, in place, zeros at the start; g of grad_dtype;
 *                       w_bf16: NULL, or for each matrix where w' goes rounded to bf16.
 * Arithmetic: the products multiply values of 11 bits (fp16 at fixed powers of two, which no entry of X, A or b A + c A A leaves, their singular values being
 * bounded) with fp32 sums; the diagonals of A and of b A + c A A are kept apart in fp32, and X is carried with 22 bits.  O's error is about 1e-3 of its
 * norm after 5 steps, in directions of any singular value.  |x| is summed in 64 bits.  Results are bit-identical from run to run and do not depend on the
 * other matrices of a call.  No tensor may overlap another of the call.
 * Workspace: mxc_orthogonalize_workspace_bytes, for both; none where every matrix has at most 64 by 576 values, either way.  Errors, found before anything is launched: MXC_ERR_SHAPE (non-positive count or sides, more
 * than MXC_ORTHOGONALIZE_MAX_COUNT matrices, sides above MXC_ORTHOGONALIZE_MAX_SIDE), MXC_ERR_UNSUPPORTED (dtype; steps outside 1..MXC_ORTHOGONALIZE_MAX_STEPS, past which the
 * rounding of small directions grows; momentum outside [0, 1), negative rms, nesterov, factors that are not finite; a matrix twice in y, w, m or w_bf16), MXC_ERR_NULL, MXC_ERR_ALIGN (16 bytes),
 * MXC_ERR_WORKSPACE, MXC_ERR_LAUNCH.
 */
enum { MXC_ORTHOGONALIZE_MAX_SIDE = 32768, MXC_ORTHOGONALIZE_MAX_STEPS = 6, MXC_ORTHOGONALIZE_MAX_COUNT = 4096 };
int mxc_orthogonalize_workspace_bytes(int count, const int *rows, const int *cols, size_t *out_bytes);
int mxc_orthogonalize(int count, const int *rows, const int *cols, const void *const *x, int dtype, int steps, void *const *y,
                      void *workspace, size_t workspace_bytes, void *hip_stream);
int mxc_muon_update(int count, const int *rows, const int *cols, float *const *w, const void *const *g, int grad_dtype, float *const *m,
                    void *const *w_bf16, double lr, double momentum, int nesterov, double wd, double rms, double grad_scale, int steps,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Workspace size in bytes that `pass` (MXC_FWD / MXC_BWD_DATA / MXC_BWD_WEIGHT)
 * needs for these arguments, written to *out_bytes (a HOST pointer).  Touches
 * no GPU state.
 */
int mxc_conv2d_workspace_bytes(int pass, int N, int C, int H, int W, int K, int R, int S,
                               int stride, int pad, int dtype, int layout, size_t *out_bytes);

/*
 * Layout conversion of a dense 4-D tensor between [n][c][h][w] and [n][h][w][c]
 * (the conversion a network does once at entry and exit when activations stay
 * NHWC between layers).  Also converts filters KCRS <-> KRSC with n=K, h=R, w=S.
 * src and dst are device pointers and must not overlap.  src_layout ==
 * dst_layout is a plain copy.
 */
int mxc_layout_convert(int n, int c, int h, int w, int dtype, int src_layout, int dst_layout,
                       const void *src, void *dst, void *hip_stream);

/* Static, NUL-terminated description of a status code (host memory, never freed). */
const char *mxc_status_string(int status);

/* Name of the kernel variant the calling thread's last successful compute call
 * chose (for logs and the bench); "" before any call.  Host memory, thread-local. */
const char *mxc_last_variant(void);

/* Library version as major*10000 + minor*100 + patch. */
int mxc_version(void);

/* Tuning aid: name of the index-th tile shape the matrix-core kernels are built in (family 0: forward /
 * backward-data implicit GEMM, family 1: backward-weight, family 2: the whole-launch implicit GEMMs - "igemm_stream"
 * for short reductions and "igemm_window" for multi-tap stride-1 layers of at most 64 channels, each one plan that
 * runs only where its filter tile fits on chip, family 3: fp32, family 4: the implicit GEMM of small problems,
 * family 5: their backward-weight, family 6: fp32 NHWC layers of whole 16-byte chunks of channels, backward-weight last,
 * family 7: dx of first layers at stride 1, family 8: the implicit GEMM of 3- and 5-column filters at stride 1 whose taps of
 * a filter row share their pixels, family 9: their backward-weight), NULL past the last.  These are the names that
 * mxc_last_variant() reports and that the tuning hooks MXC_FORCE_VARIANT=<name>[+<name of the shape for the
 * rows the last whole round leaves>] and MXC_FORCE_WGRAD=<name>[/<splits>] (environment, read per call) accept.
 * The tests walk the list; the tuning script times families 0 to 2, whose plans it tabulates: the others are chosen
 * beside a plan by time models.  Static host memory. */
const char *mxc_tile_name(int family, int index);

/* Tuning aid: the implicit GEMM (rows M, output columns Co, reduction length Kd) that the calling thread's last
 * forward or backward-data call planned - for first layers that is the GEMM on the packed operands, whose
 * dimensions the caller does not otherwise see.  The tuning script keys its table of measured plans on it.
 * Strided backward-data of other layers, a GEMM per residue class, leaves the key of any of them or as it was.
 * All three are 0 before any such call.  Host only. */
void mxc_last_plan_key(long long *M, int *Co, int *Kd);

/* Tuning aid: how often the calling thread has searched for the kernel that runs a problem.  A thread keeps what it
 * found: calls and size queries of problems it has met lately do not search, and the count stands still.  Host only. */
long long mxc_plan_searches(void);

/* Measurement aid (not part of the convolution path): enqueues one launch of a
 * register-resident loop of bf16 matrix instructions (v_mfma_f32_32x32x16_bf16, fp32
 * accumulate, no memory traffic) on `workgroups` workgroups of 256 threads, `iters`
 * iterations of four instructions per wave, and stores in *flops (host memory) the number
 * of floating-point operations that launch performs.  The caller times the launch; flops
 * over time is the matrix-pipe ceiling of this device at its sustained clock, the
 * "measured peak" that the benchmark reports beside the published one (the paper, Section 4,
 * compares on measured speed only).  `out`: device buffer of at least workgroups*256 floats
 * (16-byte aligned; receives values of no interest), caller-owned.  Errors: MXC_ERR_NULL,
 * MXC_ERR_SHAPE (non-positive counts), MXC_ERR_WORKSPACE (out too small), MXC_ERR_ALIGN,
 * MXC_ERR_LAUNCH. */
int mxc_probe_mfma(int workgroups, int iters, void *out, size_t out_bytes, double *flops, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MXC_H */
