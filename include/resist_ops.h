/*
 * resist_ops.h -- layer-level entry points of the same library: the convolution kernels that
 * resist_local_step is built from, exposed so each can be checked against the textbook
 * definition on its own; and, further down, the operators of residual blocks of dense layers (layer
 * norm, dropout, dense layers with their epilogue).  Same conventions as resist.h (status codes, caller-owned device
 * memory, caller's stream, no synchronisation).
 *
 * Layouts: activations NHWC [N][H][W][C]; filters [K][R][S][C]; outputs [N][P][Q][K] with
 * P = (H + 2*pad - R)/stride + 1.  dtype 0: all fp32 (matrix products as under compute_dtype in
 * resist.h).  dtype 1: activations and filters bf16
 * (as uint16 bit patterns), accumulation fp32, weight gradients fp32.
 * Supported: R = S in {1,3,5,7}; stride in {1,2}; 0 <= pad < R; C and K multiples of 4 (fp32) or 8
 * (bf16); the stride-2 data gradient needs even H and W; every tensor below 2 GiB.  Anything else is
 * RESIST_ESHAPE before any launch.
 */
#ifndef RESIST_OPS_H
#define RESIST_OPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t N, H, W, C; /* input activation */
  int32_t K, R, S;    /* filter           */
  int32_t stride, pad;
  int32_t dtype;      /* 0 fp32, 1 bf16   */
} resist_conv_shape;

/* Workspace (bytes) the three calls below use at most for this shape: a filter copy, or the split partial sums of the
 * weight gradient (of the kernel that needs most of those the shape could be given).  The forward call takes any, NULL
 * too, and leaves it as it is; the data gradient takes K*R*S*C elements at least, with the same results.  The two
 * gradients write it: calls that overlap in time need one each.  host. */
int resist_conv2d_workspace_bytes(const resist_conv_shape *s, int64_t *bytes);

/* y[n,p,q,k] = sum_{r,s,c} x[n, p*stride+r-pad, q*stride+s-pad, c] * w[k,r,s,c]  (zero padding) */
int resist_conv2d_forward(const resist_conv_shape *s, const void *x, const void *w, void *y,
                          void *workspace, int64_t workspace_bytes, void *hip_stream);

/* dx[n,h,w,c] = sum over (k,r,s,p,q) with h = p*stride+r-pad, w = q*stride+s-pad of
 * dy[n,p,q,k] * w[k,r,s,c] */
int resist_conv2d_dgrad(const resist_conv_shape *s, const void *dy, const void *w, void *dx,
                        void *workspace, int64_t workspace_bytes, void *hip_stream);

/* dw[k,r,s,c] = sum_{n,p,q} dy[n,p,q,k] * x[n, p*stride+r-pad, q*stride+s-pad, c]; dw is fp32 */
int resist_conv2d_wgrad(const resist_conv_shape *s, const void *dy, const void *x, float *dw,
                        void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * The stem convolution: the first layer reads the input batch as the caller passes it to
 * resist_local_step -- logical [N,C,H,W] fp32 with C <= 4 -- and runs as an implicit GEMM over the
 * R*S*C filter positions (no im2col matrix is written).  The resist_conv_shape describes the same
 * convolution (N, H, W, C of the image; K, R = S, stride, pad; dtype of the OUTPUT side: 0 fp32, 1 bf16,
 * in which case image and filter are rounded to bf16 as they become matrix operands).
 * Supported: C <= 4, K a multiple of 16 up to 128, R*S*C <= 160, tensors below 2 GiB.
 *   x   device [N][C][H][W] fp32           w   device [K][R][S][C] fp32 (the master filter)
 *   y   device [N][P][Q][K] in dtype       dy  device [N][P][Q][K] in dtype      dw  device [K][R][S][C] fp32
 * Workspace: resist_stem_conv2d_workspace_bytes (padded filter copies and the partial sums of the
 * weight gradient).
 */
int resist_stem_conv2d_workspace_bytes(const resist_conv_shape *s, int64_t *bytes);
int resist_stem_conv2d_forward(const resist_conv_shape *s, const float *x, const float *w, void *y, void *workspace,
                               int64_t workspace_bytes, void *hip_stream);
int resist_stem_conv2d_wgrad(const resist_conv_shape *s, const void *dy, const float *x, float *dw, void *workspace,
                             int64_t workspace_bytes, void *hip_stream);

/*
 * resist_conv2d_wgrad for callers that cannot allocate device memory or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same kernels and the same
 * bits as resist_conv2d_wgrad, but the split partial sums go to a static device array inside the
 * library (32 MiB per GPU, held until the process ends; resist_conv2d_wgrad_static_limit reports the
 * size).  The call allocates nothing (keep resist_profile_enable off: timing creates events).
 * RESIST_EWORKSPACE if the shape's partial sums (resist_conv2d_workspace_bytes' split part) exceed
 * the array.  Nothing in the array needs clearing between calls: every split writes its whole slice
 * before the reduction reads it.  All calls on one GPU share the array, so two calls that overlap in
 * time on one GPU (different streams, or different host threads) race; calls on one stream do not.
 */
int resist_conv2d_wgrad_static(const resist_conv_shape *s, const void *dy, const void *x, float *dw,
                               void *hip_stream);
int resist_conv2d_wgrad_static_limit(int64_t *bytes);

/*
 * Operators of a residual block of dense layers:
 *     n = layernorm(x);   h = dropout(act(n w1' + b1));   y = x + dropout(h w2' + b2)
 * and their gradients.  Same conventions; in particular every pointer is 16-byte aligned.  Rows are tokens: a matrix is M rows of
 * contiguous elements, `ld` elements from one row to the next (at least the row's length; 0: exactly that).  Activations, their
 * gradients and the weights w [N][K] (dense) are dtype 0 fp32 or 1 bf16; biases, LN parameters and statistics, and the
 * gradients of parameters are fp32.  All arithmetic is fp32 (products of fp32 operands as under compute_dtype in resist.h), with one
 * rounding where a result is stored.  M may be 0: nothing is written but the gradients of parameters, which are zero.  An output
 * may be the very tensor (pointer and stride) that it is named after with "in place" below; otherwise outputs overlap nothing.
 *
 * Activations `act`:
 *   RESIST_ACT_NONE       a(z) = z
 *   RESIST_ACT_RELU       max(z, 0), with a'(0) = 0
 *   RESIST_ACT_GELU       z Phi(z), Phi the normal distribution function
 *   RESIST_ACT_GELU_TANH  z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3)))
 *   RESIST_ACT_SILU       z / (1 + exp(-z))
 * Of infinite z all of them and their derivatives are the limits (a(-inf) = 0 but for NONE); a NaN stays one, but for RELU, which
 * takes what is not above 0 as 0, as in resist.h's layers.
 *
 * Dropout with probability 0 <= p < 1: an element is dropped (0, whatever it was) or kept and multiplied by 1/(1-p).  The mask is never
 * stored: it is a function of rng, device {seed, offset}, read when the kernel runs (a captured call draws a new mask with
 * every replay if the caller moves the offset on in between), and of the position.  With splitmix64 as in
 * resist_partition, let s be the first output of the sequence seeded with `seed`, and word(i, c) output number
 * offset + i*ceil(N/2) + c (from 0) of the sequence seeded with s.  Element (i, j) of an M x N matrix is dropped where the low (j even)
 * or high (j odd) 32 bits of word(i, j/2) are below p 2^32, rounded to a whole number.  So a call uses M*ceil(N/2) words: a
 * caller who wants independent masks moves the offset on by that.  The same rng, p, M and N give the same mask in every call
 * below.  rng may be NULL where p is 0.
 */
enum { RESIST_ACT_NONE = 0, RESIST_ACT_RELU = 1, RESIST_ACT_GELU = 2, RESIST_ACT_GELU_TANH = 3, RESIST_ACT_SILU = 4 };

/*
 * Layer norm over rows of N elements (1 <= N <= 2^24, M < 2^31):
 *   forward   mu = mean x, v = mean (x - mu)^2, r = 1/sqrt(v + eps);  y = gamma (x - mu) r + beta      [y in place of x]
 *   backward  xhat = (x - mu) r, g = gamma dy;  dx = r (g - mean g - xhat mean(g xhat)) [+ addend]     [dx in place of dy, x or addend]
 *             dgamma = sum over rows of dy xhat, dbeta = sum over rows of dy
 *   gamma, beta    device [N] or NULL (1, 0)          eps  >= 0
 *   mean, rstd     device [M]: mu and r, written by the forward pass (or NULL), read by the backward pass
 *   addend         device [M][N] or NULL: a gradient that reaches x by another path
 *   dgamma, dbeta  device [N] or NULL
 *   workspace      resist_layernorm_workspace_bytes (backward only): partial sums; calls that overlap in time need one each
 */
int resist_layernorm_workspace_bytes(int64_t M, int32_t N, int64_t *bytes);
int resist_layernorm_forward(int64_t M, int32_t N, int32_t dtype, const void *x, int64_t ldx, const float *gamma, const float *beta,
                             float eps, void *y, int64_t ldy, float *mean, float *rstd, void *hip_stream);
int resist_layernorm_backward(int64_t M, int32_t N, int32_t dtype, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                              const float *gamma, const float *mean, const float *rstd, const void *addend, int64_t ldadd, void *dx,
                              int64_t lddx, float *dgamma, float *dbeta, void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * Dropout on its own, with the residual add behind it, and its gradient, with that of an activation in front of it
 * (1 <= N <= 2^24, M < 2^31):
 *   forward   y = [residual +] drop(x)       [y in place of x or residual]
 *   backward  dx = a'(z) drop(dy)            [dx in place of dy or z]       (act RESIST_ACT_NONE: z is not read)
 */
int resist_dropout_forward(int64_t M, int32_t N, int32_t dtype, const void *x, int64_t ldx, double p, const uint64_t *rng,
                           const void *residual, int64_t ldr, void *y, int64_t ldy, void *hip_stream);
int resist_dropout_backward(int64_t M, int32_t N, int32_t dtype, const void *dy, int64_t lddy, double p, const uint64_t *rng, int32_t act,
                            const void *z, int64_t ldz, void *dx, int64_t lddx, void *hip_stream);

/*
 * Dense layer, x [M][K], w [N][K], y [M][N] (1 <= K, N <= 2^20, row strides up to 2^20, M < 2^31; of 2^38 outputs or more, beyond any
 * card's memory, a call may be refused with RESIST_ESHAPE):
 *   forward          z = x w' + bias,  y = [residual +] drop(act(z))      [y in place of residual]
 *   data gradient    dx = a'(z) drop(dz w): z, act and drop are of the layer that produced x, the gradient leaves taken
 *                    through them                                         [dx in place of z]
 *   weight gradient  dw = dz' x [N][K], db = column sums of dz [N]; db may be NULL
 * dz and y share ldy, dx and x share ldx.
 * Workspace (may be NULL where resist_linear_workspace_bytes is 0): operands laid out for the kernels, and partial sums; calls
 * that overlap in time need one each.  op: 0 forward, 1 data gradient, 2 weight gradient.  It depends on the shape alone.
 */
typedef struct {
  int64_t M;
  int32_t K, N;
  int64_t ldx, ldy;
  int32_t dtype;
} resist_linear_shape;
typedef struct {
  const float *bias;        /* device [N] or NULL */
  int32_t act;
  double p;                 /* dropout; rng device [2] */
  const uint64_t *rng;
  const void *residual;     /* device [M][N] or NULL */
  int64_t ldr;
  void *z;                  /* device [M][N] or NULL: receives z, as the gradients need it */
  int64_t ldz;
} resist_linear_epilogue;
typedef struct {
  int32_t act;              /* RESIST_ACT_NONE: z is not read */
  const void *z;            /* device [M][K] */
  int64_t ldz;
  double p;
  const uint64_t *rng;
} resist_linear_through;
int resist_linear_workspace_bytes(const resist_linear_shape *s, int32_t op, int64_t *bytes);
int resist_linear_forward(const resist_linear_shape *s, const void *x, const void *w, const resist_linear_epilogue *epilogue /* or NULL */,
                          void *y, void *workspace, int64_t workspace_bytes, void *hip_stream);
int resist_linear_dgrad(const resist_linear_shape *s, const void *dz, const void *w, const resist_linear_through *through /* or NULL */,
                        void *dx, void *workspace, int64_t workspace_bytes, void *hip_stream);
int resist_linear_wgrad(const resist_linear_shape *s, const void *dz, const void *x, float *dw, float *db, void *workspace,
                        int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RESIST_OPS_H */
