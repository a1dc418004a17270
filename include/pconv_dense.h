/*
 * pconv_dense — the dense half of a pruned network and the loss that trains it.  C ABI, part of libpconv.so, next to
 * pconv.h (whose conventions, error codes and pconv_strerror apply).
 *
 * A network whose 3x3 and 1x1 convolutions are pruned still has its fully connected layers, the 1x1 layers that are left
 * dense (on channel-minor tensors [pixels][channels] those are matrix products), its norms, and, where the pruned weights
 * are trained further (paper, section 5.1: the primal step), a loss; training against the unpruned network's outputs is
 * the usual one.  The operators here are those: matrix product with bias, activation and residual, layer norm, distillation
 * from a teacher's top logits, each with its backward pass.
 *
 * Conventions of this header
 *   - storage types: PCONV_F32, PCONV_F16 and, for the entries of this header only, PCONV_BF16; sums, statistics, biases,
 *     norm weights, losses and weight gradients are fp32; results are rounded to nearest even once, at the store;
 *   - matrices are row-major, ld* is the distance of two rows in elements, 0 = rows without gaps; gaps are neither read as
 *     values nor written.  A row stride is at least the row's length and at most 2^20 elements (PCONV_EUNSUPPORTED);
 *   - device pointers need the alignment of one element; rows that are aligned to 16 bytes are read and written in wider pieces;
 *   - outputs must not overlap inputs, unless a comment says so;
 *   - calls are asynchronous on `stream` (a hipStream_t passed as void*, NULL = the default stream) of the current device,
 *     allocate nothing and may be captured into a HIP graph.  Calls that overlap in time need workspaces of their own;
 *   - results are reproducible: every sum is taken in an order fixed by the sizes;
 *   - the sizes are checked before the pointers: a null pointer is refused (PCONV_EINVAL) only where there is work to do.
 */
#ifndef PCONV_DENSE_H
#define PCONV_DENSE_H

#include <stddef.h>
#include <stdint.h>

#include "pconv.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { PCONV_BF16 = 2 };   /* storage type of the entries of this header; the other headers' entries refuse it */

enum { PCONV_ACT_NONE = 0,
       PCONV_ACT_RELU = 1,
       PCONV_ACT_GELU = 2,       /* z * Phi(z), Phi the normal distribution */
       PCONV_ACT_GELU_TANH = 3,  /* z/2 * (1 + tanh(sqrt(2/pi) * (z + 0.044715 z^3))) */
       PCONV_ACT_SILU = 4        /* z / (1 + exp(-z)) */ };
/* (At z = -inf the last three are NaN, like the formulas; their slopes there are 0.) */

enum { PCONV_FLAG_RESIDUAL_FIRST = 8u };   /* pconv_linear: the residual is added in front of the activation */

/*
 * Matrix product with bias, activation and residual:
 *     z[m][n] = bias[n] + sum over k of x[m][k] * w[n][k]   (+ residual[m][n] with PCONV_FLAG_RESIDUAL_FIRST)
 *     y[m][n] = act(z[m][n])                                (+ residual[m][n] without it)
 *   x        device, dtype[M][K], row stride ldx
 *   w        device, dtype[N][K], row stride ldw (the layout of a fully connected layer's weights; a dense 1x1 layer's too)
 *   bias     device, float[N], or NULL
 *   residual device, dtype[M][N], row stride ldr, or NULL; may be y itself with ldr = ldy
 *   z        device, dtype[M][N], row stride ldy: receives z for the backward pass, or NULL
 *   y        device, dtype[M][N], row stride ldy
 *   M rows 0.., N 1.., K 1..;  act PCONV_ACT_*;  flags 0 or PCONV_FLAG_RESIDUAL_FIRST
 *   workspace, workspace_bytes  device scratch of pconv_linear_workspace() bytes, aligned to 16 bytes (NULL if that is 0):
 *            partial sums where few tiles of the output have to share a long K
 * M = 0 is a no-op.  PCONV_EINVAL: null pointers, bad enum or flag, a pointer that is not aligned to an element, a workspace
 * that is too small or not aligned; PCONV_ESHAPE: M < 0, N < 1 or K < 1, a row stride below the row's length;
 * PCONV_EUNSUPPORTED: M above 2^30, N, K or a row stride above 2^20.
 * The same input row gives the same output row wherever it stands in x, as long as M, N, K, the strides' and pointers'
 * alignment stay the same.
 */
int pconv_linear_workspace(int dtype, int M, int N, int K, size_t* bytes);
int pconv_linear(const void* x, long long ldx, const void* w, long long ldw, const float* bias, const void* residual, long long ldr,
                 void* z, void* y, long long ldy, int dtype, int M, int N, int K, int act, unsigned flags, void* workspace,
                 size_t workspace_bytes, void* stream);

/*
 * Gradient of the layer's input.  With dz = dL/dz, the gradient at the product's result:
 *     dx[m][k] = act'(z[m][k]) * sum over n of dz[m][n] * w[n][k]  +  add[m][k]
 *   dz   device, dtype[M][N], row stride lddz
 *   w    device, dtype[N][K], row stride ldw
 *   z    device, dtype[M][K], row stride ldz, or NULL with PCONV_ACT_NONE: the argument of the activation that made x in the layer
 *        before (its z), whose gradient the result then is: layers that follow each other need no pass of their own for it.
 *        For PCONV_ACT_RELU x itself may stand for z.  The derivative of ReLU at 0 is 0.
 *   add  device, dtype[M][K], row stride lda, or NULL: a gradient that reaches x by another way (a residual's); may be dx
 *        itself with lda = lddx
 *   dx   device, dtype[M][K], row stride lddx
 * Workspace and errors as pconv_linear's (pconv_linear_grad_input_workspace() bytes).
 */
int pconv_linear_grad_input_workspace(int dtype, int M, int N, int K, size_t* bytes);
int pconv_linear_grad_input(const void* dz, long long lddz, const void* w, long long ldw, const void* z, long long ldz, int act,
                            const void* add, long long lda, void* dx, long long lddx, int dtype, int M, int N, int K, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Gradients of the layer's weights and bias:
 *     dw[n][k] = sum over m of dz[m][n] * x[m][k],   db[n] = sum over m of dz[m][n]
 *   dz   device, dtype[M][N], row stride lddz;   x  device, dtype[M][K], row stride ldx
 *   dw   device, float[N][K];   db  device, float[N], or NULL
 * M = 0 gives zeros.  Workspace and errors as pconv_linear's (pconv_linear_grad_weight_workspace() bytes).
 */
int pconv_linear_grad_weight_workspace(int dtype, int M, int N, int K, size_t* bytes);
int pconv_linear_grad_weight(const void* dz, long long lddz, const void* x, long long ldx, float* dw, float* db, int dtype, int M,
                             int N, int K, void* workspace, size_t workspace_bytes, void* stream);

/*
 * dz[m][n] = dy[m][n] * act'(z[m][n]): the gradient in front of a layer's activation, where no pconv_linear_grad_input of a
 * layer behind it has applied the derivative already.
 *   dy, z, dz  device, dtype[M][N], row strides lddy, ldz, lddz; dz may be dy or z itself with the same row stride
 */
int pconv_activation_grad(const void* dy, long long lddy, const void* z, long long ldz, void* dz, long long lddz, int dtype, int M,
                          int N, int act, void* stream);

/*
 * Layer norm over the last axis (a row; of a channel-minor tensor [N][H][W][C]: the channels of a pixel):
 *     mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps),  y[d] = (x[d] - mean) * rstd * gamma[d] + beta[d]
 *   x, y         device, dtype[rows][D], row strides ldx, ldy; y may be x itself with the same row stride
 *   gamma, beta  device, float[D], or NULL for ones / zeros
 *   mean, rstd   device, float[rows]: receive the statistics for the backward pass, or NULL (each of its own)
 *   rows 0.., D 1.., eps >= 0
 * The variance is taken around the mean (two passes over the row, the second from registers or cache), and x - mean is good to
 * units of the row's spread, however far from 0 the row lies: equal values give beta and 1 / sqrt(eps).
 * PCONV_EINVAL also for an eps that is negative or not a number.
 */
int pconv_layer_norm(const void* x, long long ldx, const float* gamma, const float* beta, float eps, void* y, long long ldy,
                     float* mean, float* rstd, int dtype, int rows, int D, void* stream);

/*
 * The backward pass of layer norm.  With h = (x - mean) * rstd and g = dy * gamma:
 *     dx = rstd * (g - sum(g) / D - h * sum(g * h) / D),  dgamma[d] = sum over rows of dy * h,  dbeta[d] = sum over rows of dy
 *   dy, x         device, dtype[rows][D], row strides lddy, ldx
 *   mean, rstd    device, float[rows], from pconv_layer_norm.  (mean is rounded to fp32: h is off by half a unit of mean's last
 *                 place times rstd, which counts in rows whose spread is small against their level)
 *   gamma         device, float[D], or NULL for ones
 *   dx            device, dtype[rows][D], row stride lddx, or NULL; may be dy or x itself with the same row stride
 *   dgamma, dbeta device, float[D], or NULL (each of its own)
 *   workspace     device scratch of pconv_layer_norm_grad_workspace() bytes, aligned to 16 bytes; not needed (NULL) if dgamma
 *                 and dbeta are NULL
 * rows = 0 gives zeros in dgamma and dbeta.
 */
int pconv_layer_norm_grad_workspace(int dtype, int rows, int D, size_t* bytes);
int pconv_layer_norm_grad(const void* dy, long long lddy, const void* x, long long ldx, const float* gamma, const float* mean,
                          const float* rstd, void* dx, long long lddx, float* dgamma, float* dbeta, int dtype, int rows, int D,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * Distillation from a teacher's top logits.  Row r has V logits s of the network that is trained, and up to k entries
 * (index i_j, teacher's logit t_j).  With the temperature T and the row's weight w:
 *     p_j = exp(t_j / T) / sum over the row's entries of exp(t / T)      (the teacher, over what is stored of it)
 *     q_v = exp(s_v / T) / sum over all v of exp(s / T)
 *     loss[r]    = w * T^2 * sum over j of p_j * (log p_j - log q_{i_j})
 *     grad[r][v] = d loss[r] / d s_v = w * T * (q_v - sum over the j with i_j = v of p_j)
 *   logits   device, dtype[R][V], row stride ldl
 *   indices  device, int32[R][k]; an entry whose index lies outside [0, V) is not there (short lists end in -1); an index may
 *            come twice
 *   values   device, float[R][k]: the teacher's logits; -inf is a probability of 0; +inf or NaN in an entry that is there gives
 *            NaN in the row's loss and gradient.  Values of entries that are not there are not looked at
 *   weight   device, float[R], or NULL for ones
 *   loss     device, float[R], or NULL
 *   grad     device, dtype[R][V], row stride ldg, or NULL; may be logits itself with ldg = ldl
 *   stats    device, float[R][2], or NULL: receives what pconv_distill_grad needs of the row's softmax (the largest logit
 *            and the sum of exp((s - largest) / T)); zeros for a row that is left out
 *   R 0.., V 1.., k 1..1024, T > 0 and finite, log2(e) / T too (T from 4.25e-39 on; PCONV_EINVAL otherwise)
 * A row without entries, whose entries are all -inf, or of weight 0 is left out: loss and gradient 0, whatever its logits hold
 * (padding).  In other rows a logit of -inf has q = 0 (loss +inf if the teacher gives it more), +inf or NaN makes NaN.
 * loss, grad and stats are three results of one call; at least one is asked for (PCONV_EINVAL).
 */
int pconv_distill(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight, float* loss,
                  void* grad, long long ldg, float* stats, int dtype, int R, int V, int k, float temperature, void* stream);

/*
 * The gradient alone, for programs whose row weights are known only in the backward pass: grad as above, with
 * weight = dL/dloss of a pconv_distill call whose own weights were ones and which left `stats`.
 * Arguments as above; stats is read.
 */
int pconv_distill_grad(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight,
                       const float* stats, void* grad, long long ldg, int dtype, int R, int V, int k, float temperature, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PCONV_DENSE_H */
