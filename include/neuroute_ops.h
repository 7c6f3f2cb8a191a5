/*
 * neuroute_ops.h -- operators for training and serving encoders other than
 * the index file's own: residual encoders with layer norms, whose logits go
 * to nr_build_set_logits and nr_search_logits. The pairwise loss L_sim (paper
 * Sec. 3.2.2) couples every pair of a mini-batch, so all activations of a
 * batch are held at once; the 8-bit checkpoints hold them at half the bytes.
 *
 *   linear        z = x w^T + bias, y = act(z) + residual       nr_linear_forward
 *   its gradients dz = dy act'(z), dx = dz w, dw = dz^T x,
 *                 dbias = sum of dz's rows                      nr_linear_backward
 *   layer norm    xh = (x - mean) rstd, y = xh weight + bias,
 *                 rstd = (variance + eps)^-1/2, the variance
 *                 being the mean square deviation               nr_layer_norm_forward
 *   its gradients g = dy weight, dx = rstd (g - mean(g) -
 *                 xh mean(g xh)) + residual gradient, dweight =
 *                 sum dy xh, dbias = sum dy over the rows       nr_layer_norm_backward
 *   checkpoint    see below                                     nr_checkpoint8_write, _read
 *
 * Activations: none, ReLU max(z, 0) with slope [z > 0], GELU z Phi(z) with the
 * normal distribution's Phi, SiLU z / (1 + e^-z).
 *
 * Types. Matrices are row-major with any row pitch (ld, elements) and no
 * alignment beyond their element's; rows may repeat (ld = 0) where they are only
 * read. x, w, residual, z, dx and dw are fp16 or bf16 (one type a call); y and dy
 * that type or fp32; bias and dbias fp32 or that type. The layer norm takes
 * x, y, dy, dx and the residual's gradient in fp32, fp16 or bf16 (one type a
 * call), weight, bias and their gradients in fp32 or that type, mean and
 * rstd in fp32. Sums, statistics and activations are held in fp32 and rounded
 * once, at the output, except dz, which is rounded to x's type for the
 * products that make dx and dw, also where dy is fp32 (dbias sums it unrounded):
 * in bf16 their errors, 0.0017 of the norm from their own rounding, become 0.0023.
 *
 * Exponentials and reciprocals in the activations are the hardware's approximate
 * ones, and GELU's Phi is formula 7.1.26 of Abramowitz and Stegun (7.5e-8). Values
 * are good to 2^-20 |z| and slopes to 2^-19, absolutely, before their rounding; GELU's
 * lower tail so has few digits: 5e-4 of its value at z = -4, 4e-3 at -6.
 *
 * 8-bit checkpoints. Each row is cut into groups of 32 columns (the last may
 * be shorter). A group's scale is 2^e with e the least whole number in
 * [-126, 121] for which every |v| < 127.5 2^e; a value is held as
 * round(v / 2^e), ties to even, within +-127, and stands for that number
 * times 2^e (exact in bf16, and in fp16 within its range; beyond it the largest
 * finite value). The scale is stored as the byte e + 133; a group with an
 * infinity or NaN stores 255 and reads back as NaN, all of it. Codes: int8
 * [m x 32 ceil(n / 32)], the columns past n zero; scales: uint8
 * [m x ceil(n / 32)]; both contiguous, codes 16-byte aligned.
 *
 * Conventions as in neuroute.h: device pointers on `device`, asynchronous on
 * `stream` (a cudaStream_t), argument errors returned before any work.
 * Nothing is allocated: a call that needs scratch takes it from `ws` (at least
 * the bytes that the _workspace function gives, 256-byte aligned, free for
 * reuse once the stream has passed the call). No outputs may overlap inputs.
 * Results do not depend on timing: sums have a fixed order for given sizes,
 * types and alignments. m = 0 is a no-op, but gradients of parameters are
 * then zeroed. m < 2^31; 1 <= k, n < 2^24.
 */
#ifndef NEUROUTE_OPS_H
#define NEUROUTE_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "neuroute.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
enum { NR_F32 = 0, NR_F16 = 1, NR_BF16 = 2 };
/* activations */
enum { NR_ACT_NONE = 0, NR_ACT_RELU = 1, NR_ACT_GELU = 2, NR_ACT_SILU = 3 };

/* Arguments of the linear layer; every field is 8 bytes wide. A pointer that
 * is NULL leaves its part out. */
typedef struct {
  int64_t m, k, n;     /* rows, inputs, outputs */
  int64_t dtype;       /* of x, w, residual, z, dx, dw: NR_F16 or NR_BF16 */
  int64_t y_dtype;     /* of y and dy: dtype or NR_F32 */
  int64_t bias_dtype;  /* of bias and dbias: dtype or NR_F32 */
  int64_t act;
  const void *x;       /* [m x k]; backward: int8 codes if x_scale is given */
  int64_t x_ld;
  const void *x_scale; /* backward only */
  int64_t x_act;       /* backward, codes only: the layer's input is x_act(held value) */
  const void *w;       /* [n x k] */
  int64_t w_ld;
  const void *bias;    /* [n]; forward */
  const void *residual;/* [m x n]; forward */
  int64_t residual_ld;
  void *y;             /* [m x n]; forward: out */
  int64_t y_ld;
  void *z;             /* [m x n]; forward: out, or NULL; backward: in, needed
                        * unless act is none. int8 codes if z_scale is given */
  int64_t z_ld;
  void *z_scale;
  const void *dy;      /* [m x n]; backward */
  int64_t dy_ld;
  void *dx;            /* [m x k]; backward: out, or NULL */
  int64_t dx_ld;
  void *dw;            /* [n x k] contiguous; backward: out, or NULL */
  void *dbias;         /* [n]; backward: out, or NULL */
} nr_linear;

/* Scratch bytes of a call with these sizes, types, alignments and outputs, or
 * NR_ERR_INVALID_ARG, or NR_ERR_CUDA if the device is not there (both negative). */
int64_t nr_linear_forward_workspace(const nr_linear *a, int device);
int64_t nr_linear_backward_workspace(const nr_linear *a, int device);

/* Errors: NR_ERR_INVALID_ARG (sizes, types, a missing pointer, a matrix or codes
 * at an address that is no multiple of their alignment, ws_bytes too small),
 * NR_ERR_CUDA. */
nr_status nr_linear_forward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream);
nr_status nr_linear_backward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream);

/* Arguments of the layer norm; every field is 8 bytes wide. */
typedef struct {
  int64_t m, n;        /* rows and their length */
  int64_t dtype;       /* of x, y, dy, dx, residual_grad */
  int64_t w_dtype;     /* of weight, bias, dweight, dbias: dtype or NR_F32 */
  double eps;          /* forward; > 0 */
  const void *x;       /* [m x n], int8 codes if x_scale is given */
  int64_t x_ld;
  const void *x_scale;
  const void *weight;  /* [n], or NULL: ones */
  const void *bias;    /* [n], or NULL: zeros; forward */
  void *y;             /* [m x n]; forward: out */
  int64_t y_ld;
  float *mean, *rstd;  /* [m]; forward: out, or both NULL; backward: in */
  const void *dy;      /* [m x n]; backward */
  int64_t dy_ld;
  const void *residual_grad; /* [m x n], or NULL; backward: added to dx */
  int64_t residual_grad_ld;
  void *dx;            /* [m x n]; backward: out */
  int64_t dx_ld;
  void *dweight, *dbias; /* [n]; backward: out, or both NULL */
} nr_layer_norm;

/* as nr_linear_backward_workspace */
int64_t nr_layer_norm_backward_workspace(const nr_layer_norm *a, int device);
nr_status nr_layer_norm_forward(const nr_layer_norm *a, int device, void *stream);
nr_status nr_layer_norm_backward(const nr_layer_norm *a, int device, void *ws, int64_t ws_bytes,
                                 void *stream);

/* Holds x [m x n] (pitch x_ld; fp32, fp16 or bf16) in 8 bits: codes and scales
 * as described above. */
nr_status nr_checkpoint8_write(const void *x, int dtype, int64_t m, int64_t n, int64_t x_ld,
                               void *codes, void *scales, int device, void *stream);
/* y [m x n] (pitch y_ld; fp32, fp16 or bf16) = act(held values). */
nr_status nr_checkpoint8_read(const void *codes, const void *scales, int64_t m, int64_t n, int act,
                              void *y, int dtype, int64_t y_ld, int device, void *stream);

/* Waits for the device, then NR_ERR_DEVICE_CHECK if a bounded wait inside one
 * of these operators' kernels has expired on `device` since the last such call
 * (their outputs are then undefined), else NR_OK. */
nr_status nr_ops_status(int device);

/* Execution only: the limit of the bounded waits, in microseconds, for calls
 * that follow, at most 60000000 (else NR_ERR_INVALID_ARG and no change). 0
 * (default): 1 s. < 0: a wait whose phase is not complete when first tested
 * expires at once, which exercises the failure path. */
nr_status nr_ops_wait_limit(int64_t us);

#ifdef __cplusplus
}
#endif
#endif
