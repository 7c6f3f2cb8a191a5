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
 *   block norm    the norms after and before a block fused with
 *                 its gate and residual scale, see nr_block_norm nr_block_norm_forward
 *   its gradients                                               nr_block_norm_backward
 *   AdamW         a step over all parameters, see nr_adamw      nr_adamw_step, nr_adamw_read,
 *                                                               nr_grad_norm
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

/* norms */
enum { NR_NORM_NONE = 0, NR_NORM_RMS = 1, NR_NORM_LAYER = 2 };
/* gates: NR_ACT_SILU, or the logistic function */
enum { NR_ACT_SIGMOID = 4 };

/* What lies between a block's last product and the next one's first: with the
 * residual stream r, the block's output u and its gate q (the gate's argument),
 *   uh = u, u ru or (u - mean) ru  post none, RMS, layer; ru = (mean square + eps)^-1/2,
 *                                  for the layer norm of the deviations from the mean
 *   c  = uh post_weight + post_bias
 *   y  = alpha r + scale a(q) c    a(q) = 1 without a gate
 *   h  = yh weight + bias          yh of y as uh of u, by pre; none: no h
 * and, without u, y = r: then h alone is made, and y may be NULL. h is made from y before
 * its rounding. Gradients, with g = dh weight:
 *   t  = dy + ry (g - mean(g) - yh mean(g yh))  the mean for the layer norm only; dr = alpha t
 *   dq = t scale a'(q) c, its row's sum if gate_cols = 1
 *   e  = t scale a(q) post_weight, du = ru (e - mean(e) - uh mean(e uh)), as for t
 *   A = sum t a(q) uh, B = sum t a(q) over the rows: dpost_weight = scale A,
 *   dpost_bias = scale B, dscale = post_weight A + post_bias B
 *   dweight = sum dh yh, dbias = sum dh
 * Backward takes y and the statistics as forward left them, yh = (y - mean) ry. Statistics and h are of y before
 * its rounding, so that a 16-bit y moves yh by up to half a unit of y's last place times ry: little for rows around
 * zero, a quarter of a deviation in bf16 for a mean of 100 deviations. r_dtype NR_F32 has none of it to speak of. */
typedef struct {
  int64_t m, n;
  int64_t dtype;     /* of u, gate, h, dh, du, dgate: NR_F32, NR_F16 or NR_BF16 */
  int64_t r_dtype;   /* of r, y, dy, dr: dtype or NR_F32 */
  int64_t w_dtype;   /* of the vectors and their gradients: dtype or NR_F32 */
  int64_t post, pre; /* norms */
  int64_t gate_act;  /* NR_ACT_SIGMOID or NR_ACT_SILU */
  int64_t gate_cols; /* n, or 1: a gate for each row */
  double alpha;      /* in fp32's range */
  double eps;        /* forward; > 0 */
  const void *r;     /* [m x n]; forward */
  int64_t r_ld;
  const void *u;     /* [m x n], or NULL */
  int64_t u_ld;
  const void *gate;  /* [m x gate_cols], or NULL; needs u */
  int64_t gate_ld;
  const void *scale; /* [n], or NULL: ones; needs u */
  const void *post_weight, *post_bias; /* [n], or NULL: ones, zeros; need post */
  const void *weight, *bias;           /* [n], or NULL: ones, zeros; need pre */
  void *y;           /* [m x n]; forward: out; backward: in, needed with pre */
  int64_t y_ld;
  void *h;           /* [m x n]; forward: out */
  int64_t h_ld;
  float *stats;      /* [s x m], or NULL forward: of u its mean (layer) and ru, of y its mean
                      * (layer) and ry, those there are, one after the other */
  const void *dh;    /* [m x n]; backward, with pre */
  int64_t dh_ld;
  const void *dy;    /* [m x n]; backward, or NULL with pre: zeros */
  int64_t dy_ld;
  void *dr;          /* [m x n]; backward: out */
  int64_t dr_ld;
  void *du;          /* [m x n]; backward: out, with u */
  int64_t du_ld;
  void *dgate;       /* [m x gate_cols]; backward: out, with a gate */
  int64_t dgate_ld;
  void *dscale, *dpost_weight, *dpost_bias, *dweight, *dbias; /* [n]; backward: out, or NULL each */
} nr_block_norm;

/* as nr_linear_backward_workspace */
int64_t nr_block_norm_backward_workspace(const nr_block_norm *a, int device);
nr_status nr_block_norm_forward(const nr_block_norm *a, int device, void *stream);
nr_status nr_block_norm_backward(const nr_block_norm *a, int device, void *ws, int64_t ws_bytes, void *stream);

/* A parameter tensor of an AdamW step; every field is 8 bytes wide. */
typedef struct {
  int64_t n;         /* values; 0 <= n < 2^40 */
  int64_t at;        /* where its averages begin in m, v and master: a multiple of 32; from there up to the
                      * next multiple of 32 behind them the arrays are the tensor's */
  int64_t p_dtype, g_dtype;
  double decay;      /* weight decay, >= 0 */
} nr_adamw_tensor;

/* An AdamW step. With g' = g coef, coef = min(1, max_norm / (norm + 1e-6)) and norm the 2-norm of
 * all gradients (max_norm > 0; else coef = 1 and no norm is made), t = *step + 1:
 *   m' = beta1 m + (1 - beta1) g',  v' = beta2 v + (1 - beta2) g'^2
 *   p' = p (1 - lr decay) - lr / (1 - beta1^t) m' / ((v' / (1 - beta2^t))^1/2 + eps)
 * and *step = t. A norm that is infinite or NaN leaves everything as it was, *step too. Its squares are
 * added in fp32: a gradient of 2^60 or more may make it infinite, and ones below 2^-63 lose digits. A 16-bit p
 * with a master is the master's rounding, and the master is what the step reads and updates; without
 * one p' itself is rounded, and changes below half a unit of its last place are lost.
 *
 * Averages in 32 bits are fp32; m' and v' are rounded at every operation. In 8 bits, 32
 * neighbours share 2^e, the least with |x| < 2^e (2 - 1/16) for all of them, e in [-108, 127],
 * held as the byte e + 120; a group with an infinity or NaN has the byte 255 and reads as NaN.
 * With E the exponent of the value, but at least e - 6 (m) or e - 14 (v), and S = floor(|x| /
 * 2^(E-4) + d / 2^16) the code is 16 (E - e + 6 or 14) + S, at most 127 or 255, and stands for S 2^(E-4); m's
 * sign is bit 7. A v above zero has at least the code 1. So m keeps 4 bits after the leading
 * one over 7 binades and v over 15, below which steps are equal. The dither d makes the held value right on
 * average: to nearest, v would stand still, as a step changes it by a share of 1 - beta2 and half
 * a unit of its last place is 1/32 to 1/64. d is 16 bits of Philox4x32 with 7 rounds (Salmon, Moraes,
 * Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11): key seed, counter (i / 4, t), two 64-bit
 * numbers, for place i of the arrays; of word i mod 4 m has the low half and v the high half. p' is
 * made from m' and v' before they are held. */
typedef struct {
  int64_t count;
  /* host memory, free for reuse after the call: the tensors, their values (contiguous; updated) and
   * their gradients (contiguous; NULL: the tensor and its averages are left as they are) */
  const nr_adamw_tensor *tensors;
  void *const *p;
  const void *const *g;
  int64_t bits;      /* of the averages: 32 or 8 */
  float *master;     /* of the 16-bit parameters, or NULL */
  void *m, *v;       /* 16-byte aligned: float, or uint8 codes */
  void *m_scale, *v_scale; /* 8 bits: a byte for 32 places */
  int64_t *step;     /* device */
  int32_t *ticket;   /* device; zero before the first call, and left zero */
  double lr;         /* in fp32's range, as decay */
  const float *lr_at; /* device, or NULL: lr */
  double beta1, beta2; /* in [0, 1) */
  double eps;        /* > 0 */
  double max_norm;   /* 0: no clipping */
  float *norm;       /* device; out, with max_norm */
  int64_t seed;
} nr_adamw;

/* Calls on one state follow one another on a stream; a CUDA graph may hold them, as step and lr_at are
 * read on the device. Outputs do not depend on timing. */
int64_t nr_adamw_workspace(const nr_adamw *a, int device);
nr_status nr_adamw_step(const nr_adamw *a, int device, void *ws, int64_t ws_bytes, void *stream);
/* y_m[i], y_v[i] = the values that m's and v's codes i stand for, i < n (a multiple of 32), in bf16, exactly;
 * codes and outputs 16-byte aligned. */
nr_status nr_adamw_read(const void *m, const void *m_scale, const void *v, const void *v_scale, int64_t n, void *y_m, void *y_v,
                        int device, void *stream);
/* *norm = the 2-norm of all gradients a->g of a->tensors (only count, tensors' n and g_dtype, and g are read) */
nr_status nr_grad_norm(const nr_adamw *a, float *norm, int device, void *ws, int64_t ws_bytes, void *stream);

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
