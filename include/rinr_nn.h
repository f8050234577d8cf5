/* rinr_nn — operators for the network that learns from decoded batches (MI355X / gfx950).
 *
 * rinr_decode_batch (rinr.h) leaves a batch of images on the GPU.  These are the dense operators that a network of linear layers
 * on that batch needs for training and for answering: a linear layer whose bias, activation and residual are part of the product's
 * kernel, the root-mean-square norm with the residual's addition, and activations kept in 8 bits between the forward and the
 * backward pass.  RINR_ACT_SINE is the activation of the images' own models (Sec. II-A, sin(w0 z)), so that a sine MLP wider than
 * a store's models can be evaluated and trained too.
 *
 * Same conventions as rinr.h: plain C ABI, 0 or a negative RINR_E_* code, every pointer of this file is a device pointer, the caller
 * owns every buffer, nothing is allocated and nothing is waited for: kernels go to `stream` in order.  All matrices are
 * row-major with unit stride between columns; ld_* is the distance between rows in elements.  What a call writes shares no memory with what it
 * reads or with another result, but where a field says so.
 *
 * Types: RINR_T_BF16, _F16 and _F32 matrices, aligned to their element.  A packed matrix (RINR_T_PACKED8) holds 8-bit codes:
 * every 32 columns of a row (a block; the last may be shorter) share one scale byte e, the value is code * 2^(e - 127), codes are
 * -127..127, and e (1..254) is the least with which the block's largest value fits.  A block that holds an infinity or a NaN has
 * e = 255 and stands for NaN.  Codes: int8[rows][ld], ld a multiple of 32, 16-byte aligned, 0 behind the last column; scales:
 * uint8[rows][ld / 32].  Such a value has 7 significant bits, so bf16 (and f16 within its range) hold it exactly, and
 * products take it as it stands.  Beyond the range of bf16 (in f16: of f16) it stands for the largest finite number there, so that a finite block never gives an
 * infinity.
 *
 * At an infinity activations and slopes are their limits (GELU and SiLU: +inf and 1, 0 and 0); the sine's are NaN.  So a z kept in f16, infinite
 * beyond 65504, has the gradient that the finite one has, but for the sine.
 *
 * Sums (products, norms, gradients of bias and gain) are held in 32 bits.  Products of 32-bit operands take each operand as three
 * bf16 parts that add up to it and leave out what is below 2^-21 of a product; parts are cut off, so that has the product's sign.  An infinity in such an
 * operand makes results NaN where 32-bit arithmetic would keep the infinity.  Results are the same bits from call to call on one GPU.
 */
#ifndef RINR_NN_H
#define RINR_NN_H

#include "rinr.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { RINR_T_NONE = 0, RINR_T_BF16 = 1, RINR_T_F16 = 2, RINR_T_F32 = 3, RINR_T_PACKED8 = 4 };
enum { RINR_ACT_NONE = 0,
       RINR_ACT_RELU = 1,   /* max(z, 0), slope 0 at 0                 */
       RINR_ACT_GELU = 2,   /* z (1 + erf(z / sqrt 2)) / 2             */
       RINR_ACT_SILU = 3,   /* z / (1 + exp(-z))                       */
       RINR_ACT_SINE = 4 }; /* sin(w0 z)                               */
enum { RINR_NN_MAX_COLS = 32768,          /* columns of a norm's rows                          */
       RINR_NN_MAX_FEATURES = 1 << 20 };  /* inputs or outputs of a linear layer               */

/* y = act(x w' + bias) + residual. */
typedef struct {
    int64_t rows, n_in, n_out;             /* x [rows][n_in], w [n_out][n_in], y [rows][n_out]                       */
    const void *x; int64_t ld_x;           /* x_type: dtype or RINR_T_PACKED8                                        */
    const uint8_t *x_scales;               /* of a packed x, else NULL                                               */
    const void *w; int64_t ld_w;           /* dtype                                                                  */
    const float *bias;                     /* float[n_out] or NULL                                                   */
    const void *residual; int64_t ld_residual;   /* dtype [rows][n_out] or NULL; may be y itself                     */
    void *y; int64_t ld_y;                 /* dtype                                                                  */
    void *z; int64_t ld_z;                 /* what the activation is taken of, kept for the backward pass (or NULL)  */
    uint8_t *z_scales;                     /* of a packed z, else NULL                                               */
    int32_t dtype, x_type;
    int32_t z_type;                        /* RINR_T_NONE, dtype or RINR_T_PACKED8                                   */
    int32_t act;
    float w0;                              /* RINR_ACT_SINE's frequency, finite                                      */
    int32_t reserved;                      /* 0                                                                      */
} rinr_linear_args;

/* Bytes of workspace that rinr_linear needs (0: none; 0 on bad arguments): sums, where few workgroups share the
 * products' k, and x as dtype, where a large product takes a packed one. */
size_t rinr_linear_workspace_bytes(const rinr_linear_args *a);
/* workspace: 16-byte aligned device memory, in use until the call's kernels have run.  RINR_E_NULL / RINR_E_ARG (sizes, strides,
 * types;
 * y or z on top of x or w, y on part of the residual) / RINR_E_SIZE (workspace_bytes less than that) / RINR_E_ALIGN / RINR_E_HIP.  rows = 0 does nothing. */
int rinr_linear(const rinr_linear_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of y = act(z), z = x w' + bias, given dy (the residual's gradient is dy itself):
 * dz = dy act'(z), dx = dz w, dw = dz' x, dbias = sum of dz's rows.
 * With x_act, x holds what an activation was taken of (a z that the layer before kept): the layer's input was x_act(x), dw is taken
 * with that, and dx is the gradient of x before x_act: dx = (dz w) x_act'(x).
 * dx, dw, dbias: each may be NULL.  dz is rounded to dtype once, for both products; dbias is summed before that.  x_act(x) is rounded to dtype for dw, but
 * where dz is rounded too (both activations, 16 bits): there it is taken as two of dtype, so that one rounding at most adds to the result's own. */
typedef struct {
    int64_t rows, n_in, n_out;
    const void *dy; int64_t ld_dy;         /* dtype [rows][n_out]                                                    */
    const void *x; int64_t ld_x;           /* x_type: dtype or RINR_T_PACKED8; NULL where neither dw nor x_act's slope needs it */
    const uint8_t *x_scales;
    const void *w; int64_t ld_w;           /* dtype [n_out][n_in]; NULL where dx is                                  */
    const void *z; int64_t ld_z;           /* z_type: RINR_T_NONE where act is RINR_ACT_NONE                         */
    const uint8_t *z_scales;
    void *dx; int64_t ld_dx;               /* dtype [rows][n_in]                                                     */
    void *dw; int64_t ld_dw;               /* dtype [n_out][n_in]                                                    */
    float *dbias;                          /* float[n_out]                                                           */
    int32_t dtype, x_type, z_type, act, x_act;
    float w0;                              /* of both activations                                                    */
} rinr_linear_grad_args;

/* Bytes of workspace that rinr_linear_backward needs (0 on bad arguments). */
size_t rinr_linear_backward_workspace_bytes(const rinr_linear_grad_args *a);
/* RINR_E_SIZE if workspace_bytes is less than that; else as rinr_linear.  rows = 0 sets dw and dbias to 0. */
int rinr_linear_backward(const rinr_linear_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* h = x + residual, y = gain h / sqrt(mean(h^2) + eps), per row; mean and y from h in 32 bits, before h is rounded to dtype. */
typedef struct {
    int64_t rows, cols;                    /* cols 1..RINR_NN_MAX_COLS                                               */
    const void *x; int64_t ld_x;           /* dtype                                                                  */
    const void *residual; int64_t ld_residual;   /* dtype or NULL (then h is not written either)                     */
    const float *gain;                     /* float[cols]                                                            */
    void *y; int64_t ld_y;                 /* y_type: dtype or RINR_T_PACKED8                                        */
    uint8_t *y_scales;                     /* of a packed y, else NULL                                               */
    void *h; int64_t ld_h;                 /* dtype; may be x or residual; NULL: not kept                            */
    int32_t dtype, y_type;
    float eps;                             /* > 0                                                                    */
    int32_t reserved;                      /* 0                                                                      */
} rinr_norm_args;
/* RINR_E_NULL / RINR_E_ARG / RINR_E_UNSUPPORTED (cols) / RINR_E_ALIGN / RINR_E_HIP. */
int rinr_rms_norm(const rinr_norm_args *a, void *stream);

/* Gradients of y in rinr_rms_norm: with s = 1 / sqrt(mean(h^2) + eps), u = h s, g = dy gain:
 * dh = s (g - u mean(g u)) + dres (the gradient of x and of the residual alike), dgain = sum over rows of dy u. */
typedef struct {
    int64_t rows, cols;
    const void *dy; int64_t ld_dy;         /* dtype                                                                  */
    const void *h; int64_t ld_h;           /* dtype: the sum that the norm was taken of                              */
    const float *gain;
    const void *dres; int64_t ld_dres;     /* dtype: the gradient that arrives at h on another path, or NULL         */
    void *dh; int64_t ld_dh;               /* dtype; may be dy or dres                                               */
    float *dgain;                          /* float[cols] or NULL                                                    */
    int32_t dtype;
    float eps;
} rinr_norm_grad_args;
/* Bytes of workspace that rinr_rms_norm_backward needs where dgain is asked for (0 on bad arguments). */
size_t rinr_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols);
/* RINR_E_SIZE if workspace_bytes is less than that and dgain is not NULL; else as rinr_rms_norm. */
int rinr_rms_norm_backward(const rinr_norm_grad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* 8-bit checkpoints: x (dtype) to codes and scales, and back through an activation (act, w0 as above). */
int rinr_pack8(int64_t rows, int64_t cols, const void *x, int64_t ld_x, int32_t dtype, void *codes, int64_t ld, uint8_t *scales, void *stream);
int rinr_unpack8(int64_t rows, int64_t cols, const void *codes, int64_t ld, const uint8_t *scales, int32_t act, float w0, void *x, int64_t ld_x,
                 int32_t dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif
