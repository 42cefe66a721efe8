/*
 * fpsk_decoder.h - the operators on a decoder's other verified accumulators: the output projection's and the head's.
 *
 * The output projection of a layer and the head are products whose FP32 accumulators are delivered un-narrowed so that they can be
 * probed, like the QKV projection's (fpsk_attention.h).  What follows them reads the accumulators: the addition to the
 * residual stream with the next norm, whose output is the next product's operand, and on the head's logits the penalties,
 * biases and grammar masks of an answer, or the loss against a teacher's top logits with its gradient.
 *
 * The conventions of fpsk.h hold: the caller owns every buffer, nothing is allocated, every call is asynchronous on `stream`
 * without a host synchronisation, errors are return codes, nothing throws.  Strides are in ELEMENTS between rows; the elements
 * of a row are contiguous.  Types are fpsk_elem; a row may start anywhere that its type may.  Rows of 0 do nothing.  Sums, norms
 * and exponentials are FP32 in a fixed order: a call gives the same bits each time on one device.  d_status is a device int32 or
 * NULL, to which the kernels only ever write an fpsk_status other than FPSK_OK (FPSK_ERR_TIMEOUT: a device-side wait gave up, and
 * what the call wrote is not to be used).
 */
#ifndef FPSK_DECODER_H
#define FPSK_DECODER_H

#include "fpsk_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FPSK_MAX_NORM_DIM 32768

/* Residual addition and norm, row by row:  h = x + residual, stored to residual_out rounded once;
 *   y = h r w,  r = rsqrt(mean(h^2) + eps)        (from the sum in FP32, not from the stored one)
 * rounded once to y_type; or, with y_type FPSK_ELEM_E4M3, y / s rounded (ties to even, at most 448 in magnitude) with
 * s = max(max |y| / 448, 2^-126) over each group of `group` channels of the row (the last group may be shorter), 1 where the group is all
 * zeros, NaN where it holds a NaN.  A group with an infinity has that for its scale and NaN or 0 for its values. */
typedef struct {
    const void *x;               /* device, n_tokens rows of dim values of x_type                      */
    const void *residual;        /* device, residual_type; NULL: h = x                                 */
    const void *weight;          /* device, dim values of weight_type; NULL: 1                         */
    void *residual_out;          /* device, residual_type; NULL: not stored.  May be `residual`        */
    void *y;                     /* device, y_type.  May be x or residual, of the same type and stride  */
    float *scale;                /* device, ceil(dim / group) a row (1 when group = 0); with FPSK_ELEM_E4M3 only */
    int64_t x_stride, residual_stride, residual_out_stride, y_stride, scale_stride;
    int64_t n_tokens;
    int32_t dim;                 /* 1 .. FPSK_MAX_NORM_DIM                                             */
    int32_t x_type, residual_type, weight_type, y_type;
    int32_t group;               /* 0 (the whole row), 32, 64, 128 or 256                              */
    float eps;
} fpsk_add_norm;
fpsk_status fpsk_add_rms_norm(const fpsk_add_norm *a, int32_t *d_status, void *stream);

/* Its backward pass, from the sum h (residual_out, or x where there was no residual), the gradient dy of y and the gradient dh that
 * arrives at the sum from elsewhere (NULL: none).  With n = h r and g = dy w:
 *   dx = r (g - n mean(g n)) + dh       the gradient of x and of the residual alike
 *   dweight = sum over the tokens of dy n
 * (an 8-bit y passes its gradient straight through).  The workspace needs no initialisation and serves one call at a time. */
typedef struct {
    const void *h;               /* device, h_type                                                     */
    const void *dy, *dh;         /* device, grad_type                                                  */
    const void *weight;          /* device, weight_type; NULL: 1                                       */
    void *dx;                    /* device, grad_type.  May be dy or dh, of the same stride            */
    float *dweight;              /* device, dim floats, overwritten; NULL: not wanted                  */
    int64_t h_stride, dy_stride, dh_stride, dx_stride;
    int64_t n_tokens;
    int32_t dim;
    int32_t h_type, grad_type, weight_type;
    float eps;
} fpsk_add_norm_grad;
size_t fpsk_add_norm_workspace_bytes(int32_t dim);
fpsk_status fpsk_add_rms_norm_backward(const fpsk_add_norm_grad *a, void *workspace, size_t ws_bytes, int32_t *d_status, void *stream);

#define FPSK_MAX_VOCAB (1 << 23)
#define FPSK_MAX_HISTORY (1 << 28)

/* What is done to a row of logits before a token is picked, in this order, in FP32:
 *   tokens that the row's history holds:      z > 0 ? z / repetition : z * repetition     (by a product with 1 / repetition)
 *   c times behind the first prompt_len:      z -= frequency c + presence
 *   tokens of the row's list of biases:       z += the sum of their biases, in the list's order
 *   tokens whose bit of the row's mask is 0:  z = -inf, whatever the logit (NaN too)
 * stored to `out`, rounded once, and / or read for the token of the largest z (from the FP32 values; ties go to the lowest token, a NaN
 * is larger than all; -1 where every z is -inf) and the log of the sum of their exponentials. */
typedef struct {
    const void *logits;          /* device, n_rows rows of vocab values                                */
    void *out;                   /* device, out_type, or NULL.  May be logits, of the same type and stride */
    int64_t logits_stride, out_stride;
    int64_t n_rows;
    int32_t vocab;               /* 1 .. FPSK_MAX_VOCAB                                                */
    int32_t logits_type, out_type;
    int32_t history_width;
    const int32_t *history;      /* device, history_width tokens a row, prompt first, or NULL.  What is no token (-1) is passed over */
    const int32_t *history_len;  /* device, how many of them count; NULL: all                          */
    const int32_t *prompt_len;   /* device, how many of those are the prompt's; NULL: none              */
    int64_t history_stride;
    const float *repetition, *frequency, *presence;   /* device, one a row; NULL: 1, 0, 0              */
    const int32_t *bias_ptr;     /* device, n_rows + 1: row r has the entries bias_ptr[r] .. bias_ptr[r + 1] - 1, or NULL */
    const int32_t *bias_token;   /* device, n_biases.  What is no token is passed over                  */
    const float *bias_value;     /* device, n_biases                                                   */
    int64_t n_biases;
    const int32_t *mask;         /* device, n_masks rows of ceil(vocab / 32) words, bit v % 32 of word v / 32: token v is allowed */
    const int32_t *mask_row;     /* device, the mask of each row, -1: none; NULL: row r has mask r.  A mask that there is not allows
                                    nothing and sets *d_status to FPSK_ERR_PARAM                       */
    int64_t mask_stride, n_masks;
    int32_t *token;              /* device, one a row, or NULL                                         */
    float *lse;                  /* device, one a row, or NULL                                         */
} fpsk_logits;
fpsk_status fpsk_adjust_logits(const fpsk_logits *a, int32_t *d_status, void *stream);

#define FPSK_MAX_TOP 1024

/* The loss of each row of logits x against a teacher's top logits t of some tokens:
 *   q = softmax(x / temperature) over the vocabulary;  p = softmax(t / temperature) over the listed tokens when normalize, else exp(t)
 *   loss = sum_j p_j (log p_j - log q_j),   d loss / d x_v = (m q_v - p_v) / temperature,   m = sum_j p_j
 * Entries whose token is outside the vocabulary (-1) are left out, before p is normalised; a token that is listed twice counts twice;
 * an entry with t = -inf adds nothing.  A row without entries has loss 0 and gradient 0.
 * fpsk_distill_loss stores the losses, lse (of x / temperature) where wanted, and, where dlogits is given, the gradients of
 * sum_r row_weight_r loss_r, in one launch that reads the logits once.  fpsk_distill_loss_backward makes the gradients alone, from
 * the lse of the forward pass and the gradients of the rows' losses in row_weight.  A row of weight 0 is not read: its loss and lse are
 * 0 and its gradient zeros, whatever it holds. */
typedef struct {
    const void *logits;          /* device, n_rows rows of vocab values                                */
    const void *teacher_token;   /* device, `top` a row, int32 (token_bytes = 4) or int64 (8)          */
    const void *teacher_logit;   /* device, `top` a row, teacher_type                                  */
    const float *row_weight;     /* device, one a row; NULL: 1                                         */
    float *loss;                 /* device, one a row (fpsk_distill_loss)                              */
    float *lse;                  /* device, one a row; may be NULL in fpsk_distill_loss                 */
    void *dlogits;               /* device, grad_type; may be NULL in fpsk_distill_loss.  May be logits, of the same type and stride */
    int64_t logits_stride, token_stride, teacher_stride, dlogits_stride;
    int64_t n_rows;
    int32_t vocab, top;          /* 1 .. FPSK_MAX_VOCAB, 0 .. FPSK_MAX_TOP                             */
    int32_t logits_type, token_bytes, teacher_type, grad_type;
    int32_t normalize;
    float temperature;           /* positive and finite, 5e-39 at least                                */
} fpsk_distill;
fpsk_status fpsk_distill_loss(const fpsk_distill *a, int32_t *d_status, void *stream);
fpsk_status fpsk_distill_loss_backward(const fpsk_distill *a, int32_t *d_status, void *stream);
/* The two for a gradient that is not rounded at the size of the log-sum-exp: `sums` (device, two floats a row; NULL: as above) takes a
 * number M near each row's largest logit and S = sum_v exp((x_v - M) / temperature), so that lse = M / temperature + ln S.  The backward
 * pass reads them in place of lse, which may be NULL.  (From an FP32 lse a gradient is off by lse's rounding, relative: 5e-7 at 10, 3e-5
 * at 700.) */
fpsk_status fpsk_distill_loss_sums(const fpsk_distill *a, float *sums, int32_t *d_status, void *stream);
fpsk_status fpsk_distill_loss_backward_sums(const fpsk_distill *a, const float *sums, int32_t *d_status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FPSK_DECODER_H */
