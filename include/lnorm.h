/*
 * lnorm.h -- C ABI of LayerNorm over rows for AMD MI355X (gfx950), forward and backward: the norm that
 * opens and closes a sequence of the layers of astl.h (which take their own two norms themselves), with
 * the residual connection in front of it where there is one.
 *
 * Per row of C values:
 *   u  = x, or x + residual rounded to the element type and stored in `sum` (the norm is of what is stored)
 *   xh = (u - mean u) / sqrt(var u + eps)       mean and (biased) variance over the C values
 *   y  = xh * gamma + beta
 * and for a loss with gradient dy at y (and dsum at `sum`, from the rest of the residual path):
 *   g  = dy * gamma;  dx = (g - mean g - xh * mean(g * xh)) / sqrt(var u + eps) + dsum
 *   dgamma = sum over rows of dy * xh;  dbeta = sum over rows of dy
 * dx is the gradient at u, hence at x and at the residual alike.
 *
 * The conventions of gswa.h hold: `desc` is a HOST pointer, everything else a DEVICE pointer the caller
 * owns; nothing is allocated, freed or synchronised; all work is enqueued on `hip_stream`; arithmetic is in
 * fp32; gradients of parameters are fp32; a failed call has enqueued nothing.  Pointers are 16-byte aligned,
 * `ws` 256-byte aligned; the rows themselves need no alignment (any C, any stride).
 */
#ifndef LNORM_H
#define LNORM_H

#include "gswa.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LNORM_ACCUM_WGRAD = 1u << 0 /* lnorm_backward adds into dgamma and dbeta                              */
};

typedef struct lnorm_desc {
    int64_t rows;      /* > 0                                                                            */
    int32_t C;         /* values per row, 1 .. 16384                                                     */
    int32_t dtype;     /* GSWA_F32 or GSWA_BF16: x, residual, gamma, beta, y, sum, dy, dsum, dx          */
    float eps;         /* >= 0                                                                           */
    uint32_t flags;    /* LNORM_ACCUM_WGRAD                                                              */
    int64_t x_stride;  /* elements from one row of x to the next, >= C; 0 = C                            */
    int64_t y_stride;  /* the same of y and of dy                                                        */
    int64_t r_stride;  /* the same of residual, sum, dsum and dx                                         */
} lnorm_desc;

/* Scratch of lnorm_backward in bytes, a multiple of 256: a vector of 2 C partial sums for each workgroup.
 * lnorm_forward needs none. */
int lnorm_query_bytes(const lnorm_desc *desc, size_t *bwd_ws_bytes);

/*
 * residual and sum are both given or both NULL.  gamma may be NULL (ones), beta may be NULL (zeros).
 * y and sum must be disjoint, as byte ranges, from every other buffer of the call, except that sum may be x or
 * residual itself where the strides agree (the residual path updated in place).
 */
int lnorm_forward(const lnorm_desc *desc, const void *x, const void *residual, const void *gamma, const void *beta,
                  void *y, void *sum, void *hip_stream);

/*
 * x: what was normalised (the stored `sum` of the forward call where it had a residual; x_stride is ITS stride).
 * gamma may be NULL (ones); dsum may be NULL (no further gradient); dgamma and dbeta may be NULL (not wanted: ws
 * may then be NULL too), both or neither.  Statistics are computed again from x.  Parameter gradients are summed in
 * a fixed order: the same bits every run.  dx may be dy or dsum itself where the strides agree; otherwise dx,
 * dgamma, dbeta and ws must be disjoint from every other buffer.
 */
int lnorm_backward(const lnorm_desc *desc, const void *x, const void *dy, const void *gamma, const void *dsum,
                   void *dx, float *dgamma, float *dbeta, void *ws, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LNORM_H */
