/*
 * adamw.h -- C ABI of an AdamW step over many tensors at once for AMD MI355X (gfx950): what follows
 * astl_stack_backward in a training step.  Parameters in fp32, or in bf16 with or without an fp32 copy; the two
 * states in 32 bits or in 8.
 *
 * Per element, with t = 1, 2, ... the number of this step and g the gradient times the clipping factor:
 *   m' = beta1 m + (1 - beta1) g
 *   v' = beta2 v + (1 - beta2) g^2
 *   p' = p (1 - lr weight_decay) - lr / (1 - beta1^t) * m' / (sqrt(v') / sqrt(1 - beta2^t) + eps)
 * in fp32 (beta^t in fp64), p being the fp32 copy (`master`) where there is one.
 *
 * What is rounded to fewer bits and is all that the next step sees of it (8-bit states, bf16 parameters without an
 * fp32 copy) is rounded up or down at random, with the probability of the remainder: a change far below half a step, such
 * as (1 - beta2) of a second moment or most updates of a bf16 parameter, would be lost every time under rounding to
 * nearest.  The random numbers are a hash of (seed, t, element), so a run can be repeated bit by bit.
 *   element   the tensors of a plan stand one after another, each starting at a multiple of 256; e = its number there
 *   mix(x)    x ^= x >> 16;  x *= 0x9E3779B9;  x ^= x >> 15;  x *= 0x6A09E667;  x ^= x >> 16      (32 bits)
 *   key       k = mix(seed_hi ^ 0x510E527F);  k = mix(k ^ seed_lo);  k = mix(k ^ t_hi);  k = mix(k ^ t_lo);  k = mix(k ^ e_hi)
 *   h         mix(e_lo ^ k): its low 16 bits round m, its high 16 bits v;  the low 16 bits of mix(h ^ 0xBB67AE85) round p
 * The 16 bits are added below the last bit that is kept (aligned to it) and the rest is cut off.  An fp32 copy's
 * bf16 parameter is rounded to nearest.
 *
 * States in 8 bits (state_bits = 8): blocks of 256 elements of a tensor share a byte E, the biased fp32 exponent of
 * the block's largest magnitude.  An element keeps 3 bits behind its leading one: an fp32 pattern cut to its upper
 * 12 bits, T = exponent << 3 | mantissa, stored as the code c = T - 8 (E + 1) + top, so that code `top` is 2^(E + 1 - 127):
 *   m   sign bit, and c of 7 bits, top = 127: 15.75 powers of two; below code 1 it is 0
 *   v   c of 8 bits, top = 255: 31.75 powers of two; below code 1 it is code 1, or 0 if it is 0 itself
 * (c = 0 is the value 0; in the block with E = 254 codes stop below `top`; a pattern T below 1 is taken as 1).  A value is off by less than one
 * step of 2^-3 relative to its power of two, and right on average.  A block with an infinity or NaN in it has E = 255 and is NaN
 * as a whole from then on.
 * 32-bit states are plain fp32.  New states are zeros in every field of either kind.
 *
 * The conventions of gswa.h hold: `desc`, `tensors` and `plan` are HOST pointers, what they point at is DEVICE memory the caller owns;
 * nothing is allocated, freed or synchronised; all work is enqueued on `hip_stream`; a failed call has enqueued nothing.
 */
#ifndef ADAMW_H
#define ADAMW_H

#include "gswa.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    ADAMW_SKIP_NONFINITE = 1u << 0 /* a step whose `norm` is infinite or NaN changes nothing, the count of steps included */
};

typedef struct adamw_desc {
    double beta1, beta2; /* 0 <= beta < 1                                                                 */
    float eps;          /* 0, or at least 2^-126                                                          */
    int32_t state_bits; /* 32 or 8                                                                        */
    uint32_t flags;
    uint64_t seed;      /* of the random roundings                                                        */
} adamw_desc;

/* One tensor, of n contiguous elements; all pointers 16-byte aligned (m_exp and v_exp: any). */
typedef struct adamw_tensor {
    int64_t n;              /* >= 0                                                                       */
    int32_t p_dtype;        /* GSWA_F32 or GSWA_BF16                                                      */
    int32_t g_dtype;        /* GSWA_F32 or GSWA_BF16                                                      */
    float weight_decay;     /* >= 0                                                                       */
    void *p;                /* the parameter, updated                                                     */
    float *master;          /* its fp32 copy, updated, or NULL; only beside a GSWA_BF16 parameter. Then p is only written */
    const void *g;          /* its gradient                                                               */
    void *m, *v;            /* states: float[n], or uint8_t[n] codes                                      */
    uint8_t *m_exp, *v_exp; /* state_bits = 8: the byte E of every block, [(n + 255) / 256]; else NULL    */
} adamw_tensor;

/*
 * The tensors a step goes over, laid out for the device once: where they lie, not what they hold.  Filled by adamw_plan; valid as long as
 * the tensors and the buffer stay where they are.  Members are not for the caller.
 */
typedef struct adamw_plan_t {
    adamw_desc desc;
    int32_t n_tensors, each;
    int64_t chunks;   /* pieces of work                                                                   */
    int64_t blocks;   /* blocks of 256 elements                                                           */
    void *buffer;
    uint64_t check;
} adamw_plan_t;

/* Device memory of a plan in bytes, a multiple of 256. */
int adamw_query_bytes(const adamw_desc *desc, const adamw_tensor *tensors, int32_t n_tensors, size_t *plan_bytes);

/*
 * Lays the tensors out in `buffer` (256-byte aligned, of the queried size), by kernels on `hip_stream` that take the
 * tensors' places as arguments: `tensors` may go when the call returns.  Writable arrays must not overlap one another, any
 * gradient or the buffer (GSWA_EINVAL).  Two tensors may share a gradient.  At least one tensor; tensors of no elements are passed over.
 * 468 tensors take 0.06 ms of the host, four times their step: a plan is for tensors that stay where they are, gradients among them.
 */
int adamw_plan(const adamw_desc *desc, const adamw_tensor *tensors, int32_t n_tensors, void *buffer, adamw_plan_t *plan,
               void *hip_stream);

/* *norm = sqrt(sum over all gradients of g^2), summed in fp64 and in a fixed order: the same bits every run.  A gradient that two tensors share
 * counts twice. */
int adamw_norm(const adamw_plan_t *plan, float *norm, void *hip_stream);

/*
 * One step.  *step (device) is the number of steps taken so far, >= 0, and is raised by one, so that a captured step can be replayed: each plan
 * has a counter of its own.  step, norm and lr_scale lie outside the tensors and the plan's buffer.
 *   lr        learning rate; with lr_scale (device, may be NULL) it is lr * *lr_scale
 *   norm      as adamw_norm leaves it (device), or NULL.  Where *norm > max_norm the gradients are taken times max_norm / *norm;
 *             max_norm = 0: no clipping, norm is then only looked at for ADAMW_SKIP_NONFINITE
 * Calls on one plan must follow each other (they share the plan's buffer and the tensors).
 */
int adamw_step(const adamw_plan_t *plan, int64_t *step, float lr, const float *lr_scale, const float *norm, float max_norm,
               void *hip_stream);

/*
 * What 8-bit states stand for, as bf16 (which holds them whole): m_out and v_out [elements] with every tensor starting at a
 * multiple of 256 and zeros from its end to the next start; plan->blocks * 256 elements each, disjoint
 * from each other, from the tensors and from the plan's buffer.  Either may be NULL.  GSWA_EINVAL for a plan of
 * 32-bit states.
 */
int adamw_unpack(const adamw_plan_t *plan, void *m_out, void *v_out, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADAMW_H */
