/*
 * zvc_adamw.h -- C ABI of the optimizer's step (libzvc_adamw.so), AMD gfx950: AdamW over many
 * tensors in one launch, states in 32 bits or in 8.
 *
 * Step t >= 1 of a tensor's weights p from its gradient, both elementwise:
 *
 *     g = factor * gradient
 *     m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
 *     p = (1 - rate * decay) p - rate / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * in 32 bits, with g, m and v by these multiplications and additions, each rounded.  Weights of 16 bits are rounded to the nearest
 * number, so a change of less than half a unit is lost; a tensor with a 32-bit `master` keeps its weights there, and
 * d_param receives them rounded.
 *
 * States of 8 bits (state_bits = 8) hold m and r = sqrt(v) as numbers of the e4m3 format (sign, four bits of exponent with a bias of 7,
 * three of mantissa, no infinities; code 0x7F, its NaN, is not written), each block of 128 consecutive elements
 * with a scale in 32 bits: a value is its code's number times the scale.  A step writes the scale 2^(e-7) with 2^e <= the block's largest
 * finite magnitude < 2^(e+1) (e not below -95) and rounds values over the scale stochastically: up with the probability of what is cut off, in units of
 * 2^-16, so that a change too small for the format is kept on the average.  An r above 0 is never rounded to 0 (m over it would not be bounded).  What is not
 * finite is stored as the largest number, 448.  Element i of tensor number j (its place in the plan) takes half i % 8 of Philox4x32-10
 * (see zvc_ffn.h) with key = seed and counter = (i / 8, j, t low, t high), the low half of each word first; m and r take the same one.
 * So a step's result is a function of its arguments, whatever the order of work.
 *
 * Tensors, scales and steps are given by a plan, made once on the host; a step is one launch.  Conventions are those of zvc.h.
 */
#ifndef ZVC_ADAMW_H_
#define ZVC_ADAMW_H_

#include "zvc_ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One tensor; the pointers are device pointers, aligned to their elements. */
typedef struct zvc_adamw_tensor {
    void* d_param;         /* count weights */
    float* d_master;       /* null, or the weights in 32 bits (16-bit weights only) */
    const void* d_grad;    /* count gradients */
    void* d_m;             /* state_bits 32: count floats each, m and v; 8: count codes each, m and r */
    void* d_v;
    float* d_m_scale;      /* state_bits 8: ceil(count / 128) scales each; else null */
    float* d_v_scale;
    uint64_t count;        /* elements; 0 to ZVC_ADAMW_MAX_ELEMENTS */
    int32_t type;          /* of the weights: zvc_type */
    int32_t grad_type;     /* of the gradients: as the weights', or ZVC_FP32 */
    int32_t state_bits;    /* 32 or 8 */
    int32_t decays;        /* 0: no decay for this tensor */
} zvc_adamw_tensor;

#define ZVC_ADAMW_BLOCK 128
#define ZVC_ADAMW_MAX_ELEMENTS ((uint64_t)1 << 34)
#define ZVC_ADAMW_MAX_TENSORS ((size_t)1 << 20)

/* Bytes of a plan for that many tensors; 0 for more than ZVC_ADAMW_MAX_TENSORS. */
size_t zvc_adamw_plan_bytes(size_t tensors);

/* Writes a plan to HOST memory (8-byte aligned).  The caller copies these bytes to device memory, 16-byte aligned, and keeps both
 * for as long as the tensors lie where they do.  What a step writes (weights, masters, states, scales) may overlap nothing else in the plan:
 * ZVC_E_ARG; gradients may overlap each other.  All tensors together: at most 2^24 - 1 pieces of 2048 elements. */
zvc_status zvc_adamw_plan(const zvc_adamw_tensor* tensors, size_t count, void* plan, size_t bytes);

/* What changes from step to step; host memory, read during the call. */
typedef struct zvc_adamw_now {
    double rate, beta1, beta2, eps, decay, factor;   /* finite; betas in [0, 1); eps >= 0 */
    uint64_t step;                                   /* t, from 1 on */
    uint64_t seed;
    const uint64_t* d_step;     /* null, or a word that is added to `step` when the work runs (a sum of 0 counts as 1) */
    const float* d_factors;     /* null, or two floats that `rate` and `factor` are multiplied by when the work runs */
} zvc_adamw_now;

/* One step.  plan: the host's copy; d_plan: the device's.  With d_step and d_factors a captured graph goes on to the next
 * step, another rate or another scaling of the gradients at each replay. */
zvc_status zvc_adamw(const void* plan, const void* d_plan, const zvc_adamw_now* now, hipStream_t stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* ZVC_ADAMW_H_ */
