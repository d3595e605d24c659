/*
 * zvc_experts.h -- C ABI of the operators for mixtures of experts (libzvc_experts.so), AMD gfx950:
 * the router, and the experts' matrix products with their gradients.
 *
 * A token's feed-forward block is one of many: a router gives each of m tokens its `top` experts of E,
 * the rows of each expert are gathered one expert behind the other, and every product is one with a weight of its own for each of them:
 *
 *     chosen, weights, offsets, order, place  from logits                        zvc_route
 *     dlogits  from dweights                                                     zvc_route_backward
 *     y[r] = x[r] W_e^T           for offsets[e] <= r < offsets[e+1]             zvc_expert_product
 *     dx[r] = dy[r] W_e   dW_e = dy_e^T x_e                                      zvc_expert_gradients
 *
 * How many rows an expert has is known on the device alone; no call waits for it.
 *
 * Conventions are those of zvc.h and zvc_ffn.h: element types, row strides in elements (ld*), outputs that overlap
 * nothing else, products summed in 32 bits, no sums by atomics, results that do not depend on timing.
 */
#ifndef ZVC_EXPERTS_H_
#define ZVC_EXPERTS_H_

#include "zvc_ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The most experts, choices of a token, and choices of all tokens (m * top). */
#define ZVC_EXPERTS_MAX 1024
#define ZVC_EXPERTS_MAX_TOP 16
#define ZVC_EXPERTS_MAX_ENTRIES ((size_t)1 << 27)

/* Bytes of device workspace that zvc_route needs for m tokens or fewer (256-byte aligned, no initialisation).  0 for a bad size. */
size_t zvc_route_workspace_bytes(size_t m, size_t experts, size_t top);

/* The router.  d_logits: m x experts, row stride ldl.  An expert whose logit is minus infinity or a NaN is out of that token's choice.
 *   d_chosen   m x top int32: a token's experts by falling logit, equal ones by rising number; -1 where none is left
 *   d_weights  m x top floats: exp(l) over the sum of exp(l) -- of the chosen (normalize != 0) or of all experts that are
 *              not out -- and 0 beside a -1.  (A logit of plus infinity: NaNs, as the formula gives.)
 *   d_offsets  experts + 1 int64: offsets[e] to offsets[e+1] are expert e's rows; the last is the number of rows in all
 *   d_order    m * top int64: row r holds entry order[r] = token * top + choice; an expert's rows lie in rising order of their entries;
 *              -1 behind the last row
 *   d_place    m x top int64: the row of each entry, -1 where there is none
 * The outputs have contiguous rows.  top is at most experts. */
zvc_status zvc_route(const void* d_logits, size_t ldl, int32_t* d_chosen, float* d_weights, int64_t* d_offsets, int64_t* d_order,
                     int64_t* d_place, size_t m, size_t experts, size_t top, int type, int normalize, void* d_ws, size_t ws,
                     hipStream_t stream);

/* The gradient of the logits (m x experts, of their type) from that of the weights, with the choice that zvc_route made.  0 for an expert
 * that is out, or not chosen where the weights are normalized over the chosen.  A number in d_chosen that is no expert's counts as -1;
 * an expert that a token has twice gets both gradients. */
zvc_status zvc_route_backward(const float* d_dweights, const void* d_logits, size_t ldl, const int32_t* d_chosen, void* d_dlogits, size_t ldd,
                              size_t m, size_t experts, size_t top, int type, int normalize, hipStream_t stream);

/* Bytes of device workspace that zvc_expert_product (backward = 0) or zvc_expert_gradients (backward = 1) needs
 * for m rows or fewer of the same experts, n, k and type (256-byte aligned, no initialisation).  0 for a bad type or size. */
size_t zvc_expert_workspace_bytes(size_t m, size_t experts, size_t n, size_t k, int type, int backward);

/* y[r] = x[r] W_e^T.  x: m x k; y: m x n; W: experts times n x k with row stride ldw, an expert's weight sw elements behind
 * the one before it.  d_offsets: experts + 1 int64.  Rows of y before offsets[0] and from offsets[experts] on stay as they were, and so do those
 * of x unread.  An offset below the one before it counts as that one, one below 0 as 0, and one above m as m. */
zvc_status zvc_expert_product(const void* d_x, size_t ldx, const void* d_w, size_t ldw, size_t sw, const int64_t* d_offsets, void* d_y,
                              size_t ldy, size_t m, size_t experts, size_t n, size_t k, int type, void* d_ws, size_t ws, hipStream_t stream);

/* The gradients of x and W from dy, that of y.  dW: experts times n x k with strides lddw and sdw; 0 for an expert without rows.
 * Rows of dx that are no expert's stay as they were.  d_dx or d_dw may be null: that one is not computed, and the other one's last bits
 * need not be those that a call for both gives (which kernel is taken goes by what is wanted). */
zvc_status zvc_expert_gradients(const void* d_dy, size_t lddy, const void* d_x, size_t ldx, const void* d_w, size_t ldw, size_t sw,
                                const int64_t* d_offsets, void* d_dx, size_t lddx, void* d_dw, size_t lddw, size_t sdw, size_t m,
                                size_t experts, size_t n, size_t k, int type, void* d_ws, size_t ws, hipStream_t stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* ZVC_EXPERTS_H_ */
