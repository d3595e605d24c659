/*
 * zvc_ffn.h -- C ABI of the training operators beside the codec (libzvc_ffn.so), AMD gfx950.
 *
 * The codec of zvc.h takes activations that a training step keeps between its
 * forward and its backward pass.  In a transformer most of them belong to the
 * feed-forward block, and they are sparse where its gate is a ReLU and where
 * dropout acts.  These are that block's gated half and dropout, forward and
 * backward:
 *
 *     g = x Wg^T     u = x Wu^T     h = drop(act(g) * u)          zvc_glu_forward
 *     dh' = drop(dh)   du = dh' act(g)   dg = dh' u act'(g)
 *     dx = dg Wg + du Wu   dWg = dg^T x   dWu = du^T x            zvc_glu_backward
 *     y = drop(x)  or  residual + drop(x)                         zvc_dropout
 *
 * x is m x k, Wg and Wu are n x k, g, u and h are m x n, all row by row with a
 * row stride (ld*, in elements, at least the row's length).  One element type per
 * call; products are summed in 32 bits.
 *
 * drop() with probability p = drop / 2^32 writes 0 for a dropped element (also
 * where the element is an infinity or a NaN) and multiplies the others by
 * 1/(1-p).  Element i (row by row, without the strides' gaps) is dropped if
 * its 32-bit number is below `drop`.  The numbers come from a counter-based
 * generator, Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers:
 * as easy as 1, 2, 3", 2011): key = seed, counter = (i / 8, offset), each the low
 * 32-bit word first.  Of the four output words, taken as eight 16-bit halves with
 * the low one first, half i % 8 is the number's upper 16 bits; the lower 16 are
 * the same half of the counter with the top bit of i / 8 set.  So no mask is ever
 * stored: the gradient makes it again from seed and offset, and dropping inside
 * zvc_glu_forward is the same as zvc_dropout behind it.  Where `d_offset` is not
 * null, the 64-bit word there is added to `offset` when the work runs: a captured
 * graph that advances the word drops other elements at each replay.
 *
 * Conventions are those of zvc.h (device pointers, caller-owned buffers, work
 * enqueued on `stream` without waiting, arguments checked on the host before any
 * GPU call), and:
 *   - pointers are aligned to the element; calls are fastest where pointers and
 *     row strides are multiples of 16 bytes;
 *   - inputs may overlap each other; outputs overlap nothing else, but rows that
 *     interleave (two halves of one wider buffer, at the same row stride) do not
 *     overlap;
 *   - any of m, n, k may be 0: outputs that are sums over it are 0;
 *   - results do not depend on timing: no sums by atomics.  They do depend on m, n and k, which
 *     choose the kernels and so the order of sums.
 */
#ifndef ZVC_FFN_H_
#define ZVC_FFN_H_

#include "zvc.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum zvc_type { ZVC_FP32 = 0, ZVC_FP16 = 1, ZVC_BF16 = 2 } zvc_type;

/* act(g).  relu: max(g, 0), with derivative 0 at 0; silu: g / (1 + exp(-g)); gelu:
 * g times the normal distribution function of g; gelu_tanh: its approximation
 * g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2.  A NaN stays one.
 * Computed in 32 bits: relative to the value within (16 + 9 z) 2^-24, z the argument of its exp (silu |g|,
 * gelu g^2 / 2), and gelu of 16-bit types within 2^-15 more. */
typedef enum zvc_activation { ZVC_RELU = 0, ZVC_SILU = 1, ZVC_GELU = 2, ZVC_GELU_TANH = 3 } zvc_activation;

/* The largest n, k and row stride. */
#define ZVC_FFN_MAX_COLUMNS ((size_t)1 << 21)
/* The largest m, m n and m k. */
#define ZVC_FFN_MAX_ROWS ((size_t)1 << 28)
#define ZVC_FFN_MAX_ELEMENTS ((size_t)1 << 40)

/* p as the calls take it: the nearest multiple of 2^-32, in 2^-32.  p outside [0, 1] or NaN: more than 2^32, which the calls refuse. */
uint64_t zvc_dropout_fraction(double p);

/* y = drop(x), or residual + drop(x) where d_residual is not null: rows x cols
 * elements, added and scaled in 32 bits and rounded once.  d_y may be d_x or d_residual itself, at
 * the same row stride.  rows times the largest row stride: at most ZVC_FFN_MAX_ELEMENTS. */
zvc_status zvc_dropout(const void* d_x, size_t ldx, const void* d_residual, size_t ldr, void* d_y, size_t ldy,
                       size_t rows, size_t cols, int type, uint64_t drop, uint64_t seed, uint64_t offset,
                       const uint64_t* d_offset, hipStream_t stream);

/* Bytes of device workspace that zvc_glu_forward (backward = 0) or
 * zvc_glu_backward (backward = 1) needs.  `loose`: not 0 if the address or the
 * row stride of x, Wg or Wu is no multiple of 16 bytes.  The workspace must be
 * 256-byte aligned and needs no initialisation.  0 for a bad type or size.
 * For these sizes alone: fewer rows may need more, since few tiles are cut along their sums. */
size_t zvc_glu_workspace_bytes(size_t m, size_t n, size_t k, int type, int backward, int loose);

/* h = drop(act(x Wg^T) * (x Wu^T)).  Where d_gate and d_up are not null (both or
 * neither, m x n with row stride ldp) they receive what zvc_glu_backward needs of the
 * projections: g and u, but zero where h was dropped, and for relu max(g, 0) and
 * u where g > 0, zero elsewhere -- what zvc_compress makes small. */
zvc_status zvc_glu_forward(const void* d_x, size_t ldx, const void* d_wg, const void* d_wu, size_t ldw, void* d_h,
                           size_t ldh, void* d_gate, void* d_up, size_t ldp, size_t m, size_t n, size_t k, int type,
                           int activation, uint64_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset,
                           void* d_ws, size_t ws, hipStream_t stream);

/* The gradients of x, Wg and Wu from dh, that of h.  drop, seed and offset as in
 * the forward call.  d_gate and d_up as that call left them (or after a round trip through
 * the codec), or both null: then the projections are computed again, which
 * costs half as much again and keeps nothing.  dg and du are rounded to the element type between
 * the products (fp16: what is beyond 65504 there becomes an infinity, also where the gradients
 * themselves would not).  d_dx may be null, and so may both of d_dwg and d_dwu: what is null is not computed. */
zvc_status zvc_glu_backward(const void* d_dh, size_t lddh, const void* d_x, size_t ldx, const void* d_wg,
                            const void* d_wu, size_t ldw, const void* d_gate, const void* d_up, size_t ldp, void* d_dx,
                            size_t lddx, void* d_dwg, void* d_dwu, size_t lddw, size_t m, size_t n, size_t k, int type,
                            int activation, uint64_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset,
                            void* d_ws, size_t ws, hipStream_t stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* ZVC_FFN_H_ */
