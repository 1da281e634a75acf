/*
 * tessel_block_ops.h -- C ABI of the operators that the blocks of a schedule run (MI355X, gfx950).
 *
 * tessel.h searches the order of a model's forward and backward blocks from their times t and activation memory m.  The
 * operators here are what such a block of a transformer stage spends t on and keeps m for:
 *   attention over whole prompts, causal, grouped heads, packed sequences        tessel_attention_*
 *   the norms around a block with its gate and residual scale                    tessel_residual_norm_*
 *   activation checkpoints in 8 bits and their use in the backward pass          tessel_checkpoint_*, tessel_gated_*,
 *                                                                                tessel_weight_gradient
 * Conventions are those of tessel.h: every function returns TESSEL_OK or a negative TESSEL_E_* code and nothing aborts or
 * throws; the caller owns all device memory and the stream; calls are asynchronous on `hip_stream` (NULL = default stream)
 * unless stated otherwise and may be captured into a HIP graph; the library allocates no device memory.  Pointers inside
 * the structures are DEVICE pointers unless stated otherwise.  All strides count elements.  Results do not depend on
 * the order in which the GPU runs things: two calls on the same inputs give the same bits.
 * No output may overlap an input or another output, except where stated.
 */
#ifndef TESSEL_BLOCK_OPS_H
#define TESSEL_BLOCK_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "tessel.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
enum { TESSEL_BF16 = 0, TESSEL_F16 = 1, TESSEL_F32 = 2 };

/* [tokens][heads][dim], the last dimension contiguous */
typedef struct {
    void    *data;
    int64_t  token_stride;
    int64_t  head_stride;
} tessel_heads;

/* [tokens][channels], the last dimension contiguous */
typedef struct {
    void    *data;
    int64_t  stride;
} tessel_rows;

/* hipError_t of the calling thread's last call of this header that returned TESSEL_E_HIP; 0 if there was none. */
int  tessel_block_last_hip_error(void);

/* ---- attention over packed sequences ----------------------------------------------------------------------------
 * The tokens of sequence i are lengths[0] + .. + lengths[i-1] and the lengths[i] (0 or more) that follow; tokens behind the
 * last sequence belong to none.  For head h, which reads key-value head h / (heads / kv_heads), and token i of a sequence
 *     lse_i = log sum_{j <= i} exp(scale q_i . k_j),    o_i = sum_{j <= i} exp(scale q_i . k_j - lse_i) v_j.
 * A token of no sequence gets o = 0 and lse = -infinity, is read by nobody, and has gradients of 0.  Infinities and NaN reach the
 * tokens that see them by the formula and no others; in the backward pass, any token of the same sequence.
 * Products are taken in the inputs' type and summed in 32 bits; the probabilities (and, going back, the gradients of the
 * scores) are rounded to the inputs' type before the second product. */
typedef struct tessel_packing tessel_packing;   /* opaque, host memory only: the tiles of a set of lengths */

/* lengths: host array, read during the call.  Errors: INVALID_ARG (a negative length, num_sequences < 0, more tokens in the
 * sequences than total_tokens), TOOBIG (total_tokens above 2^31 - 1). */
int  tessel_packing_create(const int32_t *lengths, int32_t num_sequences, int64_t total_tokens, tessel_packing **out);
void tessel_packing_destroy(tessel_packing *p);
/* Bytes of the device table of `p` (at least 16). */
int  tessel_packing_table_bytes(const tessel_packing *p, size_t *bytes);
/* Copies the table to `table_dev` (16-byte aligned; the caller keeps it as long as `p` is used) and waits until it is there,
 * so that `p` can be used on any stream afterwards.  Not for a stream that is being captured.
 * Errors: INVALID_ARG, WORKSPACE (missing, misaligned, too small), HIP. */
int  tessel_packing_bind(tessel_packing *p, void *table_dev, size_t table_bytes, void *hip_stream);

typedef struct {
    int32_t  type;          /* TESSEL_BF16 or TESSEL_F16                                                   */
    int32_t  heads;         /* a multiple of kv_heads                                                      */
    int32_t  kv_heads;
    int32_t  dim;           /* a multiple of 8, at most 128                                                */
    float    scale;         /* 2^-100 .. 2^100                                                             */
    tessel_heads q, k, v;   /* data and strides: multiples of 16 bytes, strides not negative               */
    tessel_heads o;         /* forward: written; backward: read                                            */
    float   *lse;           /* [heads][total_tokens]; forward: written; backward: read                     */
    tessel_heads d_o;       /* backward: gradient of o                                                     */
    tessel_heads dq, dk, dv;/* backward: written                                                           */
} tessel_attention;

/* Workspaces: 16-byte aligned, contents need not be kept between calls (the forward pass needs none, and 0 bytes are asked for, unless a few
 * heads go over long sequences: their work is then split over the keys).
 * Errors: INVALID_ARG, UNSUPPORTED (type, dim), TOOBIG (more workgroups than one launch holds), WORKSPACE (also: `p` is not bound), HIP. */
int  tessel_attention_forward_workspace_bytes(const tessel_packing *p, const tessel_attention *a, size_t *bytes);
int  tessel_attention_forward(const tessel_packing *p, const tessel_attention *a, void *workspace_dev, size_t workspace_bytes,
                              void *hip_stream);
int  tessel_attention_backward_workspace_bytes(const tessel_packing *p, const tessel_attention *a, size_t *bytes);
int  tessel_attention_backward(const tessel_packing *p, const tessel_attention *a, void *workspace_dev, size_t workspace_bytes,
                               void *hip_stream);

/* ---- the norms around a block, with its gate and residual scale --------------------------------------------------
 * x is the residual stream, y what the block put out, n(z, w) = w z / sqrt(mean(z^2) + eps) over the channels of a token:
 *     u = n(y, post)  (u = y without post),    r = scale x + gate u  (gate = 1 without one),    h = n(r, pre):
 * r is the residual stream behind the block and h what the next block reads.  Everything is computed in 32 bits from the
 * inputs and rounded once, h from the r that is not yet rounded; the backward pass computes r again from x and y. */
enum { TESSEL_GATE_NONE = 0, TESSEL_GATE_CHANNEL = 1, TESSEL_GATE_TOKEN = 2 };
typedef struct {
    int32_t  type;          /* of x, y, r, h and their gradients, and of a gate for each token             */
    int32_t  gate_kind;     /* TESSEL_GATE_*: none; 32-bit [channels]; [tokens][channels]                  */
    int64_t  tokens;
    int32_t  channels;      /* at most 16384                                                               */
    float    scale;
    float    eps;           /* not negative                                                                */
    tessel_rows x, y;
    tessel_rows gate;       /* (stride: for each token's gate)                                             */
    const float *pre;       /* [channels]                                                                  */
    const float *post;      /* [channels] or NULL                                                          */
    float   *stats;         /* [2][tokens]: 1 / root mean square of y (with post) and of r; forward: written, backward: read */
    tessel_rows r, h;       /* forward: written                                                            */
    tessel_rows dr, dh;     /* backward: gradients of r (all but what comes through h) and h               */
    tessel_rows dx, dy;     /* backward: written                                                           */
    tessel_rows dgate;      /* backward, each token's gate: written                                        */
    float   *dpre, *dpost, *dgate_channel;   /* backward: [channels], written, or added to with `accumulate` */
    int32_t  accumulate;    /* backward: not 0: the gradients of the parameters are added to what is there
                               (the micro-batches of a schedule)                                           */
} tessel_residual_norm;

/* Errors: INVALID_ARG, UNSUPPORTED (type), TOOBIG (channels, tokens), WORKSPACE, HIP. */
int  tessel_residual_norm_forward(const tessel_residual_norm *a, void *hip_stream);
int  tessel_residual_norm_backward_workspace_bytes(const tessel_residual_norm *a, size_t *bytes);
int  tessel_residual_norm_backward(const tessel_residual_norm *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- activation checkpoints in 8 bits ---------------------------------------------------------------------------
 * Every group of 64 channels of a token (the last one may be shorter) is held as whole numbers times a power of two:
 *     e = the least exponent, not below that of the type, with max |x| < 127.5 2^e;    value = rint(x / 2^e),
 * ties to even, cut where value 2^e would leave the type's range.  The least exponent is -126 (bf16, f32) or -24 (f16).  A
 * power of two costs up to one of the eight bits against a scale of max|x| / 127; in return value 2^e is exact in all three types,
 * so a matrix product takes it as it is.  A group with an infinity or NaN reads back as NaN. */
#define TESSEL_CHECKPOINT_GROUP 64
typedef struct {
    int8_t  *values;           /* [tokens][channels up to the next multiple of 64], all of it written and read */
    uint8_t *exponents;        /* [tokens][ceil(channels / 64)]: e + 127; 0 marks a group that is not finite */
    int64_t  value_stride;     /* a multiple of 64, at least channels; data 16-byte aligned                */
    int64_t  exponent_stride;  /* at least ceil(channels / 64)                                             */
    int64_t  tokens;
    int32_t  channels;
    int32_t  type;             /* of what was stored                                                       */
} tessel_checkpoint;

/* Errors: INVALID_ARG, UNSUPPORTED (type), TOOBIG, HIP.  x: rows of the checkpoint's type. */
int  tessel_checkpoint_store(const tessel_checkpoint *c, const tessel_rows *x, void *hip_stream);
int  tessel_checkpoint_restore(const tessel_checkpoint *c, const tessel_rows *x, void *hip_stream);

/* The gated activation a = act(g) u of a block, computed from g and u as they are, which are kept in 8 bits:
 * SILU act(z) = z / (1 + exp(-z)), GELU act(z) = z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2.
 * Backward: dg = da u act'(g), du = da act(g) from the checkpoints' g and u; a (data may be NULL): act(g) u of those. */
enum { TESSEL_SILU = 0, TESSEL_GELU = 1 };
int  tessel_gated_forward(int act, const tessel_rows *g, const tessel_rows *u, const tessel_rows *a,
                          const tessel_checkpoint *kept_g, const tessel_checkpoint *kept_u, void *hip_stream);
int  tessel_gated_backward(int act, const tessel_rows *da, const tessel_checkpoint *kept_g, const tessel_checkpoint *kept_u,
                           const tessel_rows *dg, const tessel_rows *du, const tessel_rows *a, void *hip_stream);

/* Gradient of the weights of a product y = x w^T from the input that was kept in 8 bits:
 *     dw[n][c] = sum over tokens of dy[token][n] x[token][c]   (+ what is there, with `accumulate`),
 * dw in 32 bits, products of the checkpoint's type (bf16 or f16) summed in 32 bits. */
typedef struct {
    tessel_checkpoint x;
    tessel_rows dy;            /* [tokens][outputs], the checkpoint's type; strides here at most 2^24     */
    int32_t  outputs;
    int32_t  accumulate;
    float   *dw;               /* [outputs][channels]                                                      */
    int64_t  dw_stride;        /* at least channels                                                        */
} tessel_weight_grad;
int  tessel_weight_gradient_workspace_bytes(const tessel_weight_grad *a, size_t *bytes);
/* Errors: INVALID_ARG, UNSUPPORTED (type), TOOBIG, WORKSPACE, HIP. */
int  tessel_weight_gradient(const tessel_weight_grad *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TESSEL_BLOCK_OPS_H */
