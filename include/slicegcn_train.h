/*
 * slicegcn_train.h -- operators for models that learn their inputs and are built from blocks, beside slicegcn.h (same
 * conventions): token embeddings with their gradient, norms before and after a block fused with its gate and residual, the norm
 * over all gradients with clipping, and the optimiser step that takes the clipping along.
 *
 * Rows of tokens and of blocks are fp32, bf16 or fp16; parameters of norms, their gradients and all sums are fp32 or fp64, and a
 * result is rounded once, when it is stored.  An empty batch (n = 0) is a valid one.
 * "Rows in place": an output may lie in the rows of an input of the same call (same address and leading dimension); outputs
 * overlap no other operand and not each other.
 */
#ifndef SLICEGCN_TRAIN_H
#define SLICEGCN_TRAIN_H

#include "slicegcn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define SLICEGCN_F32 0
#define SLICEGCN_BF16 1
#define SLICEGCN_F16 2

/* ---------------------------------------------------------------------------------------
 * Token embeddings: nodes that carry a token (a category, an item) instead of raw features look up the rows that feed the
 * slice models.
 *   n            number of tokens, at most 2^31 - 1
 *   vocab        rows of the table, at most 2^31 - 2
 *   width        columns of the table and of the looked-up rows, at most 2^31 - 1024 (in a lookup 2^26 - 1024)
 *   table_type   type of the table, or of its gradient;  row_type: type of the looked-up rows, or of their gradient
 *                (equal, or one of them SLICEGCN_F32)
 *   scale        factor of every looked-up row
 *   pad          with SLICEGCN_EMBED_PAD: rows of this token (any value, -1 for instance) are zero and give no gradient
 * ids: int32, or int64 with SLICEGCN_EMBED_IDS64.  Calls are asynchronous, so a token outside [0, vocab) that is not the padding
 * cannot come back as a status: its row is NaN, and it gives no gradient. */
#define SLICEGCN_EMBED_IDS64 1u
#define SLICEGCN_EMBED_PAD 2u
#define SLICEGCN_EMBED_ACCUMULATE 4u /* backward: dTable += instead of = (a table that another layer uses too) */
typedef struct {
    int64_t n;
    int64_t vocab;
    int64_t pad;
    double scale;
    int32_t width;
    int32_t table_type;
    int32_t row_type;
    uint32_t flags;
} slicegcn_embed_desc;

/* out[i, 0:width] = scale * table[ids[i], 0:width].  out: n x width (ldo), table: vocab x width (ldt).
 * EINVAL: NULL pointer, sizes < 1 (n < 0), ld < width, unknown type or pair of types, unknown flag, scale not finite, misaligned
 * base; ERANGE: n, vocab or width too large. */
int slicegcn_embed_fwd(const slicegcn_embed_desc *desc, const void *ids, const void *table, int64_t ldt, void *out, int64_t ldo,
                       void *stream);

/* The tokens sorted, for the gradient: order[starts[t] .. starts[t + 1]) are the positions i with ids[i] = t, ascending; padding
 * and tokens outside the table are left out, so the order holds starts[vocab] positions (what lies behind them is undefined).
 * order: int32 [n]; starts: int32 [vocab + 1].  Uses n, vocab, pad and flags of desc.  Where tokens stay the same (nodes of a graph,
 * full batch) one call serves every epoch.  EINVAL, ERANGE as above; EWORKSPACE. */
size_t slicegcn_embed_sort_workspace_bytes(int64_t n, int64_t vocab); /* 0 on bad input */
int slicegcn_embed_sort(const slicegcn_embed_desc *desc, const void *ids, int32_t *order, int32_t *starts, void *ws, size_t ws_bytes,
                        void *stream);

/* dTable[t, :] = scale * sum of dOut[i, :] over the positions i of token t, in fp32 over at most 64 positions at a time and in fp64
 * over those sums, in a fixed order; every row of dTable is written (zeros without positions), or with ACCUMULATE added to (rows
 * without positions are not touched).  order, starts: from slicegcn_embed_sort with the same n and vocab.  An entry outside [0, n)
 * is skipped.  EINVAL, ERANGE as above; EWORKSPACE. */
size_t slicegcn_embed_bwd_workspace_bytes(int64_t n, int32_t width); /* 0 on bad input, and where none is needed */
int slicegcn_embed_bwd(const slicegcn_embed_desc *desc, const int32_t *order, const int32_t *starts, const void *dOut, int64_t ldo,
                       void *dTable, int64_t ldt, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------
 * Norms before and after a block, with the block's gate and the residual, in one pass over the rows.  With y the output of a
 * block, x what went round it, and u the input of the next block:
 *   p = post(y) * post_w + post_b;   h = residual * x + s * p;   u = pre(h) * pre_w + pre_b
 *   post, pre: SLICEGCN_NORM_NONE v;  SLICEGCN_NORM_RMS v / sqrt(mean v^2 + eps);  SLICEGCN_NORM_LAYER (v - mean) / sqrt(var + eps)
 *   s: 1 without gate, params->gate[column] or io->gate[row, column], each through a sigmoid with SLICEGCN_GATE_SIGMOID
 * u is formed from h before h is rounded.  Absent (NULL): x (no residual), y (h = residual * x: a first block's norm; no post and no
 * gate then), h or u in the forward pass (not stored).  A weight or bias that is NULL is one or zero; weights and biases stand
 * only where their norm is not NONE. */
#define SLICEGCN_NORM_NONE 0
#define SLICEGCN_NORM_RMS 1
#define SLICEGCN_NORM_LAYER 2
#define SLICEGCN_GATE_SIGMOID 1u
#define SLICEGCN_RESNORM_MAX_WIDTH 16384
typedef struct {
    int64_t n;
    int32_t width;
    int32_t type; /* of x, y, the gate's rows, h, u and their gradients */
    int32_t post;
    int32_t pre;
    uint32_t flags;
    double residual;
    double eps;
} slicegcn_resnorm_desc;

/* fp32 [width] each, or NULL */
typedef struct {
    const float *post_w;
    const float *post_b;
    const float *pre_w;
    const float *pre_b;
    const float *gate;
} slicegcn_resnorm_params;

typedef struct {
    void *data; /* n x width, row-major, or NULL */
    int64_t ld;
} slicegcn_rows;

/* stats: n x 4 floats (16-byte aligned), written by the forward pass (NULL: not wanted) for the backward pass: mean and
 * 1/sqrt of y's row, mean and 1/sqrt of h's row. */
typedef struct {
    slicegcn_rows x, y, gate;
    slicegcn_rows h, u;
    float *stats;
    slicegcn_rows dh, du;        /* gradients of h and u; either may be absent, not both */
    slicegcn_rows dx, dy, dgate; /* absent: not wanted */
} slicegcn_resnorm_io;

/* Gradients of the parameters, same shapes; NULL: not wanted */
typedef struct {
    float *post_w;
    float *post_b;
    float *pre_w;
    float *pre_b;
    float *gate;
} slicegcn_resnorm_grads;

/* EINVAL: NULL desc, params or io, n < 0, width < 1, ld < width, unknown type, norm or flag, residual not finite, eps not positive,
 * no x and no y, no h and no u, stats without the u they belong to; y absent with post or a gate; a parameter without its norm;
 * two gates; SIGMOID without gate; misaligned base.  EUNSUPPORTED: width > SLICEGCN_RESNORM_MAX_WIDTH. */
int slicegcn_resnorm_fwd(const slicegcn_resnorm_desc *desc, const slicegcn_resnorm_params *params, const slicegcn_resnorm_io *io,
                         void *stream);

/* Backward: from dh, du and what the forward pass read (x, y, gate, parameters, stats).  Column sums (gradients of the parameters)
 * run in fp32 over the rows a workgroup takes and in fp64 over workgroups.  EINVAL as for the forward, and for a gradient of
 * something absent, stats absent; EWORKSPACE when a parameter's gradient is wanted and ws is NULL or too small. */
size_t slicegcn_resnorm_bwd_workspace_bytes(int64_t n, int32_t width); /* 0 on bad input */
int slicegcn_resnorm_bwd(const slicegcn_resnorm_desc *desc, const slicegcn_resnorm_params *params, const slicegcn_resnorm_io *io,
                         const slicegcn_resnorm_grads *grads, void *ws, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------------
 * The norm over all elements of many tensors (a model's gradients), and clipping to it.
 *   norm   = sqrt(sum g^2) (SLICEGCN_NORM_TWO) or max |g| (SLICEGCN_NORM_MAX), squares and sums in fp64, rounded to fp32 once
 *   factor = 1 where norm <= max_norm, else max_norm / norm  (NaN where the norm is NaN; 0 where it is infinite)
 * tensors: HOST array of contiguous DEVICE tensors; count = 0 and empty tensors (data may be NULL) are valid.
 * norm, factor: DEVICE scalars. */
#define SLICEGCN_NORM_TWO 0
#define SLICEGCN_NORM_MAX 1
typedef struct {
    void *data;
    int64_t count;
    int32_t type;
    int32_t reserved; /* set it to 0; not read */
} slicegcn_tensor;

size_t slicegcn_global_norm_workspace_bytes(const slicegcn_tensor *tensors, int32_t count); /* 0 on bad input */

/* norm, and factor unless that is NULL (max_norm is not looked at then).
 * EINVAL: NULL pointer, count < 0, bad tensor, unknown kind, max_norm negative or NaN; EWORKSPACE. */
int slicegcn_global_norm(const slicegcn_tensor *tensors, int32_t count, int32_t kind, double max_norm, float *norm, float *factor,
                         void *ws, size_t ws_bytes, void *stream);

/* The same (norm and factor may each be NULL), and to[i] = factor * from[i].  `to` has the counts and types of `from`; NULL, or a
 * tensor at the same address: in place (then nothing is written where factor is 1).  Tensors overlap in no other way. */
int slicegcn_clip(const slicegcn_tensor *from, const slicegcn_tensor *to, int32_t count, int32_t kind, double max_norm, float *norm,
                  float *factor, void *ws, size_t ws_bytes, void *stream);

/* slicegcn_adam_step on factor * grad, factor a DEVICE scalar (slicegcn_global_norm's): a step on clipped gradients without a pass
 * that clips them. */
int slicegcn_adam_step_scaled(float *param, const float *grad, const float *factor, float *m, float *v, int64_t count, double lr,
                              double beta1, double beta2, double eps, double weight_decay, int32_t step, void *stream);

/* further kinds of slicegcn_profile_entry */
#define SLICEGCN_PROF_EMBED 11   /* lookup, sort and gradient; width = columns (0: sort) */
#define SLICEGCN_PROF_RESNORM 12 /* norms around a block, forward and backward; width = columns */
#define SLICEGCN_PROF_CLIP 13    /* norm over all gradients, clipping; width = tensors */

#ifdef __cplusplus
}
#endif
#endif /* SLICEGCN_TRAIN_H */
