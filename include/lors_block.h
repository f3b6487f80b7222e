/*
 * lors_block.h -- C ABI of three operators that a fine-tuning loop of gated
 * models needs beside the layer (lors.h) and the operators around it
 * (lors_train.h), for AMD MI355X (gfx950):
 *
 *   gated    H = act(G) . U, the gated half of a feed-forward block, out of two
 *            sparsity-preserved LoRA projections, and its gradients
 *   update   orthogonalised (Newton-Schulz) update directions of matrices with a
 *            short side, such as adapters, and the optimiser's step with them
 *   sample   tokens drawn from logits: temperature, top-k, top-p, min-p
 *
 * Conventions are those of lors.h: the same status codes, arguments validated on
 * the host in the order
 *   null -> dtype/format -> shape/range -> alignment -> alias -> workspace
 * before any HIP call, caller-owned buffers, no allocation of device memory, asynchronous work on
 * `stream`.  Outputs must not overlap any input, each other or the workspace
 * (LORS_ERR_ALIAS).  Arrays of no elements may be NULL.
 */
#ifndef LORS_BLOCK_H
#define LORS_BLOCK_H

#include <stddef.h>
#include <stdint.h>

#include "lors.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Version of this interface: major * 10000 + minor * 100 + patch. */
int lors_block_version(void);

/* -------------------------------------------------------------------- gated */

typedef enum lors_activation {
    LORS_ACT_SILU = 0, /* g / (1 + exp(-g)) */
    LORS_ACT_GELU = 1  /* g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2 */
} lors_activation_t;

/* One of the block's two projections, as lors_forward takes them. */
typedef struct lors_projection {
    const void* W;            /* R x C */
    const uint32_t* M_packed; /* the problem's mask format */
    const void* B;            /* R x r */
    const void* A;            /* r x C */
} lors_projection_t;

/*
 * The problem p describes both projections: they share R, C, r, scale, dtype and
 * mask format.  Limits and errors are those of lors_problem_t; the tiles of both
 * together must number below 2^31 (LORS_ERR_UNSUPPORTED).  Pointers are 16-byte
 * aligned.  An unknown activation is refused in LORS_ERR_MASK_FORMAT's place of
 * the order, with LORS_ERR_UNSUPPORTED.
 *
 * Scratch bytes of lors_gated_forward (without G and U) and, with backward != 0,
 * of lors_gated_backward: the two transposed masks, padded copies of B where r is
 * no multiple of 8, dG and dU (L x R each), and at most 64 MiB of fp32 partial sums of dX's
 * tiles that are cut over their contraction.  (size_t)-1 if p is invalid for the call.
 */
size_t lors_gated_workspace_bytes(const lors_problem_t* p, int backward);

/*
 * G = X . Wg'^T, U = X . Wu'^T, H = act(G) . U (L x R), with W' = select(M, W + s.B.A, 0)
 * rounded to the dtype, as in lors_forward.  G and U: where the projections'
 * results are kept for the backward, both or neither (LORS_ERR_NULL); NULL for
 * serving.  G and U are rounded once.  H is computed from their fp32 sums in
 * bf16 (in batches of tiles above rank 48 act(G) is rounded to bf16 before the
 * product), and from the stored G and U in fp32.  p->flags: 0, otherwise
 * LORS_ERR_UNSUPPORTED.
 */
lors_status_t lors_gated_forward(const lors_problem_t* p, int32_t activation, const void* X,
                                 const lors_projection_t* gate, const lors_projection_t* up, void* G, void* U, void* H,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * Backward from dH (L x R) and the G and U that the forward kept:
 *   dG = dH . U . act'(G), dU = dH . act(G)   (rounded to the dtype, in the workspace)
 *   dX = dG . Wg' + dU . Wu'                  (skipped if dX is NULL; rounded once)
 *   dB, dA of each projection as lors_backward's, from dG and dU: fp32,
 *   overwritten, their sums' order not fixed; bf16: the weight's gradient takes part in them
 *   to 2^-16 of itself (lors_backward: to 2^-8).
 * p->flags: 0 or LORS_FLAG_REUSE_MASK_T (the workspace still holds the transposed
 * masks of an earlier call with the same R, C, r, L and masks), otherwise
 * LORS_ERR_UNSUPPORTED.
 */
lors_status_t lors_gated_backward(const lors_problem_t* p, int32_t activation, const void* dH, const void* X,
                                  const lors_projection_t* gate, const lors_projection_t* up, const void* G,
                                  const void* U, void* dX, float* dB_gate, float* dA_gate, float* dB_up, float* dA_up,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------- update */

#define LORS_UPDATE_MAX_SIDE 128  /* of a matrix's shorter side */
#define LORS_UPDATE_MAX_STEPS 32

/*
 * The direction of a matrix v, with its shorter side taken as its rows:
 *   x = v / (|v| + eps)   (|.|: the root of the sum of squares)
 *   `steps` times:  S = x x^T,  x <- a x + (b S + c S^2) x
 * S, the product of the steps and the direction's sums are in 64 bits; the direction is
 * rounded once, to fp32, before the update.
 * momentum in [0, 1], eps >= 0 and a, b, c finite, 1 <= steps <=
 * LORS_UPDATE_MAX_STEPS; otherwise LORS_ERR_SHAPE.  In directions that v does not
 * have, S holds its own rounding, 2^-53 of its norm, which a step raises by a^2: a
 * larger a^(2 steps) than 2^38 is refused (LORS_ERR_UNSUPPORTED).
 */
typedef struct lors_update_desc {
    double momentum;
    double eps;
    double a, b, c;
    int32_t steps;
    int32_t nesterov;     /* 0 or 1 */
    int32_t grad_dtype;   /* lors_dtype_t */
    int32_t param_dtype;  /* lors_dtype_t */
    uint32_t flags;       /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_update_t;

/*
 * One matrix of a call, rows x cols, row-major and contiguous.
 * 1 <= rows, cols < 2^31 and the shorter of them at most LORS_UPDATE_MAX_SIDE
 * (LORS_ERR_UNSUPPORTED above), rows * cols < 2^40, rate and decay finite; otherwise
 * LORS_ERR_SHAPE.  Pointers are aligned to their elements.
 *   m     <- momentum . m + (1 - momentum) . grad           (in place)
 *   v      = nesterov ? momentum . m + (1 - momentum) . grad : m;   grad where m is NULL
 *   master <- (1 - decay) . master - rate . direction(v)    (in place)
 *   param  = master, rounded; rate . direction(v) where master is NULL
 * param may be NULL where master is not.
 */
typedef struct lors_update_item {
    int64_t rows;
    int64_t cols;
    const void* grad;
    float* m;
    float* master;
    void* param;
    double rate;
    double decay;
} lors_update_item_t;

/* Device scratch bytes of lors_orthogonal_update.  (size_t)-1 if the arguments are
 * invalid. */
size_t lors_orthogonal_workspace_bytes(const lors_update_t* p, const lors_update_item_t* items, int64_t count);

/*
 * One step of `count` matrices (0 .. 65535, otherwise LORS_ERR_SHAPE).  `items` is a
 * host array, read during the call.  m, master and param may not overlap anything
 * else of the call (the same array in two items: LORS_ERR_ALIAS).  Every result is a
 * function of the inputs alone, bit for bit; where a matrix's gradient holds an Inf
 * or NaN, that matrix's master and param are NaN (m where the gradient is Inf or NaN), no
 * other's.
 */
lors_status_t lors_orthogonal_update(const lors_update_t* p, const lors_update_item_t* items, int64_t count,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------- sample */

/*
 * Logits of `rows` distributions over `vocab` entries; row n starts at element
 * n . row_stride.  0 <= rows < 2^31, 1 <= vocab < 2^31, row_stride >= 0, rows . vocab <
 * 2^57; temperature and min_p finite and >= 0, top_p >= 0; otherwise LORS_ERR_SHAPE.
 * Pointers are aligned to their elements.
 *   temperature  0: the largest entry; otherwise weights w = exp((z - max z) / temperature)
 *   top_k        keep the first top_k of the entries (<= 0: all) ...
 *   top_p        ... the shortest run of those that holds top_p of their weight (>= 1: all)
 *   min_p        ... and of that the entries with w >= min_p (the largest one has w = 1)
 * Entries are ordered by logit, equal ones by index; the first is always kept.
 */
typedef struct lors_sample_desc {
    int64_t rows;
    int64_t vocab;
    int64_t row_stride;
    double temperature;
    int64_t top_k;
    double top_p;
    double min_p;
    int32_t dtype;   /* lors_dtype_t */
    uint32_t flags;  /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_sample_t;

/* Device scratch bytes of lors_sample.  (size_t)-1 if p is invalid. */
size_t lors_sample_workspace_bytes(const lors_sample_t* p);

/*
 * token[n]: the first kept entry, by index, at which the running sum of the kept
 * entries' weights exceeds u[n] (fp32 in [0, 1)) times their sum; the last kept one of
 * positive weight if none does.  logp[n] (may be NULL): log of that entry's weight over
 * the sum.  Weights and sums are in 64 bits: a weight is off by at most 2^-46 + 2^-52 .
 * |log2 w| of its value, the sums that top_p's border is found by are off by vocab . 2^-60 of
 * theirs and by 2^-46 of the largest weight.  Below 2^-1022 weights have fewer bits, below 2^-1075
 * none.
 * temperature, top_k, top_p, min_p: NULL, or device arrays of `rows` that take the
 * place of the scalars; there, a temperature that is not above 0 counts as 0, and a
 * top_p or min_p that is NaN as none.
 * -Inf entries have no weight.  A row that holds a NaN, or +Inf, or nothing but -Inf,
 * has no distribution: token -1, logp NaN.
 */
lors_status_t lors_sample(const lors_sample_t* p, const void* logits, const float* u, const float* temperature,
                          const int32_t* top_k, const float* top_p, const float* min_p, int64_t* token, float* logp,
                          void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LORS_BLOCK_H */
