/*
 * lors_train.h -- C ABI of the operators around the sparsity-preserved LoRA
 * linear (lors.h) in a fine-tuning step, for AMD MI355X (gfx950):
 *
 *   norm        z = residual + dropout(x), y = the layer norm of z, or its norm by
 *               the root mean square, and the gradients
 *   dropout     from a counter-based generator; the mask is never stored
 *   embedding   the scaled lookup of token rows, and the gradient of the table
 *   preference  log-probabilities of target tokens out of logits, the paired
 *               preference loss over sequences, and the gradient of the logits
 *
 * Conventions are those of lors.h: the same status codes (lors_status_string
 * names them), arguments validated on the host in the order
 *   null -> dtype/format -> shape/range -> alignment -> alias -> workspace
 * before any HIP call, caller-owned buffers, no allocation, asynchronous work on
 * `stream`, outputs overwritten.  Outputs must not overlap any input, each other
 * or the workspace (LORS_ERR_ALIAS).  Arrays of no elements may be NULL.
 *
 * Every array is row-major and contiguous, except that logits may have strides
 * between their rows.  Unlike lors.h, any width is accepted, and a pointer only
 * has to be aligned to its element (LORS_ERR_ALIGN); a workspace to 16 bytes.
 * The dtype (bf16 or fp32) applies to the activations, tables, weights and
 * logits.  Arithmetic is in fp32, each result rounded once (nearest-even); sums
 * are fp32 or wider.
 * Every result is a function of the inputs alone, bit for bit: no sum depends on
 * the order in which workgroups finish.
 */
#ifndef LORS_TRAIN_H
#define LORS_TRAIN_H

#include <stddef.h>
#include <stdint.h>

#include "lors.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Version of this interface: major * 10000 + minor * 100 + patch. */
int lors_train_version(void);

/*
 * Random bits: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random
 * numbers: as easy as 1, 2, 3", 2011).  Column c of row n of a tensor takes the
 * 16-bit half c % 8 (the low half of word 0 first) of the block with
 *   counter (c / 8, n, offset low, offset high), key (seed low, seed high),
 * so that a mask is recomputed from (seed, offset) alone wherever it is needed.
 * Calls that need other bits take another seed or offset.
 * `state`: NULL, or the device address (8-byte aligned) of two uint64 that the
 * kernels read: state[0] is added to the seed and state[1] to the offset.  A
 * captured graph advances its masks by writing them between replays.
 */
typedef struct lors_rng {
    uint64_t seed;
    uint64_t offset;
    const uint64_t* state;
} lors_rng_t;

/* ------------------------------------------------------------------ dropout */

/*
 * rows, cols: 0 <= rows < 2^31, 1 <= cols < 2^31 (LORS_ERR_SHAPE).
 * p: an element is dropped where its 16 bits are below t = round(65536 p), and a
 * kept one is multiplied by 65536 / (65536 - t), which keeps the expectation at
 * the p that is applied.  0 <= p and t <= 65535, otherwise LORS_ERR_SHAPE.
 */
typedef struct lors_dropout_desc {
    int64_t rows;
    int64_t cols;
    double p;
    lors_rng_t rng;
    int32_t dtype;   /* lors_dtype_t */
    uint32_t flags;  /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_dropout_t;

/*
 * Y = dropout(X) (+ residual, may be NULL): rows x cols.  Dropping is a select: a
 * dropped Inf or NaN is 0.  The gradient of X is the same call on dY without
 * residual; the residual's is dY.
 */
lors_status_t lors_dropout(const lors_dropout_t* p, const void* X, const void* residual, void* Y, void* stream);

/* --------------------------------------------------------------------- norm */

typedef enum lors_norm_kind {
    LORS_NORM_LAYER = 0, /* y = (z - mean) / sqrt(variance + eps) . weight + bias */
    LORS_NORM_RMS = 1    /* y = z / sqrt(mean of z^2 + eps) . weight + bias */
} lors_norm_kind_t;

#define LORS_NORM_MAX_COLS 32768

/*
 * 0 <= rows < 2^31, 1 <= cols <= LORS_NORM_MAX_COLS, eps finite and >= 0, p and
 * rng as in lors_dropout_t (p = 0: no dropout); otherwise LORS_ERR_SHAPE.
 * grad_dtype: the type of dweight and dbias.
 */
typedef struct lors_norm_desc {
    int64_t rows;
    int64_t cols;
    double eps;
    double p;
    lors_rng_t rng;
    int32_t dtype;       /* lors_dtype_t */
    int32_t grad_dtype;  /* lors_dtype_t */
    int32_t kind;        /* lors_norm_kind_t: LORS_ERR_MASK_FORMAT's place in the order, LORS_ERR_UNSUPPORTED */
    uint32_t flags;      /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_norm_t;

/*
 * Z = residual + dropout(X), rounded to the dtype, and Y = norm(Z) of Z as it is
 * stored, so that the call gives what lors_dropout followed by the norm alone
 * gives.  `residual`, `weight` and `bias` (cols) may be NULL.  Z is required with
 * a residual or p > 0, and must be NULL otherwise (Z is X; LORS_ERR_UNSUPPORTED).
 * mean (LORS_NORM_LAYER only; ignored otherwise) and rstd: rows fp32, what the
 * backward needs of the statistics; NULL where there is none.
 */
lors_status_t lors_norm_forward(const lors_norm_t* p, const void* X, const void* residual, const void* weight,
                                const void* bias, void* Y, void* Z, float* mean, float* rstd, void* stream);

/* Device scratch bytes of lors_norm_backward: partial sums of dweight and dbias.
 * (size_t)-1 if p is invalid. */
size_t lors_norm_workspace_bytes(const lors_norm_t* p);

/*
 * Backward.  Z: what the forward normalised (its Z, or X).  dY: gradient of Y.
 * dZ: gradient of Z from its other uses (the residual stream), or NULL.
 * With h = (Z - mean) rstd and g = dY . weight, rows by rows,
 *   d  = rstd (g - mean(g) - h mean(g h)) + dZ     (LORS_NORM_RMS: no mean(g))
 *   dX = dropout(d), dresidual = d, dweight = sum of dY h, dbias = sum of dY.
 * mean is required for LORS_NORM_LAYER.  dX is required; dresidual, dweight and
 * dbias may be NULL (with p = 0 dresidual equals dX).  The workspace is needed
 * for dweight or dbias only.
 */
lors_status_t lors_norm_backward(const lors_norm_t* p, const void* dY, const void* dZ, const void* Z,
                                 const void* weight, const float* mean, const float* rstd, void* dX, void* dresidual,
                                 void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------- embedding */

typedef enum lors_index_dtype {
    LORS_INDEX_I64 = 0,
    LORS_INDEX_I32 = 1
} lors_index_dtype_t;

/*
 * tokens >= 0, vocab >= 1, cols >= 1, each < 2^31, scale finite; otherwise
 * LORS_ERR_SHAPE; the backward takes (ceil(cols / 256) + 1) . max(vocab / 8, tokens / 32) < 2^31,
 * otherwise LORS_ERR_UNSUPPORTED.  Ids outside 0 .. vocab - 1 stand for no token (padding): their
 * row of Y is zero and they have no part in the gradient.
 * grad_dtype: the type of dE.
 */
typedef struct lors_embedding_desc {
    int64_t tokens;
    int64_t vocab;
    int64_t cols;
    float scale;
    int32_t dtype;        /* lors_dtype_t: E, Y, dY */
    int32_t grad_dtype;   /* lors_dtype_t */
    int32_t index_dtype;  /* lors_index_dtype_t: ids; otherwise LORS_ERR_DTYPE */
    uint32_t flags;       /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_embedding_t;

/* Y[t] = scale . E[ids[t]] (tokens x cols out of vocab x cols). */
lors_status_t lors_embedding_forward(const lors_embedding_t* p, const void* ids, const void* E, void* Y, void* stream);

/* Device scratch bytes of lors_embedding_backward: the tokens sorted by id, and
 * partial sums of frequent ones; 0 for a few tokens.  (size_t)-1 if p is invalid. */
size_t lors_embedding_workspace_bytes(const lors_embedding_t* p);

/*
 * dE[v] = scale . sum of dY[t] over the tokens t with ids[t] = v, in a fixed order:
 * the whole table's gradient, rows without a token zero.
 */
lors_status_t lors_embedding_backward(const lors_embedding_t* p, const void* ids, const void* dY, void* dE,
                                      void* workspace, size_t workspace_bytes, void* stream);

/* --------------------------------------------------------------- preference */

/*
 * Logits of `batch` sequences of `length` tokens over `vocab` entries: entry v of
 * token t of sequence b is element b . batch_stride + t . row_stride + v.  Targets,
 * log-probabilities and the like are batch x length, contiguous.
 * batch, length >= 0, batch . length < 2^31, 1 <= vocab < 2^31, strides >= 0;
 * otherwise LORS_ERR_SHAPE.  (batch . length) . ceil(vocab / 4096) < 2^31, otherwise
 * LORS_ERR_UNSUPPORTED.
 * A target outside 0 .. vocab - 1 (a prompt's or padding's, -100) does not count:
 * its log-probability and gradient are 0, and its row of logits is not read.
 */
typedef struct lors_logits_desc {
    int64_t batch;
    int64_t length;
    int64_t vocab;
    int64_t batch_stride;
    int64_t row_stride;
    int32_t dtype;        /* lors_dtype_t */
    int32_t index_dtype;  /* lors_index_dtype_t: targets */
    uint32_t flags;       /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_logits_t;

/* Device scratch bytes of lors_logprob_forward (partial sums of few, long rows).
 * (size_t)-1 if p is invalid. */
size_t lors_logprob_workspace_bytes(const lors_logits_t* p);

/*
 * logp = logits[target] - log of the sum of exp(logits) (fp32; 0 where the target does
 * not count).  stats (two fp32 a row, 8-byte aligned, may be NULL): the row's largest logit and the sum
 * of exp(logits - it), what the backward needs; 0, 0 where the target does not count.
 * Rows whose entries are all the type's lowest value have an even distribution; a row
 * of -Inf alone has none: NaN.
 */
lors_status_t lors_logprob_forward(const lors_logits_t* p, const void* logits, const void* targets, float* logp,
                                   float* stats, void* workspace, size_t workspace_bytes, void* stream);

/*
 * dlogits[n] = u . dlogp[n / span] . (onehot(target) - softmax(logits)): batch x length x
 * vocab, contiguous, in the logits' dtype.  `span` (1 .. length, dividing batch . length,
 * otherwise LORS_ERR_SHAPE): consecutive tokens that share one gradient, 1 for
 * one each, `length` for one a sequence.  u: the fp32 at `upstream` (device), 1 if
 * NULL.
 */
lors_status_t lors_logprob_backward(const lors_logits_t* p, const float* dlogp, int64_t span, const float* upstream,
                                    const void* logits, const void* targets, const float* stats, void* dlogits,
                                    void* stream);

/*
 * The paired preference loss.  logp: 2 pairs x length, the preferred sequences
 * first, then the rejected ones in the same order; ref: the reference's
 * log-probabilities of the same tokens; targets as above (vocab: their range).
 *   reward[b] = beta . sum over counted tokens of (logp - ref)
 *   m[i]      = reward[i] - reward[pairs + i]
 *   loss      = mean over pairs of -(1 - e) log sigmoid(m) - e log sigmoid(-m)
 *   dseq[b]   = d loss / d(sum of logp of sequence b)
 * e: label smoothing, 0 <= e <= 0.5; beta finite; pairs >= 1, length >= 0, 2 pairs . length
 * < 2^31; otherwise LORS_ERR_SHAPE.  reward and dseq: 2 pairs fp32; loss: one fp32.
 * ref NULL: a reference of 0 everywhere.  Sums over tokens and pairs and the margins are in
 * 64 bits; of many pairs (above 512, or 16384 tokens) each one's loss is rounded to fp32
 * before their mean.
 */
typedef struct lors_preference_desc {
    int64_t pairs;
    int64_t length;
    int64_t vocab;
    double beta;
    double smoothing;
    int32_t index_dtype;  /* lors_index_dtype_t: targets */
    uint32_t flags;       /* 0, otherwise LORS_ERR_UNSUPPORTED */
} lors_preference_t;

lors_status_t lors_preference(const lors_preference_t* p, const float* logp, const float* ref, const void* targets,
                              float* loss, float* reward, float* dseq, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LORS_TRAIN_H */
