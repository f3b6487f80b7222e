// C ABI of the operators around the layer: argument validation and dispatch to the
// gfx950 kernels.
//
// Validation runs entirely on the host, in the order null, dtype/format,
// shape/range, alignment, alias, workspace, before any HIP call, so every rejected
// call is free of side effects.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "abi_common.hpp"
#include "lors_train.h"
#include "train_kernels.hpp"

namespace {

using namespace lors::abi;
namespace lt = lors::train;

// 65536 p rounded: elements whose 16 bits are below it are dropped; -1 if p is out
// of range.
int32_t threshold_of(double p) {
    if (!(p >= 0.0 && p <= 1.0)) return -1;
    const double t = std::floor(p * 65536.0 + 0.5);
    return t <= 65535.0 ? static_cast<int32_t>(t) : -1;
}

lt::DropArgs drop_args(double p, const lors_rng_t& rng) {
    const int32_t t = threshold_of(p);
    return lt::DropArgs{rng.seed, rng.offset, rng.state, static_cast<uint32_t>(t),
                        static_cast<float>(65536.0 / (65536.0 - t))};
}

Array state_of(const lors_rng_t& rng) { return Array{rng.state, 16, 8}; }

}  // namespace

extern "C" {

int lors_train_version(void) { return 10000; }

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------
lors_status_t lors_dropout(const lors_dropout_t* p, const void* X, const void* residual, void* Y, void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    if (p->rows != 0 && (X == nullptr || Y == nullptr)) return LORS_ERR_NULL;
    if (!valid_dtype(p->dtype)) return LORS_ERR_DTYPE;
    if (p->rows < 0 || p->rows > kMaxExtent || p->cols < 1 || p->cols > kMaxExtent) return LORS_ERR_SHAPE;
    const int64_t es = elt_size(p->dtype), n = bytes_of(p->rows, p->cols, es);
    if (n < 0 || threshold_of(p->p) < 0) return LORS_ERR_SHAPE;
    if (p->flags != 0) return LORS_ERR_UNSUPPORTED;
    const lors_status_t st = check_arrays({{X, n, es}, {residual, n, es}, state_of(p->rng)}, {{Y, n, es}});
    if (st != LORS_OK) return st;
    const lt::DropoutArgs a{p->rows, p->cols, drop_args(p->p, p->rng), X, residual, Y};
    return from_hip(lt::launch_dropout(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------
static lors_status_t check_norm(const lors_norm_t* p) {
    if (!valid_dtype(p->dtype) || !valid_dtype(p->grad_dtype)) return LORS_ERR_DTYPE;
    if (p->kind != LORS_NORM_LAYER && p->kind != LORS_NORM_RMS) return LORS_ERR_UNSUPPORTED;
    if (p->rows < 0 || p->rows > kMaxExtent || p->cols < 1 || p->cols > LORS_NORM_MAX_COLS) return LORS_ERR_SHAPE;
    if (!std::isfinite(p->eps) || p->eps < 0.0 || threshold_of(p->p) < 0) return LORS_ERR_SHAPE;
    if (p->flags != 0) return LORS_ERR_UNSUPPORTED;
    return LORS_OK;
}

lors_status_t lors_norm_forward(const lors_norm_t* p, const void* X, const void* residual, const void* weight,
                                const void* bias, void* Y, void* Z, float* mean, float* rstd, void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    const bool sum = residual != nullptr || threshold_of(p->p) > 0;
    if (p->rows != 0 && (X == nullptr || Y == nullptr || (sum && Z == nullptr))) return LORS_ERR_NULL;
    lors_status_t st = check_norm(p);
    if (st != LORS_OK) return st;
    if (!sum && Z != nullptr) return LORS_ERR_UNSUPPORTED;
    const int64_t es = elt_size(p->dtype), n = p->rows * p->cols * es, w = p->cols * es;
    if (p->kind == LORS_NORM_RMS) mean = nullptr;
    st = check_arrays({{X, n, es}, {residual, n, es}, {weight, w, es}, {bias, w, es}, state_of(p->rng)},
                      {{Y, n, es}, {Z, n, es}, {mean, 4 * p->rows, 4}, {rstd, 4 * p->rows, 4}});
    if (st != LORS_OK) return st;
    lt::NormArgs a{};
    a.rows = p->rows;
    a.cols = p->cols;
    a.eps = static_cast<float>(p->eps);
    a.rms = p->kind == LORS_NORM_RMS;
    a.drop = drop_args(p->p, p->rng);
    a.X = X;
    a.residual = residual;
    a.weight = weight;
    a.bias = bias;
    a.Y = Y;
    a.Z = Z;
    a.mean = mean;
    a.rstd = rstd;
    return from_hip(lt::launch_norm_forward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

size_t lors_norm_workspace_bytes(const lors_norm_t* p) {
    if (p == nullptr || check_norm(p) != LORS_OK) return static_cast<size_t>(-1);
    return lt::norm_workspace_bytes(p->rows, p->cols, p->dtype == LORS_DTYPE_BF16);
}

lors_status_t lors_norm_backward(const lors_norm_t* p, const void* dY, const void* dZ, const void* Z,
                                 const void* weight, const float* mean, const float* rstd, void* dX, void* dresidual,
                                 void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    if (p->rows != 0 && (dY == nullptr || Z == nullptr || rstd == nullptr || dX == nullptr ||
                         (p->kind == LORS_NORM_LAYER && mean == nullptr)))
        return LORS_ERR_NULL;
    lors_status_t st = check_norm(p);
    if (st != LORS_OK) return st;
    if (p->kind == LORS_NORM_RMS) mean = nullptr;
    const int64_t es = elt_size(p->dtype), n = p->rows * p->cols * es, w = p->cols * es;
    const int64_t gs = elt_size(p->grad_dtype), g = p->cols * gs;
    const size_t need = dweight != nullptr || dbias != nullptr ? lt::norm_workspace_bytes(p->rows, p->cols, p->dtype == LORS_DTYPE_BF16) : 0;
    st = check_arrays({{dY, n, es}, {dZ, n, es}, {Z, n, es}, {weight, w, es}, {mean, 4 * p->rows, 4},
                       {rstd, 4 * p->rows, 4}, state_of(p->rng)},
                      {{dX, n, es}, {dresidual, n, es}, {dweight, g, gs}, {dbias, g, gs},
                       {workspace, static_cast<int64_t>(need), 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, need);
    if (st != LORS_OK) return st;
    lt::NormArgs a{};
    a.rows = p->rows;
    a.cols = p->cols;
    a.rms = p->kind == LORS_NORM_RMS;
    a.drop = drop_args(p->p, p->rng);
    a.grad_bf16 = p->grad_dtype == LORS_DTYPE_BF16;
    a.Z = const_cast<void*>(Z);
    a.weight = weight;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.dY = dY;
    a.dZ = dZ;
    a.dX = dX;
    a.dresidual = dresidual;
    a.dweight = dweight;
    a.dbias = dbias;
    a.part = static_cast<float*>(workspace);
    return from_hip(lt::launch_norm_backward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// embedding
// ---------------------------------------------------------------------------
static lors_status_t check_embedding(const lors_embedding_t* p, bool backward) {
    if (!valid_dtype(p->dtype) || !valid_dtype(p->grad_dtype) || !valid_index(p->index_dtype)) return LORS_ERR_DTYPE;
    if (p->tokens < 0 || p->tokens > kMaxExtent || p->vocab < 1 || p->vocab > kMaxExtent || p->cols < 1 ||
        p->cols > kMaxExtent)
        return LORS_ERR_SHAPE;
    if (bytes_of(p->tokens, p->cols, 4) < 0 || bytes_of(p->vocab, p->cols, 4) < 0 || !std::isfinite(p->scale))
        return LORS_ERR_SHAPE;
    if (p->flags != 0) return LORS_ERR_UNSUPPORTED;
    if (backward && !lt::embedding_groups_fit(p->tokens, p->vocab, p->cols)) return LORS_ERR_UNSUPPORTED;
    return LORS_OK;
}

lors_status_t lors_embedding_forward(const lors_embedding_t* p, const void* ids, const void* E, void* Y,
                                     void* stream) {
    if (p == nullptr || E == nullptr) return LORS_ERR_NULL;
    if (p->tokens != 0 && (ids == nullptr || Y == nullptr)) return LORS_ERR_NULL;
    lors_status_t st = check_embedding(p, false);
    if (st != LORS_OK) return st;
    const int64_t es = elt_size(p->dtype), is = index_size(p->index_dtype);
    st = check_arrays({{ids, p->tokens * is, is}, {E, p->vocab * p->cols * es, es}}, {{Y, p->tokens * p->cols * es, es}});
    if (st != LORS_OK) return st;
    lt::EmbeddingArgs a{};
    a.tokens = p->tokens;
    a.vocab = p->vocab;
    a.cols = p->cols;
    a.scale = p->scale;
    a.index64 = p->index_dtype == LORS_INDEX_I64;
    a.ids = ids;
    a.E = E;
    a.Y = Y;
    return from_hip(lt::launch_embedding_forward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

size_t lors_embedding_workspace_bytes(const lors_embedding_t* p) {
    if (p == nullptr || check_embedding(p, true) != LORS_OK) return static_cast<size_t>(-1);
    return lt::embedding_workspace_bytes(p->tokens, p->vocab, p->cols);
}

lors_status_t lors_embedding_backward(const lors_embedding_t* p, const void* ids, const void* dY, void* dE,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr || dE == nullptr) return LORS_ERR_NULL;
    if (p->tokens != 0 && (ids == nullptr || dY == nullptr)) return LORS_ERR_NULL;
    lors_status_t st = check_embedding(p, true);
    if (st != LORS_OK) return st;
    const int64_t es = elt_size(p->dtype), is = index_size(p->index_dtype), gs = elt_size(p->grad_dtype);
    const size_t need = lt::embedding_workspace_bytes(p->tokens, p->vocab, p->cols);
    st = check_arrays({{ids, p->tokens * is, is}, {dY, p->tokens * p->cols * es, es}},
                      {{dE, p->vocab * p->cols * gs, gs}, {workspace, static_cast<int64_t>(need), 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, need);
    if (st != LORS_OK) return st;
    lt::EmbeddingArgs a{};
    a.tokens = p->tokens;
    a.vocab = p->vocab;
    a.cols = p->cols;
    a.scale = p->scale;
    a.grad_bf16 = p->grad_dtype == LORS_DTYPE_BF16;
    a.index64 = p->index_dtype == LORS_INDEX_I64;
    a.ids = ids;
    a.dY = dY;
    a.dE = dE;
    a.workspace = workspace;
    return from_hip(lt::launch_embedding_backward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// preference
// ---------------------------------------------------------------------------
// batch * length when it is a count of rows, else -1.
static int64_t rows_of(int64_t batch, int64_t length) {
    if (batch < 0 || length < 0 || batch > kMaxExtent || length > kMaxExtent) return -1;
    const int64_t n = batch * length;  // below 2^62
    return n <= kMaxExtent ? n : -1;
}

// Bytes from the first to past the last logit, or -1.
static int64_t logits_bytes(const lors_logits_t* p) {
    const int64_t es = elt_size(p->dtype);
    if (p->batch == 0 || p->length == 0) return 0;
    const int64_t b = bytes_of(p->batch - 1, p->batch_stride, es), r = bytes_of(p->length - 1, p->row_stride, es);
    const int64_t v = bytes_of(p->vocab, 1, es);
    return b < 0 || r < 0 || b + r + v > kMaxBytes ? -1 : b + r + v;
}

static lors_status_t check_logits(const lors_logits_t* p) {
    if (!valid_dtype(p->dtype) || !valid_index(p->index_dtype)) return LORS_ERR_DTYPE;
    const int64_t n = rows_of(p->batch, p->length);
    if (n < 0 || p->vocab < 1 || p->vocab > kMaxExtent || p->batch_stride < 0 || p->row_stride < 0)
        return LORS_ERR_SHAPE;
    if (logits_bytes(p) < 0 || bytes_of(n, p->vocab, 4) < 0) return LORS_ERR_SHAPE;
    if (p->flags != 0 || !lt::logprob_grids_fit(n, p->vocab)) return LORS_ERR_UNSUPPORTED;
    return LORS_OK;
}

static lt::LogprobArgs logprob_args(const lors_logits_t* p, const void* logits, const void* targets) {
    lt::LogprobArgs a{};
    a.batch = p->batch;
    a.length = p->length;
    a.vocab = p->vocab;
    a.batch_stride = p->batch_stride;
    a.row_stride = p->row_stride;
    a.index64 = p->index_dtype == LORS_INDEX_I64;
    a.logits = logits;
    a.targets = targets;
    return a;
}

size_t lors_logprob_workspace_bytes(const lors_logits_t* p) {
    if (p == nullptr || check_logits(p) != LORS_OK) return static_cast<size_t>(-1);
    return lt::logprob_workspace_bytes(p->batch * p->length, p->vocab, p->dtype == LORS_DTYPE_BF16);
}

lors_status_t lors_logprob_forward(const lors_logits_t* p, const void* logits, const void* targets, float* logp,
                                   float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    const bool some = p->batch != 0 && p->length != 0;
    if (some && (logits == nullptr || targets == nullptr || logp == nullptr)) return LORS_ERR_NULL;
    lors_status_t st = check_logits(p);
    if (st != LORS_OK) return st;
    const int64_t n = p->batch * p->length, es = elt_size(p->dtype), is = index_size(p->index_dtype);
    const size_t need = lt::logprob_workspace_bytes(n, p->vocab, p->dtype == LORS_DTYPE_BF16);
    st = check_arrays({{logits, logits_bytes(p), es}, {targets, n * is, is}},
                      {{logp, 4 * n, 4}, {stats, 8 * n, 8}, {workspace, static_cast<int64_t>(need), 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, need);
    if (st != LORS_OK) return st;
    lt::LogprobArgs a = logprob_args(p, logits, targets);
    a.logp = logp;
    a.stats = stats;
    a.workspace = workspace;
    return from_hip(lt::launch_logprob_forward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

lors_status_t lors_logprob_backward(const lors_logits_t* p, const float* dlogp, int64_t span, const float* upstream,
                                    const void* logits, const void* targets, const float* stats, void* dlogits,
                                    void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    const bool some = p->batch != 0 && p->length != 0;
    if (some && (dlogp == nullptr || logits == nullptr || targets == nullptr || stats == nullptr || dlogits == nullptr))
        return LORS_ERR_NULL;
    lors_status_t st = check_logits(p);
    if (st != LORS_OK) return st;
    const int64_t n = p->batch * p->length, es = elt_size(p->dtype), is = index_size(p->index_dtype);
    if (span < 1 || (some && (span > p->length || n % span != 0))) return LORS_ERR_SHAPE;
    st = check_arrays({{dlogp, 4 * (n / span), 4}, {upstream, 4, 4}, {logits, logits_bytes(p), es},
                       {targets, n * is, is}, {stats, 8 * n, 8}},
                      {{dlogits, n * p->vocab * es, es}});
    if (st != LORS_OK) return st;
    lt::LogprobArgs a = logprob_args(p, logits, targets);
    a.dlogp = dlogp;
    a.span = span;
    a.upstream = upstream;
    a.stats = const_cast<float*>(stats);
    a.dlogits = dlogits;
    return from_hip(lt::launch_logprob_backward(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

lors_status_t lors_preference(const lors_preference_t* p, const float* logp, const float* ref, const void* targets,
                              float* loss, float* reward, float* dseq, void* stream) {
    if (p == nullptr || loss == nullptr || reward == nullptr || dseq == nullptr) return LORS_ERR_NULL;
    if (p->length != 0 && (logp == nullptr || targets == nullptr)) return LORS_ERR_NULL;
    if (!valid_index(p->index_dtype)) return LORS_ERR_DTYPE;
    if (p->pairs < 1 || p->pairs > kMaxExtent / 2 || p->vocab < 1 || p->vocab > kMaxExtent) return LORS_ERR_SHAPE;
    const int64_t n = rows_of(2 * p->pairs, p->length), is = index_size(p->index_dtype);
    if (n < 0 || !std::isfinite(p->beta) || !(p->smoothing >= 0.0 && p->smoothing <= 0.5)) return LORS_ERR_SHAPE;
    if (p->flags != 0) return LORS_ERR_UNSUPPORTED;
    const lors_status_t st = check_arrays({{logp, 4 * n, 4}, {ref, 4 * n, 4}, {targets, n * is, is}},
                                          {{loss, 4, 4}, {reward, 8 * p->pairs, 4}, {dseq, 8 * p->pairs, 4}});
    if (st != LORS_OK) return st;
    const lt::PreferenceArgs a{p->pairs,
                               p->length,
                               p->vocab,
                               p->beta,
                               p->smoothing,
                               p->index_dtype == LORS_INDEX_I64,
                               logp,
                               ref,
                               targets,
                               loss,
                               reward,
                               dseq};
    return from_hip(lt::launch_preference(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
