// Internal launcher interface between the C ABI of the operators around the layer
// (train_abi.cpp) and their kernels.  Every launcher assumes its arguments were
// validated by the ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lors {
namespace train {

// A grid of at least `blocks` workgroups: more than 2^20 go on in a second dimension
// (a launch counts its threads of one dimension in 32 bits).  Kernels take their
// number from block_id() and leave where it is past the work.
static inline dim3 grid_of(int64_t blocks) {
    const int64_t wide = (int64_t)1 << 20;
    if (blocks <= wide) return dim3((unsigned)blocks);
    return dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}

// Dropout of a launch: elements whose 16 random bits are below `below` are
// dropped (0: no dropout), the others multiplied by `factor`.
struct DropArgs {
    uint64_t seed, offset;
    const uint64_t* state;  // device, or nullptr
    uint32_t below;
    float factor;
};

struct DropoutArgs {
    int64_t rows, cols;
    DropArgs drop;
    const void* X;
    const void* residual;  // or nullptr
    void* Y;
};
hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t s);

struct NormArgs {
    int64_t rows, cols;
    float eps;
    bool rms;
    DropArgs drop;
    bool grad_bf16;
    const void* X;         // forward
    const void* residual;  // or nullptr
    const void* weight;    // or nullptr
    const void* bias;      // or nullptr
    void* Y;
    void* Z;               // or nullptr
    float* mean;           // or nullptr
    float* rstd;           // or nullptr (forward)
    const void* dY;        // backward (with Z, weight, mean, rstd)
    const void* dZ;        // or nullptr
    void* dX;
    void* dresidual;       // or nullptr
    void* dweight;         // or nullptr
    void* dbias;           // or nullptr
    float* part;           // partial sums of dweight and dbias
};
hipError_t launch_norm_forward(const NormArgs& a, bool bf16, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, bool bf16, hipStream_t s);
size_t norm_workspace_bytes(int64_t rows, int64_t cols, bool bf16);

struct EmbeddingArgs {
    int64_t tokens, vocab, cols;
    float scale;
    bool grad_bf16, index64;
    const void* ids;
    const void* E;
    void* Y;
    const void* dY;
    void* dE;
    void* workspace;
};
hipError_t launch_embedding_forward(const EmbeddingArgs& a, bool bf16, hipStream_t s);
hipError_t launch_embedding_backward(const EmbeddingArgs& a, bool bf16, hipStream_t s);
// Whether the backward's grids can count their work in 32 bits.
bool embedding_groups_fit(int64_t tokens, int64_t vocab, int64_t cols);
size_t embedding_workspace_bytes(int64_t tokens, int64_t vocab, int64_t cols);

struct LogprobArgs {
    int64_t batch, length, vocab, batch_stride, row_stride;
    bool index64;
    const void* logits;
    const void* targets;
    float* logp;
    float* stats;           // or nullptr (forward)
    void* workspace;
    const float* dlogp;     // backward (with stats)
    int64_t span;
    const float* upstream;  // or nullptr
    void* dlogits;
};
hipError_t launch_logprob_forward(const LogprobArgs& a, bool bf16, hipStream_t s);
hipError_t launch_logprob_backward(const LogprobArgs& a, bool bf16, hipStream_t s);
// Whether the grids can count their work in 32 bits.
bool logprob_grids_fit(int64_t rows, int64_t vocab);
size_t logprob_workspace_bytes(int64_t rows, int64_t vocab, bool bf16);

struct PreferenceArgs {
    int64_t pairs, length, vocab;
    double beta, smoothing;
    bool index64;
    const float* logp;
    const float* ref;  // or nullptr
    const void* targets;
    float* loss;
    float* reward;
    float* dseq;
};
hipError_t launch_preference(const PreferenceArgs& a, hipStream_t s);

}  // namespace train
}  // namespace lors
