// Internal launcher interface between the C ABI of lors_block.h (block_abi.cpp) and the
// kernels of orthogonalised updates and sampling.  Every launcher assumes its arguments
// were validated by the ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lors {
namespace block {

// One matrix of an update: d its shorter side, n its longer one; element (i, j) of
// short index i and long index j is at i * n + j (wide) or j * d + i.
struct Matrix {
    const void* grad;
    float* m;        // or nullptr
    float* master;   // or nullptr
    void* param;     // or nullptr with master
    int64_t n;
    int64_t scratch; // bytes into the workspace: partial Gram matrices, then the steps' product
    float rate, keep;
    int32_t d, wide;
};

struct UpdateArgs {
    float momentum;   // beta, and 1 - beta
    float fresh;
    bool nesterov;
    double eps, a, b, c;
    int steps;
    bool grad_bf16, param_bf16;
    uint8_t* workspace;
};

// Bytes of a matrix's scratch (a multiple of 256).
int64_t update_scratch(int64_t d, int64_t n);
// Bytes of the descriptors of many matrices, in the workspace behind their scratch.
int64_t update_table(int64_t count);
hipError_t launch_update(const UpdateArgs& a, const Matrix* matrices, int64_t count, void* table, hipStream_t s);

struct SampleArgs {
    int64_t rows, vocab, row_stride;
    double temperature;
    int64_t top_k;
    double top_p, min_p;
    const void* logits;
    const float* u;
    const float* temperatures;  // or nullptr each
    const int32_t* top_ks;
    const float* top_ps;
    const float* min_ps;
    int64_t* token;
    float* logp;                // or nullptr
    void* workspace;
};
hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t s);

}  // namespace block
}  // namespace lors
