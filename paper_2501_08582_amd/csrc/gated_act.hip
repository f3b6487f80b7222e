// The elementwise steps of a gated block: H = act(G) U where the projections ran one by
// one (fp32), and the gradients of the projections' results,
//   dG = dH U act'(G),  dU = dH act(G).
// dG and dU are rounded to bf16 there, half a step each, because they are operands of
// the matrix instructions that follow; everything before that rounding is fp32.
// Bound by HBM: one pass, five arrays of 2 bytes an element in bf16 (4096 x 13824: 566 MB
// in 91 us, 6.2 TB/s).  A lane takes units of 16 bytes, a grid's stride apart.  As
// a pass of its own it is 4 % of the backward: dX's and the gradients' kernels both read the
// results, in copies straight to LDS that compute nothing on the way.
#include "gated.hpp"
#include "train_common.hpp"

#include <algorithm>

namespace lors {
namespace {

constexpr int NT = 256;

template <typename T>
__global__ __launch_bounds__(NT) void join_kernel(const T* __restrict__ G, const T* __restrict__ U, T* __restrict__ H,
                                                  int64_t n, int gelu) {
    constexpr int N = train::kUnit<T>;
    const int64_t step = (int64_t)gridDim.x * NT * N;
    for (int64_t e = ((int64_t)blockIdx.x * NT + threadIdx.x) * N; e < n; e += step) {
        train::F<N> g = train::widen<T, N>(train::load_whole<T, N>(G + e));
        const train::F<N> u = train::widen<T, N>(train::load_whole<T, N>(U + e));
#pragma unroll
        for (int i = 0; i < N; ++i) g.v[i] = activate(g.v[i], gelu) * u.v[i];
        train::store_unit<T, N>(H + e, train::narrow<T, N>(g), N);
    }
}

template <typename T>
__global__ __launch_bounds__(NT) void split_kernel(const T* __restrict__ dH, const T* __restrict__ G,
                                                   const T* __restrict__ U, T* __restrict__ dG, T* __restrict__ dU,
                                                   int64_t n, int gelu, Clear clear) {
    constexpr int N = train::kUnit<T>;
    // the adapters' gradients, which the kernels after this one add to
#pragma unroll
    for (int k = 0; k < 4; ++k)
        for (int64_t e = (int64_t)blockIdx.x * NT + threadIdx.x; e < clear.n[k]; e += (int64_t)gridDim.x * NT) clear.p[k][e] = 0.f;
    const int64_t step = (int64_t)gridDim.x * NT * N;
    for (int64_t e = ((int64_t)blockIdx.x * NT + threadIdx.x) * N; e < n; e += step) {
        const train::F<N> d = train::widen<T, N>(train::load_whole<T, N>(dH + e));
        train::F<N> g = train::widen<T, N>(train::load_whole<T, N>(G + e));
        train::F<N> u = train::widen<T, N>(train::load_whole<T, N>(U + e));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float slope;
            const float y = activate_grad(g.v[i], gelu, slope);
            g.v[i] = d.v[i] * u.v[i] * slope;
            u.v[i] = d.v[i] * y;
        }
        train::store_unit<T, N>(dG + e, train::narrow<T, N>(g), N);
        train::store_unit<T, N>(dU + e, train::narrow<T, N>(u), N);
    }
}

dim3 grid_for(int64_t n, int unit) {
    const int64_t blocks = (n / unit + NT - 1) / NT;
    return dim3((unsigned)(blocks < 8192 ? blocks : 8192));
}

}  // namespace

// n is a multiple of a unit (8 bf16, 4 fp32): R is
hipError_t launch_gated_join(const void* G, const void* U, void* H, int64_t n, bool gelu, bool bf16, hipStream_t s) {
    if (n == 0) return hipSuccess;
    if (bf16)
        hipLaunchKernelGGL(join_kernel<uint16_t>, grid_for(n, 8), dim3(NT), 0, s, (const uint16_t*)G, (const uint16_t*)U,
                           (uint16_t*)H, n, (int)gelu);
    else
        hipLaunchKernelGGL(join_kernel<float>, grid_for(n, 4), dim3(NT), 0, s, (const float*)G, (const float*)U, (float*)H, n,
                           (int)gelu);
    return hipGetLastError();
}

hipError_t launch_gated_split(const void* dH, const void* G, const void* U, void* dG, void* dU, int64_t n, bool gelu,
                              bool bf16, const Clear& clear, hipStream_t s) {
    if (n == 0) return hipSuccess;
    // few rows of wide projections have more to clear than to split
    const int64_t zeros = clear.n[0] + clear.n[1] + clear.n[2] + clear.n[3];
    const dim3 grid = grid_for(std::max(n, zeros), bf16 ? 8 : 4);
    if (bf16)
        hipLaunchKernelGGL(split_kernel<uint16_t>, grid, dim3(NT), 0, s, (const uint16_t*)dH, (const uint16_t*)G,
                           (const uint16_t*)U, (uint16_t*)dG, (uint16_t*)dU, n, (int)gelu, clear);
    else
        hipLaunchKernelGGL(split_kernel<float>, grid, dim3(NT), 0, s, (const float*)dH, (const float*)G,
                           (const float*)U, (float*)dG, (float*)dU, n, (int)gelu, clear);
    return hipGetLastError();
}

}  // namespace lors
