// Dropout from the counter-based generator: y = keep ? factor x : 0 (+ residual).
// The mask is a function of (seed, offset, row, column), so the gradient is the
// same pass over dY and nothing is stored.
//
// Bound by memory as long as the generator keeps up: a block of Philox is 20
// products of 32 x 32 -> 64 bits (a quarter of the rate of other instructions) and
// about 60 more.  With 32 bits an element a block would cover four and, by that count,
// take 1.7 times as long as reading and writing four bf16; with 16 bits it covers
// eight, and p is resolved to 2^-16.  8192 x 14336 bf16: 94 us, 5.0 TB/s (a copy reaches 5.1);
// 777 x 1003 fp32: 4 us.
#include "train_common.hpp"

namespace lors {
namespace train {
namespace {

constexpr int NT = 256;
constexpr int kAhead = 2;  // units a thread has in flight

// A grid of 16 workgroups a CU walks the units, two of them ahead of the generator.
template <typename T>
__global__ __launch_bounds__(NT) void dropout_kernel(int64_t rows, uint32_t cols, uint32_t units, DropArgs drop,
                                                     const T* __restrict__ X, const T* __restrict__ residual,
                                                     T* __restrict__ Y) {
    constexpr int N = kUnit<T>;
    const Dropper d(drop);
    // Units in row-major order, a grid's worth apart: one division, then steps.
    const uint32_t stride = gridDim.x * NT;
    const uint32_t step_rows = stride / units, step_units = stride - step_rows * units;
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    int64_t n = t / units;
    uint32_t g = t - (uint32_t)n * units;
    while (n < rows) {
        int64_t at[kAhead];
        uint32_t row[kAhead], unit[kAhead];
        int left[kAhead];
        Raw<T, N> x[kAhead], r[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            at[i] = n * cols + (int64_t)g * N;
            row[i] = (uint32_t)n;
            unit[i] = g;
            left[i] = n < rows ? (int)min(cols - g * N, (uint32_t)N) : 0;
            if (left[i] > 0) {
                x[i] = load_unit(X + at[i], left[i]);
                if (residual != nullptr) r[i] = load_unit(residual + at[i], left[i]);
            }
            n += step_rows;
            g += step_units;
            if (g >= units) {
                g -= units;
                ++n;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (left[i] <= 0) break;
            F<N> f = widen(x[i]);
            d.apply(f, row[i], unit[i]);
            if (residual != nullptr) {
                const F<N> q = widen(r[i]);
#pragma unroll
                for (int e = 0; e < N; ++e) f.v[e] += q.v[e];
            }
            store_unit(Y + at[i], narrow<T>(f), left[i]);
        }
    }
}

template <typename T>
hipError_t launch(const DropoutArgs& a, hipStream_t s) {
    const uint32_t units = (uint32_t)((a.cols + kUnit<T> - 1) / kUnit<T>);
    // rows and units are below 2^31 and 2^29: their product fits
    const int64_t blocks = (a.rows * units + NT - 1) / NT;
    const int64_t most = 16 * (int64_t)256;
    hipLaunchKernelGGL(dropout_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(NT), 0, s, a.rows,
                       (uint32_t)a.cols, units, a.drop, (const T*)a.X, (const T*)a.residual, (T*)a.Y);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? launch<__bf16>(a, s) : launch<float>(a, s);
}

}  // namespace train
}  // namespace lors
