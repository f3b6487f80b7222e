// Norms of residual + dropout(x), and their gradients.
//
// A row is held in registers by a group of lanes: of one wave for narrow rows
// (several rows to a wave), of a whole workgroup for wide ones.  The mean is
// taken first and the variance from the deviations, so that neither cancels.
#include "train_common.hpp"

namespace lors {
namespace train {
namespace {

constexpr int kMaxWaves = 1024 / 64;

// The lanes that share a row.  LPR (8 .. 64): that many lanes of a wave; the
// workgroup of 256 threads takes 256 / LPR rows at once.  LPR = 0: the whole
// workgroup.  V units per lane; lane i of the row holds units i, i + lanes, ..
template <int LPR>
struct RowLanes {
    int lanes, slot, slots, lane;
    __device__ __forceinline__ RowLanes() {
        if constexpr (LPR == 0) {
            lanes = blockDim.x;
            slot = 0;
            slots = 1;
            lane = threadIdx.x;
        } else {
            lanes = LPR;
            slots = blockDim.x / LPR;
            slot = threadIdx.x / LPR;
            lane = threadIdx.x % LPR;
        }
    }
};

// Sums of N values over the lanes of a row, in each of them.  `lds`: kMaxWaves
// floats per value, which no wave may still read from an earlier call.
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[kMaxWaves]) {
    if constexpr (LPR != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = over_lanes<LPR>(v[i], Add());
    } else {
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = over_lanes<64>(v[i], Add());
            if ((threadIdx.x & 63) == 0) lds[i][wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float sum = 0.f;
            for (int w = 0; w < waves; ++w) sum += lds[i][w];
            v[i] = sum;
        }
    }
}

template <typename T, int LPR, int V, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(
    int64_t rows, int cols, float eps, bool rms, DropArgs drop, const T* __restrict__ X,
    const T* __restrict__ residual, const T* __restrict__ weight, const T* __restrict__ bias, T* __restrict__ Y,
    T* __restrict__ Z, float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float lds[2][1][kMaxWaves];
    const RowLanes<LPR> me;
    const int64_t n = (int64_t)block_id() * me.slots + me.slot;
    if (n >= rows) return;  // whole rows: no barrier follows for LPR != 0, and all lanes agree for LPR = 0
    const int64_t base = n * cols;
    F8 z[V];
    int left[V];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (me.lane + i * me.lanes) * kUnit;
        left[i] = min(cols - c, kUnit);
        if (left[i] <= 0) continue;
        z[i] = widen(load_unit(X + base + c, left[i]));
        Raw<T> q;
        if (residual != nullptr) q = load_unit(residual + base + c, left[i]);
        if (drop.below != 0) Dropper(drop).apply(z[i], (uint32_t)n, (uint32_t)(c / kUnit));
        if (residual != nullptr) {
            const F8 f = widen(q);
#pragma unroll
            for (int e = 0; e < kUnit; ++e) z[i].v[e] += f.v[e];
        }
        if (Z != nullptr) {
            // the sum is what the residual stream stores: normalise that
            const Raw<T> r = narrow<T>(z[i]);
            store_unit(Z + base + c, r, left[i]);
            z[i] = widen(r);
        }
#pragma unroll
        for (int e = 0; e < kUnit; ++e) sum[0] += rms ? z[i].v[e] * z[i].v[e] : z[i].v[e];  // 0 past the row
    }
    row_sums<LPR>(sum, lds[0]);
    float mu = 0.f, sq = sum[0];
    if (!rms) {
        mu = sum[0] / (float)cols;
        float dev[1] = {0.f};
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (left[i] > 0)
#pragma unroll
                for (int e = 0; e < kUnit; ++e)
                    if (e < left[i]) dev[0] += (z[i].v[e] - mu) * (z[i].v[e] - mu);
        row_sums<LPR>(dev, lds[1]);
        sq = dev[0];
    }
    const float scale = 1.f / sqrtf(sq / (float)cols + eps);
    if (me.lane == 0) {
        if (mean != nullptr && !rms) mean[n] = mu;
        if (rstd != nullptr) rstd[n] = scale;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (left[i] <= 0) continue;
        const int c = (me.lane + i * me.lanes) * kUnit;
        F8 y;
#pragma unroll
        for (int e = 0; e < kUnit; ++e) y.v[e] = (z[i].v[e] - mu) * scale;
        if (weight != nullptr) {
            const F8 w = widen(load_unit(weight + c, left[i]));
#pragma unroll
            for (int e = 0; e < kUnit; ++e) y.v[e] *= w.v[e];
        }
        if (bias != nullptr) {
            const F8 b = widen(load_unit(bias + c, left[i]));
#pragma unroll
            for (int e = 0; e < kUnit; ++e) y.v[e] += b.v[e];
        }
        store_unit(Y + base + c, narrow<T>(y), left[i]);
    }
}

template <typename T>
__device__ __forceinline__ Raw<T> ones() {
    F8 f;
#pragma unroll
    for (int e = 0; e < kUnit; ++e) f.v[e] = 1.f;
    return narrow<T>(f);
}

// A workgroup's sums, one per column, to `out`: those of its slots are added up
// in LDS first.
template <int LPR, int V>
__device__ __forceinline__ void put_row(const RowLanes<LPR>& me, F8 (&sum)[V], const int (&left)[V],
                                        float* __restrict__ out) {
    if constexpr (LPR != 0) {
        __shared__ float lds[kUnit][256];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kUnit; ++e) lds[e][threadIdx.x] = sum[i].v[e];
            __syncthreads();
            if (me.slot == 0)
                for (int k = 1; k < 256 / LPR; ++k)
#pragma unroll
                    for (int e = 0; e < kUnit; ++e) sum[i].v[e] += lds[e][k * LPR + me.lane];
        }
        if (me.slot != 0) return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (left[i] > 0) store_unit(out + (me.lane + i * me.lanes) * kUnit, narrow<float>(sum[i]), left[i]);
}

// The gradients.  A workgroup takes every gridDim.x-th group of rows and keeps its
// sums of dweight and dbias in registers; they leave as one partial row per
// workgroup, which a second launch adds up in a fixed order.
template <typename T, int LPR, int V, int NT>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(
    int64_t rows, int cols, bool rms, DropArgs drop, const T* __restrict__ dY, const T* __restrict__ dZ,
    const T* __restrict__ Z, const T* __restrict__ weight, const float* __restrict__ mean,
    const float* __restrict__ rstd, T* __restrict__ dX, T* __restrict__ dresidual, float* __restrict__ part,
    bool want_dw, bool want_db) {
    __shared__ float lds[2][2][kMaxWaves];
    const RowLanes<LPR> me;
    F8 dw[V] = {}, db[V] = {};
    Raw<T> w[V];
    int left[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (me.lane + i * me.lanes) * kUnit;
        left[i] = min(cols - c, kUnit);
        w[i] = ones<T>();
        if (weight != nullptr && left[i] > 0) w[i] = load_unit(weight + c, left[i]);
    }
    int turn = 0;
    for (int64_t n = (int64_t)blockIdx.x * me.slots + me.slot; n < rows; n += (int64_t)gridDim.x * me.slots) {
        const int64_t base = n * cols;
        const float mu = rms ? 0.f : mean[n], scale = rstd[n];
        Raw<T> z[V], y[V], q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (me.lane + i * me.lanes) * kUnit;
            if (left[i] <= 0) continue;
            z[i] = load_unit(Z + base + c, left[i]);
            y[i] = load_unit(dY + base + c, left[i]);
            if (dZ != nullptr) q[i] = load_unit(dZ + base + c, left[i]);
        }
        float sums[2] = {0.f, 0.f};  // of g, and of g h
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (left[i] <= 0) continue;
            const F8 fz = widen(z[i]), fy = widen(y[i]), fw = widen(w[i]);
#pragma unroll
            for (int e = 0; e < kUnit; ++e) {
                const float h = (fz.v[e] - mu) * scale, g = fy.v[e] * fw.v[e];  // dY is 0 past the row
                sums[0] += g;
                sums[1] += g * h;
                dw[i].v[e] += fy.v[e] * h;
                db[i].v[e] += fy.v[e];
            }
        }
        row_sums<LPR>(sums, lds[turn]);
        turn ^= 1;
        const float m1 = rms ? 0.f : sums[0] / (float)cols, m2 = sums[1] / (float)cols;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (left[i] <= 0) continue;
            const int c = (me.lane + i * me.lanes) * kUnit;
            const F8 fz = widen(z[i]), fy = widen(y[i]), fw = widen(w[i]);
            F8 d;
#pragma unroll
            for (int e = 0; e < kUnit; ++e) {
                const float h = (fz.v[e] - mu) * scale, g = fy.v[e] * fw.v[e];
                d.v[e] = scale * (g - m1 - h * m2);
            }
            if (dZ != nullptr) {
                const F8 f = widen(q[i]);
#pragma unroll
                for (int e = 0; e < kUnit; ++e) d.v[e] += f.v[e];
            }
            if (dresidual != nullptr) store_unit(dresidual + base + c, narrow<T>(d), left[i]);
            if (drop.below != 0) Dropper(drop).apply(d, (uint32_t)n, (uint32_t)(c / kUnit));
            store_unit(dX + base + c, narrow<T>(d), left[i]);
        }
    }
    // one row of dweight per workgroup, then as many of dbias
    if (want_dw) put_row<LPR, V>(me, dw, left, part + (int64_t)blockIdx.x * cols);
    if (want_db) put_row<LPR, V>(me, db, left, part + (int64_t)((want_dw ? gridDim.x : 0) + blockIdx.x) * cols);
}

// The sum of a column over the partial rows: 64 columns per workgroup, a part of
// the rows per wave, the waves' sums added in order.
constexpr int kJoinWaves = 16;
template <bool BF16>
__global__ __launch_bounds__(64 * kJoinWaves) void norm_join_kernel(const float* __restrict__ part, int prows, int cols,
                                                                    void* dweight, void* dbias) {
    __shared__ float lds[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    const float* p = part + (int64_t)blockIdx.y * prows * cols + c;
    void* out = dweight == nullptr || blockIdx.y == 1 ? dbias : dweight;
    float sum = 0.f;
    if (c < cols)
        for (int r = wave; r < prows; r += kJoinWaves) sum += p[(int64_t)r * cols];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= cols) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i) sum += lds[i][lane];
    if constexpr (BF16) ((uint16_t*)out)[c] = bf16_bits(sum);
    else ((float*)out)[c] = sum;
}

// How a row is held: lanes of a wave per row (0: a workgroup), units per lane, the
// threads of the workgroup and the most of them that its kernel is built for
// (which sets the registers each may have).
struct Plan {
    int lpr, v, most, threads;
};

Plan plan_of(int64_t cols) {
    const int units = (int)((cols + kUnit - 1) / kUnit);
    if (units <= 8) return {8, 1, 256, 256};
    if (units <= 16) return {16, 1, 256, 256};
    if (units <= 32) return {32, 1, 256, 256};
    if (units <= 64) return {64, 1, 256, 256};
    if (units <= 128) return {64, 2, 256, 256};
    const int v = units <= 1024 ? 2 : 4;
    return {0, v, units <= 2048 ? 512 : 1024, ((units + v - 1) / v + 63) / 64 * 64};
}

int64_t rows_per_group(const Plan& p) { return p.lpr == 0 ? 1 : p.threads / p.lpr; }

// Workgroups of the backward: enough to fill the chip, no more than there are
// groups of rows.
int64_t backward_groups(int64_t rows, const Plan& p) {
    const int64_t groups = (rows + rows_per_group(p) - 1) / rows_per_group(p);
    const int64_t most = 512;
    return groups < most ? groups : most;
}

template <int LPR, int V, int NT>
struct Held {
    static constexpr int lpr = LPR, v = V, nt = NT;
};

template <typename F>
hipError_t with_plan(const Plan& p, F&& f) {
    switch (p.lpr) {
        case 8: return f(Held<8, 1, 256>());
        case 16: return f(Held<16, 1, 256>());
        case 32: return f(Held<32, 1, 256>());
        case 64: return p.v == 1 ? f(Held<64, 1, 256>()) : f(Held<64, 2, 256>());
        default: break;
    }
    if (p.v == 2) return f(Held<0, 2, 512>());
    return p.most == 512 ? f(Held<0, 4, 512>()) : f(Held<0, 4, 1024>());
}

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t s) {
    const Plan p = plan_of(a.cols);
    return with_plan(p, [&](auto h) {
        using H = decltype(h);
        const int64_t rpg = rows_per_group(p);
        hipLaunchKernelGGL((norm_fwd_kernel<T, H::lpr, H::v, H::nt>),
                           grid_of((a.rows + rpg - 1) / rpg), dim3(p.threads), 0, s, a.rows, (int)a.cols,
                           a.eps, a.rms, a.drop, (const T*)a.X, (const T*)a.residual, (const T*)a.weight,
                           (const T*)a.bias, (T*)a.Y, (T*)a.Z, a.mean, a.rstd);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward(const NormArgs& a, hipStream_t s) {
    const Plan p = plan_of(a.cols);
    const int64_t groups = backward_groups(a.rows, p);
    const bool dw = a.dweight != nullptr, db = a.dbias != nullptr;
    if (groups > 0) {
        const hipError_t e = with_plan(p, [&](auto h) {
            using H = decltype(h);
            hipLaunchKernelGGL((norm_bwd_kernel<T, H::lpr, H::v, H::nt>), dim3((unsigned)groups),
                               dim3(p.threads), 0, s, a.rows, (int)a.cols, a.rms, a.drop, (const T*)a.dY,
                               (const T*)a.dZ, (const T*)a.Z, (const T*)a.weight, a.mean, a.rstd, (T*)a.dX,
                               (T*)a.dresidual, a.part, dw, db);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if (!dw && !db) return hipSuccess;
    const dim3 grid((unsigned)((a.cols + 63) / 64), dw && db ? 2 : 1);
    if (a.grad_bf16)
        hipLaunchKernelGGL(norm_join_kernel<true>, grid, dim3(64 * kJoinWaves), 0, s, a.part, (int)groups, (int)a.cols,
                           a.dweight, a.dbias);
    else
        hipLaunchKernelGGL(norm_join_kernel<false>, grid, dim3(64 * kJoinWaves), 0, s, a.part, (int)groups, (int)a.cols,
                           a.dweight, a.dbias);
    return hipGetLastError();
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int64_t cols) {
    const Plan p = plan_of(cols);
    return (size_t)(2 * 4 * backward_groups(rows, p) * cols);
}

hipError_t launch_norm_forward(const NormArgs& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? forward<__bf16>(a, s) : forward<float>(a, s);
}

hipError_t launch_norm_backward(const NormArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? backward<__bf16>(a, s) : backward<float>(a, s);
}

}  // namespace train
}  // namespace lors
