// Norms of residual + dropout(x), and their gradients.
//
// A row is held in registers by a group of lanes: of one wave for narrow rows
// (several rows to a wave), of a whole workgroup for wide ones.  The mean is
// taken first and the variance from the deviations, so that neither cancels.
// h = (z - mean) rstd; y = h weight + bias; with g = dy weight and dz the gradient of z
// from elsewhere, d = rstd (g - mean(g) - h mean(g h)) + dz (no mean(g) for the root mean
// square), dweight = sum of dy h, dbias = sum of dy over the rows.
//
// Bound by memory: every element is read and written once a pass.  4096 x 5120
// bf16 with residual and dropout 0.1: forward 38 us (168 MB, 4.4 TB/s; a copy
// reaches 5.1), backward 53 us (210 MB and 21 MB of partial sums) and 5 us to join
// them.  4 x 4096, the norm of a token: 3.7 us, all latency.
#include "train_common.hpp"

namespace lors {
namespace train {
namespace {

constexpr int kMaxWaves = 1024 / 64;

// The lanes that share a row.  LPR (8 .. 64): that many lanes of a wave; the
// workgroup of 256 threads takes 256 / LPR rows at once.  LPR = 0: the whole
// workgroup.  Lane i of a row holds its units i, i + lanes, ..
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

// Sums of K values over the lanes of a row, in each of them.  `lds`: kMaxWaves
// floats per value, which no wave may still read from an earlier call.
template <int LPR, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*lds)[kMaxWaves]) {
    if constexpr (LPR != 0) {
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] = over_lanes<LPR>(v[i], Add());
    } else {
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            v[i] = over_lanes<64>(v[i], Add());
            if ((threadIdx.x & 63) == 0) lds[i][wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float sum = 0.f;
            for (int w = 0; w < waves; ++w) sum += lds[i][w];
            v[i] = sum;
        }
    }
}

template <typename T, int LPR, int V, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(int64_t rows, int cols, float eps, bool rms, DropArgs drop,
                                                      const T* __restrict__ X, const T* __restrict__ residual,
                                                      const T* __restrict__ weight, const T* __restrict__ bias,
                                                      T* __restrict__ Y, T* __restrict__ Z, float* __restrict__ mean,
                                                      float* __restrict__ rstd) {
    constexpr int N = kUnit<T>;
    __shared__ float lds[2][1][kMaxWaves];
    const RowLanes<LPR> me;
    const int64_t n = (int64_t)block_id() * me.slots + me.slot;
    if (n >= rows) return;  // whole rows: no barrier follows for LPR != 0, and all lanes agree for LPR = 0
    const Dropper dropper(drop);
    const int64_t base = n * cols;
    Raw<T, N> x[V], r[V];
    F<N> z[V];
    int left[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (me.lane + i * me.lanes) * N;
        left[i] = min(cols - c, N);
        if (left[i] <= 0) continue;
        x[i] = load_unit(X + base + c, left[i]);
        if (residual != nullptr) r[i] = load_unit(residual + base + c, left[i]);
    }
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (left[i] <= 0) continue;
        const int c = (me.lane + i * me.lanes) * N;
        z[i] = widen(x[i]);
        if (drop.below != 0) dropper.apply(z[i], (uint32_t)n, (uint32_t)(c / N));
        if (residual != nullptr) {
            const F<N> f = widen(r[i]);
#pragma unroll
            for (int e = 0; e < N; ++e) z[i].v[e] += f.v[e];
        }
        if (Z != nullptr) {
            // the sum is what the residual stream stores: normalise that
            const Raw<T, N> q = narrow<T>(z[i]);
            store_unit(Z + base + c, q, left[i]);
            z[i] = widen(q);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[0] += rms ? z[i].v[e] * z[i].v[e] : z[i].v[e];  // 0 past the row
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
                for (int e = 0; e < N; ++e)
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
        const int c = (me.lane + i * me.lanes) * N;
        F<N> y;
#pragma unroll
        for (int e = 0; e < N; ++e) y.v[e] = (z[i].v[e] - mu) * scale;
        if (weight != nullptr) {
            const F<N> w = widen(load_unit(weight + c, left[i]));
#pragma unroll
            for (int e = 0; e < N; ++e) y.v[e] *= w.v[e];
        }
        if (bias != nullptr) {
            const F<N> b = widen(load_unit(bias + c, left[i]));
#pragma unroll
            for (int e = 0; e < N; ++e) y.v[e] += b.v[e];
        }
        store_unit(Y + base + c, narrow<T>(y), left[i]);
    }
}

// A workgroup's sums, one per column, to `out`: those of its slots are added up
// in LDS first.
template <int LPR, int V, int N>
__device__ __forceinline__ void put_row(const RowLanes<LPR>& me, F<N> (&sum)[V], const int (&left)[V],
                                        float* __restrict__ out) {
    if constexpr (LPR != 0) {
        __shared__ float lds[N][256];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < N; ++e) lds[e][threadIdx.x] = sum[i].v[e];
            __syncthreads();
            if (me.slot == 0)
                for (int k = 1; k < 256 / LPR; ++k)
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[i].v[e] += lds[e][k * LPR + me.lane];
        }
        if (me.slot != 0) return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (left[i] > 0) store_unit(out + (me.lane + i * me.lanes) * N, narrow<float>(sum[i]), left[i]);
}

// N sums of a lane in LDS, four at a time, NT apart.
template <int N, int NT>
__device__ __forceinline__ F<N> get_sums(const float4* at) {
    F<N> f;
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const float4 q = at[k * NT];
        f.v[4 * k] = q.x;
        f.v[4 * k + 1] = q.y;
        f.v[4 * k + 2] = q.z;
        f.v[4 * k + 3] = q.w;
    }
    return f;
}
template <int N, int NT>
__device__ __forceinline__ void put_sums(float4* at, const F<N>& f) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) at[k * NT] = float4{f.v[4 * k], f.v[4 * k + 1], f.v[4 * k + 2], f.v[4 * k + 3]};
}

// The gradients.  A workgroup takes every gridDim.x-th group of rows and keeps its
// sums of dweight and dbias in registers; they leave as one partial row per
// workgroup, which a second launch adds up in a fixed order.
// AHEAD: the next row is loaded before this one's sums are joined, so that memory
// works through the barrier.  Without it (rows so wide that the registers do not
// hold two) a row's second half reads it again out of the cache, and the widest
// rows' sums of dweight are in LDS (each lane's own columns; 128 KB of the 160):
// 1024 x 32768 bf16 103 us, fp32 194, against 140 and 265 with registers that spill.
template <typename T, int LPR, int V, int NT, bool AHEAD>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(int64_t rows, int cols, bool rms, DropArgs drop,
                                                      const T* __restrict__ dY, const T* __restrict__ dZ,
                                                      const T* __restrict__ Z, const T* __restrict__ weight,
                                                      const float* __restrict__ mean, const float* __restrict__ rstd,
                                                      T* __restrict__ dX, T* __restrict__ dresidual,
                                                      float* __restrict__ part, bool want_dw, bool want_db) {
    constexpr int N = kUnit<T>;
    constexpr int H = AHEAD ? V : 1;             // units that are held
    constexpr bool kInLds = V * N == 32;         // 32 sums of each kind a lane
    constexpr int W = kInLds ? 1 : V;            // units of dweight in registers
    __shared__ float4 wide[kInLds ? NT * 8 : 1];  // the lane's 32 sums of dweight, NT apart
    __shared__ float lds[2][2][kMaxWaves];
    const RowLanes<LPR> me;
    const Dropper dropper(drop);
    const int64_t step = (int64_t)gridDim.x * me.slots;
    F<N> dw[W] = {}, db[V] = {};
    int left[V];
    if constexpr (kInLds)
#pragma unroll
        for (int k = 0; k < 8; ++k) wide[k * NT + threadIdx.x] = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) left[i] = min(cols - (me.lane + i * me.lanes) * N, N);
    auto column = [&](int i) { return (me.lane + i * me.lanes) * N; };
    auto weights = [&](int i) {
        if (weight == nullptr || left[i] <= 0) {
            F<N> one;
#pragma unroll
            for (int e = 0; e < N; ++e) one.v[e] = 1.f;
            return narrow<T>(one);
        }
        return load_unit(weight + column(i), left[i]);
    };
    struct Row {
        Raw<T, N> z[H], y[H], q[H];
        float mu, scale;
    };
    auto load = [&](Row& r, int h, int i, int64_t n) {
        const int64_t at = n * cols + column(i);
        if (left[i] <= 0) return;
        r.z[h] = load_unit(Z + at, left[i]);
        r.y[h] = load_unit(dY + at, left[i]);
        if (dZ != nullptr) r.q[h] = load_unit(dZ + at, left[i]);
    };
    auto load_row = [&](Row& r, int64_t n) {
        r.mu = rms ? 0.f : mean[n];
        r.scale = rstd[n];
        if constexpr (AHEAD)
#pragma unroll
            for (int i = 0; i < V; ++i) load(r, i, i, n);
    };
    Raw<T, N> w[H];
    if constexpr (AHEAD)
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = weights(i);
    Row now, next;
    int64_t n = (int64_t)blockIdx.x * me.slots + me.slot;
    if (n < rows) load_row(now, n);
    for (int turn = 0; n < rows; turn ^= 1) {
        if (AHEAD && n + step < rows) load_row(next, n + step);
        float sums[2] = {0.f, 0.f};  // of g, and of g h
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int h = AHEAD ? i : 0;
            if constexpr (!AHEAD) {
                __builtin_amdgcn_sched_barrier(0);  // one unit after the other: the registers hold no more
                load(now, 0, i, n);
                w[0] = weights(i);
            }
            if (left[i] <= 0) continue;
            const F<N> fz = widen(now.z[h]), fy = widen(now.y[h]), fw = widen(w[h]);
            F<N>& sum = dw[kInLds ? 0 : i];
            float4* const kept = wide + (kInLds ? i * (N / 4) * NT + threadIdx.x : 0);
            if constexpr (kInLds) sum = get_sums<N, NT>(kept);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float hat = (fz.v[e] - now.mu) * now.scale, g = fy.v[e] * fw.v[e];  // dY is 0 past the row
                sums[0] += g;
                sums[1] += g * hat;
                sum.v[e] += fy.v[e] * hat;
                db[i].v[e] += fy.v[e];
            }
            if constexpr (kInLds) put_sums<N, NT>(kept, sum);
        }
        row_sums<LPR>(sums, lds[turn]);
        const float m1 = rms ? 0.f : sums[0] / (float)cols, m2 = sums[1] / (float)cols;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int h = AHEAD ? i : 0;
            if constexpr (!AHEAD) {
                __builtin_amdgcn_sched_barrier(0);  // one unit after the other: the registers hold no more
                load(now, 0, i, n);
                w[0] = weights(i);
            }
            if (left[i] <= 0) continue;
            const int64_t at = n * cols + column(i);
            const F<N> fz = widen(now.z[h]), fy = widen(now.y[h]), fw = widen(w[h]);
            F<N> d;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float hat = (fz.v[e] - now.mu) * now.scale, g = fy.v[e] * fw.v[e];
                d.v[e] = now.scale * (g - m1 - hat * m2);
            }
            if (dZ != nullptr) {
                const F<N> f = widen(now.q[h]);
#pragma unroll
                for (int e = 0; e < N; ++e) d.v[e] += f.v[e];
            }
            if (dresidual != nullptr) store_unit(dresidual + at, narrow<T>(d), left[i]);
            if (drop.below != 0) dropper.apply(d, (uint32_t)n, (uint32_t)(column(i) / N));
            store_unit(dX + at, narrow<T>(d), left[i]);
        }
        n += step;
        if constexpr (AHEAD) now = next;
        else if (n < rows) load_row(now, n);
    }
    // one row of dweight per workgroup, then as many of dbias
    if (want_dw) {
        if constexpr (kInLds) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (left[i] > 0)
                    store_unit(part + (int64_t)blockIdx.x * cols + column(i),
                               narrow<float>(get_sums<N, NT>(wide + i * (N / 4) * NT + threadIdx.x)), left[i]);
        } else {
            put_row(me, dw, left, part + (int64_t)blockIdx.x * cols);
        }
    }
    if (want_db) put_row(me, db, left, part + (int64_t)((want_dw ? gridDim.x : 0) + blockIdx.x) * cols);
}

// The sum of a column over the partial rows: 64 columns per workgroup, a part of
// the rows per wave with eight loads ahead (512 rows of 5120: 4.8 us, 11 us one by one),
// the waves' sums added in order.
constexpr int kJoinWaves = 16;
template <bool BF16>
__global__ __launch_bounds__(64 * kJoinWaves) void norm_join_kernel(const float* __restrict__ part, int prows, int cols,
                                                                    void* dweight, void* dbias) {
    __shared__ float lds[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    const float* p = part + (int64_t)blockIdx.y * prows * cols + min(c, cols - 1);
    void* out = dweight == nullptr || blockIdx.y == 1 ? dbias : dweight;
    float sum = 0.f;
#pragma unroll 8
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
// most threads that its kernel is built for (which sets the registers each may
// have), the threads of the workgroup.
struct Plan {
    int lpr, v, most, threads;
};

int64_t units_of(int64_t cols, bool bf16) {
    const int64_t per = bf16 ? kUnit<__bf16> : kUnit<float>;
    return (cols + per - 1) / per;
}

Plan narrow_plan(int64_t units) {
    if (units <= 8) return {8, 1, 256, 256};
    if (units <= 16) return {16, 1, 256, 256};
    if (units <= 32) return {32, 1, 256, 256};
    return {64, units <= 64 ? 1 : 2, 256, 256};
}

Plan wide_plan(int64_t units, int v, int most) {
    return {0, v, most, (int)((units + v - 1) / v + 63) / 64 * 64};
}

// The forward holds a row and little else: few waves with two units a lane are
// faster than many with one (4096 x 5120 bf16 with dropout and residual: 39 us against
// 42; 14336 wide, four against two units: 47 against 54).
Plan forward_plan(int64_t units) {
    if (units <= 128) return narrow_plan(units);
    if (units <= 1024) return wide_plan(units, 2, 512);
    return wide_plan(units, units <= 4096 ? 4 : 8, units <= 2048 ? 512 : 1024);
}

// The backward's sums take 64 bytes a unit beside the rows themselves: one unit a
// lane as far as it goes leaves room for twice the waves (4096 x 5120 bf16, the same: 59 us
// against 73; 2000 x 14336, two against four: 94 against 139).
Plan backward_plan(int64_t units) {
    if (units <= 128) return narrow_plan(units);
    if (units <= 640) return wide_plan(units, 1, 640);
    return wide_plan(units, units <= 1024 ? 1 : units <= 2048 ? 2 : units <= 4096 ? 4 : 8, 1024);
}

int64_t rows_per_group(const Plan& p) { return p.lpr == 0 ? 1 : p.threads / p.lpr; }

// Workgroups of the backward: what the chip holds of them (two to a CU, one of the
// largest), all with the same count of turns.
int64_t backward_groups(int64_t rows, const Plan& p) {
    const int64_t groups = (rows + rows_per_group(p) - 1) / rows_per_group(p);
    const int64_t most = p.threads > 640 ? 256 : 512;
    if (groups <= most) return groups;
    const int64_t turns = (groups + most - 1) / most;
    return (groups + turns - 1) / turns;
}

template <int LPR, int V, int NT>
struct Held {
    static constexpr int lpr = LPR, v = V, nt = NT;
};

template <typename T, bool FORWARD, typename Fn>
hipError_t with_plan(const Plan& p, Fn&& f) {
    switch (p.lpr) {
        case 8: return f(Held<8, 1, 256>());
        case 16: return f(Held<16, 1, 256>());
        case 32: return f(Held<32, 1, 256>());
        case 64: return p.v == 1 ? f(Held<64, 1, 256>()) : f(Held<64, 2, 256>());
        default: break;
    }
    if constexpr (FORWARD) {
        if (p.v == 2) return f(Held<0, 2, 512>());
        if (p.v == 4 && p.most == 512) return f(Held<0, 4, 512>());
    } else {
        if (p.v == 1) return p.most == 640 ? f(Held<0, 1, 640>()) : f(Held<0, 1, 1024>());
        if (p.v == 2) return f(Held<0, 2, 1024>());
    }
    if constexpr (sizeof(T) == 4)
        if (p.v == 8) return f(Held<0, 8, 1024>());
    return f(Held<0, 4, 1024>());
}

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t s) {
    const Plan p = forward_plan(units_of(a.cols, sizeof(T) == 2));
    return with_plan<T, true>(p, [&](auto h) {
        using H = decltype(h);
        const int64_t rpg = rows_per_group(p);
        hipLaunchKernelGGL((norm_fwd_kernel<T, H::lpr, H::v, H::nt>), grid_of((a.rows + rpg - 1) / rpg),
                           dim3(p.threads), 0, s, a.rows, (int)a.cols, a.eps, a.rms, a.drop, (const T*)a.X,
                           (const T*)a.residual, (const T*)a.weight, (const T*)a.bias, (T*)a.Y, (T*)a.Z, a.mean,
                           a.rstd);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward(const NormArgs& a, hipStream_t s) {
    const Plan p = backward_plan(units_of(a.cols, sizeof(T) == 2));
    const int64_t groups = backward_groups(a.rows, p);
    const bool dw = a.dweight != nullptr, db = a.dbias != nullptr;
    if (groups > 0) {
        const hipError_t e = with_plan<T, false>(p, [&](auto h) {
            using H = decltype(h);
            hipLaunchKernelGGL((norm_bwd_kernel<T, H::lpr, H::v, H::nt, (H::nt == 256 || H::v * kUnit<T> <= 8)>), dim3((unsigned)groups),
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
        hipLaunchKernelGGL(norm_join_kernel<true>, grid, dim3(64 * kJoinWaves), 0, s, a.part, (int)groups,
                           (int)a.cols, a.dweight, a.dbias);
    else
        hipLaunchKernelGGL(norm_join_kernel<false>, grid, dim3(64 * kJoinWaves), 0, s, a.part, (int)groups,
                           (int)a.cols, a.dweight, a.dbias);
    return hipGetLastError();
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int64_t cols, bool bf16) {
    return (size_t)(2 * 4 * backward_groups(rows, backward_plan(units_of(cols, bf16))) * cols);
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
