// Orthogonalised updates: the optimiser's step along Newton-Schulz directions of many
// matrices with a short side d <= 128 (adapters), in two passes over their data.
//
//   x = v / (|v| + eps);   steps times:  S = x x^T,  x <- a x + (b S + c S^2) x
//
// Every iterate is x_k = Q_k x_0 with Q_k a polynomial of S_0 = x_0 x_0^T, so the
// steps run on d x d matrices alone:
//   P = a I + b S + c S^2,   Q <- P Q,   S <- P S P
// (all of them symmetric, and they commute, but for rounding):
//   gram_kernel    m and v out of the gradient and the momentum; v v^T by pieces of the
//                  long side
//   steps_kernel   one workgroup a matrix: the pieces' sum, |v| out of its trace, the steps
//   apply_kernel   v again, Q v, and the update of master and param
//
// Why 64 bits: S squares the singular values.  A direction of sigma = 2e-3 of |v|
// lies at 4e-6 in S, where an error of 2^-24 of S's norm is 1.5 % of it, and the
// steps raise it by a^5 = 485 to about 1.  The matrix cores' fp64 products (half the rate of
// their fp32 ones) keep it at 1e-10, and their results come out in the layout of a
// right operand: value v of lane l is row 4v + l / 16, column l % 16, which is the
// operand of the k = 4v .. 4v + 3.  The matrices of the steps therefore never leave the
// registers; only the left operands pass through LDS.
//
// Bound by HBM for many matrices: 10 bytes an element in the first pass (bf16 gradient), 16
// in the second.  One matrix alone is bound by the steps' chain of products.
#include "block_kernels.hpp"
#include "train_common.hpp"

namespace lors {
namespace block {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;
constexpr int kBatch = 48;        // matrices of a launch: their descriptors are kernel arguments
constexpr int kPiece = 512;       // least columns (along the long side) of a workgroup
constexpr int kMostPieces = 256;

struct Batch {
    int count;
    int first[kBatch + 1];  // first workgroup of each matrix
    Matrix m[kBatch];
};

__host__ __device__ inline int64_t piece_cols(int64_t n) {
    const int64_t most = (n + kMostPieces - 1) / kMostPieces;
    const int64_t c = (most + 127) / 128 * 128;
    return c < kPiece ? kPiece : c;
}
__host__ __device__ inline int64_t pieces_of(int64_t n) { return (n + piece_cols(n) - 1) / piece_cols(n); }

// D(16x16) += A(16x4) . B(4x16): lane l holds A[l % 16][l / 16], B[l / 16][l % 16].
__device__ __forceinline__ f64x4 mfma64(double a, double b, f64x4 c) {
    return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0);
}

// The first n of N elements at p as fp32, the others 0.
template <typename T, int N>
__device__ __forceinline__ void read_some(const T* p, int n, float (&f)[N]) {
    if (n >= N) {
        const train::Packed<T, N> v = *(const train::Packed<T, N>*)p;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (sizeof(T) == 2) f[e] = bf16_bits_to_f32(v.v[e]);
            else f[e] = v.v[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        f[e] = 0.f;
        if (e < n) {
            if constexpr (sizeof(T) == 2) f[e] = bf16_bits_to_f32(p[e]);
            else f[e] = p[e];
        }
    }
}
template <typename T, int N>
__device__ __forceinline__ void write_some(T* p, int n, const float (&f)[N]) {
    train::Packed<T, N> v;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) v.v[e] = bf16_bits(f[e]);
        else v.v[e] = f[e];
    }
    if (n >= N) {
        *(train::Packed<T, N>*)p = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < n) p[e] = v.v[e];
}

__device__ __forceinline__ int most(int64_t left, int n) { return left >= n ? n : left > 0 ? (int)left : 0; }

// Matrix of this workgroup.
__device__ __forceinline__ int find(const Batch& b, int block) {
    int lo = 0, hi = b.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

struct Rule {
    float beta, fresh;
    int nesterov;
    // m <- beta m + fresh g, and v.  The second pass forms v from the m that the first
    // one stored, by the same operations: the same bits.
    __device__ __forceinline__ float moment(float m, float g) const { return fmaf(beta, m, fresh * g); }
    __device__ __forceinline__ float direction(float m, float g) const { return nesterov ? fmaf(beta, m, fresh * g) : m; }
};

// DT: 16-row blocks of the short side.  Short index i of row p of block t: 16 t + p of a
// wide matrix, DT p + t of a tall one (consecutive in memory over t).  The steps
// work on rows in the order (t, p) whatever that is.
template <int DT>
constexpr int kTiles = DT * (DT + 1) / 2;

// v of 32 columns from j0 on: lane l holds, of row l % 16 of every block, the columns
// 8 (l / 16) + e (wide) or 4 e + l / 16 (tall); any assignment does that is the same
// for every row.
template <typename T, int DT, bool WIDE>
__device__ __forceinline__ void gram_piece(const Matrix& x, const Rule& rule, int64_t j0, int64_t j1, f64x4 (&acc)[kTiles<DT>]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane & 15, h = lane >> 4;
    const T* grad = (const T*)x.grad;
    for (int64_t jb = j0 + 32 * wave; jb < j1; jb += 32 * (NT / 64)) {
        float g[DT][8], m[DT][8];
        if constexpr (WIDE) {
            const int64_t j = jb + 8 * h;
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const int i = 16 * t + p, n = i < x.d ? most(j1 - j, 8) : 0;
                read_some<T, 8>(grad + (n ? (int64_t)i * x.n + j : 0), n, g[t]);
                if (x.m != nullptr) read_some<float, 8>(x.m + (n ? (int64_t)i * x.n + j : 0), n, m[t]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t j = jb + 4 * e + h;
                const int n = j < j1 ? most(x.d - DT * p, DT) : 0;
                float a[DT], b[DT];
                read_some<T, DT>(grad + (n ? j * x.d + DT * p : 0), n, a);
                if (x.m != nullptr) read_some<float, DT>(x.m + (n ? j * x.d + DT * p : 0), n, b);
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    g[t][e] = a[t];
                    m[t][e] = x.m != nullptr ? b[t] : 0.f;
                }
            }
        }
        if (x.m != nullptr) {
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) m[t][e] = rule.moment(m[t][e], g[t][e]);
            if constexpr (WIDE) {
                const int64_t j = jb + 8 * h;
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    const int i = 16 * t + p, n = i < x.d ? most(j1 - j, 8) : 0;
                    if (n) write_some<float, 8>(x.m + (int64_t)i * x.n + j, n, m[t]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t j = jb + 4 * e + h;
                    const int n = j < j1 ? most(x.d - DT * p, DT) : 0;
                    float b[DT];
#pragma unroll
                    for (int t = 0; t < DT; ++t) b[t] = m[t][e];
                    if (n) write_some<float, DT>(x.m + j * x.d + DT * p, n, b);
                }
            }
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[t][e] = rule.direction(m[t][e], g[t][e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            double v[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) v[t] = (double)g[t][e];
            int k = 0;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int u = t; u < DT; ++u, ++k) acc[k] = mfma64(v[t], v[u], acc[k]);
        }
    }
}

template <typename T, int DT>
__global__ __launch_bounds__(NT, DT == 8 ? 1 : 2) void gram_kernel(Batch batch, Rule rule, uint8_t* __restrict__ ws) {
    constexpr int G = kTiles<DT> < 8 ? kTiles<DT> : 8;  // tiles joined at a time
    __shared__ double red[NT / 64][G][256];
    const int item = find(batch, (int)blockIdx.x);
    const Matrix x = batch.m[item];
    const int piece = (int)blockIdx.x - batch.first[item];
    const int64_t cols = piece_cols(x.n), j0 = piece * cols, j1 = j0 + cols < x.n ? j0 + cols : x.n;
    f64x4 acc[kTiles<DT>];
#pragma unroll
    for (int k = 0; k < kTiles<DT>; ++k) acc[k] = f64x4{0., 0., 0., 0.};
    if (x.wide) gram_piece<T, DT, true>(x, rule, j0, j1, acc);
    else gram_piece<T, DT, false>(x, rule, j0, j1, acc);
    // the waves' sums, in wave order
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double* out = (double*)(ws + x.scratch) + (int64_t)piece * (kTiles<DT> * 256);
#pragma unroll
    for (int k0 = 0; k0 < kTiles<DT>; k0 += G) {
        if (k0 > 0) __syncthreads();
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (k0 + k < kTiles<DT>)
#pragma unroll
                for (int v = 0; v < 4; ++v) red[wave][k][64 * v + lane] = acc[k0 + k < kTiles<DT> ? k0 + k : 0][v];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (k0 + k < kTiles<DT>) {
                double s = red[0][k][tid];
#pragma unroll
                for (int w = 1; w < NT / 64; ++w) s += red[w][k][tid];
                out[(k0 + k) * 256 + tid] = s;
            }
    }
}

// ---------------------------------------------------------------------------
// the steps: wave w holds the columns 16 w .. of every matrix
// ---------------------------------------------------------------------------
template <int DT>
struct Square {
    static constexpr int D = 16 * DT;
    static constexpr int PITCH = D + (DT > 1 ? 16 : 0);  // rows k, k + 1 on other banks
};

// L . B with L in LDS, transposed (put).  The matrices are symmetric but for rounding, and that
// part must not be transposed from step to step: it then grows (2^-53 to 2^-18 in ten
// steps, against 2^-39).
template <int DT>
__device__ __forceinline__ void times(const double* L, const f64x4 (&B)[DT], f64x4 (&out)[DT]) {
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
#pragma unroll
    for (int t = 0; t < DT; ++t) out[t] = f64x4{0., 0., 0., 0.};
#pragma unroll
    for (int kb = 0; kb < DT; ++kb)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < DT; ++t)
                out[t] = mfma64(L[(16 * kb + 4 * c + h) * Square<DT>::PITCH + 16 * t + p], B[kb][c], out[t]);
}

template <int DT>
__device__ __forceinline__ void put(double* L, const f64x4 (&B)[DT], int wave) {
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) L[(16 * wave + p) * Square<DT>::PITCH + 16 * t + 4 * v + h] = B[t][v];
}

template <int DT>
constexpr int kStepThreads = 64 * DT < NT ? NT : 64 * DT;

template <int DT>
__global__ __launch_bounds__(kStepThreads<DT>) void steps_kernel(Batch batch, double eps, double a, double b, double c, int steps,
                                                                  uint8_t* __restrict__ ws) {
    constexpr int D = Square<DT>::D, PITCH = Square<DT>::PITCH, N = kStepThreads<DT>;
    __shared__ double L[D * PITCH];
    __shared__ double trace[2];
    const Matrix x = batch.m[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, p = lane & 15, h = lane >> 4;
    const double* part = (const double*)(ws + x.scratch);
    const int64_t pieces = pieces_of(x.n);
    for (int e = tid; e < kTiles<DT> * 256; e += N) {
        double s = 0.;
#pragma unroll 8
        for (int64_t q = 0; q < pieces; ++q) s += part[q * (kTiles<DT> * 256) + e];
        int t = 0, k = e >> 8;  // tile k is (t, u)
        while (k >= DT - t) k -= DT - t++;
        const int u = t + k, row = 16 * t + 4 * ((e >> 6) & 3) + ((e >> 4) & 3), col = 16 * u + (e & 15);
        L[row * PITCH + col] = s;
        if (t != u) L[col * PITCH + row] = s;
    }
    __syncthreads();
    if (wave == 0) {
        double s = lane < D ? L[lane * PITCH + lane] : 0.;
        if (D > 64) s += L[(D > 64 ? lane + 64 : 0) * PITCH + (D > 64 ? lane + 64 : 0)];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
        if (lane == 0) trace[0] = s;
    }
    __syncthreads();
    const double inv = 1. / (sqrt(trace[0]) + eps);
    const bool works = wave < DT;
    f64x4 S[DT], P[DT], Q[DT], W[DT];
    if (works) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) S[t][v] = L[(16 * t + 4 * v + h) * PITCH + 16 * wave + p] * inv * inv;
    }
    for (int k = 0; k < steps; ++k) {
        __syncthreads();  // every wave is done with the left operand
        if (works) put<DT>(L, S, wave);
        __syncthreads();
        if (works) {
            times<DT>(L, S, P);
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    P[t][v] = fma(c, P[t][v], fma(b, S[t][v], t == wave && 4 * v + h == p ? a : 0.));
        }
        __syncthreads();
        if (works) put<DT>(L, P, wave);
        __syncthreads();
        if (works) {
            if (k == 0) {
#pragma unroll
                for (int t = 0; t < DT; ++t) Q[t] = P[t];
            } else {
                times<DT>(L, Q, W);
#pragma unroll
                for (int t = 0; t < DT; ++t) Q[t] = W[t];
            }
            if (k + 1 < steps) {
                times<DT>(L, S, W);
                times<DT>(L, W, S);
            }
        }
    }
    double* out = (double*)(ws + x.scratch) + pieces * (kTiles<DT> * 256);
    if (works) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) out[(16 * wave + p) * D + 16 * t + 4 * v + h] = Q[t][v] * inv;
    }
}

// ---------------------------------------------------------------------------
// the direction and the update
// ---------------------------------------------------------------------------

// 64 columns from jb on: lane l holds, of the rows k = 4c + l / 16 of every block, the
// columns 4 (l % 16) + e (wide) or 16 e + l % 16 (tall).  Results come out where the
// operands lay.
template <typename T, typename TP, int DT, bool WIDE>
__device__ __forceinline__ void apply_piece(const Matrix& x, const Rule& rule, int64_t j0, int64_t j1, const double* L) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane & 15, h = lane >> 4;
    const T* grad = (const T*)x.grad;
    for (int64_t jb = j0 + 64 * wave; jb < j1; jb += 64 * (NT / 64)) {
        float v[DT][4][4];  // [block][c][e]
        // where (c, t or e)'s run of elements starts, and how many of it exist
        auto run = [&](int c, int k, int& n) {
            if constexpr (WIDE) {  // k: block; 4 columns
                const int i = 16 * k + 4 * c + h;
                n = i < x.d ? most(j1 - (jb + 4 * p), 4) : 0;
                return n ? (int64_t)i * x.n + jb + 4 * p : 0;
            } else {  // k: e; DT rows
                const int64_t j = jb + 16 * k + p;
                const int i = DT * (4 * c + h);
                n = j < j1 ? most(x.d - i, DT) : 0;
                return n ? j * x.d + i : 0;
            }
        };
        constexpr int K = WIDE ? DT : 4, E = WIDE ? 4 : DT;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                int n;
                const int64_t at = run(c, k, n);
                float g[E], m[E];
                read_some<T, E>(grad + at, n, g);
                if (x.m != nullptr) {
                    read_some<float, E>(x.m + at, n, m);
#pragma unroll
                    for (int e = 0; e < E; ++e) g[e] = rule.direction(m[e], g[e]);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (WIDE) v[k][c][e] = g[e];
                    else v[e][c][k] = g[e];
                }
            }
        constexpr int EG = DT == 8 ? 2 : 4;  // columns sets at a time
#pragma unroll
        for (int e0 = 0; e0 < 4; e0 += EG) {
            f64x4 o[EG][DT];
#pragma unroll
            for (int e = 0; e < EG; ++e)
#pragma unroll
                for (int t = 0; t < DT; ++t) o[e][t] = f64x4{0., 0., 0., 0.};
#pragma unroll
            for (int kb = 0; kb < DT; ++kb)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    double r[EG];
#pragma unroll
                    for (int e = 0; e < EG; ++e) r[e] = (double)v[kb][c][e0 + e];
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const double l = L[(16 * kb + 4 * c + h) * Square<DT>::PITCH + 16 * t + p];
#pragma unroll
                        for (int e = 0; e < EG; ++e) o[e][t] = mfma64(l, r[e], o[e][t]);
                    }
                }
            // the later sets still need their own operands: only these columns change
#pragma unroll
            for (int e = 0; e < EG; ++e)
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[t][c][e0 + e] = (float)o[e][t][c];
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                int n;
                const int64_t at = run(c, k, n);
                float d[E], w[E];
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = v[WIDE ? k : e][c][WIDE ? e : k];
                if (n == 0) continue;
                if (x.master != nullptr) {
                    read_some<float, E>(x.master + at, n, w);
#pragma unroll
                    for (int e = 0; e < E; ++e) w[e] = fmaf(-x.rate, d[e], x.keep * w[e]);
                    write_some<float, E>(x.master + at, n, w);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) w[e] = x.rate * d[e];
                }
                if (x.param != nullptr) write_some<TP, E>((TP*)x.param + at, n, w);
            }
    }
}

template <typename T, typename TP, int DT>
__global__ __launch_bounds__(NT, DT == 8 ? 1 : 2) void apply_kernel(Batch batch, Rule rule, const uint8_t* __restrict__ ws) {
    constexpr int D = Square<DT>::D, PITCH = Square<DT>::PITCH;
    __shared__ double L[D * PITCH];
    const int item = find(batch, (int)blockIdx.x);
    const Matrix x = batch.m[item];
    const int piece = (int)blockIdx.x - batch.first[item];
    const int64_t cols = piece_cols(x.n), j0 = piece * cols, j1 = j0 + cols < x.n ? j0 + cols : x.n;
    const double* Q = (const double*)(ws + x.scratch) + pieces_of(x.n) * (kTiles<DT> * 256);
    for (int e = threadIdx.x; e < D * D; e += NT) L[e / D * PITCH + e % D] = Q[e];
    __syncthreads();
    if (x.wide) apply_piece<T, TP, DT, true>(x, rule, j0, j1, L);
    else apply_piece<T, TP, DT, false>(x, rule, j0, j1, L);
}

int blocks_of(int64_t d) { return d <= 16 ? 1 : d <= 32 ? 2 : d <= 64 ? 4 : 8; }

template <int DT>
hipError_t launch_batch(const UpdateArgs& a, const Batch& b, hipStream_t s) {
    const Rule rule{a.momentum, a.fresh, (int)a.nesterov};
    const dim3 grid((unsigned)b.first[b.count]);
    if (a.grad_bf16) hipLaunchKernelGGL((gram_kernel<uint16_t, DT>), grid, dim3(NT), 0, s, b, rule, a.workspace);
    else hipLaunchKernelGGL((gram_kernel<float, DT>), grid, dim3(NT), 0, s, b, rule, a.workspace);
    hipLaunchKernelGGL((steps_kernel<DT>), dim3(b.count), dim3(kStepThreads<DT>), 0, s, b, a.eps, a.a, a.b, a.c, a.steps, a.workspace);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(NT), 0, s, b, rule, (const uint8_t*)a.workspace); };
    if (a.grad_bf16) {
        if (a.param_bf16) run(apply_kernel<uint16_t, uint16_t, DT>);
        else run(apply_kernel<uint16_t, float, DT>);
    } else {
        if (a.param_bf16) run(apply_kernel<float, uint16_t, DT>);
        else run(apply_kernel<float, float, DT>);
    }
    return hipGetLastError();
}

}  // namespace

int64_t update_scratch(int64_t d, int64_t n) {
    const int64_t dt = blocks_of(d);
    return 8 * (pieces_of(n) * (dt * (dt + 1) / 2 * 256) + 256 * dt * dt);
}

hipError_t launch_update(const UpdateArgs& a, const Matrix* matrices, int64_t count, hipStream_t s) {
    hipError_t e = hipSuccess;
    for (int dt = 1; dt <= 8 && e == hipSuccess; dt *= 2) {
        Batch b{};
        for (int64_t i = 0; i <= count && e == hipSuccess; ++i) {
            const bool fits = i < count && blocks_of(matrices[i].d) == dt;
            if (fits) {
                b.m[b.count] = matrices[i];
                b.first[b.count + 1] = b.first[b.count] + (int)pieces_of(matrices[i].n);
                ++b.count;
            }
            if (b.count == kBatch || (i == count && b.count > 0)) {
                e = dt == 1 ? launch_batch<1>(a, b, s) : dt == 2 ? launch_batch<2>(a, b, s) : dt == 4 ? launch_batch<4>(a, b, s)
                                                                                               : launch_batch<8>(a, b, s);
                b.count = 0;
            }
        }
    }
    return e;
}

}  // namespace block
}  // namespace lors
