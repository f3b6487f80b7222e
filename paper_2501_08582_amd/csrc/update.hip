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
//   sum_kernel     the pieces' sum
//   steps_kernel   one workgroup a matrix: |v| out of the trace, the steps (sides above 64:
//                  start_kernel and product_kernel, a launch for each product)
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
// Bound by memory for many matrices: 10 bytes an element in the first pass (bf16 gradient: it,
// m twice), 16 in the second (it, m, master twice, param).  112 adapters of rank 16 (10
// million elements) take 86 us: 26 in the first pass (3.9 TB/s), 6 + 7 in the sum and the
// steps, 35 in the second pass (4.6 TB/s), 7 for the descriptors.  Of rank 64 (50 million, 452 us): 147 (3.4 TB/s),
// 15, 45, 254 (3.2 TB/s).  One matrix alone is bound by the steps' chain of products: 64 x 14336
// takes 70 us, of which 42 are the steps' 17 products of 64 x 64 (4096 cycles of one
// compute unit's matrix cores each: 29 us).
#include <type_traits>

#include "block_kernels.hpp"
#include "train_common.hpp"

namespace lors {
namespace block {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;
constexpr int kBatch = 48;        // matrices whose descriptors are kernel arguments
constexpr int kPiece = 256;       // least columns (along the long side) of a workgroup
constexpr int kMostPieces = 256;
constexpr int kNarrow = 96;       // at most as many pieces of the second pass in a launch take a quarter of their columns a turn

struct Batch {
    int count;
    int first[kBatch];  // first workgroup of each matrix
    Matrix m[kBatch];
};

// The matrices of a launch: a batch, or more of them in the workspace (table_kernel).
struct Table {
    int* first;
    Matrix* m;
};
struct Source {
    Table table;
    int count;
    bool many;
    Batch batch;
};

__host__ __device__ inline int64_t piece_cols(int64_t n) {
    const int64_t most = (n + kMostPieces - 1) / kMostPieces;
    const int64_t c = (most + 255) / 256 * 256;  // turns of 64 columns of four waves
    return c < kPiece ? kPiece : c;
}
__host__ __device__ inline int64_t pieces_of(int64_t n) { return (n + piece_cols(n) - 1) / piece_cols(n); }

// D(16x16) += A(16x4) . B(4x16): lane l holds A[l % 16][l / 16], B[l / 16][l % 16].
__device__ __forceinline__ f64x4 mfma64(double a, double b, f64x4 c) {
    return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0);
}

// Pointers out of a descriptor: the compiler is told that they are to global memory (it
// would use flat accesses, which wait for LDS operations too).
#ifdef __HIP_DEVICE_COMPILE__
#define LORS_GLOBAL __attribute__((address_space(1)))
#else
#define LORS_GLOBAL
#endif
template <typename T>
using Global = LORS_GLOBAL T*;

// Where a run of elements starts: FULL ones at an element that the whole wave shares and 32 bits
// of a lane's own (one register for all runs of a turn), others anywhere.
struct Place {
    int64_t base;
    uint32_t lane;
};
template <typename T>
__device__ __forceinline__ Global<T> at_place(T* p, const Place& at) {
    return (Global<T>)((LORS_GLOBAL char*)(Global<T>)(p + at.base) + (uint64_t)(at.lane * (uint32_t)sizeof(T)));
}

// The first n of N elements at p as fp32, the others 0.
template <typename T, int N>
__device__ __forceinline__ void read_some(Global<const T> p, int n, float (&f)[N]) {
    if (n >= N) {
        const train::Packed<T, N> v = *(Global<const train::Packed<T, N>>)p;
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
__device__ __forceinline__ void write_some(Global<T> p, int n, const float (&f)[N]) {
    train::Packed<T, N> v;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) v.v[e] = bf16_bits(f[e]);
        else v.v[e] = f[e];
    }
    if (n >= N) {
        *(Global<train::Packed<T, N>>)p = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < n) p[e] = v.v[e];
}

__device__ __forceinline__ int most(int64_t left, int n) { return left >= n ? n : left > 0 ? (int)left : 0; }

// Matrix of this workgroup, and the workgroup's number in it.
__device__ __forceinline__ int find(const int* first, int count, int block) {
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// A workgroup's descriptor, which all lanes load alike, into scalar registers.
__device__ __forceinline__ Matrix uniform(const Matrix& x) {
    uint32_t w[sizeof(Matrix) / 4];
    __builtin_memcpy(w, &x, sizeof(Matrix));
#pragma unroll
    for (uint32_t& e : w) e = __builtin_amdgcn_readfirstlane(e);
    Matrix out;
    __builtin_memcpy(&out, w, sizeof(Matrix));
    return out;
}
__device__ __forceinline__ Matrix matrix_of(const Source& s, int block, int& piece) {
    if (s.many) {
        const int i = find(s.table.first, s.count, block);
        piece = __builtin_amdgcn_readfirstlane(block - s.table.first[i]);
        return uniform(s.table.m[i]);
    }
    const int i = find(s.batch.first, s.count, block);
    piece = block - s.batch.first[i];
    return s.batch.m[i];
}
__device__ __forceinline__ Matrix matrix_at(const Source& s, int i) { return uniform(s.many ? s.table.m[i] : s.batch.m[i]); }

struct Rule {
    float beta, fresh;
    int nesterov, grad_bf16, param_bf16;
    // m <- beta m + fresh g, and v.  The second pass forms v from the m that the first
    // one stored, by the same operations: the same bits.
    __device__ __forceinline__ float moment(float m, float g) const { return fmaf(beta, m, fresh * g); }
    __device__ __forceinline__ float direction(float m, float g) const { return nesterov ? fmaf(beta, m, fresh * g) : m; }
};

// DT: 16-row blocks of the short side.  Row p = 4c + h of block t is the short index i = 16 t + p of a
// wide matrix and 4 DT h + DT c + t of a tall one: there a lane of the second pass (h its
// row of 16 lanes) holds 4 DT consecutive elements, one of the first pass DT.  The
// steps work on rows in the order (t, p), whatever that is.
template <int DT>
constexpr int kTiles = DT * (DT + 1) / 2;
// Columns of a lane in a turn of the first pass (the widest short side has registers for four).
template <int DT>
constexpr int kEach = DT >= 6 ? 4 : 8;
// The widest short side's 36 tiles are more than a wave's accumulators: there two waves read the
// same columns, wave w takes the tiles of w's parity, and the even one stores m, once
// both have read it.  (All 36 in one wave: 377 registers spilled; 128 x 4096 in
// 96 us, against 29.)
template <int DT>
constexpr int kShare = DT == 8 ? 2 : 1;
template <int DT>
constexpr int kOwn = kTiles<DT> / kShare<DT>;

// FULL: the turn's columns exist and rows are read in whole vectors (read_whole): every
// lane loads, from the last row that exists where its own does not, and takes 0 instead.
// Without branches around them all loads of a turn are in flight together.
template <typename T, int N>
__device__ __forceinline__ void read_whole(Global<const T> p, bool some, float (&f)[N]) {
    const train::Packed<T, N> v = *(Global<const train::Packed<T, N>>)p;
    if constexpr (sizeof(T) * N == 2) {
        // (else the load writes the upper half of a register, and waits for what it held)
        uint32_t w = v.v[0];
        asm("" : "+v"(w));
        f[0] = some ? bf16_bits_to_f32(w) : 0.f;
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) f[e] = some ? bf16_bits_to_f32(v.v[e]) : 0.f;
        else f[e] = some ? v.v[e] : 0.f;
    }
}
// The gradient's, of either type.
template <int N, bool FULL>
__device__ __forceinline__ void read_grad(const void* p, bool bf16, const Place& at, int n, float (&f)[N]) {
    if (bf16) {
        if constexpr (FULL) read_whole<uint16_t, N>(at_place((const uint16_t*)p, at), n > 0, f);
        else read_some<uint16_t, N>(at_place((const uint16_t*)p, at), n, f);
    } else {
        if constexpr (FULL) read_whole<float, N>(at_place((const float*)p, at), n > 0, f);
        else read_some<float, N>(at_place((const float*)p, at), n, f);
    }
}

template <int DT, bool WIDE, bool FULL>
__device__ __forceinline__ void gram_turn(const Matrix& x, const Rule& rule, int64_t jb, int64_t j1, f64x4 (&acc)[kOwn<DT>]) {
    const int part = kShare<DT> == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kShare<DT>;
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
    // run k of a lane: where it starts and how many of its elements exist
    constexpr int N = kEach<DT>, K = WIDE ? DT : N, E = WIDE ? N : DT;
    auto run = [&](int k, int& n) -> Place {
        if constexpr (WIDE) {  // k: block; N columns
            const int i = 16 * k + p;
            const int64_t j = jb + N * h;
            n = i < x.d ? (FULL ? N : most(j1 - j, N)) : 0;
            if (FULL) return {(16 * k < x.d ? 16 * k * x.n : 0) + jb, (i < x.d ? (uint32_t)(p * x.n) : 0u) + N * h};
            return {n ? (int64_t)i * x.n + j : 0, 0};
        } else {  // k: column; DT rows
            const int64_t j = jb + 4 * k + h;
            const int i = 4 * DT * (p & 3) + DT * (p >> 2);
            n = FULL ? (i < x.d ? DT : 0) : j < j1 ? most(x.d - i, DT) : 0;
            if (FULL) return {(jb + 4 * k) * x.d, (uint32_t)(h * x.d + (i < x.d ? i : 0))};
            return {n ? j * x.d + i : 0, 0};
        }
    };
    // (the branches on what a matrix has stand around whole loops of loads, not inside)
    float g[K][E];
    auto gradients = [&](bool bf16) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int n;
            const Place at = run(k, n);
            read_grad<E, FULL>(x.grad, bf16, at, n, g[k]);
        }
    };
    if (rule.grad_bf16) gradients(true);
    else gradients(false);
    if (x.m != nullptr) {
        float m[K][E];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int n;
            const Place at = run(k, n);
            if constexpr (FULL) read_whole<float, E>(at_place(x.m, at), n > 0, m[k]);
            else read_some<float, E>(at_place(x.m, at), n, m[k]);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                m[k][e] = rule.moment(m[k][e], g[k][e]);
                g[k][e] = rule.direction(m[k][e], g[k][e]);
            }
        if constexpr (kShare<DT> > 1) {  // the other wave has its m
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        }
        if (part == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                int n;
                const Place at = run(k, n);
                if (n > 0) write_some<float, E>(at_place(x.m, at), FULL ? E : n, m[k]);
            }
    }
    auto products = [&](auto part_tag) {
        constexpr int PART = decltype(part_tag)::value;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            double v[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) v[t] = (double)g[WIDE ? t : e][WIDE ? e : t];
            int k = 0;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int u = t; u < DT; ++u, ++k)
                    if (k % kShare<DT> == PART) acc[k / kShare<DT>] = mfma64(v[t], v[u], acc[k / kShare<DT>]);
        }
    };
    if (part == 0) products(std::integral_constant<int, 0>{});
    else products(std::integral_constant<int, kShare<DT> - 1>{});
}

// v of 4 N columns a turn: lane l holds, of row l % 16 of every block, the columns N (l / 16) + e
// (wide) or 4 e + l / 16 (tall); any assignment does that is the same for every row.
template <int DT, bool WIDE>
__device__ __forceinline__ void gram_piece(const Matrix& x, const Rule& rule, int64_t j0, int64_t j1, f64x4 (&acc)[kOwn<DT>]) {
    const bool whole = WIDE ? x.n < (int64_t)1 << 26 : x.d % DT == 0;  // (a lane's own offset fits 32 bits)
    constexpr int C = 4 * kEach<DT>;
    constexpr int SETS = NT / 64 / kShare<DT>;  // turns at a time; where they hold a barrier, all waves take as many
    const int set = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kShare<DT>;
#pragma unroll 1
    for (int64_t ja = j0; ja < j1; ja += C * SETS) {
        const int64_t jb = ja + C * set;
        if (kShare<DT> == 1 && jb >= j1) break;
        if (whole && jb + C <= j1) gram_turn<DT, WIDE, true>(x, rule, jb, j1, acc);
        else gram_turn<DT, WIDE, false>(x, rule, jb, j1, acc);
    }
}

template <int DT>
__global__ __launch_bounds__(NT, DT >= 6 ? 1 : 2) void gram_kernel(Source src, Rule rule, uint8_t* __restrict__ ws) {
    constexpr int G = kOwn<DT> < 8 ? kOwn<DT> : 8;  // tiles joined at a time
    constexpr int SHARE = kShare<DT>;
    __shared__ double red[NT / 64][G][256];
    int piece;
    const Matrix x = matrix_of(src, (int)blockIdx.x, piece);
    const int64_t cols = piece_cols(x.n), j0 = piece * cols, j1 = j0 + cols < x.n ? j0 + cols : x.n;
    f64x4 acc[kOwn<DT>];
#pragma unroll
    for (int k = 0; k < kOwn<DT>; ++k) acc[k] = f64x4{0., 0., 0., 0.};
    if (x.wide) gram_piece<DT, true>(x, rule, j0, j1, acc);
    else gram_piece<DT, false>(x, rule, j0, j1, acc);
    // the waves' sums, in wave order
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double* out = (double*)(ws + x.scratch) + (int64_t)piece * (kTiles<DT> * 256);
#pragma unroll
    for (int k0 = 0; k0 < kOwn<DT>; k0 += G) {
        if (k0 > 0) __syncthreads();
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (k0 + k < kOwn<DT>)
#pragma unroll
                for (int v = 0; v < 4; ++v) red[wave][k][64 * v + lane] = acc[k0 + k < kOwn<DT> ? k0 + k : 0][v];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (k0 + k < kOwn<DT>)
#pragma unroll
                for (int q = 0; q < SHARE; ++q) {
                    double s = red[q][k][tid];
#pragma unroll
                    for (int w = q + SHARE; w < NT / 64; w += SHARE) s += red[w][k][tid];
                    out[(SHARE * (k0 + k) + q) * 256 + tid] = s;
                }
    }
}

// The pieces' sum, in their order, into the first piece's place: one entry a thread.
__global__ __launch_bounds__(NT) void sum_kernel(Source src, int entries, uint8_t* __restrict__ ws) {
    const Matrix x = matrix_at(src, (int)blockIdx.x);
    const int e = blockIdx.y * NT + threadIdx.x;
    double* part = (double*)(ws + x.scratch) + e;
    const int64_t pieces = pieces_of(x.n);
    if (pieces == 1) return;
    double s = 0.;
#pragma unroll 16
    for (int64_t q = 0; q < pieces; ++q) s += part[q * entries];
    part[0] = s;
}

// ---------------------------------------------------------------------------
// the steps: wave w holds the columns 16 w .. of every matrix
// ---------------------------------------------------------------------------
template <int DT>
struct Square {
    static constexpr int D = 16 * DT;
    static constexpr int PITCH = D + (DT % 2 == 0 ? 16 : 0);  // rows k, k + 1 on other banks
    // Element (row, col) of a left operand in LDS: the 16 columns of a tile in the order that
    // the row's number gives, so that the writes of 16 rows' column (put) fall on 16 places as the
    // reads of a row do.  (In one order for all rows the writes met on one bank: 4200 cycles at 64 x
    // 64, as long as a product.)
    static __device__ __forceinline__ int at(int row, int col) { return row * PITCH + (col ^ (row & 15)); }
};

// L . B with L in LDS, transposed (put).  The matrices are symmetric but for rounding, and that
// part must not be transposed from step to step: it then grows (2^-53 to 2^-18 in ten
// steps, against 2^-39).
template <int DT>
__device__ __forceinline__ void read_left(const double* L, int group, double (&l)[DT]) {
    const int lane = threadIdx.x & 63;
    const double* row = L + Square<DT>::at(4 * group + (lane >> 4), lane & 15);
#pragma unroll
    for (int t = 0; t < DT; ++t) l[t] = row[16 * t];
}
// The same of a matrix that stands in LDS row by row (apply_kernel, whose copy is written so).
template <int DT>
__device__ __forceinline__ void read_plain(const double* L, int group, double (&l)[DT]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < DT; ++t) l[t] = L[(4 * group + (lane >> 4)) * Square<DT>::PITCH + 16 * t + (lane & 15)];
}
// (The left operands of four columns of L are read while the products of the four before run; the
// barriers keep the compiler from reading all of L ahead, for which there are no registers.)
template <int DT>
__device__ __forceinline__ void times(const double* L, const f64x4 (&B)[DT], f64x4 (&out)[DT]) {
    double l[2][DT];
    read_left<DT>(L, 0, l[0]);
#pragma unroll
    for (int t = 0; t < DT; ++t) out[t] = f64x4{0., 0., 0., 0.};
#pragma unroll
    for (int g = 0; g < 4 * DT; ++g) {
        if (g + 1 < 4 * DT) read_left<DT>(L, g + 1, l[(g + 1) & 1]);
#pragma unroll
        for (int t = 0; t < DT; ++t) out[t] = mfma64(l[g & 1][t], B[g >> 2][g & 3], out[t]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int DT>
__device__ __forceinline__ void put(double* L, const f64x4 (&B)[DT], int wave) {
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) L[Square<DT>::at(16 * wave + p, 16 * t + 4 * v + h)] = B[t][v];
}


template <int DT>
__global__ __launch_bounds__(NT) void steps_kernel(Source src, double eps, double a, double b, double c, int steps,
                                                                  uint8_t* __restrict__ ws) {
    using Left = Square<DT>;
    constexpr int D = Left::D, N = NT;
    __shared__ double L[D * Left::PITCH];
    __shared__ double trace[2];
    const Matrix x = matrix_at(src, (int)blockIdx.x);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, p = lane & 15, h = lane >> 4;
    const double* part = (const double*)(ws + x.scratch);
    const int64_t pieces = pieces_of(x.n);
    for (int e = tid; e < kTiles<DT> * 256; e += N) {
        const double s = part[e];
        int t = 0, k = e >> 8;  // tile k is (t, u)
        while (k >= DT - t) k -= DT - t++;
        const int u = t + k, row = 16 * t + 4 * ((e >> 6) & 3) + ((e >> 4) & 3), col = 16 * u + (e & 15);
        L[Left::at(row, col)] = s;
        if (t != u) L[Left::at(col, row)] = s;
    }
    __syncthreads();
    if (wave == 0) {
        double s = lane < D ? L[Left::at(lane, lane)] : 0.;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
        if (lane == 0) trace[0] = s;
    }
    __syncthreads();
    const double inv = 1. / (sqrt(trace[0]) + eps);
    const bool works = wave < DT;
    double* out = (double*)(ws + x.scratch) + pieces * (kTiles<DT> * 256);
    f64x4 S[DT], Q[DT], W[DT];
    if (works) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) S[t][v] = L[Left::at(16 * t + 4 * v + h, 16 * wave + p)] * inv * inv;
    }
    for (int k = 0; k < steps; ++k) {
        __syncthreads();  // every wave is done with the left operand
        if (works) put<DT>(L, S, wave);
        __syncthreads();
        if (works) {  // W = P
            times<DT>(L, S, W);
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    W[t][v] = fma(c, W[t][v], fma(b, S[t][v], t == wave && 4 * v + h == p ? a : 0.));
        }
        __syncthreads();
        if (works) {
            put<DT>(L, W, wave);
            if (k == 0)
#pragma unroll
                for (int t = 0; t < DT; ++t) Q[t] = W[t];
        }
        __syncthreads();
        if (works) {
            if (k > 0) {
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

// 16 EC columns from jb on: lane l holds, of the rows p = 4c + l / 16 of every block, the
// columns EC (l % 16) + e (wide) or 16 e + l % 16 (tall).  Results come out where the
// operands lay.  FULL as above; where there are registers for them (AHEAD), the
// master's values are on their way during the products.
template <int DT, bool WIDE, bool FULL, int EC>
__device__ __forceinline__ void apply_turn(const Matrix& x, const Rule& rule, int64_t jb, int64_t j1, const double* L) {
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
    float v[DT][4][EC];  // [block][c][e]
    // runs of E consecutive elements: (block k, c) over e, or column e = k over c and the block
    constexpr int K = WIDE ? 4 * DT : EC, E = WIDE ? EC : 4 * DT;
    auto run = [&](int k, int& n) -> Place {
        if constexpr (WIDE) {
            const int i0 = 16 * (k >> 2) + 4 * (k & 3), i = i0 + h;
            const int64_t j = jb + EC * p;
            n = i < x.d ? (FULL ? EC : most(j1 - j, EC)) : 0;
            if (FULL) return {(i0 < x.d ? i0 * x.n : 0) + jb, (uint32_t)(h * x.n) + EC * p};
            return {n ? (int64_t)i * x.n + j : 0, 0};
        } else {
            const int64_t j = jb + 16 * k + p;
            const int i = 4 * DT * h;
            n = FULL ? (i < x.d ? E : 0) : j < j1 ? most(x.d - i, E) : 0;
            if (FULL) return {(jb + 16 * k) * x.d, (uint32_t)(p * x.d + (i < x.d ? i : 0))};
            return {n ? j * x.d + i : 0, 0};
        }
    };
    auto value = [&](int k, int e) -> float& {
        if constexpr (WIDE) return v[k >> 2][k & 3][e];
        else return v[e % DT][e / DT][k];
    };
    auto gradients = [&](bool bf16) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int n;
            const Place at = run(k, n);
            float g[E];
            read_grad<E, FULL>(x.grad, bf16, at, n, g);
#pragma unroll
            for (int e = 0; e < E; ++e) value(k, e) = g[e];
        }
    };
    if (rule.grad_bf16) gradients(true);
    else gradients(false);
    if (x.m != nullptr)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int n;
            const Place at = run(k, n);
            float m[E];
            if constexpr (FULL) read_whole<float, E>(at_place(x.m, at), n > 0, m);
            else read_some<float, E>(at_place(x.m, at), n, m);
#pragma unroll
            for (int e = 0; e < E; ++e) value(k, e) = rule.direction(m[e], value(k, e));
        }
    constexpr bool AHEAD = FULL && DT < 4;
    float old[AHEAD ? K : 1][E];
    if constexpr (AHEAD)
        if (x.master != nullptr)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                int n;
                const Place at = run(k, n);
                read_whole<float, E>(at_place(x.master, at), true, old[k]);
            }
    constexpr int EG = EC == 1 || DT >= 6 ? 1 : DT >= 3 ? 2 : 4;  // sets of columns at a time, for the registers
#pragma unroll
    for (int e0 = 0; e0 < EC; e0 += EG) {
        f64x4 o[EG][DT];
#pragma unroll
        for (int e = 0; e < EG; ++e)
#pragma unroll
            for (int t = 0; t < DT; ++t) o[e][t] = f64x4{0., 0., 0., 0.};
        double l[2][DT];
        read_plain<DT>(L, 0, l[0]);
#pragma unroll
        for (int g = 0; g < 4 * DT; ++g) {
            if (g + 1 < 4 * DT) read_plain<DT>(L, g + 1, l[(g + 1) & 1]);
            double r[EG];
#pragma unroll
            for (int e = 0; e < EG; ++e) r[e] = (double)v[g >> 2][g & 3][e0 + e];
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < EG; ++e) o[e][t] = mfma64(l[g & 1][t], r[e], o[e][t]);
            __builtin_amdgcn_sched_barrier(0);
        }
        // (the other sets need their own columns only)
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
        for (int e = 0; e < E; ++e) value(k, e) *= x.rate;
    if (x.master != nullptr) {
        constexpr int RUNS = WIDE ? 4 : EC == 1 || DT >= 6 ? 1 : 2;  // runs of the master in flight
#pragma unroll
        for (int k0 = 0; k0 < K; k0 += RUNS) {
            float before[RUNS][E];
#pragma unroll
            for (int q = 0; q < RUNS; ++q) {
                int n;
                const Place at = run(k0 + q, n);
                if constexpr (AHEAD) {
#pragma unroll
                    for (int e = 0; e < E; ++e) before[q][e] = old[AHEAD ? k0 + q : 0][e];
                } else if constexpr (FULL) {
                    read_whole<float, E>(at_place(x.master, at), true, before[q]);
                } else {
                    read_some<float, E>(at_place(x.master, at), n, before[q]);
                }
            }
#pragma unroll
            for (int q = 0; q < RUNS; ++q) {
                int n;
                const Place at = run(k0 + q, n);
                float w[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    w[e] = fmaf(x.keep, before[q][e], -value(k0 + q, e));
                    value(k0 + q, e) = w[e];
                }
                if (n > 0) write_some<float, E>(at_place(x.master, at), FULL ? E : n, w);
            }
        }
    }
    auto params = [&](auto* to) {
        using TP = std::remove_pointer_t<decltype(to)>;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int n;
            const Place at = run(k, n);
            float w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = value(k, e);
            if (n > 0) write_some<TP, E>(at_place(to, at), FULL ? E : n, w);
        }
    };
    if (x.param != nullptr) {
        if (rule.param_bf16) params((uint16_t*)x.param);
        else params((float*)x.param);
    }
}

// Whether the whole turns of a matrix are FULL ones: rows four by four (tall: vectors of 4 DT) exist or do
// not, and a lane's own offset fits 32 bits.  All else are edges, which another launch takes.
__host__ __device__ inline bool whole_rows(bool wide, int64_t d, int64_t n, int dt) {
    return wide ? d % 4 == 0 && n < (int64_t)1 << 26 : d % (4 * dt) == 0;
}

template <int DT, bool WIDE, bool FULL, int EC>
__global__ __launch_bounds__(NT, DT >= 6 ? 1 : 2) void apply_kernel(Source src, Rule rule, int64_t cols, const uint8_t* __restrict__ ws) {
    constexpr int D = Square<DT>::D, PITCH = Square<DT>::PITCH;
    __shared__ __attribute__((aligned(16))) double L[D * PITCH];
    int piece;
    const Matrix x = matrix_of(src, (int)blockIdx.x, piece);
    const int64_t end = FULL ? x.n / 64 * 64 : x.n;
    int64_t j0 = piece * cols;
    if (!FULL && whole_rows(WIDE, x.d, x.n, DT)) j0 += x.n / 64 * 64;
    const int64_t j1 = j0 + cols < end ? j0 + cols : end;
    const double* Q = (const double*)(ws + x.scratch) + pieces_of(x.n) * (kTiles<DT> * 256);
    typedef double f64x2 __attribute__((ext_vector_type(2)));
    for (int e = 2 * threadIdx.x; e < D * D; e += 2 * NT) *(f64x2*)(L + e / D * PITCH + e % D) = *(const f64x2*)(Q + e);
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll 1
    for (int64_t jb = j0 + 16 * EC * wave; jb < j1; jb += 16 * EC * (NT / 64))
        apply_turn<DT, WIDE, FULL, EC>(x, rule, jb, j1, L);
}

int blocks_of(int64_t d) { return d <= 16 ? 1 : d <= 32 ? 2 : d <= 48 ? 3 : d <= 64 ? 4 : d <= 96 ? 6 : 8; }

// The steps of sides above 64, whose products are 8 to 14 us of one compute unit's: each of
// them a launch in which a wave takes a tile of the result, and the matrices in the
// workspace.  P is a left operand alone and kept transposed, S in both forms, so that every
// operand is read in rows of 16 doubles.  14 launches of 6 us in place of one of 333 for the five
// steps; 128 x 4096 takes 141 us in place of 395.
template <int DT>
struct Wide {
    static constexpr int D = 16 * DT;
    double *q, *spare, *s, *st, *pt, *w, *inv;  // q: what apply_kernel reads
    __device__ __forceinline__ Wide(uint8_t* ws, const Matrix& x) {
        q = (double*)(ws + x.scratch) + pieces_of(x.n) * (kTiles<DT> * 256);
        spare = q + D * D;
        s = spare + D * D;
        st = s + D * D;
        pt = st + D * D;
        w = pt + D * D;
        inv = w + D * D;
    }
};

// S_0 out of the pieces' sum (tiles (t, u), t <= u, of 16 x 16 each).
template <int DT>
__global__ __launch_bounds__(NT) void start_kernel(Source src, double eps, uint8_t* __restrict__ ws) {
    constexpr int D = 16 * DT;
    const Matrix x = matrix_at(src, (int)blockIdx.x / DT);
    const int panel = blockIdx.x % DT, tid = threadIdx.x, lane = tid & 63;
    const Wide<DT> m(ws, x);
    const double* part = (const double*)(ws + x.scratch);
    auto entry = [&](int row, int col) {
        const int i = row < col ? row : col, j = row < col ? col : row, t = i >> 4, u = j >> 4;
        const int k = t * DT - t * (t - 1) / 2 + u - t;
        // (within a diagonal tile the two halves differ by rounding alone: the upper one)
        return part[256 * k + 16 * (i & 15) + (j & 15)];
    };
    double trace = entry(lane, lane);
    if (lane + 64 < D) trace += entry(lane + 64, lane + 64);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) trace += __shfl_xor(trace, o);
    const double inv = 1. / (sqrt(trace) + eps);
    for (int e = tid; e < D * 16; e += NT) {
        const int row = e >> 4, col = 16 * panel + (e & 15);
        const double v = entry(row, col) * inv * inv;
        m.s[row * D + col] = v;
        m.st[row * D + col] = v;
    }
    if (panel == 0 && tid == 0) *m.inv = inv;
}

// Part of a step: 0  P = a I + b S + c S^2 (of the first step also Q), 1  Q <- P Q, or W = P S in
// workgroups from `split` on, 2  S <- P W.  The last step's Q is divided by |v| and stands
// transposed, a left operand's way.
struct Step {
    int part, first, last, split, odd;  // odd: Q comes from q and goes to spare
    double a, b, c;
};
template <int DT>
constexpr int kParts = DT * ((DT + 3) / 4);  // workgroups of a product: 16 columns and up to four tiles of rows each
template <int DT>
__global__ __launch_bounds__(NT) void product_kernel(Source src, Step step, uint8_t* __restrict__ ws) {
    constexpr int D = 16 * DT;
    int id = blockIdx.x;
    const bool second = step.part == 1 && id >= step.split;
    if (second) id -= step.split;
    const Matrix x = matrix_at(src, id / kParts<DT>);
    id %= kParts<DT>;
    const Wide<DT> m(ws, x);
    const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = 16 * (id % DT) + p, t = 4 * (id / DT) + wave;
    if (t >= DT) return;
    double* const from = step.odd ? m.q : m.spare;
    double* const to = step.odd ? m.spare : m.q;
    const double* left = (step.part == 0 ? m.st : m.pt) + 16 * t + p;
    const double* right = (step.part == 0 || second ? m.s : step.part == 1 ? from : m.w) + col;
    double l[4 * DT], r[4 * DT];
#pragma unroll
    for (int g = 0; g < 4 * DT; ++g) {
        l[g] = left[(4 * g + h) * D];
        r[g] = right[(4 * g + h) * D];
    }
    const double inv = step.last ? *m.inv : 1.;
    __builtin_amdgcn_sched_barrier(0);  // all loads in flight together
    f64x4 acc = {0., 0., 0., 0.}, other = {0., 0., 0., 0.};  // two chains, each product waits for its own
#pragma unroll
    for (int g = 0; g < 4 * DT; g += 2) {
        acc = mfma64(l[g], r[g], acc);
        other = mfma64(l[g + 1], r[g + 1], other);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int row = 16 * t + 4 * v + h;
        double y = acc[v] + other[v];
        if (step.part == 0) {
            y = fma(step.c, y, fma(step.b, right[row * D], row == col ? step.a : 0.));
            m.pt[col * D + row] = y;
            if (step.first) to[step.last ? col * D + row : row * D + col] = y * inv;
        } else if (step.part == 1) {
            if (second) m.w[row * D + col] = y;
            else to[step.last ? col * D + row : row * D + col] = y * inv;
        } else {
            m.s[row * D + col] = y;
            m.st[col * D + row] = y;
        }
    }
}

template <int DT>
void launch_steps(const UpdateArgs& a, const Source& src, hipStream_t s) {
    if constexpr (DT <= 4) {
        hipLaunchKernelGGL((steps_kernel<DT>), dim3(src.count), dim3(NT), 0, s, src, a.eps, a.a, a.b, a.c, a.steps, a.workspace);
    } else {
        const int panels = src.count * kParts<DT>;
        hipLaunchKernelGGL((start_kernel<DT>), dim3(src.count * DT), dim3(NT), 0, s, src, a.eps, a.workspace);
        for (int k = 0; k < a.steps; ++k) {
            const bool first = k == 0, last = k + 1 == a.steps;
            // Q after the last step stands in q, after the one before it in spare
            Step step{0, first, last, first ? 0 : panels, (a.steps - 1 - k) % 2, a.a, a.b, a.c};
            hipLaunchKernelGGL((product_kernel<DT>), dim3(panels), dim3(NT), 0, s, src, step, a.workspace);
            step.part = 1;
            const int products = (first ? 0 : 1) + (last ? 0 : 1);
            if (products > 0) hipLaunchKernelGGL((product_kernel<DT>), dim3(products * panels), dim3(NT), 0, s, src, step, a.workspace);
            step.part = 2;
            if (!last) hipLaunchKernelGGL((product_kernel<DT>), dim3(panels), dim3(NT), 0, s, src, step, a.workspace);
        }
    }
}

// The launches over one size's matrices: 0 the first pass, 1 + 2 (tall) + (edges) the second's.
constexpr int kLaunches = 5;
struct Plan {
    int64_t cols[kLaunches];  // columns of a workgroup
};
// Columns that a launch takes of a matrix, and its workgroups there.
template <int DT>
__host__ __device__ inline int64_t cols_in(const Matrix& x, int launch) {
    if (launch == 0) return x.n;
    const bool wide = launch <= 2, full = launch % 2 == 1;
    if ((x.wide != 0) != wide) return 0;
    const bool whole = whole_rows(wide, x.d, x.n, DT);
    return full ? (whole ? x.n / 64 * 64 : 0) : whole ? x.n % 64 : x.n;
}
template <int DT>
__host__ __device__ inline int blocks_in(const Matrix& x, int launch, const Plan& plan) {
    if (launch == 0) return (int)pieces_of(x.n);
    return (int)((cols_in<DT>(x, launch) + plan.cols[launch] - 1) / plan.cols[launch]);
}

// The descriptors of more matrices than a batch holds go to the workspace, one wave for 60
// of them, with every launch's first workgroups.
constexpr int kUpload = 60;
struct Upload {
    int count, at, total;
    int base[kLaunches];
    Matrix m[kUpload];
};
static_assert(sizeof(Upload) + sizeof(Plan) + sizeof(Table) <= 4096, "kernel arguments");
template <int DT>
__global__ __launch_bounds__(64) void table_kernel(Upload u, Plan plan, Table t) {
    const int i = threadIdx.x;
    const bool have = i < u.count;
    const Matrix x = u.m[have ? i : 0];
    if (have) t.m[u.at + i] = x;
#pragma unroll
    for (int l = 0; l < kLaunches; ++l) {
        const int own = have ? blocks_in<DT>(x, l, plan) : 0;
        int upto = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o);
            if (i >= o) upto += y;
        }
        if (have) t.first[(int64_t)l * u.total + u.at + i] = u.base[l] + upto - own;
    }
}

// The matrices of one size of the short side.
template <int DT>
hipError_t launch_size(const UpdateArgs& a, const Matrix* matrices, int64_t count, Table table, hipStream_t s) {
    const Rule rule{a.momentum, a.fresh, (int)a.nesterov, (int)a.grad_bf16, (int)a.param_bf16};
    auto mine = [](const Matrix& x) { return blocks_of(x.d) == DT; };
    int total = 0;
    int64_t turns[kLaunches] = {};
    for (int64_t i = 0; i < count; ++i) {
        if (!mine(matrices[i])) continue;
        ++total;
        for (int l = 1; l < kLaunches; ++l) turns[l] += (cols_in<DT>(matrices[i], l) + kPiece - 1) / kPiece;
    }
    if (total == 0) return hipSuccess;
    // Columns of a workgroup of the second pass: its copy of Q is worth several turns of them where
    // there are workgroups enough; where they are few, a quarter of the columns a lane, since
    // a turn's products are 7 us at side 64 (64 x 14336: 11.2 us against 16.5).
    Plan plan{};
    bool narrow[kLaunches] = {};
    for (int l = 1; l < kLaunches; ++l) {
        narrow[l] = turns[l] <= kNarrow;
        if (narrow[l]) {
            plan.cols[l] = kPiece / 4;
            continue;
        }
        int64_t each = turns[l] / 512;
        each = each < 1 ? 1 : each > 8 ? 8 : each;
        while (turns[l] / each + count > (int64_t)1 << 23) each *= 2;  // (a grid's threads are counted in 32 bits)
        plan.cols[l] = each * kPiece;
    }
    Source src[kLaunches] = {};
    int blocks[kLaunches] = {};
    const bool many = total > kBatch;
    Upload u{};
    u.total = total;
    for (int64_t i = 0, at = 0; i < count; ++i) {
        if (!mine(matrices[i])) continue;
        if (many) u.m[u.count++] = matrices[i];
        for (int l = 0; l < kLaunches; ++l) {
            if (!many) {
                src[l].batch.m[at] = matrices[i];
                src[l].batch.first[at] = blocks[l];
            }
            blocks[l] += blocks_in<DT>(matrices[i], l, plan);
        }
        ++at;
        if (many && (u.count == kUpload || at == total)) {
            u.at = (int)at - u.count;
            hipLaunchKernelGGL((table_kernel<DT>), dim3(1), dim3(64), 0, s, u, plan, table);
            for (int l = 0; l < kLaunches; ++l) u.base[l] = blocks[l];
            u.count = 0;
        }
    }
    for (int l = 0; l < kLaunches; ++l) {
        src[l].table = Table{table.first + (many ? (int64_t)l * total : 0), table.m};
        src[l].count = total;
        src[l].many = many;
    }
    hipLaunchKernelGGL((gram_kernel<DT>), dim3(blocks[0]), dim3(NT), 0, s, src[0], rule, a.workspace);
    hipLaunchKernelGGL(sum_kernel, dim3(total, kTiles<DT>), dim3(NT), 0, s, src[0], kTiles<DT> * 256, a.workspace);
    launch_steps<DT>(a, src[0], s);
    auto apply = [&](int l, auto wide_tag, auto full_tag) {
        constexpr bool WIDE = decltype(wide_tag)::value, FULL = decltype(full_tag)::value;
        if (blocks[l] > 0 && narrow[l])
            hipLaunchKernelGGL((apply_kernel<DT, WIDE, FULL, 1>), dim3(blocks[l]), dim3(NT), 0, s, src[l], rule, plan.cols[l],
                               (const uint8_t*)a.workspace);
        else if (blocks[l] > 0)
            hipLaunchKernelGGL((apply_kernel<DT, WIDE, FULL, 4>), dim3(blocks[l]), dim3(NT), 0, s, src[l], rule, plan.cols[l],
                               (const uint8_t*)a.workspace);
    };
    apply(1, std::true_type{}, std::true_type{});
    apply(3, std::false_type{}, std::true_type{});
    apply(2, std::true_type{}, std::false_type{});
    apply(4, std::false_type{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace

int64_t update_scratch(int64_t d, int64_t n) {
    const int64_t dt = blocks_of(d);
    // (the steps of the wide sides keep six matrices and |v| there, in 256 bytes of its own)
    return 8 * (pieces_of(n) * (dt * (dt + 1) / 2 * 256) + (dt > 4 ? 6 * 256 * dt * dt + 32 : 256 * dt * dt));
}

int64_t update_table(int64_t count) { return count > kBatch ? count * (int64_t)(sizeof(Matrix) + kLaunches * sizeof(int)) : 0; }

hipError_t launch_update(const UpdateArgs& a, const Matrix* matrices, int64_t count, void* table, hipStream_t s) {
    Table t{};
    t.m = (Matrix*)table;
    t.first = (int*)(t.m + (table != nullptr ? count : 0));
    hipError_t e = launch_size<1>(a, matrices, count, t, s);
    if (e == hipSuccess) e = launch_size<2>(a, matrices, count, t, s);
    if (e == hipSuccess) e = launch_size<3>(a, matrices, count, t, s);
    if (e == hipSuccess) e = launch_size<4>(a, matrices, count, t, s);
    if (e == hipSuccess) e = launch_size<6>(a, matrices, count, t, s);
    if (e == hipSuccess) e = launch_size<8>(a, matrices, count, t, s);
    return e;
}

}  // namespace block
}  // namespace lors
