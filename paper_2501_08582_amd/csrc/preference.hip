// Log-probabilities of target tokens, the paired preference loss over them, and
// the gradient of the logits.
//
// The logits are what costs: the forward reads each row once, keeping a running
// maximum and the sum of exponentials below it, and the backward reads it again
// and writes the gradient.  Rows whose target does not count are not read.  (The
// loss of a pair needs all its tokens before the first gradient, so two reads it
// is.)
//   logp = x[target] - top - log(sum),  dx = c (onehot - exp(x - top) / sum)
//
// Bound by memory: 8192 x 65536 bf16, 86 % of the rows counted: forward 154 us (0.92 GB,
// 6.0 TB/s), backward 345 us (0.92 GB read, 1.07 written, 5.8 TB/s).  1028 x 50021 fp32:
// 35 and 59 us.
#include <algorithm>

#include "train_common.hpp"

namespace lors {
namespace train {
namespace {

constexpr int NT = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNone = -__builtin_inff();

template <bool I64>
__device__ __forceinline__ uint32_t target_of(const void* targets, int64_t n, uint32_t vocab) {
    if constexpr (I64) {
        const uint64_t v = ((const uint64_t*)targets)[n];
        return v < vocab ? (uint32_t)v : ~0u;
    } else {
        const uint32_t v = ((const uint32_t*)targets)[n];
        return v < vocab ? v : ~0u;
    }
}

// 2^x by the hardware's instruction: results below 2^-126 are 0, which is far
// below what a term of a sum next to 1 or a probability is rounded to.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// e^t for t <= 0 where the result is an output of type T.  t log2(e) in fp32 is off by
// up to 2^-24 of itself, t of -16 by 1e-6 of the result: nothing next to bf16's
// rounding, more than fp32's, for which the product's remainder is put back.
constexpr float kLog2eRest = 1.92596299e-8f;  // log2(e) - kLog2e
template <typename T>
__device__ __forceinline__ float exp_below(float t) {
    const float x = t * kLog2e, y = exp2_hw(x);
    if constexpr (sizeof(T) == 2) return y;
    const float rest = __builtin_fmaf(t, kLog2e, -x) + t * kLog2eRest;
    // -Inf, and products past fp32's range, have no remainder: their result is 0
    return y == 0.f ? 0.f : __builtin_fmaf(y, rest * 0.69314718f, y);
}

// t log2(e) for the terms of a sum.  With the constant in fp32 alone every term is off
// by the same 1.3e-8 t, which does not average out: the logarithms of a sequence's
// sums are off by 7e-8 each, and its reward by as many as it has tokens.  (The small
// product first: added to the rounded large one it would be lost.)
__device__ __forceinline__ float times_log2e(float t) { return __builtin_fmaf(t, kLog2e, t * kLog2eRest); }

// The sum of exp(x - top) over what was seen, with top the largest of it.
struct Running {
    float top = kNone, sum = 0.f;

    template <int B, int N>
    __device__ __forceinline__ void add(const F<N> (&x)[B]) {
        float m = x[0].v[0];
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) m = fmaxf(m, x[i].v[e]);
        if (m > top) rescale(m);
        const float ref = top == kNone ? 0.f : top;  // all -Inf so far: they add nothing
        float s[N] = {};
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) s[e] += exp2_hw(times_log2e(x[i].v[e] - ref));
        sum += (s[0] + s[1]) + (s[2] + s[3]);
        if constexpr (N == 8) sum += (s[4] + s[5]) + (s[6] + s[7]);
    }

    __device__ __forceinline__ void rescale(float to) {
        // below a top of -Inf the sum is 0, or NaN where a NaN was among the entries: it stays
        sum = top == kNone ? sum : sum * exp2_hw((top - to) * kLog2e);
        top = to;
    }
};

// A row of logits in memory, and its last unit past the whole ones.
template <typename T>
__device__ __forceinline__ F<kUnit<T>> logits_unit(const T* row, uint32_t u, uint32_t vocab) {
    constexpr int N = kUnit<T>;
    const int left = (int)min(vocab - u * N, (uint32_t)N);
    F<N> f = widen(load_unit(row + (int64_t)u * N, left));
#pragma unroll
    for (int e = 1; e < N; ++e)
        if (e >= left) f.v[e] = kNone;
    return f;
}

// The row's results: `top` and `sum` apart, because a sum of them loses the logarithm
// next to a large `top` (a row whose entries are all the type's lowest value).
__device__ __forceinline__ void finish(float x, Running r, int64_t n, float* logp, float2* stats) {
    logp[n] = (float)((double)x - (double)r.top - log((double)r.sum));
    if (stats != nullptr) stats[n] = float2{r.top, r.sum};
}

__device__ __forceinline__ void finish_uncounted(int64_t n, float* logp, float2* stats) {
    logp[n] = 0.f;
    if (stats != nullptr) stats[n] = float2{0.f, 0.f};
}

struct Rows {
    uint32_t count, length, vocab;
    int64_t batch_stride, row_stride;
    __device__ __forceinline__ int64_t offset(uint32_t n) const {
        const uint32_t b = n / length;
        return b * batch_stride + (n - b * length) * row_stride;
    }
};

// An element takes a conversion, half a maximum, a difference, a product and an fma, an
// exponential (a quarter of the rate) and a sum, 9.5 of the chip's instructions: by that count
// three quarters of the time that the two bytes of a bf16 take.  A whole row of one
// compute unit is bound by them: 131072 entries are 8 us of the kernel's 9.7.
// A row's `splits` workgroups of W threads take a run of it each; with splits > 1 their (top, sum) go to
// `part` and logprob_join_kernel finishes.
template <typename T, bool I64, int W>
__global__ __launch_bounds__(W) void logprob_fwd_kernel(Rows rows, uint32_t splits, const T* __restrict__ logits,
                                                         const void* __restrict__ targets, float* __restrict__ logp,
                                                         float2* __restrict__ stats, float2* __restrict__ part) {
    constexpr int N = kUnit<T>;
    __shared__ float2 waves[W / 64];
    const uint32_t n = block_id() / splits, split = block_id() - n * splits;
    if (n >= rows.count) return;
    const uint32_t target = target_of<I64>(targets, n, rows.vocab);
    if (target == ~0u) {
        if (threadIdx.x == 0 && splits == 1) finish_uncounted(n, logp, stats);
        return;
    }
    const T* row = logits + rows.offset(n);
    const float picked = (float)row[target];  // ahead: nothing waits for it at the end
    const uint32_t units = (rows.vocab + N - 1) / N, per = (units + splits - 1) / splits;
    const uint32_t begin = min(split * per, units), end = min(begin + per, units);
    const uint32_t whole = min(end, rows.vocab / N);
    Running r;
    uint32_t u = begin + threadIdx.x;
    constexpr int kBatch = W == 1024 ? 8 : 4;  // units in flight: few rows have few waves to wait beside them
    for (; u + (kBatch - 1) * W < whole; u += kBatch * W) {
        Raw<T, N> raw[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) raw[i] = load_whole<T, N>(row + (int64_t)(u + i * W) * N);
        F<N> x[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i] = widen(raw[i]);
        r.add(x);
    }
    for (; u < end; u += W) {
        const F<N> x[1] = {logits_unit(row, u, rows.vocab)};
        r.add(x);
    }
    // lanes, then waves
    r.rescale(over_lanes<64>(r.top, Max()));
    r.sum = over_lanes<64>(r.sum, Add());
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = float2{r.top, r.sum};
    __syncthreads();
    if (threadIdx.x != 0) return;
    float top = kNone;
#pragma unroll
    for (int w = 0; w < W / 64; ++w) top = fmaxf(top, waves[w].x);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < W / 64; ++w) {
        Running q{waves[w].x, waves[w].y};
        q.rescale(top);
        sum += q.sum;
    }
    r.top = top;
    r.sum = sum;
    if (splits > 1) part[block_id()] = float2{top, sum};
    else finish(picked, r, n, logp, stats);
}

// One wave per row joins its splits.
template <typename T, bool I64>
__global__ __launch_bounds__(64) void logprob_join_kernel(Rows rows, uint32_t splits, const T* __restrict__ logits,
                                                          const void* __restrict__ targets,
                                                          const float2* __restrict__ part, float* __restrict__ logp,
                                                          float2* __restrict__ stats) {
    const uint32_t n = block_id();
    if (n >= rows.count) return;
    const uint32_t target = target_of<I64>(targets, n, rows.vocab);
    if (target == ~0u) {
        if (threadIdx.x == 0) finish_uncounted(n, logp, stats);
        return;
    }
    Running r;
    for (uint32_t i = threadIdx.x; i < splits; i += 64) {
        const float2 p = part[(int64_t)n * splits + i];
        Running q{p.x, p.y};
        const float top = fmaxf(r.top, q.top);
        r.rescale(top);
        q.rescale(top);
        r.sum += q.sum;
    }
    r.rescale(over_lanes<64>(r.top, Max()));
    r.sum = over_lanes<64>(r.sum, Add());
    if (threadIdx.x == 0) finish((float)logits[rows.offset(n) + target], r, n, logp, stats);
}

// dlogits = c (onehot - exp(x - top) / sum); a workgroup takes `kPart` units of a row.
constexpr int kPart = 4;
template <typename T, bool I64>
__global__ __launch_bounds__(NT) void logprob_bwd_kernel(Rows rows, uint32_t parts, uint32_t span,
                                                         const float* __restrict__ dlogp,
                                                         const float* __restrict__ upstream,
                                                         const T* __restrict__ logits, const void* __restrict__ targets,
                                                         const float2* __restrict__ stats, T* __restrict__ dlogits) {
    constexpr int N = kUnit<T>;
    const uint32_t n = block_id() / parts, first = (block_id() - n * parts) * (kPart * NT) + threadIdx.x;
    if (n >= rows.count) return;
    const uint32_t target = target_of<I64>(targets, n, rows.vocab);
    const uint32_t units = (rows.vocab + N - 1) / N;
    T* out = dlogits + (int64_t)n * rows.vocab;
    if (target == ~0u) {
#pragma unroll
        for (int i = 0; i < kPart; ++i) {
            const uint32_t u = first + i * NT;
            if (u < units)
                stream_unit(out + (int64_t)u * N, Raw<T, N>{}, (int)min(rows.vocab - u * N, (uint32_t)N));
        }
        return;
    }
    const T* row = logits + rows.offset(n);
    const float c = dlogp[n / span] * (upstream != nullptr ? *upstream : 1.f);
    const float2 st = stats[n];
    const float top = st.x, down = -c / st.y;
    Raw<T, N> x[kPart];
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
        const uint32_t u = first + i * NT;
        if (u < units) x[i] = load_unit(row + (int64_t)u * N, (int)min(rows.vocab - u * N, (uint32_t)N));
    }
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
        const uint32_t u = first + i * NT;
        if (u >= units) break;
        F<N> f = widen(x[i]);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f.v[e] = down * exp_below<T>(f.v[e] - top);
            if (u * N + e == target) f.v[e] += c;
        }
        stream_unit(out + (int64_t)u * N, narrow<T>(f), (int)min(rows.vocab - u * N, (uint32_t)N));
    }
}

// ---------------------------------------------------------------------------
// the loss over pairs of sequences
// ---------------------------------------------------------------------------
__device__ __forceinline__ double log_sigmoid(double x) { return fmin(x, 0.0) - log1p(exp(-fabs(x))); }

__device__ __forceinline__ double pair_loss(double margin, double e) {
    const double l = -(1.0 - e) * log_sigmoid(margin);
    return e == 0.0 ? l : l - e * log_sigmoid(-margin);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

constexpr int kWaves = 16;
constexpr int kOnePairs = 512;

// sum[side] += logp - ref over the tokens begin, begin + step, .. < end of both
// sequences of pair i.
template <bool I64>
__device__ __forceinline__ void add_pair(double (&sum)[2], int64_t i, int64_t pairs, int64_t length, uint32_t vocab,
                                         const float* logp, const float* ref, const void* targets, int64_t begin,
                                         int64_t end, int step) {
#pragma unroll 4
    for (int64_t t = begin; t < end; t += step) {
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const int64_t at = (side * pairs + i) * length + t;
            const double d = (double)logp[at] - (ref != nullptr ? (double)ref[at] : 0.0);
            sum[side] += target_of<I64>(targets, at, vocab) != ~0u ? d : 0.0;
        }
    }
}

// The rewards of pair i from its sums, and dseq of its preferred sequence; its loss is
// returned.  The margin is a small difference of rewards that may be large: it exists
// in 64 bits only.
__device__ __forceinline__ double finish_pair(double won, double lost, int64_t i, int64_t pairs, double beta, double e,
                                              float* reward, float* dseq) {
    won *= beta;
    lost *= beta;
    const double margin = won - lost;
    reward[i] = (float)won;
    reward[pairs + i] = (float)lost;
    dseq[i] = (float)(beta / (double)pairs * (e * exp(log_sigmoid(margin)) - (1.0 - e) * exp(log_sigmoid(-margin))));
    return pair_loss(margin, e);
}

// Few tokens: one workgroup for all pairs, each cut into `segs` runs of tokens so
// that every wave has one, then a thread to a pair.
template <bool I64>
__global__ __launch_bounds__(64 * kWaves) void preference_one_kernel(int pairs, int64_t length, uint32_t vocab,
                                                                     double beta, double e, int segs,
                                                                     const float* __restrict__ logp,
                                                                     const float* __restrict__ ref,
                                                                     const void* __restrict__ targets,
                                                                     float* __restrict__ loss,
                                                                     float* __restrict__ reward,
                                                                     float* __restrict__ dseq) {
    __shared__ double sums[2][kOnePairs];
    __shared__ double totals[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int item = wave; item < pairs * segs; item += kWaves) {
        const int i = item / segs, seg = item - i * segs;
        double s[2] = {0.0, 0.0};
        add_pair<I64>(s, i, pairs, length, vocab, logp, ref, targets, length * seg / segs + lane,
                      length * (seg + 1) / segs, 64);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            s[side] = wave_sum(s[side]);
            if (lane == 0) sums[side][item] = s[side];
        }
    }
    __syncthreads();
    double total = 0.0;
    for (int i = threadIdx.x; i < pairs; i += 64 * kWaves) {
        double s[2] = {0.0, 0.0};
        for (int seg = 0; seg < segs; ++seg)
#pragma unroll
            for (int side = 0; side < 2; ++side) s[side] += sums[side][i * segs + seg];
        total += finish_pair(s[0], s[1], i, pairs, beta, e, reward, dseq);
        dseq[pairs + i] = -dseq[i];
    }
    total = wave_sum(total);
    if (lane == 0) totals[wave] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    total = 0.0;
    for (int w = 0; w < kWaves; ++w) total += totals[w];
    *loss = (float)(total / (double)pairs);
}

// Many: a workgroup to a pair.  Its loss, rounded to fp32 (2^-24 of it, as the mean will
// be), waits in the place of the rejected sequence's dseq, which is the preferred one's
// negated: preference_mean_kernel takes the mean and puts that there.
template <bool I64>
__global__ __launch_bounds__(64 * kWaves) void preference_kernel(int64_t pairs, int64_t length, uint32_t vocab,
                                                                 double beta, double e, const float* __restrict__ logp,
                                                                 const float* __restrict__ ref,
                                                                 const void* __restrict__ targets,
                                                                 float* __restrict__ reward,
                                                                 float* __restrict__ dseq) {
    __shared__ double lds[2][kWaves];
    for (int64_t i = blockIdx.x; i < pairs; i += gridDim.x) {
        double s[2] = {0.0, 0.0};
        add_pair<I64>(s, i, pairs, length, vocab, logp, ref, targets, threadIdx.x, length, 64 * kWaves);
        __syncthreads();  // the sums of the pair before are read
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            s[side] = wave_sum(s[side]);
            if ((threadIdx.x & 63) == 0) lds[side][threadIdx.x >> 6] = s[side];
        }
        __syncthreads();
        if (threadIdx.x != 0) continue;
        s[0] = s[1] = 0.0;
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int side = 0; side < 2; ++side) s[side] += lds[side][w];
        dseq[pairs + i] = (float)finish_pair(s[0], s[1], i, pairs, beta, e, reward, dseq);
    }
}

__global__ __launch_bounds__(64 * kWaves) void preference_mean_kernel(int64_t pairs, float* __restrict__ dseq,
                                                                      float* __restrict__ loss) {
    __shared__ double lds[kWaves];
    double total = 0.0;
    for (int64_t i = threadIdx.x; i < pairs; i += 64 * kWaves) {
        total += (double)dseq[pairs + i];
        dseq[pairs + i] = -dseq[i];
    }
    total = wave_sum(total);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    total = 0.0;
    for (int w = 0; w < kWaves; ++w) total += lds[w];
    *loss = (float)(total / (double)pairs);
}

constexpr int64_t kPartCols = 4096;  // the fewest entries of a row that a workgroup takes
constexpr int64_t kManyRows = 512, kRowBytes = 256 << 10, kFewGroups = 512;
constexpr int64_t kOneMost = 16384;  // tokens of both sides that one workgroup sums

// How the forward takes its rows.  Many rows fill the chip with workgroups of 256
// threads each.  A few take 1024 threads each, and very long ones of them several
// workgroups, whose sums a second launch joins.  A call of two launches costs its caller
// 15.5 us at least, one of one launch 11.3; in a captured graph the second costs less.  4 rows,
// us a call, and in a graph:
//   bf16: 131072 entries whole 11.3, 9.7; 200064 whole 13.0, 13.4, in pieces of 128 KB 15.5, 8.7;
//   256000 whole 17.3, 17.7, pieces of 128 KB 15.4, 10.2; 393213 whole 28.3, 28.8, pieces of
//   256 KB 19.7, 19.9, of 128 KB 15.7, 11.0;
//   fp32: 131072 whole 11.4, 9.8, pieces of 256 KB 15.7, 8.8; 262141 whole 17.2, 17.5, 16.3, 11.0.
// Smaller pieces lose where rows times pieces come to fill the chip: 64 x 1000000 bf16 31.5 in
// pieces of 256 KB, 35.5 of 128 KB; 200 x 256000 25.9 whole, 32.4 of 128 KB.
struct FwdPlan {
    int threads;
    uint32_t splits;
};
FwdPlan fwd_plan(int64_t rows, int64_t vocab, bool bf16) {
    if (rows >= kManyRows) return {NT, 1};
    const int64_t pieces = vocab * (bf16 ? 2 : 4) / kRowBytes, room = rows > 0 ? kFewGroups / rows : 1;
    const int64_t splits = pieces < room ? pieces : room;
    return {1024, (uint32_t)(splits > 1 ? splits : 1)};
}

Rows rows_of(const LogprobArgs& a) {
    return Rows{(uint32_t)(a.batch * a.length), (uint32_t)a.length, (uint32_t)a.vocab, a.batch_stride, a.row_stride};
}

template <typename T, bool I64>
hipError_t forward(const LogprobArgs& a, hipStream_t s) {
    const int64_t rows = a.batch * a.length;
    const FwdPlan p = fwd_plan(rows, a.vocab, sizeof(T) == 2);
    const uint32_t splits = p.splits;
    if (p.threads == NT)
        hipLaunchKernelGGL((logprob_fwd_kernel<T, I64, NT>), grid_of(rows), dim3(NT), 0, s, rows_of(a), splits,
                           (const T*)a.logits, a.targets, a.logp, (float2*)a.stats, (float2*)a.workspace);
    else
        hipLaunchKernelGGL((logprob_fwd_kernel<T, I64, 1024>), grid_of(rows * splits), dim3(1024), 0, s, rows_of(a),
                           splits, (const T*)a.logits, a.targets, a.logp, (float2*)a.stats, (float2*)a.workspace);
    if (splits > 1)
        hipLaunchKernelGGL((logprob_join_kernel<T, I64>), grid_of(rows), dim3(64), 0, s, rows_of(a), splits,
                           (const T*)a.logits, a.targets, (const float2*)a.workspace, a.logp, (float2*)a.stats);
    return hipGetLastError();
}

template <typename T, bool I64>
hipError_t backward(const LogprobArgs& a, hipStream_t s) {
    const int64_t rows = a.batch * a.length;
    constexpr int64_t cols = kUnit<T> * kPart * NT;
    const uint32_t parts = (uint32_t)((a.vocab + cols - 1) / cols);
    hipLaunchKernelGGL((logprob_bwd_kernel<T, I64>), grid_of(rows * parts), dim3(NT), 0, s, rows_of(a), parts,
                       (uint32_t)a.span, a.dlogp, a.upstream, (const T*)a.logits, a.targets, (const float2*)a.stats, (T*)a.dlogits);
    return hipGetLastError();
}

template <bool I64>
hipError_t preference(const PreferenceArgs& a, hipStream_t s) {
    const dim3 block(64 * kWaves);
    if (2 * a.pairs * a.length <= kOneMost && a.pairs <= kOnePairs) {
        const int segs = a.pairs >= kWaves ? 1 : kWaves / (int)a.pairs;
        hipLaunchKernelGGL(preference_one_kernel<I64>, dim3(1), block, 0, s, (int)a.pairs, a.length,
                           (uint32_t)a.vocab, a.beta, a.smoothing, segs, a.logp, a.ref, a.targets, a.loss, a.reward,
                           a.dseq);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(preference_kernel<I64>, dim3((unsigned)std::min<int64_t>(a.pairs, 65536)), block, 0, s,
                       a.pairs, a.length, (uint32_t)a.vocab, a.beta, a.smoothing, a.logp, a.ref, a.targets, a.reward,
                       a.dseq);
    hipLaunchKernelGGL(preference_mean_kernel, dim3(1), dim3(64 * kWaves), 0, s, a.pairs, a.dseq, a.loss);
    return hipGetLastError();
}

}  // namespace

bool logprob_grids_fit(int64_t rows, int64_t vocab) {
    return rows * ((vocab + kPartCols - 1) / kPartCols) < (int64_t)1 << 31;
}

size_t logprob_workspace_bytes(int64_t rows, int64_t vocab, bool bf16) {
    const uint32_t splits = fwd_plan(rows, vocab, bf16).splits;
    return splits > 1 ? (size_t)(rows * splits * sizeof(float2)) : 0;
}

hipError_t launch_logprob_forward(const LogprobArgs& a, bool bf16, hipStream_t s) {
    if (a.batch * a.length == 0) return hipSuccess;
    if (bf16) return a.index64 ? forward<__bf16, true>(a, s) : forward<__bf16, false>(a, s);
    return a.index64 ? forward<float, true>(a, s) : forward<float, false>(a, s);
}

hipError_t launch_logprob_backward(const LogprobArgs& a, bool bf16, hipStream_t s) {
    if (a.batch * a.length == 0) return hipSuccess;
    if (bf16) return a.index64 ? backward<__bf16, true>(a, s) : backward<__bf16, false>(a, s);
    return a.index64 ? backward<float, true>(a, s) : backward<float, false>(a, s);
}

hipError_t launch_preference(const PreferenceArgs& a, hipStream_t s) {
    return a.index64 ? preference<true>(a, s) : preference<false>(a, s);
}

}  // namespace train
}  // namespace lors
