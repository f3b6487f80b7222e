// Scaled embedding lookup, and the gradient of its table.
//
// The gradient needs, for every row of the table, the tokens that took it.  Among a
// few tokens a row finds its own.  More are sorted by id first, by counting for
// short batches and by digits for long ones.  Then every row of the gradient is written once, its zeros and its
// sums alike, and each sum runs over the tokens in their order, so that the
// result does not depend on which workgroup is faster.
//
// The lookup is bound by memory: 8192 x 4096 bf16 22 us (107 MB with the rows that tokens
// share read once or twice, 4.9 TB/s).  So is the writing of the gradient: 32768 x 4096 from
// 8192 tokens 71 us (322 MB, 4.5 TB/s), 131072 x 4096 from 16384 tokens 228 us (1.17 GB, 5.1
// TB/s).  The sort before it is a chain of waits: 19 us for 8192 or 16384 tokens, 7 for 1501.
#include <algorithm>
#include <utility>

#include "train_common.hpp"

namespace lors {
namespace train {
namespace {

constexpr int NT = 256;

// A token's id as the sort sees it: ids that stand for no token come last, as
// `vocab`.
template <bool I64>
__device__ __forceinline__ uint32_t id_of(const void* ids, int64_t t, uint32_t vocab) {
    if constexpr (I64) {
        const uint64_t v = ((const uint64_t*)ids)[t];
        return v < vocab ? (uint32_t)v : vocab;
    } else {
        const uint32_t v = ((const uint32_t*)ids)[t];
        return v < vocab ? v : vocab;
    }
}

// ---------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------
constexpr int kAhead = 4;  // units a thread has in flight

template <typename T, bool I64>
__global__ __launch_bounds__(NT) void lookup_kernel(int64_t tokens, uint32_t vocab, uint32_t cols, uint32_t units,
                                                    float scale, const void* __restrict__ ids,
                                                    const T* __restrict__ E, T* __restrict__ Y) {
    constexpr int N = kUnit<T>;
    // units in row-major order, a grid's worth apart: one division, then steps
    const uint32_t stride = gridDim.x * NT;
    const uint32_t step_rows = stride / units, step_units = stride - step_rows * units;
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    int64_t n = t / units;
    uint32_t g = t - (uint32_t)n * units;
    while (n < tokens) {
        int64_t at[kAhead];
        uint32_t id[kAhead], col[kAhead];
        int left[kAhead];
        Raw<T, N> x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            col[i] = g * N;
            at[i] = n * cols + col[i];
            left[i] = n < tokens ? (int)min(cols - col[i], (uint32_t)N) : 0;
            id[i] = n < tokens ? id_of<I64>(ids, n, vocab) : vocab;
            n += step_rows;
            g += step_units;
            if (g >= units) {
                g -= units;
                ++n;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            x[i] = Raw<T, N>{};
            if (id[i] < vocab) x[i] = load_unit(E + (int64_t)id[i] * cols + col[i], left[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (left[i] <= 0) break;
            F<N> f = widen(x[i]);
#pragma unroll
            for (int e = 0; e < N; ++e) f.v[e] *= scale;
            if (id[i] >= vocab) f = F<N>{};
            store_unit(Y + at[i], narrow<T>(f), left[i]);
        }
    }
}

// ---------------------------------------------------------------------------
// tokens sorted by (id, token): pairs {id, token}
// ---------------------------------------------------------------------------

// By counting: a token's place is the number of tokens that come before it.  A
// workgroup places 64 tokens, one per lane.  Its waves share the comparisons: each
// takes a run of the ids, 64 in a register, and hands them to all lanes one at a
// time through a scalar.  Three instructions a comparison of 64 tokens, no memory
// (ids read out of LDS: twice as long).  1501 tokens 6.6 us, 4096 10, 8192 16.5.
constexpr int kRankWaves = 16;

template <bool I64>
__global__ __launch_bounds__(64 * kRankWaves) void rank_kernel(int tokens, uint32_t vocab, const void* __restrict__ ids,
                                                               uint2* __restrict__ sorted) {
    __shared__ int count[kRankWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = blockIdx.x, i = group * 64 + lane;
    const uint32_t mine = i < tokens ? id_of<I64>(ids, i, vocab) : vocab;
    int before = 0;
    const int groups = (tokens + 63) / 64;
    const int begin = groups * wave / kRankWaves, end = groups * (wave + 1) / kRankWaves;
    auto ids_of = [&](int g) {  // ids above all past the last token
        const int j = g * 64 + lane;
        return g < end && j < tokens ? id_of<I64>(ids, j, vocab) : ~0u;
    };
    uint32_t next = ids_of(begin);
    for (int g = begin; g < end; ++g) {
        const uint32_t keys = next;
        next = ids_of(g + 1);
        // earlier tokens of the same id come before, later ones do not
        if (g < group) {
#pragma unroll
            for (int j = 0; j < 64; ++j) before += (uint32_t)__builtin_amdgcn_readlane((int)keys, j) <= mine;
        } else if (g > group) {
#pragma unroll
            for (int j = 0; j < 64; ++j) before += (uint32_t)__builtin_amdgcn_readlane((int)keys, j) < mine;
        } else {
#pragma unroll
            for (int j = 0; j < 64; ++j) {
                const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)keys, j);
                before += k < mine || (k == mine && j < lane);
            }
        }
    }
    count[wave][lane] = before;
    __syncthreads();
    if (wave != 0 || i >= tokens) return;
    int place = 0;
#pragma unroll
    for (int w = 0; w < kRankWaves; ++w) place += count[w][lane];
    sorted[place] = uint2{mine, (uint32_t)i};
}

// By digits of 9 bits, the lowest first.  A workgroup takes a tile of tokens and
// places them behind those of lower digits and of earlier tiles, in their order.
// For that it needs the digits of all tiles: of a short batch it counts them
// itself, of a long one they are counted by a launch before.
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = kDigits;  // one thread per digit where tiles are joined
constexpr int kSortWaves = kSortThreads / 64;

// A tile is Q tokens a thread; its last one is short.
template <int Q>
constexpr int kTile = kSortThreads * Q;

// Token i's pair: from the ids for the first digit, then from the pairs `in`.
template <bool FIRST, bool I64>
__device__ __forceinline__ uint2 pair_of(int64_t i, uint32_t vocab, const void* ids, const uint2* in) {
    if constexpr (FIRST) return uint2{id_of<I64>(ids, i, vocab), (uint32_t)i};
    else return in[i];
}
__device__ __forceinline__ uint32_t digit_of(uint2 pair, int shift) { return (pair.x >> shift) & (kDigits - 1); }

template <int Q, bool FIRST, bool I64>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(int64_t tokens, uint32_t vocab, int shift,
                                                                   const void* __restrict__ ids,
                                                                   const uint2* __restrict__ in,
                                                                   uint32_t* __restrict__ counts) {
    __shared__ uint32_t count[kDigits];
    count[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int64_t i = (int64_t)blockIdx.x * kTile<Q> + q * kSortThreads + threadIdx.x;
        if (i < tokens) atomicAdd(&count[digit_of(pair_of<FIRST, I64>(i, vocab, ids, in), shift)], 1u);
    }
    __syncthreads();
    counts[(int64_t)blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

// The counts of many tiles become the places' starts: of every tile and digit the tokens
// of that digit in earlier tiles, and in a last row those of all.  A lane to a digit, a run of
// tiles to a wave, kScanAhead of them in flight.  Without it every workgroup of the
// placement reads all tiles' counts, which grows with the square of the tokens.
constexpr int kScanWaves = 16;
constexpr int kScanAhead = 8;

__global__ __launch_bounds__(64 * kScanWaves) void digit_scan_kernel(int64_t tiles, uint32_t* __restrict__ counts) {
    __shared__ uint32_t total[kScanWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t begin = tiles * wave / kScanWaves, end = tiles * (wave + 1) / kScanWaves;
    uint32_t* const column = counts + blockIdx.x * 64 + lane;
    auto load = [&](uint32_t (&c)[kScanAhead], int64_t b) {
#pragma unroll
        for (int i = 0; i < kScanAhead; ++i) c[i] = b + i < end ? column[(b + i) * kDigits] : 0;
    };
    uint32_t sum = 0;
    for (int64_t b = begin; b < end; b += kScanAhead) {
        uint32_t c[kScanAhead];
        load(c, b);
#pragma unroll
        for (int i = 0; i < kScanAhead; ++i) sum += c[i];
    }
    total[wave][lane] = sum;
    __syncthreads();
    uint32_t at = 0;
    for (int w = 0; w < wave; ++w) at += total[w][lane];
    for (int64_t b = begin; b < end; b += kScanAhead) {
        uint32_t c[kScanAhead];
        load(c, b);
#pragma unroll
        for (int i = 0; i < kScanAhead; ++i) {
            if (b + i < end) column[(b + i) * kDigits] = at;
            at += c[i];
        }
    }
    if (wave == kScanWaves - 1) column[tiles * kDigits] = at;
}

// SELF: counts is not there.  scanned: digit_scan_kernel has made starts of them.
template <int Q, bool SELF, bool FIRST, bool I64>
__global__ __launch_bounds__(kSortThreads) void digit_place_kernel(int64_t tokens, uint32_t vocab, int shift,
                                                                   bool scanned, const void* __restrict__ ids,
                                                                   const uint2* __restrict__ in,
                                                                   const uint32_t* __restrict__ counts,
                                                                   uint2* __restrict__ out) {
    __shared__ uint32_t place[kSortWaves][kDigits];
    __shared__ uint32_t wave_total[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tile = (int64_t)blockIdx.x * kTile<Q>;
    const int64_t first = tile + wave * (kTile<Q> / kSortWaves);  // a wave's tokens are consecutive
    uint2 pair[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int64_t i = first + q * 64 + lane;
        pair[q] = i < tokens ? pair_of<FIRST, I64>(i, vocab, ids, in) : uint2{~0u, ~0u};
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) place[w][threadIdx.x] = 0;
    uint32_t all = 0, earlier = 0;  // of this thread's digit: the tokens in all tiles, and in earlier ones
    if constexpr (SELF) {
        __shared__ uint32_t others[2][kDigits];  // in earlier tiles, in this one and later ones
        others[0][threadIdx.x] = others[1][threadIdx.x] = 0;
        __syncthreads();
#pragma unroll 8
        for (int64_t i = threadIdx.x; i < tokens; i += kSortThreads)
            atomicAdd(&others[i >= tile][digit_of(pair_of<FIRST, I64>(i, vocab, ids, in), shift)], 1u);
        __syncthreads();
        earlier = others[0][threadIdx.x];
        all = earlier + others[1][threadIdx.x];
    } else {
        if (scanned) {
            earlier = counts[(int64_t)blockIdx.x * kDigits + threadIdx.x];
            all = counts[(int64_t)gridDim.x * kDigits + threadIdx.x];
        } else {
#pragma unroll 4
            for (uint32_t b = 0; b < gridDim.x; ++b) {
                const uint32_t c = counts[(int64_t)b * kDigits + threadIdx.x];
                all += c;
                if (b < blockIdx.x) earlier += c;
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (first + q * 64 + lane < tokens) atomicAdd(&place[wave][digit_of(pair[q], shift)], 1u);
    uint32_t run = all;  // inclusive sum over the lower digits of the wave
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(run, d);
        if (lane >= d) run += up;
    }
    if (lane == 63) wave_total[wave] = run;
    __syncthreads();
    uint32_t at = run - all + earlier;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w)
        if (w < wave) at += wave_total[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = place[w][threadIdx.x];
        place[w][threadIdx.x] = at;
        at += c;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const bool real = first + q * 64 + lane < tokens;
        const uint32_t digit = digit_of(pair[q], shift);
        uint64_t same = __ballot(real);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t set = __ballot((digit >> b) & 1u);
            same &= (digit >> b) & 1u ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        uint32_t base = 0;
        if (real && before == 0) base = atomicAdd(&place[wave][digit], (uint32_t)__popcll(same));
        base = __shfl(base, real ? __ffsll((unsigned long long)same) - 1 : 0);
        if (real) out[base + before] = pair[q];
    }
}

// ---------------------------------------------------------------------------
// the gradient's rows
// ---------------------------------------------------------------------------

// Columns go to groups of TL lanes, a unit each; a group of a whole wave keeps
// what all its lanes agree on in scalar registers.
template <int TL>
__device__ __forceinline__ uint32_t uniform(uint32_t v) {
    if constexpr (TL == 64) return (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
    else return v;
}

// The first position whose id is at least v.  A wave looks at 64 positions at a
// time (every lane has to take part), a smaller group halves.
template <int TL>
__device__ __forceinline__ uint32_t lower_bound(const uint2* __restrict__ sorted, uint32_t tokens, uint32_t v) {
    uint32_t lo = 0, hi = tokens;
    while (lo < hi) {
        if constexpr (TL == 64) {
            const uint32_t step = (hi - lo + 63) / 64;
            const uint32_t probe = lo + ((threadIdx.x & 63) + 1) * step - 1;
            const uint32_t below = __popcll(__ballot(probe < hi && sorted[min(probe, hi - 1)].x < v));
            lo = uniform<TL>(min(lo + below * step, hi));
            hi = uniform<TL>(min(hi, lo + step - 1));
        } else {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (sorted[mid].x < v) lo = mid + 1;
            else hi = mid;
        }
    }
    return lo;
}

// Sorted positions of a partial sum.  A token that is a fifteenth of 8192 has 17 of
// them; one that is all of them 256 (the whole gradient then takes 96 us in place of
// 78; with partial sums of 16, 120).
constexpr uint32_t kChunk = 32;
// Rows of the table per group, and of dY in flight.  With inputs that change from
// call to call (lookup and gradient, us): 8 x 8 122 at 8192 tokens into 32768 x 4096, 304
// at 16384 into 131072 x 4096, 54 at 1501 into 50021 x 771 fp32; 4 rows 129, 308, 50; 16
// rows 124, 314, 57; 16 in flight 120, 307, 51, but 59 against 52 with 32768 tokens of
// 32768 ids.  (Units counted from the row's start; from the cache line's, below, 8 x 8 takes
// 47 in the last case.)
constexpr uint32_t kRows = 8;
constexpr int kBatch = 8;

// acc += the units of dY's tokens pair[0 .. n), n <= kBatch, in order.
template <typename T, int N>
__device__ __forceinline__ void add_tokens(F<N>& acc, const uint2 (&pair)[kBatch], int n, const T* __restrict__ dY,
                                           int64_t cols, int64_t col, int left) {
    Raw<T, N> r[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
        if (i < n) r[i] = load_unit<T, N>(dY + (int64_t)pair[i].y * cols + col, left);
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
        if (i < n) {
            const F<N> f = widen(r[i]);
#pragma unroll
            for (int e = 0; e < N; ++e) acc.v[e] += f.v[e];
        }
}

// Sums of the chunks that belong to one id as a whole, so that no row of the table
// has a long chain of tokens (8192 tokens: 9 us).
template <typename T, int N, int TL>
__global__ __launch_bounds__(NT) void chunk_kernel(uint32_t chunks, uint32_t vocab, int64_t cols, uint32_t tiles,
                                                   const uint2* __restrict__ sorted, const T* __restrict__ dY,
                                                   float* __restrict__ part) {
    const uint32_t group = block_id() * (NT / TL) + uniform<TL>(threadIdx.x / TL);
    const uint32_t chunk = group / tiles;
    if (chunk >= chunks) return;
    const int64_t col = ((int64_t)(group - chunk * tiles) * TL + threadIdx.x % TL) * N;
    const int left = (int)min(cols - col, (int64_t)N);
    const uint2* s = sorted + (int64_t)chunk * kChunk;
    uint2 pair[kChunk / kBatch][kBatch];  // all at once: a chunk is two waits on memory
#pragma unroll
    for (uint32_t i = 0; i < kChunk; ++i) pair[i / kBatch][i % kBatch] = s[i];
    const uint32_t id = pair[0][0].x;
    if (left <= 0 || id != pair[kChunk / kBatch - 1][kBatch - 1].x || id >= vocab) return;
    F<N> acc = {};
#pragma unroll
    for (uint32_t b = 0; b < kChunk / kBatch; ++b) add_tokens(acc, pair[b], kBatch, dY, cols, col, left);
    store_unit(part + chunk * cols + col, narrow<float>(acc), left);
}

// A lane's part of a row of the gradient: elements first .. first + n - 1.  Its units
// are those of what it writes, N elements of G being 16 bytes.  SHIFT: rows start
// anywhere in a cache line of 128 bytes, and the units are counted from the line's
// start: no line but a row's first and last is written by two waves, and those two go
// through the cache, where their parts meet.  Lookup and gradient of 1501 tokens into
// 50021 rows, against units counted from the row's start: x 771 fp32 48.5 us (55.8),
// x 1544 bf16 45.8 (54.6); x 1541 bf16 73.8 both ways (a row that starts at an odd element
// ends in units written one element at a time); 768 fp32, where nothing shifts, 46.
// Lanes without a part stay (the search needs all of them): they read the row's
// first unit, and store nothing.
template <typename G, bool SHIFT>
struct Part {
    static constexpr int N = kUnit<G>;
    static constexpr uint32_t kLine = 128 / sizeof(G);
    int64_t first;
    int n;
    bool real, inner;  // inner: all of the part's line is this row's
    __device__ __forceinline__ Part(int64_t unit, uint32_t v, int64_t cols, uint32_t phase) {
        const uint32_t before = SHIFT ? (v * (uint32_t)cols + phase) & (kLine - 1) : 0;
        const int64_t c = unit * N - before, end = min(c + N, cols);
        first = c > 0 ? c : 0;
        real = first < end;
        inner = !SHIFT || (unit * N >= (before != 0 ? kLine : 0) && unit * N < ((cols + before) & ~(int64_t)(kLine - 1)));
        if (!real) first = 0;
        n = (int)((real ? end : min((int64_t)N, cols)) - first);
    }
    __device__ __forceinline__ void store(G* row, const F<N>& f) const {
        if (!real) return;
        if (inner) stream_unit(row + first, narrow<G>(f), n);
        else store_unit(row + first, narrow<G>(f), n);
    }
};

// Elements from the start of a cache line to p.
template <typename G>
__device__ __forceinline__ uint32_t phase_of(const G* p) {
    return (uint32_t)((uintptr_t)p / sizeof(G)) & (Part<G, true>::kLine - 1);
}

template <typename T, typename G, int TL, bool SHIFT>
__global__ __launch_bounds__(NT) void rows_kernel(uint32_t tokens, uint32_t vocab, int64_t cols, uint32_t tiles,
                                                  uint32_t per, float scale, const uint2* __restrict__ sorted,
                                                  const T* __restrict__ dY, const float* __restrict__ part,
                                                  G* __restrict__ dE) {
    constexpr int N = kUnit<G>;
    const uint32_t group = block_id() * (NT / TL) + uniform<TL>(threadIdx.x / TL);
    const uint32_t v0 = group / tiles * per;
    if (v0 >= vocab) return;
    const int64_t unit = (int64_t)(group % tiles) * TL + threadIdx.x % TL;
    const uint32_t phase = phase_of(dE);
    uint32_t pos = lower_bound<TL>(sorted, tokens, v0);
    uint32_t next = pos < tokens ? uniform<TL>(sorted[pos].x) : ~0u;
    for (uint32_t v = v0; v < min(v0 + per, vocab); ++v) {
        const Part<G, SHIFT> at(unit, v, cols, phase);
        F<N> acc = {};
        while (next == v) {
            if (pos % kChunk == 0 && tokens - pos >= kChunk && sorted[pos + kChunk - 1].x == v) {
                // whole chunks of a frequent token: their sums are there
                const uint32_t n = (lower_bound<TL>(sorted, tokens, v + 1) - pos) / kChunk;
                const float* p = part + (int64_t)(pos / kChunk) * cols + at.first;
#pragma unroll 8
                for (uint32_t i = 0; i < n; ++i) {
                    const F<N> f = widen(load_unit<float, N>(p + i * cols, at.n));
#pragma unroll
                    for (int e = 0; e < N; ++e) acc.v[e] += f.v[e];
                }
                pos += n * kChunk;
            } else {
                // up to the next chunk: the tokens of v come first
                const int room = (int)min(min(kChunk - pos % kChunk, tokens - pos), (uint32_t)kBatch);
                uint2 pair[kBatch];
                int n = 0;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    pair[i] = i < room ? sorted[pos + i] : uint2{~0u, 0u};
                    n += pair[i].x == v;
                }
                add_tokens(acc, pair, n, dY, cols, at.first, at.n);
                pos += n;
            }
            next = pos < tokens ? uniform<TL>(sorted[pos].x) : ~0u;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) acc.v[e] *= scale;
        at.store(dE + (int64_t)v * cols, acc);
    }
}

// The same without a sort, for up to 64 Q tokens: a wave holds all ids, Q to a lane,
// and takes each row's tokens from the lanes that have its id, in order.  One launch
// in place of three: 100 or 256 tokens into 2000 x 512 8.2 us a call against 14.5, into
// 32768 x 4096 50 against 56.  What it lacks is the partial sums of a frequent token: 256
// tokens of one id take 31 us against 14, 512 (with 8 ids a lane) 60 against 14, which is
// why it ends at 256.
constexpr int kFewIds = 4;
template <typename T, typename G, bool I64, bool SHIFT>
__global__ __launch_bounds__(NT) void rows_few_kernel(int tokens, uint32_t vocab, int64_t cols, uint32_t tiles,
                                                      uint32_t per, float scale, const void* __restrict__ ids,
                                                      const T* __restrict__ dY, G* __restrict__ dE) {
    constexpr int N = kUnit<G>;
    const int lane = threadIdx.x & 63;
    const uint32_t group = block_id() * (NT / 64) + uniform<64>(threadIdx.x >> 6);
    const uint32_t v0 = group / tiles * per;
    if (v0 >= vocab) return;
    uint32_t key[kFewIds];  // `vocab` and all ones are no row's id
#pragma unroll
    for (int q = 0; q < kFewIds; ++q) key[q] = q * 64 + lane < tokens ? id_of<I64>(ids, q * 64 + lane, vocab) : ~0u;
    const int64_t unit = (int64_t)(group % tiles) * 64 + lane;
    const uint32_t phase = phase_of(dE);
    for (uint32_t v = v0; v < min(v0 + per, vocab); ++v) {
        const Part<G, SHIFT> at(unit, v, cols, phase);
        F<N> acc = {};
#pragma unroll
        for (int q = 0; q < kFewIds; ++q) {
            uint64_t mine = __ballot(key[q] == v);
            while (mine != 0) {
                uint2 pair[kBatch];
                int n = 0;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    pair[i].y = q * 64 + __ffsll((unsigned long long)mine) - 1;
                    n += mine != 0;
                    mine &= mine - 1;
                }
                add_tokens(acc, pair, n, dY, cols, at.first, at.n);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) acc.v[e] *= scale;
        at.store(dE + (int64_t)v * cols, acc);
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// How many tokens are sorted by counting, by digits that every workgroup counts, by
// digits in short tiles.  Whole gradient, us:
//   a table of 64 rows: 4096 tokens 20.7 by counting, 20.9 by digits; 6144 26 and 22;
//   65536 in tiles of 1024 32, 131072 in tiles of 4096 37.
//   Digits counted by every workgroup, or by a launch, into 64 x 64 bf16: 4224 tokens 34
//   and 36, 6144 39.5 and 40.5, 8192 41 and 42; into 775 x 735 fp32: 22 and 23.5, 25.3 and
//   24.6, 29 and 25.3; into 32768 x 4096 bf16: 63 and 64, 64 and 64, 64 and 61.
//   Counts scanned by a launch, or all read by every workgroup, into 512 x 8: 131072
//   tokens (32 tiles) 87 and 85, 262144 (64) 94 and 95, 524288 106 and 115, 4194304 349 and
//   471; the latter goes on with the square.
constexpr int64_t kFewMost = 64 * kFewIds;  // tokens that are not sorted
constexpr int64_t kRankMost = 4096;
constexpr int64_t kSelfMost = 6144;
constexpr int64_t kShortMost = 65536;
constexpr int64_t kUnscannedTiles = 64;  // more tiles than these have their counts scanned

int digit_passes(int64_t vocab) {
    int bits = 1;
    while ((vocab >> bits) != 0) ++bits;  // the ids go up to `vocab`
    return (bits + kDigitBits - 1) / kDigitBits;
}

int64_t tiles_of(int64_t tokens) {
    const int64_t tile = tokens <= kShortMost ? kTile<2> : kTile<8>;
    return (tokens + tile - 1) / tile;
}

// The workspace: two arrays of pairs, the digits' counts of every tile, the partial
// sums.
struct Layout {
    size_t sorted, other, counts, part, bytes;
};
Layout layout_of(int64_t tokens, int64_t cols) {
    Layout w{};
    if (tokens <= kFewMost) return w;
    const size_t pairs = up256((size_t)tokens * sizeof(uint2));
    const bool digits = tokens > kRankMost;
    w.other = pairs;
    w.counts = digits ? 2 * pairs : pairs;
    w.part = w.counts + (tokens > kSelfMost ? (size_t)(tiles_of(tokens) + 1) * kDigits * 4 : 0);  // a last row when scanned
    w.bytes = w.part + up256((size_t)(tokens / kChunk) * cols * 4);
    return w;
}

template <int Q, bool SELF, bool FIRST, bool I64>
void digit_pass(const EmbeddingArgs& a, int shift, const uint2* in, uint32_t* counts, uint2* out, hipStream_t s) {
    const int64_t tiles = tiles_of(a.tokens);
    const dim3 grid((unsigned)tiles), block(kSortThreads);
    const bool scan = !SELF && tiles > kUnscannedTiles;
    if constexpr (!SELF)
        hipLaunchKernelGGL((digit_count_kernel<Q, FIRST, I64>), grid, block, 0, s, a.tokens, (uint32_t)a.vocab, shift,
                           a.ids, in, counts);
    if (scan)
        hipLaunchKernelGGL(digit_scan_kernel, dim3(kDigits / 64), dim3(64 * kScanWaves), 0, s, tiles, counts);
    hipLaunchKernelGGL((digit_place_kernel<Q, SELF, FIRST, I64>), grid, block, 0, s, a.tokens, (uint32_t)a.vocab,
                       shift, scan, a.ids, in, counts, out);
}

// The sorted pairs, in one of the two arrays.
template <int Q, bool SELF, bool I64>
const uint2* sort_digits(const EmbeddingArgs& a, uint2* to, uint2* other, uint32_t* counts, hipStream_t s) {
    const int passes = digit_passes(a.vocab);
    digit_pass<Q, SELF, true, I64>(a, 0, nullptr, counts, to, s);
    for (int p = 1; p < passes; ++p) {
        digit_pass<Q, SELF, false, I64>(a, p * kDigitBits, to, counts, other, s);
        std::swap(to, other);
    }
    return to;
}

template <bool I64>
const uint2* sort(const EmbeddingArgs& a, const Layout& w, hipStream_t s) {
    uint8_t* ws = (uint8_t*)a.workspace;
    uint2* to = (uint2*)(ws + w.sorted);
    if (a.tokens <= kRankMost) {
        hipLaunchKernelGGL(rank_kernel<I64>, dim3((unsigned)((a.tokens + 63) / 64)), dim3(64 * kRankWaves), 0, s,
                           (int)a.tokens, (uint32_t)a.vocab, a.ids, to);
        return to;
    }
    uint2* other = (uint2*)(ws + w.other);
    uint32_t* counts = (uint32_t*)(ws + w.counts);
    if (a.tokens <= kSelfMost) return sort_digits<2, true, I64>(a, to, other, counts, s);
    return a.tokens <= kShortMost ? sort_digits<2, false, I64>(a, to, other, counts, s)
                                  : sort_digits<8, false, I64>(a, to, other, counts, s);
}

// Rows of the table per group: kRows where that makes 32 groups a CU, fewer of a
// small table, whose rows have many tokens each (lookup and gradient, 15000 tokens into
// 775 x 735 fp32 60 us against 82 with kRows, 30000 into 300 x 512 bf16 43 against 70).
uint32_t rows_per_group(int64_t vocab, int64_t tiles) {
    uint32_t per = kRows;
    while (per > 1 && (vocab + per - 1) / per * tiles < 8192) per /= 2;
    return per;
}

// Whether rows of the gradient start inside cache lines, and the tiles of a row then:
// a row and what its first line has before it.
template <typename G>
bool shifted(const EmbeddingArgs& a) {
    return a.cols * sizeof(G) % 128 != 0 || (uintptr_t)a.dE % 128 != 0;
}
template <typename G>
uint32_t row_tiles(const EmbeddingArgs& a, int64_t width, bool shift) {
    return (uint32_t)((a.cols + (shift ? Part<G, true>::kLine - 1 : 0) + width - 1) / width);
}

template <typename T, typename G, int TL, bool SHIFT>
hipError_t sums(const EmbeddingArgs& a, const uint2* sorted, float* part, hipStream_t s) {
    // fewer groups than 2^32: checked where the call is
    constexpr int N = kUnit<G>;
    const uint32_t tiles = (uint32_t)((a.cols + TL * N - 1) / (TL * N));
    const uint32_t chunks = (uint32_t)(a.tokens / kChunk);
    const int64_t per = NT / TL;
    const int64_t chunk_blocks = ((int64_t)chunks * tiles + per - 1) / per;
    const uint32_t wide = row_tiles<G>(a, TL * N, SHIFT), rows = rows_per_group(a.vocab, wide);
    const int64_t row_blocks = ((a.vocab + rows - 1) / rows * wide + per - 1) / per;
    if (chunks > 0)
        hipLaunchKernelGGL((chunk_kernel<T, N, TL>), grid_of(chunk_blocks), dim3(NT), 0, s, chunks,
                           (uint32_t)a.vocab, a.cols, tiles, sorted, (const T*)a.dY, part);
    hipLaunchKernelGGL((rows_kernel<T, G, TL, SHIFT>), grid_of(row_blocks), dim3(NT), 0, s, (uint32_t)a.tokens,
                       (uint32_t)a.vocab, a.cols, wide, rows, a.scale, sorted, (const T*)a.dY, part, (G*)a.dE);
    return hipGetLastError();
}

template <typename T, typename G>
hipError_t backward(const EmbeddingArgs& a, hipStream_t s) {
    if (a.tokens <= kFewMost) {
        const bool shift = shifted<G>(a);
        const uint32_t tiles = row_tiles<G>(a, 64 * kUnit<G>, shift);
        const uint32_t per = rows_per_group(a.vocab, tiles);
        const int64_t blocks = ((a.vocab + per - 1) / per * tiles + NT / 64 - 1) / (NT / 64);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid_of(blocks), dim3(NT), 0, s, (int)a.tokens, (uint32_t)a.vocab, a.cols, tiles, per,
                               a.scale, a.ids, (const T*)a.dY, (G*)a.dE);
        };
        if (shift) launch(a.index64 ? rows_few_kernel<T, G, true, true> : rows_few_kernel<T, G, false, true>);
        else launch(a.index64 ? rows_few_kernel<T, G, true, false> : rows_few_kernel<T, G, false, false>);
        return hipGetLastError();
    }
    const Layout w = layout_of(a.tokens, a.cols);
    const uint2* sorted = a.index64 ? sort<true>(a, w, s) : sort<false>(a, w, s);
    float* part = (float*)((uint8_t*)a.workspace + w.part);
    const int64_t units = (a.cols + kUnit<G> - 1) / kUnit<G>;
    if (units <= 8) return sums<T, G, 8, false>(a, sorted, part, s);
    if (units <= 16) return sums<T, G, 16, false>(a, sorted, part, s);
    return shifted<G>(a) ? sums<T, G, 64, true>(a, sorted, part, s) : sums<T, G, 64, false>(a, sorted, part, s);
}

template <typename T>
hipError_t forward(const EmbeddingArgs& a, hipStream_t s) {
    const uint32_t units = (uint32_t)((a.cols + kUnit<T> - 1) / kUnit<T>);
    const int64_t blocks = (a.tokens * units + NT - 1) / NT, most = 16 * (int64_t)256;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (a.index64)
        hipLaunchKernelGGL((lookup_kernel<T, true>), grid, dim3(NT), 0, s, a.tokens, (uint32_t)a.vocab,
                           (uint32_t)a.cols, units, a.scale, a.ids, (const T*)a.E, (T*)a.Y);
    else
        hipLaunchKernelGGL((lookup_kernel<T, false>), grid, dim3(NT), 0, s, a.tokens, (uint32_t)a.vocab,
                           (uint32_t)a.cols, units, a.scale, a.ids, (const T*)a.E, (T*)a.Y);
    return hipGetLastError();
}

}  // namespace

bool embedding_groups_fit(int64_t tokens, int64_t vocab, int64_t cols) {
    const int64_t rows = std::max((vocab + kRows - 1) / kRows, tokens / kChunk);
    // tiles of 256 columns at least, one more for the line that a row starts in; narrower groups have one
    return ((cols + 255) / 256 + 1) * rows < (int64_t)1 << 31;
}

size_t embedding_workspace_bytes(int64_t tokens, int64_t, int64_t cols) { return layout_of(tokens, cols).bytes; }

hipError_t launch_embedding_forward(const EmbeddingArgs& a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    return bf16 ? forward<__bf16>(a, s) : forward<float>(a, s);
}

hipError_t launch_embedding_backward(const EmbeddingArgs& a, bool bf16, hipStream_t s) {
    if (bf16) return a.grad_bf16 ? backward<__bf16, __bf16>(a, s) : backward<__bf16, float>(a, s);
    return a.grad_bf16 ? backward<float, __bf16>(a, s) : backward<float, float>(a, s);
}

}  // namespace train
}  // namespace lors
