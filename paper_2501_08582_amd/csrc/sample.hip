// Tokens out of logits: temperature, top-k, top-p, min-p, one given random number a row.
//
// One workgroup a row, in passes over it (the later ones out of the L2):
//   1  the largest logit and its first place, and whether the row has a distribution
//   2  with top-k or top-p: counts and weights w = exp((z - max) / T) by bins of z
//   3  the elements of the bin that holds the border, sorted: the last kept entry
//   4  sums of the kept weights by runs of entries in their order; the run that holds
//      u times the whole, and in it the token
// Every filter keeps a run of one order (logit, then index), so what is kept is
// what stands no later in it than one entry: a 64-bit number each, the ordered bits of
// the logit above the inverted index.  Equal logits need no case of their own.
// Bins hold fixed-point sums, whose order of addition does not matter, each in a unit of
// its own weights' size, so that a far tail counts as exactly as the head; the sums over bins and
// those of pass 4 are fp64 in a fixed order.  A bin of more entries than are sorted at a time is cut
// again, by those numbers.
// Rows of bf16 (sample_values) need no sort: 11777 values hold every logit but those below
// 2^-30 and from 2^16 on (rows with such take the passes above), so that
//   A  counts each value's entries in LDS; from the counts, a weight per value (one exp each,
//      not one an entry), the filters' border and how many entries of its value are kept
//   B  sums the kept weights by runs, as pass 4, out of the table of weights
// The row is read twice and sorted never.
//
// One workgroup a row, because the passes wait for each other: a second launch or a grid's
// barrier costs what splitting a row would save.  Bound by that workgroup's own work: 131072
// entries alone 37 us (about a third each of A, the border, B and the end), 256 such rows, one to a
// compute unit, 47 (67 MB: 14 at a copy's rate); 37 rows of 50021 fp32 with top-p 59, whose fixed-point
// sums take a 64-bit exp an entry, 46 with top-k alone.  1024 lanes leave 128 registers each, of which the
// bf16 kernel, with the passes for other rows in it, spills 36 and the fp32 one 7.  A row of bf16 with
// one entry outside the table's values takes those passes: 84 us alone, 256 of 131072 entries 206.
#include "block_kernels.hpp"
#include "train_common.hpp"

namespace lors {
namespace block {
namespace {

constexpr int NT = 1024;
constexpr int kWaves = NT / 64;
constexpr int kBins = 2 * NT;
constexpr int kSorted = NT;   // entries that are sorted at a time
constexpr int kRuns = 1024;   // at most, of pass 4
constexpr float kBinsPerNat = 64.f;

// The order of a logit: larger for larger ones; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t place_of(float z, uint32_t i) { return (uint64_t)order_of(z) << 32 | (uint32_t)~i; }

struct Shared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t list[kSorted];
    double runs[kRuns];
    uint64_t wave64[2 * kWaves];
    uint64_t found[3];
    double whole, before;
    uint32_t listed;
    int bin;
};

// Inclusive sums over the workgroup's threads of a and b.
template <class A, class B>
__device__ __forceinline__ void scan2(A& a, B& b, Shared& s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const A x = __shfl_up(a, o);
        const B y = __shfl_up(b, o);
        if (lane >= o) {
            a += x;
            b += y;
        }
    }
    __syncthreads();
    A* wa = (A*)s.wave64;
    B* wb = (B*)(s.wave64 + kWaves);
    if (lane == 63) {
        wa[wave] = a;
        wb[wave] = b;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        a += wa[w];
        b += wb[w];
    }
}

// s.list descending; n entries, the others 0 and at its end.
__device__ __forceinline__ void sort_list(Shared& s, uint32_t n) {
    const int tid = threadIdx.x;
    if (tid >= (int)n) s.list[tid] = 0;
    const uint32_t size = n <= 2 ? 2 : 1u << (32 - __clz((int)(n - 1)));
    for (uint32_t w = 2; w <= size; w <<= 1)
        for (uint32_t o = w >> 1; o > 0; o >>= 1) {
            __syncthreads();
            const int j = tid ^ (int)o;
            if (j > tid && tid < (int)size) {
                const uint64_t x = s.list[tid], y = s.list[j];
                if ((x < y) == (w == size || (tid & w) == 0)) {
                    s.list[tid] = y;
                    s.list[j] = x;
                }
            }
        }
    __syncthreads();
}

// 2^t for t <= 0, to 2^-46 of its value: 2^f on |f| <= 1/2 by its Taylor series (the next
// term is 2^-47).  A weight takes this many 64-bit operations, 14, of about 45 that a
// division and the library's exp take.  Times 2^more.
__device__ __forceinline__ double power_of_two(double t, int more = 0) {
    if (!(t > -1080.)) return 0.;  // (below every number: half of the least is 2^-1075)
    const double n = rint(t), x = (t - n) * 0.693147180559945309417;
    double y = 1. / 39916800.;
    y = fma(y, x, 1. / 3628800.);
    y = fma(y, x, 1. / 362880.);
    y = fma(y, x, 1. / 40320.);
    y = fma(y, x, 1. / 5040.);
    y = fma(y, x, 1. / 720.);
    y = fma(y, x, 1. / 120.);
    y = fma(y, x, 1. / 24.);
    y = fma(y, x, 1. / 6.);
    y = fma(y, x, 0.5);
    y = fma(y, x, 1.);
    y = fma(y, x, 1.);
    return ldexp(y, (int)n + more);
}

template <typename T>
struct Row {
    static constexpr int U = train::kUnit<T>;
    static constexpr int AHEAD = 4;  // units in flight in a lane
    const T* at;
    uint32_t V;
    // Unit i of U entries, and how many of them exist.  One past the row reads the last whole
    // unit: no load stands behind a branch, and all of a turn are in flight together.
    __device__ __forceinline__ train::Raw<T, U> unit(uint32_t i, int& n) const {
        const uint32_t units = V / U;
        n = i < units ? U : i == units ? (int)(V % U) : 0;
        if (units == 0) return train::Raw<T, U>{};
        return train::load_whole<T, U>(at + (uint64_t)(i < units ? i : units - 1) * U);
    }
    // (the row's last, where it is not whole)
    __device__ __forceinline__ void edge(int n, train::Raw<T, U>& raw) const {
        if (n > 0 && n < U) raw = train::load_unit<T, U>(at + (uint64_t)(V / U) * U, n);
    }
    // f(logit, index, whether it exists) over the elements of this thread, every lane of a
    // wave at the same time
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        const uint32_t wave0 = threadIdx.x & ~63u, all = (V + U - 1) / U;
        for (uint32_t i0 = 0; i0 + wave0 < all; i0 += AHEAD * NT) {
            train::Raw<T, U> raw[AHEAD];
            int n[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) raw[q] = unit(i0 + q * NT + threadIdx.x, n[q]);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const uint32_t i = (i0 + q * NT + threadIdx.x) * U;  // (of one that exists: below 2^31)
                edge(n[q], raw[q]);
                const train::F<U> z = train::widen<T, U>(raw[q]);
#pragma unroll
                for (int e = 0; e < U; ++e) f(z.v[e], i + e, e < n[q]);
            }
        }
    }
};

// Appends q of the lanes that hold one: one addition a wave.  s.listed counts all, the
// list holds the first kSorted.
__device__ __forceinline__ void append(Shared& s, bool some, uint64_t q) {
    const uint64_t mask = __ballot(some);
    if (mask == 0) return;
    const int lane = threadIdx.x & 63, leader = __ffsll((unsigned long long)mask) - 1;
    uint32_t at = 0;
    if (lane == leader) at = atomicAdd(&s.listed, (uint32_t)__popcll(mask));
    at = __shfl(at, leader) + __popcll(mask & ((1ull << lane) - 1));
    if (some && at < kSorted) s.list[at] = q;
}

// Any logits: passes as above.
template <typename T>
__device__ __forceinline__ void sample_row(const SampleArgs& a, int64_t n, Shared& s) {
    constexpr int U = Row<T>::U;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Row<T> row{(const T*)a.logits + n * a.row_stride, (uint32_t)a.vocab};
    const double T0 = a.temperatures != nullptr ? (double)a.temperatures[n] : a.temperature;
    const int64_t k0 = a.top_ks != nullptr ? a.top_ks[n] : a.top_k;
    const double p0 = a.top_ps != nullptr ? (double)a.top_ps[n] : a.top_p;
    const double low0 = a.min_ps != nullptr ? (double)a.min_ps[n] : a.min_p;
    const double low = low0 > 0. ? low0 : 0.;  // (NaN: none)
    const double u = (double)a.u[n];

    // ---- pass 1
    uint64_t best = 0;
    bool broken = false;  // NaN or +Inf
    row.each([&](float z, uint32_t i, bool some) {
        broken |= some && !(z < INFINITY);
        const uint64_t q = some ? place_of(z, i) : 0;
        best = q > best ? q : best;
    });
    if (broken) best = ~0ull;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t x = __shfl_xor(best, o);
        best = x > best ? x : best;
    }
    if (lane == 0) s.wave64[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = s.wave64[w] > best ? s.wave64[w] : best;
    const float top = logit_of((uint32_t)(best >> 32));
    const bool none = best == ~0ull || !(top > -INFINITY);
    if (none || !(T0 > 0.) || k0 == 1 || low > 1.) {
        if (tid == 0) {
            a.token[n] = none ? -1 : (int64_t)(uint32_t)~(uint32_t)best;
            if (a.logp != nullptr) a.logp[n] = none ? NAN : 0.f;
        }
        return;
    }
    // (bounded: the largest logit itself has the weight 1 at any temperature)
    const double topd = (double)top, rate = fmin(1.44269504088896340736 / T0, 1e300);
    // (finite z; T0 of Inf gives every one the same)
    auto weight = [&](float z) { return power_of_two(((double)z - topd) * rate); };

    // ---- passes 2 and 3: the last kept place
    uint64_t last = 0;  // everything
    const uint64_t k = k0 > 0 && k0 < (int64_t)row.V ? (uint64_t)k0 : 0;
    const bool by_mass = p0 < 1.;
    if (k != 0 || by_mass) {
        // A weight of bin b is below 2^-raise(b) (by 2^-16 of it at most above), and the integers of
        // a bin are its weights times 2^(bits + raise(b)): their sum stays below 2^63, and an
        // entry's rounding is 2^-bits of it.  The last bin's entries may be smaller: those that
        // round to nothing are 2^-78 or less (at temperatures above 2^-120, below which `per` is cut).
        const int bits = 62 - (32 - __clz((int)row.V));
        auto raise = [](int b) { return b * 1477 >> 16; };  // b / kBinsPerNat nats in powers of two, rounded down
        auto fixed = [&](float z, int up) {
            return z > -INFINITY ? (uint64_t)(power_of_two(((double)z - topd) * rate, bits + up) + 0.5) : 0ull;
        };
        // (halves: no difference of them overflows; finite: the largest logit's bin is 0)
        const float per = fminf((float)(2. * kBinsPerNat / T0), 3e38f);
        // the entries in [lo, hi] by a level of bins; the first level goes by the logits
        uint64_t lo = 0, hi = ~0ull;
        auto bin_of = [&](float z, uint64_t q, int shift) {
            if (shift < 0) {
                const float y = (0.5f * top - 0.5f * z) * per;  // no later for larger logits
                return y < (float)(kBins - 1) ? (int)y : kBins - 1;
            }
            return (int)((hi - q) >> shift);
        };
        for (int filter = k != 0 ? 0 : 1; filter < (by_mass ? 2 : 1); ++filter) {
            // the border: of the entries in their order, the first k, or those before which
            // less than `goal` lies.  The first filter needs no weights (a 64-bit exp an entry: the
            // second takes those of what the first kept), the second no counts: bins of
            // no weight hold nothing that it keeps.
            const bool counts = filter == 0;
            const uint64_t from = last;
            lo = 0;
            hi = ~0ull;
            int shift = -1, up = 0;  // up: of all entries in [lo, hi], behind the first level
            uint64_t count0 = 0;
            double mass0 = 0., goal = 0.;
            uint32_t listed = 0;
            for (;;) {
                for (int b = tid; b < kBins; b += NT) {
                    s.mass[b] = 0;
                    s.count[b] = 0;
                }
                if (tid == 0) {
                    s.listed = 0;
                    s.bin = -1;
                    s.found[0] = ~0ull;
                    s.found[1] = 0;
                }
                __syncthreads();
                row.each([&](float z, uint32_t i, bool some) {
                    const uint64_t q = place_of(z, i);
                    if (!some || q < lo || q > hi || q < from) return;
                    const int b = bin_of(z, q, shift);
                    if (counts) atomicAdd(&s.count[b], 1u);
                    else atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)fixed(z, shift < 0 ? raise(b) : up));
                });
                __syncthreads();
                const uint32_t c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
                auto mass_of = [&](int b) { return ldexp((double)s.mass[b], -bits - (shift < 0 ? raise(b) : up)); };
                const double m0 = counts ? 0. : mass_of(2 * tid), m1 = counts ? 0. : mass_of(2 * tid + 1), both = m0 + m1;
                uint64_t c = (uint64_t)c0 + c1;
                double m = both;
                scan2(c, m, s);
                if (filter == 1 && shift < 0) {  // the whole of what is kept so far
                    __syncthreads();
                    if (tid == NT - 1) s.whole = m;
                    __syncthreads();
                    goal = p0 * s.whole;
                    __syncthreads();
                }
                // the border's bin: the last that is not empty and in front of which too little lies
                const uint64_t cb[2] = {count0 + c - c0 - c1, count0 + c - c1};
                const double mb0 = mass0 + (m - both), mb[2] = {mb0, mb0 + m0};
                const bool in0 = counts ? c0 != 0 && cb[0] < k : m0 != 0. && (mb[0] < goal || mb[0] == 0.);
                const bool in1 = counts ? c1 != 0 && cb[1] < k : m1 != 0. && (mb[1] < goal || mb[1] == 0.);
                if (in0 || in1) atomicMax(&s.bin, 2 * tid + (in1 ? 1 : 0));
                __syncthreads();
                const int bin = s.bin;
                if (2 * tid == (bin & ~1)) {
                    s.found[2] = cb[bin & 1];
                    s.before = mb[bin & 1];
                }
                __syncthreads();
                const uint64_t inside = counts ? s.count[bin] : 0;
                // top-k of few: all up to the border, which the rest is found among
                const bool whole = counts && shift < 0 && s.found[2] + inside <= kSorted;
                row.each([&](float z, uint32_t i, bool some) {
                    const uint64_t q = place_of(z, i);
                    bool in = some && q >= lo && q <= hi && q >= from;
                    if (in) {
                        const int b = bin_of(z, q, shift);
                        in = whole ? b <= bin : b == bin;
                    }
                    append(s, in, q);
                });
                __syncthreads();
                listed = s.listed;
                if (whole) {
                    sort_list(s, listed);
                    // entry `tid` of the order; what top-k, top-p and min-p keep of it
                    const uint64_t q = s.list[tid];
                    const float z = logit_of((uint32_t)(q >> 32));
                    const bool first_k = tid < (int)listed && (uint64_t)tid < k && z > -INFINITY;
                    const double w = first_k ? weight(z) : 0.;
                    double sum = w;
                    uint64_t nothing = 0;
                    scan2(nothing, sum, s);
                    __syncthreads();
                    if (tid == NT - 1) s.whole = sum;
                    __syncthreads();
                    const double limit = p0 * s.whole;
                    const bool in = first_k && w >= low && (!by_mass || sum - w < limit || tid == 0);
                    if (tid == 0) s.bin = NT;
                    __syncthreads();
                    if (!in) atomicMin(&s.bin, tid);
                    s.runs[tid] = w;
                    __syncthreads();
                    const int kept_n = s.bin;  // the first entries of the order
                    // by index: the list holds the inverted index above the place in the order
                    s.list[tid] = (q & 0xFFFFFFFFull) << 32 | (uint32_t)tid;
                    __syncthreads();
                    sort_list(s, (uint32_t)kept_n);
                    const uint64_t e = s.list[tid];
                    const bool some = tid < kept_n;
                    const double mine = some ? s.runs[(uint32_t)e] : 0.;
                    double upto = mine;
                    scan2(upto, nothing, s);
                    __syncthreads();
                    if (tid == NT - 1) s.runs[0] = upto;
                    if (tid == 0) s.bin = kSorted;
                    __syncthreads();
                    const double all = s.runs[0];
                    if (some && mine > 0. && upto > u * all) atomicMin(&s.bin, tid);
                    __syncthreads();
                    if (s.bin == kSorted) {  // none exceeds it: the last of positive weight
                        __syncthreads();
                        if (tid == 0) s.bin = -1;
                        __syncthreads();
                        if (mine > 0.) atomicMax(&s.bin, tid);
                        __syncthreads();
                    }
                    if (tid == s.bin) {
                        a.token[n] = (int64_t)(uint32_t)~(uint32_t)(e >> 32);
                        if (a.logp != nullptr) a.logp[n] = (float)log(mine / all);
                    }
                    return;
                }
                count0 = s.found[2];
                mass0 = s.before;
                if (shift < 0) up = raise(bin);
                if (listed <= kSorted) break;
                // too many: their range, and another level
                uint64_t least = ~0ull, most = 0;
                row.each([&](float z, uint32_t i, bool some) {
                    const uint64_t q = place_of(z, i);
                    if (!some || q < lo || q > hi || q < from || bin_of(z, q, shift) != bin) return;
                    least = q < least ? q : least;
                    most = q > most ? q : most;
                });
                atomicMin((unsigned long long*)&s.found[0], (unsigned long long)least);
                atomicMax((unsigned long long*)&s.found[1], (unsigned long long)most);
                __syncthreads();
                lo = s.found[0];
                hi = s.found[1];
                const uint64_t range = hi - lo;  // above kSorted
                shift = 64 - __clzll((long long)range) - 11;
                if (shift < 0) shift = 0;
                __syncthreads();
            }
            sort_list(s, listed);
            const uint64_t q = s.list[tid];
            const bool some = tid < (int)listed;
            const float z = logit_of((uint32_t)(q >> 32));
            const double own = some && !counts && z > -INFINITY ? weight(z) : 0.;
            uint64_t c = some ? 1 : 0;
            double m = own;
            scan2(c, m, s);
            const double ahead = mass0 + (m - own);
            const bool in = some && (counts ? count0 + c - 1 < k : ahead < goal || ahead == 0.);
            if (tid == 0) s.bin = -1;
            __syncthreads();
            if (in) atomicMax(&s.bin, tid);
            __syncthreads();
            if (s.bin == tid) s.found[0] = q;
            __syncthreads();
            last = s.found[0];
            __syncthreads();
        }
    }

    // ---- pass 4
    constexpr int AHEAD = Row<T>::AHEAD;
    const uint64_t blocks = ((uint64_t)row.V + 64 * U - 1) / (64 * U);
    const uint32_t reps = (uint32_t)((blocks + kRuns - 1) / kRuns);  // blocks of a run
    const int runs = (int)((blocks + reps - 1) / reps);
    auto kept = [&](float z, uint32_t i) {
        if (!(z > -INFINITY) || place_of(z, i) < last) return 0.;
        const double w = weight(z);
        return w >= low ? w : 0.;
    };
    // this lane's U elements of a block, and their weights
    auto load = [&](uint64_t block, int& m) {
        train::Raw<T, U> raw = row.unit((uint32_t)(block * 64 + lane), m);
        row.edge(m, raw);
        return raw;
    };
    auto weigh = [&](const train::Raw<T, U>& raw, int m, uint64_t block, double (&w)[U]) {
        const train::F<U> z = train::widen<T, U>(raw);
#pragma unroll
        for (int e = 0; e < U; ++e) w[e] = e < m ? kept(z.v[e], (uint32_t)((block * 64 + lane) * U) + e) : 0.;
    };
    for (int r0 = wave; r0 < runs; r0 += AHEAD * kWaves) {
        double sum[AHEAD] = {};
        for (uint32_t b = 0; b < reps; ++b) {
            train::Raw<T, U> raw[AHEAD];
            int m[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const uint32_t block = (r0 + q * kWaves) * reps + b;  // (of a run past the last: past the row)
                raw[q] = row.unit(block * 64 + lane, m[q]);
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                double w[U];
                row.edge(m[q], raw[q]);
                weigh(raw[q], m[q], (uint64_t)(r0 + q * kWaves) * reps + b, w);
#pragma unroll
                for (int e = 0; e < U; ++e) sum[q] += w[e];
            }
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1)
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) sum[q] += __shfl_xor(sum[q], o);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
            if (lane == 0 && r0 + q * kWaves < runs) s.runs[r0 + q * kWaves] = sum[q];
    }
    __syncthreads();
    if (wave != 0) return;
    // sums before each run: up to 16 consecutive ones a lane
    const int per_lane = (runs + 63) / 64;
    double part = 0.;
    for (int e = 0; e < per_lane; ++e) {
        const int r = lane * per_lane + e;
        if (r < runs) part += s.runs[r];
    }
    double upto_lane = part;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double x = __shfl_up(upto_lane, o);
        if (lane >= o) upto_lane += x;
    }
    const double whole = __shfl(upto_lane, 63);
    const double goal = u * whole;
    // the first run at whose end the sum exceeds the goal; else the last of positive weight
    int first = runs, positive = -1;
    double base = 0., run = __shfl_up(upto_lane, 1);
    if (lane == 0) run = 0.;
    double at_first = 0.;
    for (int e = 0; e < per_lane; ++e) {
        const int r = lane * per_lane + e;
        if (r >= runs) break;
        const double w = s.runs[r];
        if (w > 0.) positive = r;
        if (first == runs && run + w > goal && w > 0.) {
            first = r;
            at_first = run;
        }
        run += w;
    }
    int chosen = first;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_xor(chosen, o), y = __shfl_xor(positive, o);
        chosen = x < chosen ? x : chosen;
        positive = y > positive ? y : positive;
    }
    const bool over = chosen == runs;  // u times the whole is not below it
    if (over) chosen = positive;
    const uint64_t owner = __ballot(!over && first == chosen);
    if (owner != 0) base = __shfl(at_first, __ffsll((unsigned long long)owner) - 1);
    int64_t token = -1;
    double weight_of = 0.;
    for (uint32_t b = 0; b < reps; ++b) {
        double w[U];
        int m;
        const uint64_t block = (uint64_t)chosen * reps + b;
        const train::Raw<T, U> raw = load(block, m);
        weigh(raw, m, block, w);
        double sum = 0.;
#pragma unroll
        for (int e = 0; e < U; ++e) sum += w[e];
        double upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        const double end = __shfl(upto, 63);
        double run2 = base + (upto - sum);
        int mine = -1, final_ = -1;
        double wm = 0., wf = 0.;
#pragma unroll
        for (int e = 0; e < U; ++e) {
            run2 += w[e];
            if (w[e] > 0.) {
                final_ = e;
                wf = w[e];
                if (mine < 0 && run2 > goal) {
                    mine = e;
                    wm = w[e];
                }
            }
        }
        const uint64_t hit = over ? 0 : __ballot(mine >= 0), some = __ballot(final_ >= 0);
        if (hit != 0) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            token = (int64_t)((block * 64 + l) * U) + __shfl(mine, l);
            weight_of = __shfl(wm, l);
            break;
        }
        if (some != 0) {  // where no entry exceeds the goal, the last one
            const int l = 63 - __clzll((long long)some);
            token = (int64_t)((block * 64 + l) * U) + __shfl(final_, l);
            weight_of = __shfl(wf, l);
        }
        base += end;
    }
    if (lane == 0) {
        a.token[n] = token;
        if (a.logp != nullptr) a.logp[n] = (float)log(weight_of / whole);
    }
}

// bf16 logits of 2^-30 <= |z| < 2^16, 0 and -Inf: few enough values to count the entries of
// each, which takes no arithmetic an entry, no search and no sort:
//   A  counts by value; with them the largest, the weights, the borders of every filter and
//      the kept weight, all on the values; a border that cuts a value's entries keeps the
//      first of them by index
//   B  sums of the kept entries' weights (out of a table) by runs, and the token
struct Values {
    static constexpr int kLeast = (127 - 30) << 7, kSpan = 46 << 7;  // magnitudes' bits
    static constexpr int kZero = kSpan, kEach = (2 * kSpan + NT) / NT, kCount = kEach * NT;
    double weight[kCount];
    uint32_t count[kCount];
    double runs[kRuns + kRuns / 16];  // run r at r + r / 16: 16 consecutive ones a lane, on other banks
    uint32_t ties[kRuns + kRuns / 16];
    static __device__ __forceinline__ int place(int r) { return r + (r >> 4); }
    uint64_t wave64[2 * kWaves];
    double mass;
    uint32_t before;
    int first, border, quota, odd;
    // descending: the larger values first; -1: -Inf, -2: not one of these values
    static __device__ __forceinline__ int bin_of(uint32_t b) {
        const uint32_t m = b & 0x7FFFu, d = m - kLeast;
        if (d < (uint32_t)kSpan) return (b & 0x8000u) ? kZero + 1 + (int)d : kZero - 1 - (int)d;
        return m == 0 ? kZero : b == 0xFF80u ? -1 : -2;
    }
    // The same of two logits, 16 bits each, where both lie in the span; false otherwise.  Packed
    // 16-bit integers: four instructions an entry, of which the passes over a row consist.
    typedef short two __attribute__((ext_vector_type(2)));
    typedef unsigned short utwo __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ bool bins_of(uint32_t b, uint32_t& bins) {
        const utwo m = __builtin_bit_cast(utwo, b & 0x7FFF7FFFu), d = m - (utwo)(unsigned short)kLeast;
        const two neg = __builtin_bit_cast(two, b) >> (two)15;  // -1 for negative ones
        const two t = __builtin_bit_cast(two, d) ^ ~neg;        // ~d or d: kZero - 1 - d, kZero + 1 + d
        bins = __builtin_bit_cast(uint32_t, t - neg + (two)(short)kZero);
        return d[0] < kSpan && d[1] < kSpan;
    }
    static __device__ __forceinline__ float value_of(int bin) {
        const uint32_t m = bin == kZero ? 0u : bin < kZero ? (uint32_t)(kLeast + kZero - 1 - bin) : 0x8000u | (uint32_t)(kLeast + bin - kZero - 1);
        return bf16_bits_to_f32(m);
    }
};
static_assert(Values::kCount > 2 * Values::kSpan, "every value has a bin");
static_assert(sizeof(Values) <= 160 * 1024, "LDS");
static_assert(train::kUnit<uint16_t> == 8, "sums of a unit");

template <class V>
__device__ __forceinline__ void scan_values(double& a, uint64_t& b, V& s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double x = __shfl_up(a, o);
        const uint64_t y = __shfl_up(b, o);
        if (lane >= o) {
            a += x;
            b += y;
        }
    }
    __syncthreads();
    double* wa = (double*)s.wave64;
    if (lane == 63) {
        wa[wave] = a;
        s.wave64[kWaves + wave] = b;
    }
    __syncthreads();
    double pa = 0.;
    for (int w = 0; w < wave; ++w) {
        pa += wa[w];
        b += s.wave64[kWaves + w];
    }
    a += pa;
}

// Sums over a wave's lanes of four values at a time: lane l gets that of value l / 16.  Seven
// exchanges, of which four stay in rows of 16 lanes, against 24 one by one.
template <typename A>
__device__ __forceinline__ A other_lane(A v, int ctrl_step) {  // 0 .. 3: the rows' butterfly
    uint32_t w[sizeof(A) / 4];
    __builtin_memcpy(w, &v, sizeof(A));
#pragma unroll
    for (uint32_t& x : w)
        x = (uint32_t)(ctrl_step == 0   ? __builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true)
                       : ctrl_step == 1 ? __builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true)
                       : ctrl_step == 2 ? __builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true)
                                        : __builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));
    __builtin_memcpy(&v, w, sizeof(A));
    return v;
}
template <typename A>
__device__ __forceinline__ A sum_of_four(const A (&v)[4]) {
    const bool upper = threadIdx.x & 32, odd = threadIdx.x & 16;
    A x = (upper ? v[2] : v[0]) + __shfl_xor(upper ? v[0] : v[2], 32);
    A y = (upper ? v[3] : v[1]) + __shfl_xor(upper ? v[1] : v[3], 32);
    A z = (odd ? y : x) + __shfl_xor(odd ? x : y, 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) z += other_lane(z, k);
    return z;
}

// false (every thread): the row holds other values
__device__ __forceinline__ bool sample_values(const SampleArgs& a, int64_t n, Values& s) {
    using R = Row<uint16_t>;
    constexpr int U = R::U, AHEAD = 4, E = Values::kEach;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t V = (uint32_t)a.vocab;
    const uint16_t* at = (const uint16_t*)a.logits + n * a.row_stride;
    const double T0 = a.temperatures != nullptr ? (double)a.temperatures[n] : a.temperature;
    const int64_t k0 = a.top_ks != nullptr ? a.top_ks[n] : a.top_k;
    const double p0 = a.top_ps != nullptr ? (double)a.top_ps[n] : a.top_p;
    const double low0 = a.min_ps != nullptr ? (double)a.min_ps[n] : a.min_p;
    const double u = (double)a.u[n];

    auto bits_at = [](const train::Raw<uint16_t, U>& raw, int e) {  // (e need not be known: no indexing of registers)
        const uint32_t lo = e & 2 ? raw.w[1] : raw.w[0], hi = e & 2 ? raw.w[3] : raw.w[2];
        return (e & 4 ? hi : lo) >> (16 * (e & 1)) & 0xFFFFu;
    };
    // Units of U entries of the row that exist whole; loads past them read the last one, so that no load
    // stands behind a branch and all of a turn are in flight together.
    const uint32_t units = V / U, left = V % U;
    if (units == 0) return false;
    auto unit = [&](uint32_t i) {
        const uint32_t from = i < units ? i : units - 1;
        return train::load_whole<uint16_t, U>((const uint16_t*)((const uint8_t*)at + from * (uint32_t)(2 * U)));
    };
    // ---- A
    for (int e = tid; e < Values::kCount; e += NT) s.count[e] = 0;
    if (tid == 0) {
        s.odd = 0;
        s.first = Values::kCount;
        s.border = -1;
    }
    __syncthreads();
    bool odd = false;
    for (uint32_t i0 = 0; i0 < units; i0 += AHEAD * NT) {
        train::Raw<uint16_t, U> raw[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) raw[q] = unit(i0 + q * NT + tid);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            if (i0 + q * NT + tid >= units) break;
            uint32_t bins[U / 2];
            bool plain = true;
#pragma unroll
            for (int e = 0; e < U / 2; ++e) plain &= Values::bins_of(raw[q].w[e], bins[e]);
            if (plain) {
#pragma unroll
                for (int e = 0; e < U / 2; ++e) {
                    atomicAdd(&s.count[bins[e] & 0xFFFFu], 1u);
                    atomicAdd(&s.count[bins[e] >> 16], 1u);
                }
            } else {
                for (int e = 0; e < U; ++e) {
                    const int bin = Values::bin_of(bits_at(raw[q], e));
                    if (bin >= 0) atomicAdd(&s.count[bin], 1u);
                    odd |= bin == -2;
                }
            }
        }
    }
    if (tid < left) {
        const int bin = Values::bin_of(at[V - left + tid]);
        if (bin >= 0) atomicAdd(&s.count[bin], 1u);
        odd |= bin == -2;
    }
    if (odd) s.odd = 1;
    __syncthreads();
    if (s.odd) return false;
    // the largest value
    uint32_t c[E];
    int first = Values::kCount;
#pragma unroll
    for (int e = E - 1; e >= 0; --e) {
        c[e] = s.count[E * tid + e];
        if (c[e] != 0) first = E * tid + e;
    }
    if (first < Values::kCount) atomicMin(&s.first, first);
    __syncthreads();
    first = s.first;
    if (first == Values::kCount) {  // -Inf alone
        if (tid == 0) {
            a.token[n] = -1;
            if (a.logp != nullptr) a.logp[n] = NAN;
        }
        return true;
    }
    const bool greedy = !(T0 > 0.) || k0 == 1 || low0 > 1.;
    const double top = (double)Values::value_of(first), rate = greedy ? 0. : fmin(1.44269504088896340736 / T0, 1e300);
    double w[E], mass = 0.;
    uint64_t count = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        w[e] = 0.;
        if (__ballot(c[e] != 0) != 0)  // (most waves' values are not in the row)
            w[e] = c[e] != 0 ? power_of_two(((double)Values::value_of(E * tid + e) - top) * rate) : 0.;
        s.weight[E * tid + e] = w[e];
        mass += (double)c[e] * w[e];
        count += c[e];
    }
    const double own_mass = mass;
    const uint64_t own_count = count;
    scan_values(mass, count, s);
    const double mass0 = mass - own_mass;  // before this thread's values (the same sums in every pass over them)
    const uint64_t count0 = count - own_count;
    // top-k: the value that holds the k-th entry
    const uint64_t k = greedy ? 1 : k0 > 0 && k0 < (int64_t)V ? (uint64_t)k0 : ~0ull;
    auto find = [&](auto test) {  // the last value with entries that passes, and what lies before it
        double m = mass0;
        uint64_t t = count0;
        int mine = -1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (c[e] != 0 && test(m, t, w[e])) mine = e;
            m += (double)c[e] * w[e];
            t += c[e];
        }
        if (mine >= 0) atomicMax(&s.border, E * tid + mine);
        __syncthreads();
        if (s.border / E == tid) {
            m = mass0;
            t = count0;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (E * tid + e < s.border) {
                    m += (double)c[e] * w[e];
                    t += c[e];
                }
            s.mass = m;
            s.before = (uint32_t)t;
        }
        __syncthreads();
    };
    find([&](double, uint64_t t, double) { return t < k; });
    int border = s.border;
    uint64_t quota = k - s.before < s.count[border] ? k - s.before : s.count[border];
    if (p0 < 1. && !greedy) {
        const double goal = p0 * (s.mass + (double)quota * s.weight[border]);
        const int last = border;
        __syncthreads();
        if (tid == 0) s.border = -1;
        __syncthreads();
        find([&](double m, uint64_t t, double) { return m < goal || t == 0; });
        if (s.border < last) {
            border = s.border;
            quota = s.count[border];
        }
        if (s.border <= last) {  // the entries i of it with mass + i w < goal
            const double wb = s.weight[border], m = s.mass;
            double q = ceil((goal - m) / wb);  // right to one entry: its rounding is 2^-52 of at most 2^31
            if (!(m + (q - 1.) * wb < goal)) q -= 1.;
            else if (m + q * wb < goal) q += 1.;
            if (!(q >= 1.)) q = 1.;
            if (q < (double)quota) quota = (uint64_t)q;
        }
    }
    if (low0 > 0. && !greedy) {
        const int last = border;
        __syncthreads();
        if (tid == 0) s.border = -1;
        __syncthreads();
        find([&](double, uint64_t t, double x) { return x >= low0 || t == 0; });
        if (s.border < last) {
            border = s.border;
            quota = s.count[border];
        }
    }
    __syncthreads();
    // entries of the values before `border`, and the first `quota` of its own
    const double wb = s.weight[border];
    if (quota == s.count[border]) {
        ++border;
        quota = 0;
    }
    // what is not kept weighs nothing, so that pass B asks no questions
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (E * tid + e >= border) s.weight[E * tid + e] = 0.;
    __syncthreads();

    // ---- B
    const uint64_t blocks = ((uint64_t)V + 64 * U - 1) / (64 * U);
    const uint32_t reps = (uint32_t)((blocks + kRuns - 1) / kRuns);  // blocks of a run
    const int runs = (int)((blocks + reps - 1) / reps);
    auto load = [&](uint64_t block, int& m) {
        const uint64_t i = (block * 64 + lane) * U;
        m = i < V ? (V - i < U ? (int)(V - i) : U) : 0;
        return train::load_unit<uint16_t, U>(m ? at + i : at, m);
    };
    auto bin_at = [&](const train::Raw<uint16_t, U>& raw, int e, int m) { return e < m ? Values::bin_of(bits_at(raw, e)) : -1; };
    constexpr int BEHIND = 4;  // runs of a wave at a time (sum_of_four)
    for (int r0 = wave; r0 < runs; r0 += BEHIND * kWaves) {
        double sum[BEHIND] = {};
        uint32_t ties[BEHIND] = {};
        for (uint32_t b = 0; b < reps; ++b) {
            // (blocks past the row's, and those of runs past the last, have no unit)
            auto index = [&](int q) { return ((r0 + q * kWaves) * reps + b) * 64u + lane; };
            train::Raw<uint16_t, U> raw[BEHIND];
#pragma unroll
            for (int q = 0; q < BEHIND; ++q) raw[q] = unit(index(q));
#pragma unroll
            for (int q = 0; q < BEHIND; ++q) {
                const uint32_t i = index(q);
                if (i >= units) {
                    for (uint32_t e = 0; i == units && e < left; ++e) {
                        const int bin = Values::bin_of(at[V - left + e]);
                        if (bin >= 0) sum[q] += s.weight[bin];
                        ties[q] += bin == border ? 1 : 0;
                    }
                    continue;
                }
                uint32_t bins[U / 2];
                bool plain = true;
#pragma unroll
                for (int e = 0; e < U / 2; ++e) plain &= Values::bins_of(raw[q].w[e], bins[e]);
                if (plain) {
                    // most entries lie behind the border: a unit of those alone is left out
                    Values::utwo least = __builtin_bit_cast(Values::utwo, bins[0]);
#pragma unroll
                    for (int e = 1; e < U / 2; ++e) least = __builtin_elementwise_min(least, __builtin_bit_cast(Values::utwo, bins[e]));
                    if (least[0] > border && least[1] > border) continue;
                    double x[U];
#pragma unroll
                    for (int e = 0; e < U; ++e) x[e] = s.weight[bins[e >> 1] >> (16 * (e & 1)) & 0xFFFFu];
                    sum[q] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                    if (quota != 0)
#pragma unroll
                        for (int e = 0; e < U; ++e) ties[q] += (int)(bins[e >> 1] >> (16 * (e & 1)) & 0xFFFFu) == border ? 1 : 0;
                } else {
                    for (int e = 0; e < U; ++e) {
                        const int bin = Values::bin_of(bits_at(raw[q], e));
                        if (bin >= 0) sum[q] += s.weight[bin];
                        ties[q] += bin == border ? 1 : 0;
                    }
                }
            }
        }
        const int mine = r0 + (lane >> 4) * kWaves;
        const double all = sum_of_four(sum);
        const uint32_t tied = quota != 0 ? sum_of_four(ties) : 0;
        if ((lane & 15) == 0 && mine < runs) {
            s.runs[Values::place(mine)] = all;
            s.ties[Values::place(mine)] = tied;
        }
    }
    __syncthreads();
    if (wave != 0) return true;
    // sums before each run: up to 16 consecutive ones a lane; a run's ties count while the quota lasts
    const int each = (runs + 63) / 64;
    uint32_t tied = 0;
    for (int e = 0; e < each; ++e) tied += lane * each + e < runs ? s.ties[Values::place(lane * each + e)] : 0;
    uint64_t ties0 = tied;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up(ties0, o);
        if (lane >= o) ties0 += x;
    }
    ties0 -= tied;
    auto of_run = [&](int r, uint64_t& t) {
        const uint64_t left = t < quota ? quota - t : 0, here = s.ties[Values::place(r)];
        t += here;
        return s.runs[Values::place(r)] + (double)(left < here ? left : here) * wb;
    };
    double part = 0.;
    uint64_t t = ties0;
    for (int e = 0; e < each; ++e)
        if (lane * each + e < runs) part += of_run(lane * each + e, t);
    double upto_lane = part;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double x = __shfl_up(upto_lane, o);
        if (lane >= o) upto_lane += x;
    }
    const double whole = __shfl(upto_lane, 63), goal = u * whole;
    double run = __shfl_up(upto_lane, 1), base = 0.;
    if (lane == 0) run = 0.;
    int chosen = runs, positive = -1;
    double at_first = 0.;
    uint64_t ties_first = 0, ties_last = 0;
    t = ties0;
    for (int e = 0; e < each; ++e) {
        const int r = lane * each + e;
        if (r >= runs) break;
        const uint64_t before = t;
        const double x = of_run(r, t);
        if (x > 0.) {
            positive = r;
            ties_last = before;
            if (chosen == runs && run + x > goal) {
                chosen = r;
                at_first = run;
                ties_first = before;
            }
        }
        run += x;
    }
    int best = chosen, end_run = positive;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_xor(best, o), y = __shfl_xor(end_run, o);
        best = x < best ? x : best;
        end_run = y > end_run ? y : end_run;
    }
    const bool over = best == runs;  // u times the whole is not below it: the last entry of weight
    const uint64_t owner = __ballot(over ? positive == end_run : chosen == best);
    const int who = __ffsll((unsigned long long)owner) - 1;
    base = __shfl(at_first, who);
    uint64_t seen = __shfl(over ? ties_last : ties_first, who);
    if (over) best = end_run;
    int64_t token = -1;
    double weight_of = 0.;
    for (uint32_t b = 0; b < reps; ++b) {
        int m;
        const uint64_t block = (uint64_t)best * reps + b;
        const train::Raw<uint16_t, U> raw = load(block, m);
        uint32_t own = 0;
#pragma unroll
        for (int e = 0; e < U; ++e) own += bin_at(raw, e, m) == border ? 1 : 0;
        uint32_t upto_ties = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(upto_ties, o);
            if (lane >= o) upto_ties += x;
        }
        uint64_t rank = seen + upto_ties - own;
        double x[U], sum = 0.;
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int bin = bin_at(raw, e, m);
            x[e] = bin >= 0 && bin < border ? s.weight[bin] : bin == border && rank < quota ? wb : 0.;
            rank += bin == border ? 1 : 0;
            sum += x[e];
        }
        seen += __shfl(upto_ties, 63);
        double upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double y = __shfl_up(upto, o);
            if (lane >= o) upto += y;
        }
        const double end = __shfl(upto, 63);
        double run2 = base + (upto - sum);
        int mine = -1, final_ = -1;
        double wm = 0., wf = 0.;
#pragma unroll
        for (int e = 0; e < U; ++e) {
            run2 += x[e];
            if (x[e] > 0.) {
                final_ = e;
                wf = x[e];
                if (mine < 0 && run2 > goal) {
                    mine = e;
                    wm = x[e];
                }
            }
        }
        const uint64_t hit = over ? 0 : __ballot(mine >= 0), some = __ballot(final_ >= 0);
        if (hit != 0) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            token = (int64_t)((block * 64 + l) * U) + __shfl(mine, l);
            weight_of = __shfl(wm, l);
            break;
        }
        if (some != 0) {  // where no entry exceeds the goal, the last one
            const int l = 63 - __clzll((long long)some);
            token = (int64_t)((block * 64 + l) * U) + __shfl(final_, l);
            weight_of = __shfl(wf, l);
        }
        base += end;
    }
    if (lane == 0) {
        a.token[n] = token;
        if (a.logp != nullptr) a.logp[n] = (float)log(weight_of / whole);
    }
    return true;
}

template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
    const int64_t n = train::block_id();
    if (n >= a.rows) return;
    if constexpr (sizeof(T) == 2) {
        __shared__ union {
            Values v;
            Shared s;
        } m;
        if (sample_values(a, n, m.v)) return;
        __syncthreads();
        sample_row<T>(a, n, m.s);
    } else {
        __shared__ Shared s;
        sample_row<T>(a, n, s);
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    const dim3 grid = train::grid_of(a.rows);
    if (bf16) hipLaunchKernelGGL(sample_kernel<uint16_t>, grid, dim3(NT), 0, s, a);
    else hipLaunchKernelGGL(sample_kernel<float>, grid, dim3(NT), 0, s, a);
    return hipGetLastError();
}

}  // namespace block
}  // namespace lors
