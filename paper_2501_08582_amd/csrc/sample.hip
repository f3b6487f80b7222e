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
// Bins hold fixed-point sums, whose order of addition does not matter; the sums of pass 4
// are fp64 in a fixed order.  A bin of more entries than are sorted at a time is cut again,
// by those numbers.
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
    uint64_t found[4];
    uint32_t listed;
    int bin;
};

// Inclusive sums over the workgroup's threads of a and b.
__device__ __forceinline__ void scan2(uint64_t& a, uint64_t& b, Shared& s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up(a, o), y = __shfl_up(b, o);
        if (lane >= o) {
            a += x;
            b += y;
        }
    }
    __syncthreads();
    if (lane == 63) {
        s.wave64[wave] = a;
        s.wave64[kWaves + wave] = b;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        a += s.wave64[w];
        b += s.wave64[kWaves + w];
    }
}

template <typename T>
struct Row {
    static constexpr int U = train::kUnit<T>;
    const T* at;
    uint32_t V;
    // f(logit, index) over the elements of this thread
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        for (uint64_t i = (uint64_t)threadIdx.x * U; i < V; i += (uint64_t)NT * U) {
            const int n = V - i < U ? (int)(V - i) : U;
            const train::F<U> z = train::widen<T, U>(train::load_unit<T, U>(at + i, n));
#pragma unroll
            for (int e = 0; e < U; ++e)
                if (e < n) f(z.v[e], (uint32_t)i + e);
        }
    }
};

template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
    __shared__ Shared s;
    constexpr int U = Row<T>::U;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t n = train::block_id();
    if (n >= a.rows) return;
    const Row<T> row{(const T*)a.logits + n * a.row_stride, (uint32_t)a.vocab};
    const double T0 = a.temperatures != nullptr ? (double)a.temperatures[n] : a.temperature;
    const int64_t k0 = a.top_ks != nullptr ? a.top_ks[n] : a.top_k;
    const double p0 = a.top_ps != nullptr ? (double)a.top_ps[n] : a.top_p;
    const double low0 = a.min_ps != nullptr ? (double)a.min_ps[n] : a.min_p;
    const double low = low0 > 0. ? low0 : 0.;  // (NaN: none)

    // ---- pass 1
    uint64_t best = 0;
    bool broken = false;  // NaN or +Inf
    row.each([&](float z, uint32_t i) {
        broken |= !(z < INFINITY);
        const uint64_t q = place_of(z, i);
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
    const double topd = (double)top;
    auto weight = [&](float z) { return exp(((double)z - topd) / T0); };

    // ---- passes 2 and 3: the last kept place
    uint64_t last = 0;  // everything
    const uint64_t k = k0 > 0 && k0 < (int64_t)row.V ? (uint64_t)k0 : 0;
    const bool by_mass = p0 < 1.;
    if (k != 0 || by_mass) {
        const int bits = 62 - (32 - __clz((int)row.V));  // of a fixed-point weight: their sum stays below 2^62
        const double unit = ldexp(1., bits);
        auto fixed = [&](float z) { return z > -INFINITY ? (uint64_t)(weight(z) * unit + 0.5) : 0ull; };
        const float per = (float)(kBinsPerNat / T0);
        // a level of bins: the entries in (lo, hi], those before it, the shift of the later levels
        uint64_t lo = 0, hi = ~0ull;
        auto bin_of = [&](float z, uint64_t q, int shift) {
            if (shift < 0) {
                const float y = (top - z) * per;  // no later for larger logits
                return y < (float)(kBins - 1) ? (int)y : kBins - 1;
            }
            return (int)((hi - q) >> shift);
        };
        uint64_t total = 0;  // of what the filter before kept
        for (int filter = k != 0 ? 0 : 1; filter < (by_mass ? 2 : 1); ++filter) {
            // the border: of the entries in their order, the first `rank`, or those before
            // which less than `goal` lies
            const uint64_t floor_ = last;
            lo = 0;
            hi = ~0ull;
            int shift = -1;
            uint64_t count0 = 0, mass0 = 0;
            double goal = 0.;
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
                row.each([&](float z, uint32_t i) {
                    const uint64_t q = place_of(z, i);
                    if (q < lo || q > hi || q < floor_) return;
                    const int b = bin_of(z, q, shift);
                    atomicAdd(&s.count[b], 1u);
                    if (by_mass) atomicAdd((unsigned long long*)&s.mass[b], (unsigned long long)fixed(z));
                });
                __syncthreads();
                const uint32_t c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
                const uint64_t m0 = s.mass[2 * tid], m1 = s.mass[2 * tid + 1];
                uint64_t c = (uint64_t)c0 + c1, m = m0 + m1;
                scan2(c, m, s);
                if (filter == 1 && shift < 0) {  // the whole of what is kept so far
                    if (k == 0) {
                        __syncthreads();
                        if (tid == NT - 1) s.found[2] = m;
                        __syncthreads();
                        total = s.found[2];
                    }
                    goal = p0 * (double)total;
                }
                // the border's bin: the last that is not empty and in front of which too little lies
                const uint64_t cb[2] = {count0 + c - c0 - c1, count0 + c - c1}, mb[2] = {mass0 + m - m0 - m1, mass0 + m - m1};
                const uint32_t cs[2] = {c0, c1};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool in = cs[e] != 0 && (filter == 0 ? cb[e] < k : (double)mb[e] < goal || cb[e] == 0);
                    if (in) atomicMax(&s.bin, 2 * tid + e);
                }
                __syncthreads();
                const int bin = s.bin;
                if (2 * tid == (bin & ~1)) {
                    s.found[2] = cb[bin & 1];
                    s.found[3] = mb[bin & 1];
                }
                __syncthreads();
                const uint32_t inside = s.count[bin];
                count0 = s.found[2];
                mass0 = s.found[3];
                if (inside <= kSorted) {
                    row.each([&](float z, uint32_t i) {
                        const uint64_t q = place_of(z, i);
                        if (q < lo || q > hi || q < floor_ || bin_of(z, q, shift) != bin) return;
                        s.list[atomicAdd(&s.listed, 1u)] = q;
                    });
                    break;
                }
                // too many: their range, and another level
                uint64_t least = ~0ull, most = 0;
                row.each([&](float z, uint32_t i) {
                    const uint64_t q = place_of(z, i);
                    if (q < lo || q > hi || q < floor_ || bin_of(z, q, shift) != bin) return;
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
            __syncthreads();
            const uint32_t listed = s.listed;
            if (tid >= (int)listed) s.list[tid] = 0;
            // descending
            for (int w = 2; w <= kSorted; w <<= 1)
                for (int o = w >> 1; o > 0; o >>= 1) {
                    __syncthreads();
                    const int j = tid ^ o;
                    if (j > tid) {
                        const uint64_t x = s.list[tid], y = s.list[j];
                        if ((x < y) == ((tid & w) == 0)) {
                            s.list[tid] = y;
                            s.list[j] = x;
                        }
                    }
                }
            __syncthreads();
            const uint64_t q = s.list[tid];
            const bool some = tid < (int)listed;
            uint64_t c = some ? 1 : 0, m = some && by_mass ? fixed(logit_of((uint32_t)(q >> 32))) : 0;
            const uint64_t own = m;
            scan2(c, m, s);
            const bool in = some && (filter == 0 ? count0 + c - 1 < k : (double)(mass0 + m - own) < goal || count0 + c == 1);
            if (tid == 0) s.bin = -1;
            __syncthreads();
            if (in) atomicMax(&s.bin, tid);
            __syncthreads();
            if (s.bin == tid) {
                s.found[0] = q;
                s.found[1] = mass0 + m;
            }
            __syncthreads();
            last = s.found[0];
            total = s.found[1];
            __syncthreads();
        }
    }

    // ---- pass 4
    const uint64_t blocks = ((uint64_t)row.V + 64 * U - 1) / (64 * U);
    const uint32_t reps = (uint32_t)((blocks + kRuns - 1) / kRuns);  // blocks of a run
    const int runs = (int)((blocks + reps - 1) / reps);
    auto kept = [&](float z, uint32_t i) {
        if (!(z > -INFINITY) || place_of(z, i) < last) return 0.;
        const double w = weight(z);
        return w >= low ? w : 0.;
    };
    // this lane's U elements of a block: their weights
    auto load = [&](uint64_t block, double (&w)[U]) {
        const uint64_t i = (block * 64 + lane) * U;
        const int m = i < row.V ? (row.V - i < U ? (int)(row.V - i) : U) : 0;
        train::F<U> z{};
        if (m > 0) z = train::widen<T, U>(train::load_unit<T, U>(row.at + i, m));
#pragma unroll
        for (int e = 0; e < U; ++e) w[e] = e < m ? kept(z.v[e], (uint32_t)i + e) : 0.;
    };
    for (int r = wave; r < runs; r += kWaves) {
        double sum = 0.;
        for (uint32_t b = 0; b < reps; ++b) {
            double w[U];
            load((uint64_t)r * reps + b, w);
#pragma unroll
            for (int e = 0; e < U; ++e) sum += w[e];
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) s.runs[r] = sum;
    }
    __syncthreads();
    if (wave != 0) return;
    // sums before each run: 16 consecutive ones a lane
    double part = 0.;
    for (int e = 0; e < kRuns / 64; ++e) {
        const int r = lane * (kRuns / 64) + e;
        if (r < runs) part += s.runs[r];
    }
    double upto_lane = part;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double x = __shfl_up(upto_lane, o);
        if (lane >= o) upto_lane += x;
    }
    const double whole = __shfl(upto_lane, 63);
    const double goal = (double)a.u[n] * whole;
    // the first run at whose end the sum exceeds the goal; else the last of positive weight
    int first = runs, positive = -1;
    double base = 0., run = __shfl_up(upto_lane, 1);
    if (lane == 0) run = 0.;
    double at_first = 0.;
    for (int e = 0; e < kRuns / 64; ++e) {
        const int r = lane * (kRuns / 64) + e;
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
        const uint64_t block = (uint64_t)chosen * reps + b;
        load(block, w);
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
