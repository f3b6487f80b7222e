// Device-side building blocks of the operators around the layer: units of
// elements, the counter-based generator, reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.hpp"
#include "train_kernels.hpp"

namespace lors {
namespace train {

// Number of the workgroup in a grid_of().
__device__ __forceinline__ uint32_t block_id() { return blockIdx.y * gridDim.x + blockIdx.x; }

// Consecutive elements of a row that a lane takes at a time: one 16-byte vector.
// Every kernel here works in such units, so that the lanes of a wave access one
// run of memory whatever the type; rows of odd widths only differ in their last
// unit.
template <typename T>
constexpr int kUnit = 16 / sizeof(T);

template <int N>
struct F {
    float v[N];
};

// N elements as they are stored.  A row of an odd width starts at any multiple of
// the element's size: the loads and stores below are written for that alignment,
// and gfx950 executes them as whole vectors at any address.
template <typename T, int N>
struct Raw {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
};
template <typename T, int N>
struct alignas(sizeof(T)) Packed {
    T v[N];
};

template <typename T, int N>
__device__ __forceinline__ Raw<T, N> load_whole(const T* p) {
    return __builtin_bit_cast(Raw<T, N>, *(const Packed<T, N>*)p);
}

template <typename T, int N>
__device__ __forceinline__ F<N> widen(const Raw<T, N>& r) {
    F<N> f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 2) f.v[e] = __uint_as_float(e & 1 ? r.w[e >> 1] & 0xFFFF0000u : r.w[e >> 1] << 16);
        else f.v[e] = __uint_as_float(r.w[e]);
    }
    return f;
}

template <typename T, int N>
__device__ __forceinline__ Raw<T, N> narrow(const F<N>& f) {
    Raw<T, N> r;
#pragma unroll
    for (int i = 0; i < Raw<T, N>::kWords; ++i) {
        if constexpr (sizeof(T) == 2) r.w[i] = pack_bf16x2(f.v[2 * i], f.v[2 * i + 1]);
        else r.w[i] = __float_as_uint(f.v[i]);
    }
    return r;
}

// The first n (1 .. N) elements at p, the others 0.
template <typename T, int N>
__device__ __forceinline__ Raw<T, N> load_unit(const T* p, int n) {
    if (n >= N) return load_whole<T, N>(p);
    Raw<T, N> r{};
#pragma unroll
    for (int e = 0; e < N - 1; ++e)
        if (e < n) {
            if constexpr (sizeof(T) == 2) r.w[e >> 1] |= (uint32_t)((const uint16_t*)p)[e] << (16 * (e & 1));
            else r.w[e] = ((const uint32_t*)p)[e];
        }
    return r;
}
template <typename T>
__device__ __forceinline__ Raw<T, kUnit<T>> load_unit(const T* p, int n) {
    return load_unit<T, kUnit<T>>(p, n);
}

template <typename T, int N>
__device__ __forceinline__ void store_unit(T* p, const Raw<T, N>& r, int n) {
    if (n >= N) {
        *(Packed<T, N>*)p = __builtin_bit_cast(Packed<T, N>, r);
        return;
    }
#pragma unroll
    for (int e = 0; e < N - 1; ++e)
        if (e < n) {
            if constexpr (sizeof(T) == 2) ((uint16_t*)p)[e] = (uint16_t)(r.w[e >> 1] >> (16 * (e & 1)));
            else ((uint32_t*)p)[e] = r.w[e];
        }
}

// The same past the caches, for results that no cache could hold until they are
// read.
template <typename T, int N>
__device__ __forceinline__ void stream_unit(T* p, const Raw<T, N>& r, int n) {
    typedef uint32_t words __attribute__((ext_vector_type(Raw<T, N>::kWords)));
    typedef words words_any __attribute__((aligned(sizeof(T))));
    if (n >= N) __builtin_nontemporal_store(__builtin_bit_cast(words, r), (words_any*)p);
    else store_unit<T, N>(p, r, n);
}

// ---------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011): ten rounds of two 32 x 32
// -> 64 bit products over a 128-bit counter, the key raised by two constants
// between rounds.
// ---------------------------------------------------------------------------
__device__ __forceinline__ u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                        uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// The generator of one launch: its key and offset after the state on the device.
struct Dropper {
    uint32_t k0, k1, o0, o1, below;
    float factor;

    __device__ __forceinline__ explicit Dropper(const DropArgs& d) {
        uint64_t seed = d.seed, offset = d.offset;
        if (d.state != nullptr) {
            seed += d.state[0];
            offset += d.state[1];
        }
        k0 = (uint32_t)seed;
        k1 = (uint32_t)(seed >> 32);
        o0 = (uint32_t)offset;
        o1 = (uint32_t)(offset >> 32);
        below = d.below;
        factor = d.factor;
    }

    // Unit g of row n, kept elements times the factor.  A block's 16-bit halves are
    // one unit of bf16 and two of fp32.
    template <int N>
    __device__ __forceinline__ void apply(F<N>& f, uint32_t n, uint32_t g) const {
        const u32x4 w = philox(g / (8 / N), n, o0, o1, k0, k1);
        const bool upper = N == 4 && (g & 1);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint32_t bits = upper ? u16_at(w, (e + 4) & 7) : u16_at(w, e);
            f.v[e] = bits >= below ? f.v[e] * factor : 0.f;
        }
    }
};

// ---------------------------------------------------------------------------
// Reductions
// ---------------------------------------------------------------------------

// v of another lane of the wave by a DPP control word (every lane has a source).
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), kCtrl, 0xF, 0xF, true));
}
// v of lane ^ 16 and of lane ^ 32.
__device__ __forceinline__ float swap16(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)__float_as_uint(v), (16 << 10) | 31));
}
__device__ __forceinline__ float swap32(float v) { return __shfl_xor(v, 32); }

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// op over each aligned group of W lanes (8 .. 64), in every lane of it.
// DPP: 0xB1 lane ^ 1, 0x4E lane ^ 2, 0x141 the lanes of eight reversed (each quad
// holds one value by then), 0x140 the row of 16 reversed.
template <int W, class Op>
__device__ __forceinline__ float over_lanes(float v, Op op) {
    v = op(v, dpp<0xB1>(v));
    v = op(v, dpp<0x4E>(v));
    v = op(v, dpp<0x141>(v));
    if constexpr (W >= 16) v = op(v, dpp<0x140>(v));
    if constexpr (W >= 32) v = op(v, swap16(v));
    if constexpr (W >= 64) v = op(v, swap32(v));
    return v;
}

}  // namespace train
}  // namespace lors
