// Device-side building blocks of the operators around the layer: units of eight
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

// Eight consecutive elements of a row: one 16-byte vector of bf16, two of fp32.
// Every kernel here works in such units: they are what the generator's blocks
// cover, and rows of odd widths only differ in their last one.
constexpr int kUnit = 8;

struct F8 {
    float v[kUnit];
};

// A unit as it is stored.  A row of an odd width starts at any multiple of the
// element's size; the loads and stores below are written for that alignment,
// and gfx950 executes them as 16-byte accesses at any address.
template <typename T>
struct Raw;
template <>
struct Raw<__bf16> {
    u32x4 a;
};
template <>
struct Raw<float> {
    u32x4 a, b;
};

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ Raw<__bf16> load_whole(const __bf16* p) { return {*(const u32x4_any*)p}; }
__device__ __forceinline__ Raw<float> load_whole(const float* p) {
    return {*(const u32x4_any4*)p, *(const u32x4_any4*)(p + 4)};
}

__device__ __forceinline__ F8 widen(Raw<__bf16> r) {
    F8 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f.v[2 * e] = __uint_as_float(r.a[e] << 16);
        f.v[2 * e + 1] = __uint_as_float(r.a[e] & 0xFFFF0000u);
    }
    return f;
}
__device__ __forceinline__ F8 widen(Raw<float> r) {
    F8 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f.v[e] = __uint_as_float(r.a[e]);
        f.v[4 + e] = __uint_as_float(r.b[e]);
    }
    return f;
}

// The first n (1 .. 8) elements at p, the others 0.
template <typename T>
__device__ __forceinline__ Raw<T> load_unit(const T* p, int n) {
    if (n >= kUnit) return load_whole(p);
    Raw<T> r{};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < kUnit - 1; ++e)
            if (e < n) r.a[e >> 1] |= (uint32_t)((const uint16_t*)p)[e] << (16 * (e & 1));
    } else {
#pragma unroll
        for (int e = 0; e < kUnit - 1; ++e)
            if (e < n) (e < 4 ? r.a : r.b)[e & 3] = __float_as_uint(p[e]);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ Raw<T> narrow(const F8& f) {
    if constexpr (sizeof(T) == 2) {
        return {u32x4{pack_bf16x2(f.v[0], f.v[1]), pack_bf16x2(f.v[2], f.v[3]), pack_bf16x2(f.v[4], f.v[5]),
                      pack_bf16x2(f.v[6], f.v[7])}};
    } else {
        Raw<float> r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            r.a[e] = __float_as_uint(f.v[e]);
            r.b[e] = __float_as_uint(f.v[4 + e]);
        }
        return r;
    }
}

__device__ __forceinline__ void store_whole(__bf16* p, Raw<__bf16> r) { *(u32x4_any*)p = r.a; }
__device__ __forceinline__ void store_whole(float* p, Raw<float> r) {
    *(u32x4_any4*)p = r.a;
    *(u32x4_any4*)(p + 4) = r.b;
}

template <typename T>
__device__ __forceinline__ void store_unit(T* p, Raw<T> r, int n) {
    if (n >= kUnit) {
        store_whole(p, r);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < kUnit - 1; ++e)
            if (e < n) ((uint16_t*)p)[e] = (uint16_t)u16_at(r.a, e);
    } else {
#pragma unroll
        for (int e = 0; e < kUnit - 1; ++e)
            if (e < n) p[e] = __uint_as_float((e < 4 ? r.a : r.b)[e & 3]);
    }
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

    // Unit g of row n, kept elements times the factor.
    __device__ __forceinline__ void apply(F8& f, uint32_t n, uint32_t g) const {
        const u32x4 w = philox(g, n, o0, o1, k0, k1);
#pragma unroll
        for (int e = 0; e < kUnit; ++e) f.v[e] = u16_at(w, e) >= below ? f.v[e] * factor : 0.f;
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
