// The two projections of a gated block, H = act(G) * U with G = X . Wg'^T and
// U = X . Wu'^T, as the tile kernels see them: the gate is the kernel's own
// projection, the other one comes in a pair.  Alone: a projection by itself.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace lors {

struct Alone {};
static inline Alone alone_of(const LayerArgs&) { return {}; }

// forward: G and U may be null (serving)
struct Gated {
    const uint16_t* W;
    const uint32_t* M;
    const uint16_t *B, *A;
    uint16_t *G, *U;
    int gelu;
};

static inline Gated pair_of(const LayerArgs& a) {
    const SecondArgs& q = *a.second;
    return {(const uint16_t*)q.W, q.M, (const uint16_t*)q.B, (const uint16_t*)q.A, (uint16_t*)q.G, (uint16_t*)q.U, (int)q.gelu};
}

// backward (dX, and the adapters' gradients)
struct GatedGrad {
    const uint16_t *dY, *W;
    const uint32_t* Mt;
    const uint16_t *B, *A;
    float *dB, *dA;
};

static inline GatedGrad grad_pair_of(const LayerArgs& a) {
    const SecondArgs& q = *a.second;
    return {(const uint16_t*)q.dY, (const uint16_t*)q.W, q.Mt, (const uint16_t*)q.B, (const uint16_t*)q.A, q.dB, q.dA};
}

// Token parts that a logical tile of a thin grid is cut into: of a batch below one tile only
// those that hold tokens.  (Empty workgroups between those with work leave the latter on a part of
// the CUs, to which they are dealt in turn: 64 tokens, 11008 x 4096, rank 16, 149 us
// against 59.)
__host__ __device__ static inline int token_parts(int64_t L, int tm) {
    const int64_t most = thin_span(tm) / tm, parts = (L + tm - 1) / tm;
    return (int)(parts < most ? parts : most);
}

// GELU's (1 + tanh(x)) / 2 = 1 / (1 + exp(-2x)) for x = k (g + 0.044715 g^3), without the difference that
// cancels below zero (1 + tanh(x) is 2^-24 at g = -5, a rounding of tanh): `s`, and 1 - s in
// `rest`, both of full relative accuracy, and x's slope.
__device__ __forceinline__ float gelu_gate(float g, float& rest, float& slope) {
    constexpr float k = 0.797884560802865356f;  // sqrt(2 / pi)
    const float g2 = g * g;
    const float x = k * g * (1.f + 0.044715f * g2);
    slope = k * (1.f + 0.134145f * g2);
    const float e = __expf(-2.f * fabsf(x)), big = 1.f / (1.f + e), small = e * big;  // no overflow
    rest = x < 0.f ? big : small;
    return x < 0.f ? small : big;
}

// SiLU g / (1 + exp(-g)), or GELU g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2.  Where exp(-g)
// overflows (g below -88) SiLU is -0, as its limit is.
__device__ __forceinline__ float activate(float g, int gelu) {
    if (gelu) {
        float rest, slope;
        return g * gelu_gate(g, rest, slope);
    }
    return g / (1.f + __expf(-g));
}

// act(g), and its derivative in `d`
__device__ __forceinline__ float activate_grad(float g, int gelu, float& d) {
    if (gelu) {
        float rest, slope;
        const float s = gelu_gate(g, rest, slope), bend = s * rest;
        d = s + (bend != 0.f ? 2.f * g * bend * slope : 0.f);  // (the slope may have overflown where the bend is 0)
        return g * s;
    }
    const float y = 1.f / (1.f + __expf(-g));
    d = y * (1.f + g * (1.f - y));
    return g * y;
}

}  // namespace lors
