// C ABI of the gated block, orthogonalised updates and sampling: argument validation
// and dispatch to the gfx950 kernels.
//
// Validation runs entirely on the host, in the order null, dtype/format,
// shape/range, alignment, alias, workspace, before any HIP call, so every rejected
// call is free of side effects.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "abi_common.hpp"
#include "block_kernels.hpp"
#include "kernels.hpp"
#include "lors_block.h"

namespace {

using namespace lors::abi;

int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

// ---------------------------------------------------------------------------
// gated
// ---------------------------------------------------------------------------
lors_status_t check_gated(const lors_problem_t* p, int32_t activation, uint32_t flags) {
    lors_status_t st = lors::check_problem(p);
    if (st == LORS_ERR_DTYPE || st == LORS_ERR_MASK_FORMAT) return st;
    if (activation != LORS_ACT_SILU && activation != LORS_ACT_GELU) return LORS_ERR_UNSUPPORTED;
    if (st != LORS_OK) return st;
    if ((p->flags & ~flags) != 0u) return LORS_ERR_UNSUPPORTED;
    // both projections' tiles in one grid: the forward's, the adapters' gradients'
    const int64_t rt = (p->R + 255) / 256;
    if (2 * rt * ((p->C + 255) / 256) > kMaxExtent || 2 * rt * ((p->L + 255) / 256) > kMaxExtent) return LORS_ERR_UNSUPPORTED;
    return LORS_OK;
}

// The backward's scratch: both transposed masks, both padded B's, dG, dU, and the fp32
// partial sums of dX's tiles that are cut over the K-steps of both projections (whole
// tiles, so ranks up to 64).
struct GatedScratch {
    int64_t mt, pad, grad, split, total;
    explicit GatedScratch(const lors_problem_t* p) {
        const bool bf16 = p->dtype == LORS_DTYPE_BF16;
        const int64_t rp = (p->r + 7) / 8 * 8;
        mt = bf16 ? round256(p->C * ((p->R + 31) / 32) * 4) : 0;
        pad = bf16 && rp != p->r ? round256(2 * p->R * rp) : 0;
        grad = round256(p->L * p->R * elt_size(p->dtype));
        split = bf16 && rp <= 64 ? lors::split_part_bytes(lors::gated_dx_split(p->L, p->R, p->C)) : 0;
        total = 2 * (mt + pad + grad) + split;
    }
};

int64_t gated_forward_bytes(const lors_problem_t* p) {
    return p->dtype == LORS_DTYPE_BF16 ? 0 : 2 * round256(p->L * p->R * 4);
}

bool complete(const lors_projection_t* q) {
    return q != nullptr && q->W != nullptr && q->M_packed != nullptr && q->B != nullptr && q->A != nullptr;
}

lors::LayerArgs gated_args(const lors_problem_t* p, int32_t activation, const void* X, const lors_projection_t* gate,
                           const lors_projection_t* up, lors::SecondArgs& second) {
    lors::LayerArgs a{};
    a.R = p->R;
    a.C = p->C;
    a.L = p->L;
    a.r = p->r;
    a.r_grad = p->r;
    a.scale = p->scale;
    a.two_four = p->mask_format == LORS_MASK_2_4;
    a.X = X;
    a.W = gate->W;
    a.M = gate->M_packed;
    a.B = gate->B;
    a.A = gate->A;
    second = lors::SecondArgs{};
    second.W = up->W;
    second.M = up->M_packed;
    second.B = up->B;
    second.A = up->A;
    second.gelu = activation == LORS_ACT_GELU;
    a.second = &second;
    return a;
}

// The launchers of one projection, on the second one of a.
lors::LayerArgs second_alone(const lors::LayerArgs& a) {
    lors::LayerArgs b = a;
    const lors::SecondArgs& q = *a.second;
    b.W = q.W;
    b.M = q.M;
    b.Mt = q.Mt;
    b.B = q.B;
    b.A = q.A;
    b.dY = q.dY;
    b.dB = q.dB;
    b.dA = q.dA;
    b.second = nullptr;
    return b;
}

// ---------------------------------------------------------------------------
// update
// ---------------------------------------------------------------------------
constexpr int64_t kMostMatrices = 65535;  // of up to 256 workgroups each, 256 threads: below 2^32

// Checks in the documented order, up to the range of the extents.
lors_status_t check_update(const lors_update_t* p, const lors_update_item_t* items, int64_t count) {
    if (p == nullptr || (count > 0 && items == nullptr)) return LORS_ERR_NULL;
    if (count > kMostMatrices) return LORS_ERR_SHAPE;
    for (int64_t i = 0; i < count; ++i)
        if (items[i].grad == nullptr || (items[i].master == nullptr && items[i].param == nullptr)) return LORS_ERR_NULL;
    if (!valid_dtype(p->grad_dtype) || !valid_dtype(p->param_dtype)) return LORS_ERR_DTYPE;
    if (count < 0 || !(p->momentum >= 0.0 && p->momentum <= 1.0) || !std::isfinite(p->eps) || p->eps < 0.0 ||
        !std::isfinite(p->a) || !std::isfinite(p->b) || !std::isfinite(p->c) || p->steps < 1 ||
        p->steps > LORS_UPDATE_MAX_STEPS || (p->nesterov != 0 && p->nesterov != 1))
        return LORS_ERR_SHAPE;
    for (int64_t i = 0; i < count; ++i) {
        const lors_update_item_t& q = items[i];
        if (q.rows < 1 || q.cols < 1 || q.rows > kMaxExtent || q.cols > kMaxExtent || q.rows * q.cols >= int64_t(1) << 40 ||
            !std::isfinite(q.rate) || !std::isfinite(q.decay))
            return LORS_ERR_SHAPE;
    }
    if (p->flags != 0 || 2 * p->steps * std::log2(std::fabs(p->a)) > 38.0) return LORS_ERR_UNSUPPORTED;
    for (int64_t i = 0; i < count; ++i)
        if (std::min(items[i].rows, items[i].cols) > LORS_UPDATE_MAX_SIDE) return LORS_ERR_UNSUPPORTED;
    return LORS_OK;
}

int64_t scratch_of(const lors_update_item_t& q) {
    return lors::block::update_scratch(std::min(q.rows, q.cols), std::max(q.rows, q.cols));
}

// What a call reads or writes, to find overlaps by a sort.
struct Span {
    uintptr_t lo, hi;
    bool out;
};

// Whether an output overlaps anything else: in the order of their starts, a span meets an
// earlier one where it starts before the furthest end so far.
bool any_overlap(Span* s, int64_t n) {
    std::sort(s, s + n, [](const Span& x, const Span& y) { return x.lo < y.lo; });
    uintptr_t ends = 0, out_ends = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (s[i].lo < (s[i].out ? ends : out_ends)) return true;
        ends = std::max(ends, s[i].hi);
        if (s[i].out) out_ends = std::max(out_ends, s[i].hi);
    }
    return false;
}

}  // namespace

extern "C" {

int lors_block_version(void) { return 10000; }

size_t lors_gated_workspace_bytes(const lors_problem_t* p, int backward) {
    if (p == nullptr || check_gated(p, LORS_ACT_SILU, backward ? LORS_FLAG_REUSE_MASK_T : 0u) != LORS_OK)
        return static_cast<size_t>(-1);
    return static_cast<size_t>(backward ? GatedScratch(p).total : gated_forward_bytes(p));
}

lors_status_t lors_gated_forward(const lors_problem_t* p, int32_t activation, const void* X,
                                 const lors_projection_t* gate, const lors_projection_t* up, void* G, void* U, void* H,
                                 void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr || !complete(gate) || !complete(up)) return LORS_ERR_NULL;
    if (p->L != 0 && (X == nullptr || H == nullptr || (G == nullptr) != (U == nullptr))) return LORS_ERR_NULL;
    lors_status_t st = check_gated(p, activation, 0u);
    if (st != LORS_OK) return st;
    const int64_t es = elt_size(p->dtype), R = p->R, C = p->C, L = p->L, r = p->r;
    const int64_t m = static_cast<int64_t>(lors_mask_packed_bytes(R, C)), y = L * R * es;
    const bool bf16 = p->dtype == LORS_DTYPE_BF16, save = G != nullptr;
    const int64_t need = save ? 0 : gated_forward_bytes(p);
    st = check_arrays({{X, L * C * es, 16}, {gate->W, R * C * es, 16}, {gate->M_packed, m, 16}, {gate->B, R * r * es, 16},
                       {gate->A, r * C * es, 16}, {up->W, R * C * es, 16}, {up->M_packed, m, 16}, {up->B, R * r * es, 16},
                       {up->A, r * C * es, 16}},
                      {{H, y, 16}, {G, y, 16}, {U, y, 16}, {need ? workspace : nullptr, need, 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, static_cast<size_t>(need));
    if (st != LORS_OK || L == 0) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    lors::SecondArgs second;
    lors::LayerArgs a = gated_args(p, activation, X, gate, up, second);
    if (bf16) {
        a.Y = H;
        second.G = G;
        second.U = U;
        return from_hip(lors::launch_gated_fwd_bf16(a, s));
    }
    a.Y = save ? G : workspace;
    lors::LayerArgs b = second_alone(a);
    b.Y = save ? U : static_cast<uint8_t*>(workspace) + need / 2;
    hipError_t e = lors::launch_fwd_f32(a, s);
    if (e == hipSuccess) e = lors::launch_fwd_f32(b, s);
    if (e == hipSuccess) e = lors::launch_gated_join(a.Y, b.Y, H, L * R, second.gelu, false, s);
    return from_hip(e);
}

lors_status_t lors_gated_backward(const lors_problem_t* p, int32_t activation, const void* dH, const void* X,
                                  const lors_projection_t* gate, const lors_projection_t* up, const void* G,
                                  const void* U, void* dX, float* dB_gate, float* dA_gate, float* dB_up, float* dA_up,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr || !complete(gate) || !complete(up)) return LORS_ERR_NULL;
    if (dB_gate == nullptr || dA_gate == nullptr || dB_up == nullptr || dA_up == nullptr) return LORS_ERR_NULL;
    if (p->L != 0 && (dH == nullptr || X == nullptr || G == nullptr || U == nullptr)) return LORS_ERR_NULL;
    lors_status_t st = check_gated(p, activation, LORS_FLAG_REUSE_MASK_T);
    if (st != LORS_OK) return st;
    const int64_t es = elt_size(p->dtype), R = p->R, C = p->C, L = p->L, r = p->r;
    const int64_t m = static_cast<int64_t>(lors_mask_packed_bytes(R, C)), y = L * R * es;
    const GatedScratch ws(p);
    st = check_arrays({{dH, y, 16}, {G, y, 16}, {U, y, 16}, {X, L * C * es, 16}, {gate->W, R * C * es, 16},
                       {gate->M_packed, m, 16}, {gate->B, R * r * es, 16}, {gate->A, r * C * es, 16}, {up->W, R * C * es, 16},
                       {up->M_packed, m, 16}, {up->B, R * r * es, 16}, {up->A, r * C * es, 16}},
                      {{dX, L * C * es, 16}, {dB_gate, R * r * 4, 16}, {dA_gate, r * C * 4, 16}, {dB_up, R * r * 4, 16},
                       {dA_up, r * C * 4, 16}, {workspace, ws.total, 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, static_cast<size_t>(ws.total));
    if (st != LORS_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = p->dtype == LORS_DTYPE_BF16;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    lors::SecondArgs second;
    lors::LayerArgs a = gated_args(p, activation, X, gate, up, second);
    a.dX = dX;
    a.dB = dB_gate;
    a.dA = dA_gate;
    second.dB = dB_up;
    second.dA = dA_up;
    a.Mt = reinterpret_cast<const uint32_t*>(at);
    second.Mt = reinterpret_cast<const uint32_t*>(at + ws.mt);
    a.b_pad = ws.pad ? at + 2 * ws.mt : nullptr;
    second.b_pad = ws.pad ? at + 2 * ws.mt + ws.pad : nullptr;
    void* dG = at + 2 * (ws.mt + ws.pad);
    void* dU = static_cast<uint8_t*>(dG) + ws.grad;
    a.dY = dG;
    second.dY = dU;
    a.split_ws = ws.split ? static_cast<uint8_t*>(dU) + ws.grad : nullptr;
    hipError_t e = hipSuccess;
    if (L == 0) {
        e = lors::launch_zero2_f32(dB_gate, R * r, dA_gate, r * C, s);
        if (e == hipSuccess) e = lors::launch_zero2_f32(dB_up, R * r, dA_up, r * C, s);
        return from_hip(e);
    }
    // which also clears dB and dA for the atomics of the adapters' gradients
    const lors::Clear clear{{dB_gate, dA_gate, dB_up, dA_up}, {R * r, r * C, R * r, r * C}};
    e = lors::launch_gated_split(dH, G, U, dG, dU, L * R, second.gelu, bf16, clear, s);
    if (bf16) {
        if ((p->flags & LORS_FLAG_REUSE_MASK_T) == 0u) {
            if (e == hipSuccess) e = lors::launch_mask_transpose(a.M, R, C, a.two_four, const_cast<uint32_t*>(a.Mt), s);
            if (e == hipSuccess)
                e = lors::launch_mask_transpose(second.M, R, C, a.two_four, const_cast<uint32_t*>(second.Mt), s);
        }
        if (e == hipSuccess) e = lors::launch_gated_dx_bf16(a, s);
        if (e == hipSuccess) e = lors::launch_gated_g_bf16(a, s);
        return from_hip(e);
    }
    const lors::LayerArgs b = second_alone(a);
    if (e == hipSuccess && dX != nullptr) e = lors::launch_gated_dx_f32(a, s);
    if (e == hipSuccess) e = lors::launch_g_f32(a, s);
    if (e == hipSuccess) e = lors::launch_g_f32(b, s);
    return from_hip(e);
}

size_t lors_orthogonal_workspace_bytes(const lors_update_t* p, const lors_update_item_t* items, int64_t count) {
    if (check_update(p, items, count) != LORS_OK) return static_cast<size_t>(-1);
    int64_t need = 0;
    for (int64_t i = 0; i < count; ++i) need += scratch_of(items[i]);
    return static_cast<size_t>(need + lors::block::update_table(count));
}

lors_status_t lors_orthogonal_update(const lors_update_t* p, const lors_update_item_t* items, int64_t count,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    const lors_status_t st = check_update(p, items, count);
    if (st != LORS_OK || count == 0) return st;
    const int64_t gs = elt_size(p->grad_dtype), ps = elt_size(p->param_dtype);
    std::unique_ptr<Span[]> spans(new (std::nothrow) Span[4 * count + 1]);
    std::unique_ptr<lors::block::Matrix[]> matrices(new (std::nothrow) lors::block::Matrix[count]);
    if (!spans || !matrices) return LORS_ERR_HIP;
    int64_t n = 0, need = 0;
    auto span = [&](const void* at, int64_t bytes, bool out) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(at);
        if (at != nullptr && bytes > 0) spans[n++] = Span{lo, lo + static_cast<uintptr_t>(bytes), out};
    };
    for (int64_t i = 0; i < count; ++i) {
        const lors_update_item_t& q = items[i];
        const int64_t size = q.rows * q.cols;
        const lors_status_t at = check_alignment({{q.grad, 0, gs}, {q.m, 0, 4}, {q.master, 0, 4}, {q.param, 0, ps}});
        if (at != LORS_OK) return at;
        span(q.grad, size * gs, false);
        span(q.m, size * 4, true);
        span(q.master, size * 4, true);
        span(q.param, size * ps, true);
        matrices[i] = lors::block::Matrix{q.grad, q.m, q.master, q.param, std::max(q.rows, q.cols), need, static_cast<float>(q.rate),
                                          static_cast<float>(1.0 - q.decay), static_cast<int32_t>(std::min(q.rows, q.cols)),
                                          q.rows <= q.cols ? 1 : 0};
        need += scratch_of(q);
    }
    const int64_t table = lors::block::update_table(count), at = need;
    need += table;
    if (check_alignment({{workspace, 0, 16}}) != LORS_OK) return LORS_ERR_ALIGN;
    span(workspace, need, true);
    if (any_overlap(spans.get(), n)) return LORS_ERR_ALIAS;
    if (check_workspace(workspace, workspace_bytes, static_cast<size_t>(need)) != LORS_OK) return LORS_ERR_WORKSPACE;
    const lors::block::UpdateArgs a{static_cast<float>(p->momentum),
                                    static_cast<float>(1.0 - p->momentum),
                                    p->nesterov != 0,
                                    p->eps,
                                    p->a,
                                    p->b,
                                    p->c,
                                    p->steps,
                                    p->grad_dtype == LORS_DTYPE_BF16,
                                    p->param_dtype == LORS_DTYPE_BF16,
                                    static_cast<uint8_t*>(workspace)};
    return from_hip(lors::block::launch_update(a, matrices.get(), count, table ? a.workspace + at : nullptr,
                                               static_cast<hipStream_t>(stream)));
}

static lors_status_t check_sample(const lors_sample_t* p) {
    if (!valid_dtype(p->dtype)) return LORS_ERR_DTYPE;
    if (p->rows < 0 || p->rows > kMaxExtent || p->vocab < 1 || p->vocab > kMaxExtent || p->row_stride < 0 ||
        p->rows * p->vocab >= int64_t(1) << 57)
        return LORS_ERR_SHAPE;
    if (p->rows > 0 && bytes_of(p->rows, p->row_stride, 4) < 0) return LORS_ERR_SHAPE;
    if (!std::isfinite(p->temperature) || p->temperature < 0.0 || !(p->top_p >= 0.0) || !std::isfinite(p->min_p) || p->min_p < 0.0)
        return LORS_ERR_SHAPE;
    return p->flags != 0 ? LORS_ERR_UNSUPPORTED : LORS_OK;
}

size_t lors_sample_workspace_bytes(const lors_sample_t* p) {
    return p == nullptr || check_sample(p) != LORS_OK ? static_cast<size_t>(-1) : 0;
}

lors_status_t lors_sample(const lors_sample_t* p, const void* logits, const float* u, const float* temperature,
                          const int32_t* top_k, const float* top_p, const float* min_p, int64_t* token, float* logp,
                          void* workspace, size_t workspace_bytes, void* stream) {
    if (p == nullptr) return LORS_ERR_NULL;
    if (p->rows != 0 && (logits == nullptr || u == nullptr || token == nullptr)) return LORS_ERR_NULL;
    lors_status_t st = check_sample(p);
    if (st != LORS_OK) return st;
    const int64_t es = elt_size(p->dtype), n = p->rows;
    const int64_t z = n == 0 ? 0 : ((n - 1) * p->row_stride + p->vocab) * es;
    const size_t need = lors_sample_workspace_bytes(p);
    st = check_arrays({{logits, z, es}, {u, 4 * n, 4}, {temperature, 4 * n, 4}, {top_k, 4 * n, 4}, {top_p, 4 * n, 4}, {min_p, 4 * n, 4}},
                      {{token, 8 * n, 8}, {logp, 4 * n, 4}, {workspace, static_cast<int64_t>(need), 16}});
    if (st == LORS_OK) st = check_workspace(workspace, workspace_bytes, need);
    if (st != LORS_OK) return st;
    const lors::block::SampleArgs a{n,           p->vocab, p->row_stride, p->temperature, p->top_k, p->top_p, p->min_p, logits,
                                    u,           temperature, top_k,      top_p,          min_p,    token,    logp,     workspace};
    return from_hip(lors::block::launch_sample(a, p->dtype == LORS_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
