// Host-side argument checks that the C ABIs of lors_train.h and lors_block.h share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "lors_block.h"
#include "lors_train.h"

namespace lors {

// The layer's checks of a problem (abi.cpp), in the documented order.
lors_status_t check_problem(const lors_problem_t* p);

namespace abi {

constexpr int64_t kMaxExtent = (int64_t(1) << 31) - 1;
// Largest byte count of any one argument: every count is checked against it
// before it is formed, and sums of a few stay far from overflow.
constexpr int64_t kMaxBytes = int64_t(1) << 60;

// a * b * es when it is at most kMaxBytes (es in 1 .. 8), else -1.
static inline int64_t bytes_of(int64_t a, int64_t b, int64_t es) {
    int64_t ab = 0, abe = 0;
    if (a < 0 || b < 0 || __builtin_mul_overflow(a, b, &ab) || __builtin_mul_overflow(ab, es, &abe) ||
        abe > kMaxBytes)
        return -1;
    return abe;
}

static inline bool valid_dtype(int32_t d) { return d == LORS_DTYPE_BF16 || d == LORS_DTYPE_F32; }
static inline bool valid_index(int32_t d) { return d == LORS_INDEX_I64 || d == LORS_INDEX_I32; }
static inline int64_t elt_size(int32_t dtype) { return dtype == LORS_DTYPE_BF16 ? 2 : 4; }
static inline int64_t index_size(int32_t dtype) { return dtype == LORS_INDEX_I64 ? 8 : 4; }

// One array of a call: where it is, its bytes, the alignment it needs.
struct Array {
    const void* p;
    int64_t bytes;
    int64_t align;
};

static inline lors_status_t check_alignment(std::initializer_list<Array> arrays) {
    for (const Array& a : arrays)
        if (reinterpret_cast<uintptr_t>(a.p) % static_cast<uintptr_t>(a.align) != 0) return LORS_ERR_ALIGN;
    return LORS_OK;
}

static inline bool overlap(const Array& a, const Array& b) {
    if (a.p == nullptr || b.p == nullptr || a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t la = reinterpret_cast<uintptr_t>(a.p), lb = reinterpret_cast<uintptr_t>(b.p);
    return la < lb + static_cast<uintptr_t>(b.bytes) && lb < la + static_cast<uintptr_t>(a.bytes);
}

// No output over an input or another output.
static inline lors_status_t check_alias(std::initializer_list<Array> in, std::initializer_list<Array> out) {
    for (const Array* o = out.begin(); o != out.end(); ++o) {
        for (const Array& i : in)
            if (overlap(*o, i)) return LORS_ERR_ALIAS;
        for (const Array* q = out.begin(); q != o; ++q)
            if (overlap(*o, *q)) return LORS_ERR_ALIAS;
    }
    return LORS_OK;
}

static inline lors_status_t check_arrays(std::initializer_list<Array> in, std::initializer_list<Array> out) {
    lors_status_t st = check_alignment(in);
    if (st == LORS_OK) st = check_alignment(out);
    if (st == LORS_OK) st = check_alias(in, out);
    return st;
}

static inline lors_status_t check_workspace(const void* ws, size_t given, size_t need) {
    return need > 0 && (ws == nullptr || given < need) ? LORS_ERR_WORKSPACE : LORS_OK;
}

static inline lors_status_t from_hip(hipError_t e) { return e == hipSuccess ? LORS_OK : LORS_ERR_HIP; }

}  // namespace abi
}  // namespace lors
