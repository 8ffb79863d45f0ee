// Host-side checks and small helpers of the calls on matrices of any element type.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "dqrm.h"
#include "dqrm_host.hpp"

namespace dqrm_host {

#define DQRM_HIP_CHECK(expr)                                         \
    do {                                                             \
        hipError_t e_ = (expr);                                      \
        if (e_ != hipSuccess) return dqrm_host::hip_fail(e_, #expr); \
    } while (0)

#define DQRM_CHECK(expr)                 \
    do {                                 \
        const int32_t rc_ = (expr);      \
        if (rc_ != DQRM_OK) return rc_;  \
    } while (0)

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t x, int64_t d) { return (x + d - 1) / d; }

constexpr int64_t kMaxDim = 2147483647LL - 1024; // rows, columns and row strides' limit
constexpr int64_t kMaxBlocks = 1 << 22;          // of one launch, with up to 512 threads each (a launch has to have fewer than 2^32)

inline size_t size_of(int32_t dtype) { return dtype == DQRM_F32 ? 4 : 2; }

// f(Elem type) for a dtype that has been checked
template <typename F>
void with_type(int32_t dtype, F f)
{
    if (dtype == DQRM_F32)
        f(std::integral_constant<int, DQRM_F32>{});
    else if (dtype == DQRM_BF16)
        f(std::integral_constant<int, DQRM_BF16>{});
    else
        f(std::integral_constant<int, DQRM_F16>{});
}

inline bool known_type(int32_t dtype) { return dtype == DQRM_F32 || dtype == DQRM_BF16 || dtype == DQRM_F16; }

inline int32_t check_shape(int32_t dtype, int64_t rows, int64_t cols)
{
    if (!known_type(dtype)) return DQRM_ERR_INVALID_ARG;
    if (rows < 0 || cols < 0) return DQRM_ERR_INVALID_ARG;
    if (rows > kMaxDim || cols > kMaxDim) return DQRM_ERR_UNSUPPORTED;
    return DQRM_OK;
}

// a matrix of elements: there if it has any, at its elements' alignment, rows that do not overlap
inline int32_t check_matrix(const void *p, int64_t ld, int32_t dtype, int64_t rows, int64_t cols)
{
    if (rows == 0 || cols == 0) return DQRM_OK;
    if (!p || !aligned(p, size_of(dtype)) || (rows > 1 && ld < cols)) return DQRM_ERR_INVALID_ARG;
    if (rows > 1 && (ld > (int64_t)1 << 40 || ld > ((int64_t)1 << 48) / rows)) return DQRM_ERR_UNSUPPORTED;
    return DQRM_OK;
}

inline int32_t check_mx(const dqrm_mxfp4_t *q, int64_t rows, int64_t cols)
{
    if (!q || q->rows != rows || q->cols != cols) return DQRM_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return DQRM_OK;
    if (!q->codes || !q->scales || !aligned(q->codes, 16) || !aligned(q->scales, 4)) return DQRM_ERR_INVALID_ARG;
    return DQRM_OK;
}

inline int32_t check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return DQRM_OK;
    if (!ws || !aligned(ws, 256)) return DQRM_ERR_INVALID_ARG;
    return have < need ? DQRM_ERR_WORKSPACE_TOO_SMALL : DQRM_OK;
}

inline int num_cus()
{
    static const int n = [] {
        int dev = 0, v = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v < 1) return 256;
        return v;
    }();
    return n;
}

} // namespace dqrm_host
