// The last step of the softmax cross entropy's forward: the tiles' parts of each row to its lse and its loss (gfx950, wave64).
#pragma once

#include "dqrm_device.hpp"

namespace dqrm {

// maximum and sum of powers of two of two parts of a row; one without classes is (-infinity, 0)
__device__ __forceinline__ float2 xent_join_parts(float2 a, float2 b)
{
    const float most = fmaxf(a.x, b.x), base = most == -__builtin_inff() ? 0.0f : most;
    return make_float2(most, a.y * __builtin_amdgcn_exp2f(a.x - base) + b.y * __builtin_amdgcn_exp2f(b.x - base));
}

// ROWS rows to a workgroup (16; 1 where there are few rows: 782 tiles of 16 rows 9.5 and 3.3 us), 256 / ROWS lanes to a row with the tiles in
// turn, eight loads at a time on their way; then their results in pairs.  A sum is at least 1 (its largest power) and at most the classes.
template <int ROWS>
__global__ __launch_bounds__(256) void xent_join_kernel(const float2 *parts, int64_t tiles, int64_t stride, int64_t rows, const float *at,
                                                        const int64_t *targets, int64_t classes, float *loss, float *lse)
{
    constexpr int slices = 256 / ROWS;
    __shared__ float2 s[slices][ROWS == 1 ? 1 : ROWS + 1];
    const int in = threadIdx.x % ROWS, slice = threadIdx.x / ROWS;
    const int64_t r = (int64_t)blockIdx.x * ROWS + in;
    float2 v = make_float2(-__builtin_inff(), 0.0f);
    if (r < rows) {
        constexpr int ahead = 8;
        for (int64_t k = slice; k < tiles; k += slices * ahead) {
            float2 x[ahead];
#pragma unroll
            for (int i = 0; i < ahead; ++i) x[i] = parts[min(k + slices * i, tiles - 1) * stride + r];
#pragma unroll
            for (int i = 0; i < ahead; ++i)
                if (k + slices * i < tiles) v = xent_join_parts(v, x[i]);
        }
    }
    s[slice][in] = v;
#pragma unroll
    for (int h = slices / 2; h >= 1; h /= 2) {
        __syncthreads();
        if (slice < h) s[slice][in] = v = xent_join_parts(v, s[slice + h][in]);
    }
    if (slice != 0 || r >= rows) return;
    // The maximum less the target's logit before the sum's logarithm is added: a loss far below the logits keeps its bits.  In 64 bits up to the one
    // rounding of each; of a sum of 1 and little more the logarithm too.
    constexpr double kLn2 = 0.693147180559945309;
    const bool none = v.x == -__builtin_inff() && v.y == 0.0f; // (no classes left; a NaN stays)
    const double rest = log2((double)v.y);
    lse[r] = none ? v.x : (float)(((double)v.x + rest) * kLn2);
    const int64_t t = targets[r];
    float l = 0.0f;
    if (t >= classes) report(DQRM_ERR_INDEX_OUT_OF_RANGE, -1, t);
    if (t >= 0 && t < classes) l = none ? __builtin_inff() : (float)(((double)v.x - (double)at[r] + rest) * kLn2);
    loss[r] = l;
}

} // namespace dqrm
