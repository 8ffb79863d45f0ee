// Products of MXFP4 matrices: C[m][n] = act(sum over k of A[m][k] B[n][k] + bias[n]) (gfx950, wave64).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 codes of a row from each lane, one block with one scale byte: lane l holds row l % 32,
// block l / 32 of the 64 values.  Sums are held in 32 bits.
#pragma once

#include "dqrm_mx.hpp"

namespace dqrm_mx {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
constexpr int kFp4 = 4; // the instruction's number for E2M1 operands

__device__ __forceinline__ v16f mfma_32x32x64(uint4 a, uint4 b, v16f c, unsigned scale_a, unsigned scale_b)
{
    const v8i va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, c, kFp4, kFp4, 0, (int)scale_a, 0, (int)scale_b);
}

struct MatmulArgs {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    int64_t m, n, k;
    const float *bias; // [n] or null
    int relu;
    void *c;
    int64_t ldc;
};

// One wave to 32 by 32 outputs, operands straight from memory.
template <int DT>
__global__ __launch_bounds__(64) void matmul_simple_kernel(MatmulArgs g)
{
    using T = elem_t<DT>;
    const int lane = threadIdx.x, half = lane >> 5;
    const int64_t m0 = (int64_t)blockIdx.y * 32, n0 = (int64_t)blockIdx.x * 32;
    const int64_t ra = min(m0 + (lane & 31), g.m - 1), rb = min(n0 + (lane & 31), g.n - 1);
    const int64_t groups = groups_of(g.k);
    const uint8_t *pa = g.a_codes + ra * groups * 64 + half * 16, *pb = g.b_codes + rb * groups * 64 + half * 16;
    const uint8_t *sa = g.a_scales + ra * groups * 4 + half, *sb = g.b_scales + rb * groups * 4 + half;
    v16f acc = {};
    for (int64_t i = 0; i < groups * 2; ++i)
        acc = mfma_32x32x64(*reinterpret_cast<const uint4 *>(pa + i * 32), *reinterpret_cast<const uint4 *>(pb + i * 32), acc, sa[i * 2], sb[i * 2]);
    const int64_t n = n0 + (lane & 31);
    if (n >= g.n) return;
    const float bias = g.bias ? g.bias[n] : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t m = m0 + 8 * (i / 4) + 4 * half + i % 4;
        float v = acc[i] + bias;
        if (g.relu) v = v < 0.0f ? 0.0f : v; // (a NaN stays)
        if (m < g.m) static_cast<T *>(g.c)[m * g.ldc + n] = (T)v;
    }
}

} // namespace dqrm_mx
