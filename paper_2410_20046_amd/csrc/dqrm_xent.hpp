// Softmax cross entropy of a linear classifier, without its logits in memory (gfx950, wave64).
//
//   l[i][j] = scale x_i . w_j + bias_j, lse_i = log sum_j exp l[i][j], loss_i = lse_i - l[i][target_i]
//   d[i][j] = grad_i (exp(l[i][j] - lse_i) - (1 if j = target_i)), dx = scale d w, dw = scale d^T x, dbias_j = sum_i d[i][j]
//
// Forward, a tile of logits stays in registers and leaves as each row's maximum and sum of exponentials over the tile's classes, which
// xent_join_kernel joins.  Backward, the tile is computed again and leaves as d for some classes at a time, which two more products read.
// Exponentials are powers of two (logits times log2 e).  A lane has one row of a block of 32 and 16 classes of each.
#pragma once

#include "dqrm_xent_gemm.hpp"

namespace dqrm_xent {

constexpr float kLog2e = 1.44269504088896341f;

// by its bias in powers of two (that of float's lowest value is -infinity too)
__device__ __forceinline__ bool taken_out(float bias) { return bias * kLog2e == -__builtin_inff(); }

struct Classifier {
    Products g;
    const float *bias; // [n] or null
    float scale2;      // scale times log2 e
    const int64_t *targets;
    int64_t first; // the products' first class
};

// a logit that is -infinity of itself, not by its class's bias
__device__ __forceinline__ float no_infinity(float l) { return l == -__builtin_inff() ? __builtin_nanf("") : l; }

// The tile's logits, in powers of two, in place of its sums; classes past the last one -infinity, and those that are taken out whatever their sums are.
// CHECKED: other infinities are NaNs, whose rows' lse is one then (+infinity comes to that by itself; a gradient's have their lse's).
template <typename S, bool CHECKED>
__device__ __forceinline__ void logits(const Classifier &c, v16f (&acc)[S::TM][S::TN], int64_t n0)
{
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
        float b[16];
        bool out = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t n = n0 + j * 32 + q * 8 + half * 4;
            struct Four { float v[4]; } f{};
            if (c.bias) {
                if (n + 4 <= c.g.n) {
                    __builtin_memcpy(&f, c.bias + n, sizeof(f));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) f.v[i] = n + i < c.g.n ? c.bias[n + i] : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = n + i < c.g.n ? f.v[i] * kLog2e : -__builtin_inff();
                b[q * 4 + i] = v;
                out |= v == -__builtin_inff();
            }
        }
#pragma unroll
        for (int t = 0; t < S::TM; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][j][i] = __builtin_fmaf(acc[t][j][i], c.scale2, b[i]);
        if constexpr (CHECKED) {
            float least = 0.0f;
#pragma unroll
            for (int t = 0; t < S::TM; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) least = fminf(least, acc[t][j][i]);
            out |= least == -__builtin_inff();
        }
        if (__any(out)) {
#pragma unroll
            for (int t = 0; t < S::TM; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][j][i] = b[i] == -__builtin_inff() ? b[i] : CHECKED ? no_infinity(acc[t][j][i]) : acc[t][j][i];
        }
    }
}

// f(t, j, i) for the place of the target's class of the lane's row, where the wave's tile has it; target: [TM], relative to the wave's first class
template <typename S, typename F>
__device__ __forceinline__ void at_target(const int (&target)[S::TM], F f)
{
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < S::TM; ++t) {
        if (!__any(target[t] >= 0)) continue;
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (target[t] == j * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) f(t, j, i);
    }
}

// the row's target as a place among the wave's classes from n0 on, -1: not there
template <typename S>
__device__ __forceinline__ int place_of_target(int64_t target, int64_t n0)
{
    const int64_t at = target - n0;
    return at >= 0 && at < S::TN * 32 ? (int)at : -1;
}

__device__ __forceinline__ float power2(float v) { return __builtin_amdgcn_exp2f(v); }

// exp(l - lse) of logits in powers of two: power2(l2 - lse2) factor.  lse times log2 e is not a number of 32 bits: what is left of it is in
// the factor, which a row's gradient takes with it (and 1, a target's place, its inverse).  Where lse's own rounding is a power and more, nothing is.
struct RowLse {
    float lse2, factor, inverse;
};
__device__ __forceinline__ RowLse lse_of(float lse)
{
    constexpr float kLow = 1.92596303e-8f; // log2 e less kLog2e
    const float lse2 = lse * kLog2e;
    const float rest = fminf(fmaxf(__builtin_fmaf(lse, kLow, __builtin_fmaf(lse, kLog2e, -lse2)), -1.0f), 1.0f);
    return {lse2, power2(-rest), power2(rest)};
}

// maximum and sum of two parts of a row; a part without classes is (-infinity, 0)
__device__ __forceinline__ float2 join_parts(float2 a, float2 b)
{
    const float most = fmaxf(a.x, b.x), base = most == -__builtin_inff() ? 0.0f : most;
    return make_float2(most, a.y * power2(a.x - base) + b.y * power2(b.x - base));
}

struct FwdArgs {
    Classifier c;
    float2 *parts; // [tiles of classes][rows]: maximum, sum of powers
    float *at;     // [rows]: the target's logit
    unsigned first_tile;
};

// The tile of 256 by 256 is bound by the matrix instructions, 8192 rows, 131072 classes, width 4096 in bf16 6.7-6.9 ms, 1.3 PFLOP/s; its exponentials, in
// nobody's shadow, are a twentieth of it.  Tiles of few rows by the classes' bytes: 16 rows, 200003 classes, width 1024 in bf16 78-83 us, 5.1 TB/s.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::per_simd) void xent_fwd_kernel(FwdArgs a)
{
    static_assert(S::WN * S::BM * sizeof(float2) <= S::lds_bytes);
    __shared__ __align__(1024) char lds[S::lds_bytes];
    const Products &g = a.c.g;
    const Place at = place_of(g);
    const int64_t m0 = (int64_t)at.tm * S::BM, n0 = (int64_t)at.tn * S::BN;
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    v16f acc[S::TM][S::TN];
    multiply_tile<T, S, false, false, false>(g, lds, m0, n0, 0, (int)(g.stages * g.pairs), at.tn, acc);
    logits<S, true>(a.c, acc, n0 + wn * S::TN * 32);
    const int64_t row0 = m0 + wm * S::TM * 32 + (lane & 31);
    int target[S::TM];
#pragma unroll
    for (int t = 0; t < S::TM; ++t)
        target[t] = place_of_target<S>(row0 + t * 32 < g.m ? a.c.targets[row0 + t * 32] : -1, a.c.first + n0 + wn * S::TN * 32);
    at_target<S>(target, [&](int t, int j, int i) { a.at[row0 + t * 32] = acc[t][j][i]; });
    float2 *s_part = reinterpret_cast<float2 *>(lds); // [WN][BM]
#pragma unroll
    for (int t = 0; t < S::TM; ++t) {
        float most = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, acc[t][j][i]);
        most = fmaxf(most, __shfl_xor(most, 32, kWaveSize));
        const float base = most == -__builtin_inff() ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            float part = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) part += power2(acc[t][j][i] - base);
            sum += part;
        }
        sum += __shfl_xor(sum, 32, kWaveSize);
        if (lane < 32) s_part[wn * S::BM + (wm * S::TM + t) * 32 + lane] = make_float2(most, sum);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < S::BM; r += S::threads) {
        if (m0 + r >= g.m) break;
        float2 p = s_part[r];
#pragma unroll
        for (int w = 1; w < S::WN; ++w) p = join_parts(p, s_part[w * S::BM + r]);
        a.parts[(int64_t)(a.first_tile + at.tn) * g.m + m0 + r] = p;
    }
}

// ---- a few rows -----------------------------------------------------------------------------------------------------------
// A few requests: w is read once, as it is (fp32 without planes, rows at any alignment), and multiplied with the rows of x, which are in LDS, in
// 32-bit fused products.  `lanes` of a wave take a class, 8 values each at a time, and then add up; a group of lanes keeps the maximum and
// sum of its classes.
struct FewArgs {
    const void *x, *w;
    int64_t ldx, ldw, rows, classes, width;
    const float *bias;
    float scale2;
    const int64_t *targets;
    int64_t per_block; // classes
    int lanes, padded; // of a class; width up to a multiple of 8 lanes
    float2 *parts;     // [workgroups][part_rows], from the first of these rows on
    float *at;
    int64_t part_rows;
};

// Bound by w's bytes: 457731 classes of width 1172 in fp32 (2.15 GB), 2 rows 401 us, 5.4 TB/s, 4 rows 424; 1000 classes of width 16, with the join, 7.3
// from a graph.  Of aligned 16-bit values the tiles are faster (200003 of width 1024 in bfloat16: 82 and 116 us).
template <int DT, int M>
__global__ __launch_bounds__(256) void xent_rows_fwd_kernel(FewArgs a)
{
    using T = elem_t<DT>;
    constexpr int together = M <= 2 ? 4 : 2; // classes of a group, whose loads are on their way together
    extern __shared__ __align__(16) float s_x[]; // [M][padded]
    __shared__ float2 s_part[4][M];
    const int width = (int)a.width;
    for (int i = threadIdx.x; i < M * a.padded; i += 256) {
        const int r = i / a.padded, c = i - r * a.padded;
        s_x[i] = r < a.rows && c < width ? (float)static_cast<const T *>(a.x)[r * a.ldx + c] : 0.0f;
    }
    __syncthreads();
    const int groups = 256 / a.lanes, group = threadIdx.x / a.lanes, lane = threadIdx.x - group * a.lanes;
    const int64_t first = (int64_t)blockIdx.x * a.per_block, last = min(first + a.per_block, a.classes);
    int64_t target[M];
    float most[M], sum[M];
#pragma unroll
    for (int m = 0; m < M; ++m) target[m] = m < a.rows ? a.targets[m] : -1, most[m] = -__builtin_inff(), sum[m] = 0.0f;
    for (int64_t j = first; j < last; j += groups * together) {
        float acc[together][M] = {};
        const T *row[together];
        int64_t cls[together];
#pragma unroll
        for (int k = 0; k < together; ++k) {
            cls[k] = j + k * groups + group;
            row[k] = static_cast<const T *>(a.w) + min(cls[k], a.classes - 1) * a.ldw;
        }
        for (int c = lane * kChunk; c < width; c += a.lanes * kChunk) {
            Vec8<T> w[together];
#pragma unroll
            for (int k = 0; k < together; ++k) w[k] = load_vec(row[k], c, width, false);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                float x[kChunk];
                __builtin_memcpy(x, __builtin_assume_aligned(&s_x[m * a.padded + c], 16), sizeof(x));
#pragma unroll
                for (int k = 0; k < together; ++k)
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) acc[k][m] = __builtin_fmaf((float)w[k].v[i], x[i], acc[k][m]);
            }
        }
        for (int d = 1; d < a.lanes; d *= 2) {
#pragma unroll
            for (int k = 0; k < together; ++k)
#pragma unroll
                for (int m = 0; m < M; ++m) acc[k][m] += __shfl_xor(acc[k][m], d, kWaveSize);
        }
#pragma unroll
        for (int k = 0; k < together; ++k) {
            const float b = cls[k] >= last ? -__builtin_inff() : a.bias ? a.bias[cls[k]] * kLog2e : 0.0f;
#pragma unroll
            for (int m = 0; m < M; ++m) acc[k][m] = b == -__builtin_inff() ? b : no_infinity(__builtin_fmaf(acc[k][m], a.scale2, b));
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float top = most[m];
#pragma unroll
            for (int k = 0; k < together; ++k) {
                top = fmaxf(top, acc[k][m]);
                if (cls[k] == target[m] && cls[k] < last && lane == 0) a.at[m] = acc[k][m];
            }
            const float base = top == -__builtin_inff() ? 0.0f : top;
            sum[m] *= power2(most[m] - base);
#pragma unroll
            for (int k = 0; k < together; ++k) sum[m] += power2(acc[k][m] - base);
            most[m] = top;
        }
    }
    // the wave's groups, then the waves
#pragma unroll
    for (int m = 0; m < M; ++m) {
        float2 p = make_float2(most[m], sum[m]);
        for (int d = a.lanes; d < kWaveSize; d *= 2) p = join_parts(p, make_float2(__shfl_xor(p.x, d, kWaveSize), __shfl_xor(p.y, d, kWaveSize)));
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6][m] = p;
    }
    __syncthreads();
    if ((int)threadIdx.x < a.rows) {
        float2 p = s_part[0][threadIdx.x];
        for (int w = 1; w < 4; ++w) p = join_parts(p, s_part[w][threadIdx.x]);
        a.parts[blockIdx.x * a.part_rows + threadIdx.x] = p;
    }
}

struct GradArgs {
    Classifier c;
    const float *lse, *grad;
    const uint64_t *live;  // rows that have a gradient, a bit each
    const float *most;     // the largest |grad|: d is held in units of it, times `by`
    float by;
    char *d;               // [planes] in blocks: rows and classes up to multiples of 64, what is past the last ones zeros
    int64_t plane, rows, cols; // bytes; values
    int planes;
    float *sums; // [tiles of rows][classes of the piece]: d's column sums, or null
};

// v summed over the 32 lanes of a half wave, for 16 values of a lane: lane l ends with the sum of value l / 2 % 16 (in pairs of lanes)
__device__ __forceinline__ float sum_over_rows(const float (&v)[16])
{
    const int lane = threadIdx.x & 63;
    float a[8], b[4], c[2], d;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool up = lane & 16;
        a[i] = (up ? v[i + 8] : v[i]) + __shfl_xor(up ? v[i] : v[i + 8], 16, kWaveSize);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool up = lane & 8;
        b[i] = (up ? a[i + 4] : a[i]) + __shfl_xor(up ? a[i] : a[i + 4], 8, kWaveSize);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool up = lane & 4;
        c[i] = (up ? b[i + 2] : b[i]) + __shfl_xor(up ? b[i] : b[i + 2], 4, kWaveSize);
    }
    d = (lane & 2 ? c[1] : c[0]) + __shfl_xor(lane & 2 ? c[0] : c[1], 2, kWaveSize);
    return d + __shfl_xor(d, 1, kWaveSize);
}

// As the forward, then d's bytes: 8192 rows, 32768 classes, width 4096 in bf16 1.81-1.83 ms, 1.2 PFLOP/s, with 0.5 GB of d.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::per_simd) void xent_grad_kernel(GradArgs a)
{
    constexpr int out_bytes = S::waves * TileOut<T, S, To::blocks>::wave_bytes, sum_bytes = S::WM * S::BN * (int)sizeof(float);
    static_assert(out_bytes <= S::lds_bytes && sum_bytes <= S::lds_bytes);
    __shared__ __align__(1024) char lds[S::lds_bytes];
    const Products &g = a.c.g;
    const Place at = place_of(g);
    const int64_t m0 = (int64_t)at.tm * S::BM, n0 = (int64_t)at.tn * S::BN;
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN, half = lane >> 5;
    v16f acc[S::TM][S::TN];
    multiply_tile<T, S, false, false, false>(g, lds, m0, n0, 0, (int)(g.stages * g.pairs), at.tn, acc);
    logits<S, false>(a.c, acc, n0 + wn * S::TN * 32);
    const int64_t row0 = m0 + wm * S::TM * 32 + (lane & 31);
    const float most = *a.most;
    int target[S::TM];
#pragma unroll
    for (int t = 0; t < S::TM; ++t) {
        const int64_t row = row0 + t * 32;
        const bool live = row < g.m && (a.live[row >> 6] >> (row & 63)) & 1;
        const RowLse lse = lse_of(live ? a.lse[row] : 0.0f);
        const float grad = live ? a.grad[row] / most * lse.factor : 0.0f;
        target[t] = place_of_target<S>(live ? a.c.targets[row] : -1, a.c.first + n0 + wn * S::TN * 32);
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][j][i] = power2(acc[t][j][i] - lse.lse2);
        // (the target's place before the gradient's factor)
        if (__any(target[t] >= 0)) {
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (target[t] == j * 32 + (i >> 2) * 8 + half * 4 + (i & 3)) acc[t][j][i] -= lse.inverse;
        }
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][j][i] *= grad;
        // (a row without a gradient is zeros, whatever its logits are)
        if (__any(!live)) {
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][j][i] = live ? acc[t][j][i] : 0.0f;
        }
    }
    if (a.sums) {
        float *s_sum = reinterpret_cast<float *>(lds); // [WM][BN]
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[i] = acc[0][j][i];
#pragma unroll
                for (int t = 1; t < S::TM; ++t) v[i] += acc[t][j][i];
            }
            const float sum = sum_over_rows(v);
            const int i = (lane >> 1) & 15; // ... of which value: bits 8, 4, 2, 1 of it came with lane bits 16, 8, 4, 2
            if (!(lane & 1)) s_sum[wm * S::BN + (wn * S::TN + j) * 32 + (i >> 2) * 8 + half * 4 + (i & 3)] = sum;
        }
        __syncthreads();
        for (int n = threadIdx.x; n < S::BN; n += S::threads) {
            float sum = s_sum[n];
#pragma unroll
            for (int w = 1; w < S::WM; ++w) sum += s_sum[w * S::BN + n];
            if (n0 + n < g.n) a.sums[(int64_t)at.tm * g.n + n0 + n] = sum * most;
        }
        __syncthreads();
    }
    for (int plane = 0; plane < a.planes; ++plane) {
        using Out = TileOut<T, S, To::blocks>;
        Out::run(reinterpret_cast<T *>(a.d + plane * a.plane), a.cols, acc, lds + wave * Out::wave_bytes, m0 + wm * S::TM * 32, n0 + wn * S::TN * 32, a.rows,
                 a.cols, a.by);
        if (plane + 1 == a.planes) break;
#pragma unroll
        for (int t = 0; t < S::TM; ++t)
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][j][i] -= (float)(T)acc[t][j][i]; // (exact)
    }
}

// ---- few logits of long sums ------------------------------------------------------------------------------------------------
// Where a few tiles are all the logits, their sums are cut into slices (xent_sums_kernel: [slices][rows][classes] in 32 bits) and what follows
// reads them.  Bound by the launches' and the stages' latency: 233 rows, 27 classes, width 5541 in fp32, forward 28 us, 234 without slices.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::per_simd) void xent_sums_kernel(Products g, float *sums)
{
    using Out = TileOut<float, S, To::rows>;
    static_assert(S::waves * Out::wave_bytes <= S::lds_bytes);
    __shared__ __align__(1024) char lds[S::lds_bytes];
    const Place at = place_of(g);
    const int64_t m0 = (int64_t)at.tm * S::BM, n0 = (int64_t)at.tn * S::BN;
    const int wave = (int)uniform(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    const int all = (int)(g.stages * g.pairs), first = (int)(at.slice * g.stages_per_slice), last = min(all, first + (int)g.stages_per_slice);
    v16f acc[S::TM][S::TN];
    multiply_tile<T, S, false, false, false>(g, lds, m0, n0, first, last, at.tm + at.tn + at.slice, acc);
    Out::run(sums + (int64_t)at.slice * g.m * g.n, g.n, acc, lds + wave * Out::wave_bytes, m0 + wm * S::TM * 32, n0 + wn * S::TN * 32, g.m, g.n, 1.0f);
}

struct SumsArgs {
    const float *sums;
    int slices, classes;
    int64_t rows;
    const float *bias;
    float scale2;
    const int64_t *targets;
    // loss
    float2 *parts; // [1024s of classes][rows]
    float *at;
    // gradient
    const float *lse, *grad, *most;
    const uint64_t *live;
    float by;
    char *d; // in blocks of 64 by 64
    int64_t plane, pitch;
    float *dbias; // [64s of rows][classes], or null
};

// a logit, in powers of two
__device__ __forceinline__ float logit_of(const SumsArgs &a, int64_t r, int c)
{
    const float b = a.bias ? a.bias[c] * kLog2e : 0.0f;
    if (b == -__builtin_inff()) return b;
    const float *from = a.sums + r * a.classes + c;
    const int64_t slice = a.rows * a.classes;
    float v = 0.0f;
    constexpr int ahead = 8; // loads in flight
    int s = 0;
    for (; s + ahead <= a.slices; s += ahead) {
        float x[ahead];
#pragma unroll
        for (int i = 0; i < ahead; ++i) x[i] = from[(s + i) * slice];
#pragma unroll
        for (int i = 0; i < ahead; ++i) v += x[i];
    }
    for (; s < a.slices; ++s) v += from[s * slice];
    return no_infinity(__builtin_fmaf(v, a.scale2, b));
}

// 1024 classes of a row to a workgroup.
constexpr int kSumsClasses = 1024;
static __global__ __launch_bounds__(256) void xent_sums_loss_kernel(SumsArgs a)
{
    __shared__ float2 s_part[4];
    const int64_t r = blockIdx.x, target = a.targets[r];
    const int first = blockIdx.y * kSumsClasses, last = min(first + kSumsClasses, a.classes);
    float2 v = make_float2(-__builtin_inff(), 0.0f);
    for (int c = first + (int)threadIdx.x; c < last; c += 256) {
        const float l = logit_of(a, r, c);
        if (c == target) a.at[r] = l;
        v = join_parts(v, make_float2(l, l == -__builtin_inff() ? 0.0f : 1.0f));
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = join_parts(v, make_float2(__shfl_xor(v.x, d, kWaveSize), __shfl_xor(v.y, d, kWaveSize)));
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) a.parts[blockIdx.y * a.rows + r] = join_parts(join_parts(s_part[0], s_part[1]), join_parts(s_part[2], s_part[3]));
}

// A block of 64 rows by 64 classes of d to a workgroup, 16 classes of a row to a thread.
template <int DT>
__global__ __launch_bounds__(256) void xent_sums_grad_kernel(SumsArgs a)
{
    using Q = std::conditional_t<DT == DQRM_F16, _Float16, __bf16>;
    constexpr int planes = DT == DQRM_F32 ? 3 : 1;
    __shared__ float s_d[64][65];
    const int row = threadIdx.x >> 2, from = (threadIdx.x & 3) * 16, c0 = blockIdx.x * kBlock;
    const int64_t r = (int64_t)blockIdx.y * kBlock + row;
    const bool live = r < a.rows && (a.live[blockIdx.y] >> row) & 1;
    const RowLse lse = lse_of(live ? a.lse[r] : 0.0f);
    const float most = *a.most, grad = live ? a.grad[r] / most * lse.factor : 0.0f;
    const int64_t target = live ? a.targets[r] : -1;
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = c0 + from + i;
        v[i] = 0.0f;
        if (live && c < a.classes) v[i] = (power2(logit_of(a, r, c) - lse.lse2) - (c == target ? lse.inverse : 0.0f)) * grad;
        s_d[row][from + i] = v[i];
    }
    char *to = a.d + ((int64_t)blockIdx.y * (a.pitch / (kBlock * 2)) + blockIdx.x) * kBlockBytes + row * (kBlock * 2) + from * 2;
#pragma unroll
    for (int k = 0; k < planes; ++k) {
        struct alignas(16) Many { Q v[16]; } f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            f.v[i] = (Q)(v[i] * a.by);
            v[i] -= (float)f.v[i]; // (more than one plane: by is 1)
        }
        *reinterpret_cast<Many *>(to + k * a.plane) = f;
    }
    if (!a.dbias) return;
    __syncthreads();
    const int c = c0 + (int)threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.classes) return;
    float sum = 0.0f;
    for (int i = 0; i < 64; ++i) sum += s_d[i][threadIdx.x];
    a.dbias[(int64_t)blockIdx.y * a.classes + c] = sum * most;
}

struct OutArgs {
    Products g;
    void *c; // the result, or [slices][m][n] of 32-bit sums
    int64_t ldc;
    float scale;
    const float *by; // and times this, or null
};

// A gradient's product, B with k as the rows.  ADD: to the sums of the pieces before.  Bound by the matrix instructions, whose operands take two
// transposing reads each: 8192 rows, 32768 classes, width 4096 in bf16, dx 1.97-2.09 ms, 1.1 PFLOP/s, dw 1.92-1.96, 1.1 (torch's products of
// these sizes: 1.13 and 1.01).
template <typename T, typename TO, typename S, bool A_BY_K, bool ADD>
__global__ __launch_bounds__(S::threads, S::per_simd) void xent_out_kernel(OutArgs a)
{
    using Out = TileOut<TO, S, ADD ? To::sums : To::rows>;
    static_assert(S::waves * Out::wave_bytes <= S::lds_bytes);
    __shared__ __align__(1024) char lds[S::lds_bytes];
    const Products &g = a.g;
    const Place at = place_of(g);
    const int64_t m0 = (int64_t)at.tm * S::BM, n0 = (int64_t)at.tn * S::BN;
    const int wave = (int)uniform(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    const int all = (int)(g.stages * g.pairs), first = (int)(at.slice * g.stages_per_slice), last = min(all, first + (int)g.stages_per_slice);
    v16f acc[S::TM][S::TN];
    multiply_tile<T, S, A_BY_K, true, true>(g, lds, m0, n0, first, last, at.tm + at.tn + at.slice, acc);
    const float by = a.by ? a.scale * *a.by : a.scale;
    Out::run(static_cast<TO *>(a.c) + (int64_t)at.slice * g.m * g.n, a.ldc, acc, lds + wave * Out::wave_bytes, m0 + wm * S::TM * 32, n0 + wn * S::TN * 32, g.m, g.n,
             by);
}

// The slices' sums (`all` values apart) in turn, times the factors, rounded: bound by their bytes.  One value to a thread, less than 2^31 in all.
template <typename TO>
__global__ __launch_bounds__(256) void xent_out_join_kernel(const float *sums, unsigned slices, int64_t all, unsigned m, dqrm::FastDiv n, TO *c, int64_t ldc,
                                                            float scale, const float *by)
{
    const unsigned at = blockIdx.x * 256 + threadIdx.x, r = n.div(at);
    if (r >= m) return;
    float v = 0.0f;
    constexpr unsigned ahead = 8; // loads in flight
    unsigned s = 0;
    for (; s + ahead <= slices; s += ahead) {
        float x[ahead];
#pragma unroll
        for (unsigned i = 0; i < ahead; ++i) x[i] = sums[(int64_t)(s + i) * all + at];
#pragma unroll
        for (unsigned i = 0; i < ahead; ++i) v += x[i];
    }
    for (; s < slices; ++s) v += sums[(int64_t)s * all + at];
    c[r * ldc + (at - r * n.d)] = (TO)(v * (by ? scale * *by : scale));
}

// A matrix as the products take it: 16-bit values, rows padded with zeros to a multiple of 64; fp32 as three bfloat16 planes.
struct PackArgs {
    const void *x;
    int64_t ldx, rows, cols;
    char *out;
    int64_t plane, pitch; // bytes
};

// a float as three bfloat16, whose sum it is exactly (of 2^-110 and more); ANY: one that would round to infinity is cut instead
template <bool ANY = true>
__device__ __forceinline__ void split(float v, __bf16 (&p)[3])
{
    p[0] = (__bf16)v;
    if (ANY && __builtin_isinf((float)p[0])) {
        const unsigned cut = __float_as_uint(v) & 0xFFFF0000u;
        p[0] = (__bf16)__uint_as_float(cut);
    }
    float rest = v - (float)p[0];
    p[1] = (__bf16)rest;
    rest -= (float)p[1];
    p[2] = (__bf16)rest;
}

template <int DT>
__global__ __launch_bounds__(256) void xent_pack_kernel(PackArgs a, dqrm::FastDiv per_row)
{
    using T = elem_t<DT>;
    const unsigned at = blockIdx.x * 256 + threadIdx.x, r = per_row.div(at), chunk = at - r * per_row.d;
    if (r >= a.rows) return;
    const Vec8<T> v = load_vec(static_cast<const T *>(a.x) + r * a.ldx, (int64_t)chunk * kChunk, a.cols, false);
    char *to = a.out + r * a.pitch + (int64_t)chunk * 16;
    if constexpr (DT == DQRM_F32) {
        struct alignas(16) Eight { __bf16 v[kChunk]; } p[3];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            __bf16 s[3];
            split(v.v[i], s);
            p[0].v[i] = s[0], p[1].v[i] = s[1], p[2].v[i] = s[2];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<Eight *>(to + k * a.plane) = p[k];
    } else {
        __builtin_memcpy(__builtin_assume_aligned(to, 16), &v, 16);
    }
}

// The largest of 1024 threads' values; thread 0 gets it
__device__ __forceinline__ unsigned largest(unsigned v)
{
    __shared__ unsigned s[16];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, d, kWaveSize));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < 16; ++i) v = max(v, s[i]);
    return v;
}

// The gradients' unit: the largest of them (of the finite ones; 1 if there is none).  d in units of it: where all rows weigh the same, as in a
// mean, the targets' places are close to -1 and lose nothing by their rounding; and fp16, times 2^14, has all its bits down to 2^-28 of the unit
// and none below 2^-39.
__device__ __forceinline__ float unit_of(unsigned bits) { return bits ? __uint_as_float(bits) : 1.0f; }

// Which rows have a gradient, a bit each, and the bits of the largest |grad| of a workgroup's rows; of all rows, by a single workgroup, as the unit.
static __global__ __launch_bounds__(1024) void xent_rows_kernel(const int64_t *targets, int64_t classes, const float *lse, const float *grad, int64_t rows,
                                                                uint64_t *live, unsigned *most, float *unit)
{
    unsigned top = 0;
    for (int64_t r = (int64_t)blockIdx.x * 1024 + threadIdx.x; r - (threadIdx.x & 63) < rows; r += (int64_t)gridDim.x * 1024) {
        bool has = false;
        if (r < rows) {
            const float g = grad[r];
            has = targets[r] >= 0 && targets[r] < classes && g != 0.0f && lse[r] != -__builtin_inff();
            if (has && abs_bits(g) < 0x7F800000u) top = max(top, abs_bits(g));
        }
        const uint64_t word = __ballot(has);
        if ((threadIdx.x & 63) == 0) live[r >> 6] = word;
    }
    top = largest(top);
    if (threadIdx.x == 0 && gridDim.x == 1) *unit = unit_of(top);
    if (threadIdx.x == 0 && gridDim.x > 1) most[blockIdx.x] = top;
}

// ... of several workgroups
static __global__ __launch_bounds__(1024) void xent_unit_kernel(const unsigned *most, int n, float *unit)
{
    const unsigned top = largest((int)threadIdx.x < n ? most[threadIdx.x] : 0u);
    if (threadIdx.x == 0) *unit = unit_of(top);
}

// Which classes are not taken out.
static __global__ __launch_bounds__(256) void xent_classes_kernel(const float *bias, int64_t classes, uint64_t *live)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const uint64_t word = __ballot(j < classes && !taken_out(bias[min(j, classes - 1)]));
    if ((threadIdx.x & 63) == 0 && j < classes) live[j >> 6] = word;
}

} // namespace dqrm_xent
