// Layer norm forward and backward (gfx950, wave64).
//
//   mean = sum x / n, var = sum (x - mean)^2 / n, rstd = 1 / sqrt(var + eps), xhat = (x - mean) rstd, y = xhat gamma + beta
//   g = dy gamma, dx = rstd (g - mean(g) - xhat mean(g xhat)), dgamma = sum over rows of dy xhat, dbeta = sum over rows of dy
//
// All in 32 bits; the variance is taken about the mean, from values that are still in registers.
#pragma once

#include "dqrm_mx.hpp"

namespace dqrm_mx {

struct NormArgs {
    const void *x;
    int64_t ldx, rows, cols;
    const float *gamma, *beta; // or null: 1 and 0
    float eps;
    void *y; // or null
    int64_t ldy;
    float *mean, *rstd;      // or null
    uint8_t *codes, *scales; // MXFP4 of y (before its rounding to the element type), or null
};

// sum over the TPR threads of a row; every one of them gets it.  TPR > 64: over the waves of a workgroup by way of s_part (a place
// to each wave of the workgroup), which the next call must not take again before another barrier (two places in turn will do).
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*s_part)[N])
{
#pragma unroll
    for (int d = (TPR < kWaveSize ? TPR : kWaveSize) / 2; d >= 1; d >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d, kWaveSize);
    }
    if constexpr (TPR > kWaveSize) {
        constexpr int waves = TPR / kWaveSize; // of a row
        const int wave = threadIdx.x / kWaveSize, first = wave & ~(waves - 1);
        if ((threadIdx.x & (kWaveSize - 1)) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s_part[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = s_part[first][i];
#pragma unroll
            for (int w = 1; w < waves; ++w) t += s_part[first + w][i];
            v[i] = t;
        }
    }
}

template <typename I>
__device__ __forceinline__ void load_gain(const float *p, I c, I cols, float without, float (&v)[kChunk])
{
    if (p) {
        load_chunk(p, c, cols, v);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = without;
    }
}

// TPR threads to a row, CH chunks of 8 values to a thread: the row stays in registers (8 <= cols <= TPR * CH * 8), and so do the
// columns' gain and offset for all rows of a workgroup.  The next row is requested before this one's sums, whose waits would leave the
// memory idle.  Bound by its bytes, one read and one write: 16384 x 8192 bfloat16 (537 MB) 95 us, 5.6 TB/s; a small one by its launch and
// a row's latency (128 x 64 float 3.6 us).
template <int DT, int TPR, int CH, int BLOCK>
__global__ __launch_bounds__(BLOCK, 4) void norm_fwd_kernel(NormArgs a)
{
    using T = elem_t<DT>;
    constexpr int rows_per_block = BLOCK / TPR;
    __shared__ float s_part[2][BLOCK / kWaveSize][1];
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * rows_per_block;
    const int cols = (int)a.cols;
    const int64_t cp = codes_pitch(cols), sp = scales_pitch(cols);
    // (a group past the last row works on that row and writes nothing)
    auto row_of = [&](int64_t r) { return static_cast<const T *>(a.x) + min(r, a.rows - 1) * a.ldx; };
    auto column = [&](int j) { return (j * TPR + t) * kChunk; };
    int64_t r = (int64_t)blockIdx.x * rows_per_block + threadIdx.x / TPR;
    Raw<T> next[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) next[j] = load_raw(row_of(r), column(j), cols);
    float gamma[CH][kChunk], beta[CH][kChunk];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        load_gain(a.gamma, column(j), cols, 1.0f, gamma[j]);
        load_gain(a.beta, column(j), cols, 0.0f, beta[j]);
    }
    for (; r - threadIdx.x / TPR < a.rows; r += step) {
        const bool own = r < a.rows;
        float x[CH][kChunk];
        float sum[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            values_of(next[j], column(j), cols, x[j]);
            sum[0] += ((x[j][0] + x[j][1]) + (x[j][2] + x[j][3])) + ((x[j][4] + x[j][5]) + (x[j][6] + x[j][7]));
        }
        {
#pragma unroll
            for (int j = 0; j < CH; ++j) next[j] = load_raw(row_of(r + step), column(j), cols);
        }
        row_sums<TPR>(sum, s_part[0]);
        const float mean = sum[0] / (float)cols;
        float sq[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) x[j][i] -= mean;
            if (column(j) + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = column(j) + i < cols ? x[j][i] : 0.0f;
            }
            sq[0] += ((x[j][0] * x[j][0] + x[j][1] * x[j][1]) + (x[j][2] * x[j][2] + x[j][3] * x[j][3])) +
                     ((x[j][4] * x[j][4] + x[j][5] * x[j][5]) + (x[j][6] * x[j][6] + x[j][7] * x[j][7]));
        }
        row_sums<TPR>(sq, s_part[1]);
        const float rstd = 1.0f / sqrtf(sq[0] / (float)cols + a.eps);
        if (!own) continue;
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = column(j);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) x[j][i] = x[j][i] * rstd * gamma[j][i] + beta[j][i];
            // (past the row's end 0, also where rstd is infinite or a NaN: the padding of the codes)
            if (c + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = c + i < cols ? x[j][i] : 0.0f;
            }
            if (a.y && c < cols) store_chunk<true>(static_cast<T *>(a.y) + r * a.ldy, c, cols, x[j]);
            if (a.codes && c < cp * 2) write_chunk(a.codes + r * cp, a.scales + r * sp, (unsigned)(c / kChunk), x[j]);
        }
    }
}

// Rows of any length, a workgroup to each: three passes over the row, the second and third from the caches.  Each pass waits for its
// loads: 2000 x 40000 bfloat16 118 to 136 us (320 MB, 2.4 to 2.7 TB/s).
template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_long_kernel(NormArgs a)
{
    using T = elem_t<DT>;
    __shared__ float s_part[2][BLOCK / kWaveSize][1];
    const int64_t r = blockIdx.x;
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    const int64_t step = BLOCK * kChunk, end = groups_of(a.cols) * kRowPad;
    float sum[1] = {0.0f}, sq[1] = {0.0f};
    float x[kChunk];
    for (int64_t c = (int64_t)threadIdx.x * kChunk; c < a.cols; c += step) {
        load_chunk(row, c, a.cols, x);
        sum[0] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    row_sums<BLOCK>(sum, s_part[0]);
    const float mean = sum[0] / (float)a.cols;
    for (int64_t c = (int64_t)threadIdx.x * kChunk; c < a.cols; c += step) {
        load_chunk(row, c, a.cols, x);
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) q += c + i < a.cols ? (x[i] - mean) * (x[i] - mean) : 0.0f;
        sq[0] += q;
    }
    row_sums<BLOCK>(sq, s_part[1]);
    const float rstd = 1.0f / sqrtf(sq[0] / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    if (!a.y && !a.codes) return;
    for (int64_t c = (int64_t)threadIdx.x * kChunk; c < end; c += step) {
        float g[kChunk], b[kChunk];
        load_chunk(row, c, a.cols, x);
        load_gain(a.gamma, c, a.cols, 1.0f, g);
        load_gain(a.beta, c, a.cols, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) x[i] = c + i < a.cols ? (x[i] - mean) * rstd * g[i] + b[i] : 0.0f;
        if (a.y && c < a.cols) store_chunk(static_cast<T *>(a.y) + r * a.ldy, c, a.cols, x);
        if (a.codes) write_chunk(a.codes + r * codes_pitch(a.cols), a.scales + r * scales_pitch(a.cols), (unsigned)(c / kChunk), x);
    }
}

struct NormBwdArgs {
    const void *dy, *x;
    int64_t lddy, ldx, rows, cols;
    const float *mean, *rstd, *gamma; // gamma or null: 1
    void *dx;                         // or null
    int64_t lddx;
    // the workgroups' sums for dgamma and dbeta, or null: [blocks][2][cols] in the workspace, or those of the only workgroup in place
    float *sum_gamma, *sum_beta;
    int64_t block_stride;
};

// The row of dy and of x in registers, the next one on its way; a thread has the same columns in every row of its workgroup's
// slice, and keeps their sums, so that x and dy are read once for dx, dgamma and dbeta together.  Bound by its bytes, two reads and a
// write: 16001 x 8190 bfloat16 (786 MB) 140 us, 5.6 TB/s, and 8 for the join of the workgroups' sums.
template <int DT, int TPR, int CH, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_kernel(NormBwdArgs a)
{
    using T = elem_t<DT>;
    constexpr int rows_per_block = BLOCK / TPR;
    __shared__ float s_part[2][BLOCK / kWaveSize][2];
    const int t = threadIdx.x % TPR;
    const int cols = (int)a.cols;
    const float inv_n = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * rows_per_block;
    auto column = [&](int j) { return (j * TPR + t) * kChunk; };
    int64_t r = (int64_t)blockIdx.x * rows_per_block + threadIdx.x / TPR;
    Raw<T> next_dy[CH], next_x[CH];
    float next_mean = 0.0f, next_rstd = 0.0f;
    // (a group past the last row works on that row with a gradient of 0)
    auto request = [&](int64_t at) {
        const int64_t q = min(at, a.rows - 1);
        next_mean = a.mean[q], next_rstd = a.rstd[q];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            next_dy[j] = load_raw(static_cast<const T *>(a.dy) + q * a.lddy, column(j), cols);
            next_x[j] = load_raw(static_cast<const T *>(a.x) + q * a.ldx, column(j), cols);
        }
    };
    request(r);
    float dg[CH][kChunk] = {}, db[CH][kChunk] = {}, gamma[CH][kChunk];
#pragma unroll
    for (int j = 0; j < CH; ++j) load_gain(a.gamma, column(j), cols, 1.0f, gamma[j]);
    int turn = 0;
    for (; r - threadIdx.x / TPR < a.rows; r += step) {
        const bool own = r < a.rows;
        const float mean = next_mean, rstd = next_rstd;
        float dy[CH][kChunk], xh[CH][kChunk];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            values_of(next_dy[j], column(j), cols, dy[j]);
            values_of(next_x[j], column(j), cols, xh[j]);
        }
        request(r + step);
        if (own) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) xh[j][i] = (xh[j][i] - mean) * rstd;
                if (column(j) + kChunk > cols) {
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) xh[j][i] = column(j) + i < cols ? xh[j][i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    dg[j][i] += dy[j][i] * xh[j][i];
                    db[j][i] += dy[j][i];
                    dy[j][i] *= gamma[j][i];
                    s[0] += dy[j][i];
                    s[1] += dy[j][i] * xh[j][i];
                }
            }
        }
        if (!a.dx) continue;
        row_sums<TPR>(s, s_part[turn]); // (two places in turn: no wave overwrites what another still reads)
        turn ^= 1;
        if (own) {
            const float c0 = s[0] * inv_n, c1 = s[1] * inv_n;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) dy[j][i] = rstd * (dy[j][i] - c0 - xh[j][i] * c1);
                if (column(j) < cols) store_chunk<true>(static_cast<T *>(a.dx) + r * a.lddx, column(j), cols, dy[j]);
            }
        }
    }
    if (!a.sum_gamma) return;
    float *out[2] = {a.sum_gamma + blockIdx.x * a.block_stride, a.sum_beta + blockIdx.x * a.block_stride};
    if constexpr (rows_per_block == 1) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = column(j);
            if (c < cols) {
                store_chunk(out[0], c, cols, dg[j]);
                store_chunk(out[1], c, cols, db[j]);
            }
        }
    } else {
        // the rows' groups of the workgroup are added in turn
        __shared__ float s_acc[rows_per_block][TPR * kChunk];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kChunk; ++i) s_acc[threadIdx.x / TPR][t * kChunk + i] = k ? db[j][i] : dg[j][i];
                __syncthreads();
                for (int c = threadIdx.x; c < TPR * kChunk; c += BLOCK) {
                    float v = s_acc[0][c];
                    for (int w = 1; w < rows_per_block; ++w) v += s_acc[w][c];
                    const int64_t col = (int64_t)j * TPR * kChunk + c;
                    if (col < a.cols) out[k][col] = v;
                }
            }
        }
    }
}

// Rows of any length: dx from two passes over the row, a workgroup to each (2000 x 40000 bfloat16 215 us, with the sums below
// and their join 285: 480 MB, 1.7 TB/s).
template <int DT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_long_kernel(NormBwdArgs a)
{
    using T = elem_t<DT>;
    __shared__ float s_part[BLOCK / kWaveSize][2];
    const int64_t r = blockIdx.x;
    const float mean = a.mean[r], rstd = a.rstd[r], inv_n = 1.0f / (float)a.cols;
    const T *pdy = static_cast<const T *>(a.dy) + r * a.lddy, *px = static_cast<const T *>(a.x) + r * a.ldx;
    float s[2] = {0.0f, 0.0f};
    float dy[kChunk], x[kChunk], g[kChunk];
    for (int64_t c = (int64_t)threadIdx.x * kChunk; c < a.cols; c += BLOCK * kChunk) {
        load_chunk(pdy, c, a.cols, dy);
        load_chunk(px, c, a.cols, x);
        load_gain(a.gamma, c, a.cols, 1.0f, g);
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            const float gi = c + i < a.cols ? dy[i] * g[i] : 0.0f;
            s0 += gi;
            s1 += c + i < a.cols ? gi * ((x[i] - mean) * rstd) : 0.0f;
        }
        s[0] += s0, s[1] += s1;
    }
    row_sums<BLOCK>(s, s_part);
    for (int64_t c = (int64_t)threadIdx.x * kChunk; c < a.cols; c += BLOCK * kChunk) {
        load_chunk(pdy, c, a.cols, dy);
        load_chunk(px, c, a.cols, x);
        load_gain(a.gamma, c, a.cols, 1.0f, g);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) x[i] = rstd * (dy[i] * g[i] - s[0] * inv_n - (x[i] - mean) * rstd * (s[1] * inv_n));
        store_chunk(static_cast<T *>(a.dx) + r * a.lddx, c, a.cols, x);
    }
}

// ... and the sums over a slice of rows, eight columns to a thread, the loads of four rows on their way at a time (rows of fewer than 8
// values: of one).
template <int DT, bool SHORT>
__global__ __launch_bounds__(256) void norm_bwd_columns_kernel(NormBwdArgs a, int64_t rows_per_slice)
{
    using T = elem_t<DT>;
    constexpr int together = SHORT ? 1 : 4;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kChunk;
    if (c >= a.cols) return;
    const int64_t r0 = (int64_t)blockIdx.y * rows_per_slice, r1 = min(r0 + rows_per_slice, a.rows);
    float dg[kChunk] = {}, db[kChunk] = {};
    for (int64_t r = r0; r < r1; r += together) {
        float dy[together][kChunk], x[together][kChunk], mean[together], rstd[together];
        if constexpr (SHORT) {
            load_chunk(static_cast<const T *>(a.dy) + r * a.lddy, c, a.cols, dy[0]);
            load_chunk(static_cast<const T *>(a.x) + r * a.ldx, c, a.cols, x[0]);
            mean[0] = a.mean[r], rstd[0] = a.rstd[r];
        } else {
            Raw<T> raw_dy[together], raw_x[together];
#pragma unroll
            for (int k = 0; k < together; ++k) {
                const int64_t q = min(r + k, r1 - 1);
                raw_dy[k] = load_raw(static_cast<const T *>(a.dy) + q * a.lddy, c, a.cols);
                raw_x[k] = load_raw(static_cast<const T *>(a.x) + q * a.ldx, c, a.cols);
                mean[k] = a.mean[q], rstd[k] = a.rstd[q];
            }
#pragma unroll
            for (int k = 0; k < together; ++k) {
                values_of(raw_dy[k], c, a.cols, dy[k]);
                values_of(raw_x[k], c, a.cols, x[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < together; ++k) {
            if (r + k >= r1) break;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) dg[i] += c + i < a.cols ? dy[k][i] * ((x[k][i] - mean[k]) * rstd[k]) : 0.0f, db[i] += dy[k][i];
        }
    }
    store_chunk(a.sum_gamma + blockIdx.y * a.block_stride, c, a.cols, dg);
    store_chunk(a.sum_beta + blockIdx.y * a.block_stride, c, a.cols, db);
}

} // namespace dqrm_mx
