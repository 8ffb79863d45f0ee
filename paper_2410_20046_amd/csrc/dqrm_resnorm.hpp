// The join of a block with its residual stream, and the norms around it, forward and backward (gfx950, wave64).
//
//   out = res_scale r + gate N1(u), y = N2(out);  N(v) = (v - mean) rstd gamma + beta, rstd = 1 / sqrt(sum (v - mean)^2 / n + eps), a layer
//   norm's mean = sum v / n, an RMS norm's mean = 0
//   With z the normalised values: of y's gradient dy, e = dy gamma2, g = dout + rstd2 (e - mean(e) - z2 mean(e z2)) (RMS: without mean(e)),
//   dr = res_scale g, and the same with e = g gate gamma1 gives du.  The vectors' gradients follow from four sums over rows:
//   S0 = sum g, S1 = sum g z1, S2 = sum dy z2, S3 = sum dy; dgamma1 = gate S1, dbeta1 = gate S0, dgate = gamma1 S1 + beta1 S0, dgamma2 = S2,
//   dbeta2 = S3 (no N1: z1 = u, dgate = S1).
//
// All in 32 bits but for the layer norm's sums, which are in 64.  N2 sees out before its rounding.
#pragma once

#include "dqrm_norm.hpp"

namespace dqrm_resnorm {

using namespace dqrm_mx;

struct Params {
    int post, pre; // DQRM_NORM_*
    const float *post_gamma, *post_beta, *gate, *pre_gamma, *pre_beta; // or null: 1 and 0
    float res_scale, post_eps, pre_eps;
};

struct FwdArgs {
    Params p;
    const void *u, *r;
    int64_t ldu, ldr, rows, cols;
    void *out, *y; // y or null
    int64_t ldo, ldy;
    float *stats;            // [4][all_rows], from this launch's first row on; or null
    int64_t all_rows;
    uint8_t *codes, *scales; // MXFP4 of y, or null
};

// A chunk on its way.  Rows of fewer than 8 values (SHORT) are loaded value by value.
template <bool SHORT, typename T>
__device__ __forceinline__ Raw<T> request(const T *row, int c, int cols)
{
    if constexpr (SHORT) {
        const Vec8<T> v = load_vec(row, c, cols, false);
        Raw<T> raw;
        __builtin_memcpy(&raw, &v, sizeof(v));
        return raw;
    } else {
        return load_raw(row, c, cols);
    }
}
template <bool SHORT, typename T>
__device__ __forceinline__ void arrived(const Raw<T> &raw, int c, int cols, float (&v)[kChunk])
{
    if constexpr (SHORT) {
        Vec8<T> t;
        __builtin_memcpy(&t, &raw, sizeof(t));
        to_float(t, v);
    } else {
        values_of(raw, c, cols, v);
    }
}

__device__ __forceinline__ float sum8(const float (&v)[kChunk]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ float squares8(const float (&v)[kChunk])
{
    return ((v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3])) + ((v[4] * v[4] + v[5] * v[5]) + (v[6] * v[6] + v[7] * v[7]));
}

// ---- sums over the threads of a row -------------------------------------------------------------------------------------
// Lanes add what a lane 8, 4, 2, 1 places on in their 16 has (after each of these steps the values repeat with that period, so all lanes
// get the same bits), then rows of 16 and halves of the wave are exchanged: no step goes through LDS.
__device__ __forceinline__ float moved(float v, int how)
{
    switch (how) {
    case 8: return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, true));
    case 4: return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xF, 0xF, true));
    case 2: return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xF, 0xF, true));
    default: return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xF, 0xF, true));
    }
}
__device__ __forceinline__ double moved(double v, int how)
{
    return __hiloint2double(__float_as_int(moved(__int_as_float(__double2hiint(v)), how)), __float_as_int(moved(__int_as_float(__double2loint(v)), how)));
}
// v of this row of 16 lanes and of its neighbour, of this half and of the other one: in the same order in both
__device__ __forceinline__ float with_other_row(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap((unsigned)__float_as_int(v), (unsigned)__float_as_int(v), false, false);
    return __int_as_float((int)r[0]) + __int_as_float((int)r[1]);
}
__device__ __forceinline__ float with_other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap((unsigned)__float_as_int(v), (unsigned)__float_as_int(v), false, false);
    return __int_as_float((int)r[0]) + __int_as_float((int)r[1]);
}
__device__ __forceinline__ double with_other_row(double v)
{
    const auto h = __builtin_amdgcn_permlane16_swap((unsigned)__double2hiint(v), (unsigned)__double2hiint(v), false, false);
    const auto l = __builtin_amdgcn_permlane16_swap((unsigned)__double2loint(v), (unsigned)__double2loint(v), false, false);
    return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}
__device__ __forceinline__ double with_other_half(double v)
{
    const auto h = __builtin_amdgcn_permlane32_swap((unsigned)__double2hiint(v), (unsigned)__double2hiint(v), false, false);
    const auto l = __builtin_amdgcn_permlane32_swap((unsigned)__double2loint(v), (unsigned)__double2loint(v), false, false);
    return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}

// Sums over the TPR threads of a row; every one of them gets them.  TPR > 64: over the row's waves by way of s_part (a place to each wave of
// the workgroup), which the next call must not take again before another barrier.
template <int TPR, int N, typename V>
__device__ __forceinline__ void totals(V (&v)[N], V (*s_part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] += moved(v[i], 8);
        v[i] += moved(v[i], 4);
        v[i] += moved(v[i], 2);
        v[i] += moved(v[i], 1);
        if constexpr (TPR > 16) v[i] = with_other_half(with_other_row(v[i]));
    }
    if constexpr (TPR > kWaveSize) {
        constexpr int waves = TPR / kWaveSize; // of a row
        const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x / kWaveSize;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s_part[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = s_part[(wave & ~(waves - 1)) + (lane & (waves - 1))][i];
            if constexpr (waves > 8) v[i] += moved(v[i], 8);
            if constexpr (waves > 4) v[i] += moved(v[i], 4);
            if constexpr (waves > 2) v[i] += moved(v[i], 2);
            v[i] += moved(v[i], 1);
        }
    }
}

// Places for a row's sums of the waves
template <int WAVES>
struct Parts {
    double layer[WAVES][2];
    float rms[WAVES][1];
};

// Mean and rstd of a row's values v (0 past its end) over its TPR threads.  One reduction: a thread takes the mean m of its own n values, and
// their squares about it; the sums over threads of n m and of n m^2 + squares are in 64 bits, where the difference that the variance is
// loses 2^-52 of the mean's square, less than the values' own rounding makes of it.
template <int TPR, int CH, int WAVES, typename F>
__device__ __forceinline__ void statistics(int kind, float eps, int cols, const float (&v)[CH][kChunk], Parts<WAVES> &parts, float &mean, float &rstd, F column)
{
    if (kind == DQRM_NORM_LAYER) {
        float own = 0.0f, squares = 0.0f;
        int n = 0;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            own += sum8(v[j]);
            n += min(max(cols - column(j), 0), kChunk);
        }
        own = n == CH * kChunk ? own * (1.0f / (CH * kChunk)) : n > 0 ? own / (float)n : 0.0f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float d[kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) d[i] = v[j][i] - own;
            if (column(j) + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) d[i] = column(j) + i < cols ? d[i] : 0.0f;
            }
            squares += squares8(d);
        }
        const double weight = (double)n * (double)own;
        double sum[2] = {weight, fma(weight, (double)own, (double)squares)};
        totals<TPR>(sum, parts.layer);
        const double inv_n = 1.0 / cols, middle = sum[0] * inv_n, var = sum[1] * inv_n - middle * middle;
        mean = (float)middle;
        rstd = 1.0f / sqrtf((var < 0.0 ? 0.0f : (float)var) + eps); // (a NaN stays)
    } else {
        float sq[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) sq[0] += squares8(v[j]);
        totals<TPR>(sq, parts.rms);
        mean = 0.0f;
        rstd = 1.0f / sqrtf(sq[0] / (float)cols + eps);
    }
}

// Where the columns' vectors are for all rows of a workgroup
enum class Gains { registers, lds, memory };

// TPR threads to a row, CH chunks of 8 values to a thread, the next rows of u and r requested before this one's sums.  Bound by its bytes, two
// reads and two writes, where a copy has 5.0 TB/s: with two layer norms, all five vectors and the statistics 65536 x 1024 bfloat16 106 us, 5.1 TB/s, 32768 x 4096 224-238 us, 4.5-4.8; wide rows by the two
// reductions' latency as well, for as many rows as are in a CU's registers: 16384 x 8192 233-257 us as the matrices lie, 4.2-4.6.  With MXFP4 codes by
// their conversion and stores of four bytes to a lane as well: 16384 x 8192 266 us, 4.3 TB/s, 32768 x 4096 324, 3.5, 65536 x 1024 141, 4.1.
template <int DT, int TPR, int CH, int BLOCK, bool SHORT, Gains GAINS, bool CODES>
__global__ __launch_bounds__(BLOCK) void resnorm_fwd_kernel(FwdArgs a)
{
    using T = elem_t<DT>;
    constexpr bool held = GAINS == Gains::registers;
    constexpr int rows_per_block = BLOCK / TPR;
    __shared__ Parts<BLOCK / kWaveSize> s_parts[2][2]; // (two rows in turn: no wave overwrites what another still reads)
    const int t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * rows_per_block;
    const int cols = (int)a.cols;
    const int64_t cp = codes_pitch(cols), sp = scales_pitch(cols);
    auto column = [&](int j) { return (j * TPR + t) * kChunk; };
    int64_t r = (int64_t)blockIdx.x * rows_per_block + threadIdx.x / TPR;
    constexpr int ahead = CH == 1 ? 2 : 1; // rows on their way
    Raw<T> next_u[ahead][CH], next_r[ahead][CH];
    // (a group past the last row works on that row and writes nothing)
    auto ask = [&](int slot, int64_t at) {
        const int64_t q = min(at, a.rows - 1);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            next_u[slot][j] = request<SHORT>(static_cast<const T *>(a.u) + q * a.ldu, column(j), cols);
            next_r[slot][j] = request<SHORT>(static_cast<const T *>(a.r) + q * a.ldr, column(j), cols);
        }
    };
#pragma unroll
    for (int k = 0; k < ahead; ++k) ask(k, r + k * step);
    // gate N1(u) = z (gate gamma1) + gate beta1
    // which: 0 gate gamma1, 1 gate beta1, 2 gamma2, 3 beta2
    auto fetch = [&](int which, int c, float(&v)[kChunk]) {
        load_gain(which == 0 ? a.p.post_gamma : which == 1 ? a.p.post_beta : which == 2 ? a.p.pre_gamma : a.p.pre_beta, c, cols, which & 1 ? 0.0f : 1.0f, v);
        if (which < 2 && a.p.gate) {
            float gate[kChunk];
            load_gain(a.p.gate, c, cols, 1.0f, gate);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] *= gate[i];
        } // (a gate of 1 otherwise)
    };
    constexpr int in_lds = GAINS == Gains::lds ? TPR * CH * kChunk : 1;
    __shared__ __align__(16) float s_gains[4][in_lds];
    float gains[4][held ? CH : 1][kChunk];
    if constexpr (held) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) fetch(k, column(j), gains[k][j]);
    } else if constexpr (GAINS == Gains::lds) {
        for (int c = threadIdx.x * kChunk; c < in_lds; c += BLOCK * kChunk)
            for (int k = 0; k < 4; ++k) {
                float v[kChunk];
                fetch(k, c, v);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) s_gains[k][c + i] = v[i];
            }
        __syncthreads();
    }
    auto gain_of = [&](int which, int j, float(&v)[kChunk]) {
        int c = column(j);
        asm volatile("" : "+v"(c)); // (a load of this row: taken out of the loop over rows, the vectors would be in registers after all)
        if constexpr (held) {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = gains[which][j][i];
        } else if constexpr (GAINS == Gains::lds) {
            __builtin_memcpy(v, __builtin_assume_aligned(&s_gains[which][c], 16), sizeof(v));
        } else {
            fetch(which, c, v);
        }
    };
    auto one_row = [&](int slot, int turn) __attribute__((always_inline)) {
        const bool own = r < a.rows;
        float v[CH][kChunk];
        Raw<T> res[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            arrived<SHORT>(next_u[slot][j], column(j), cols, v[j]);
            res[j] = next_r[slot][j];
        }
        ask(slot, r + ahead * step);
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (a.p.post != DQRM_NORM_NONE) statistics<TPR>(a.p.post, a.p.post_eps, cols, v, s_parts[turn][0], mean1, rstd1, column);
        const auto joined = [&](float u, float r, float gain, float offset) { return a.p.res_scale * r + ((u - mean1) * rstd1 * gain + offset); };
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float x[kChunk], gain[kChunk], offset[kChunk];
            arrived<SHORT>(res[j], column(j), cols, x);
            gain_of(0, j, gain);
            gain_of(1, j, offset);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[j][i] = joined(v[j][i], x[i], gain[i], offset[i]);
            if (column(j) + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[j][i] = column(j) + i < cols ? v[j][i] : 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (a.p.pre != DQRM_NORM_NONE) statistics<TPR>(a.p.pre, a.p.pre_eps, cols, v, s_parts[turn][1], mean2, rstd2, column);
        // (out may be r's or u's memory: a thread stores the values that it alone has taken from there; what else its last vector held it
        // has dropped)
#pragma unroll
        for (int j = 0; j < CH; ++j)
            if (own && column(j) < cols) store_chunk<true>(static_cast<T *>(a.out) + r * a.ldo, column(j), cols, v[j]);
        if (a.p.pre != DQRM_NORM_NONE) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = column(j);
                float gamma[kChunk], beta[kChunk];
                gain_of(2, j, gamma);
                gain_of(3, j, beta);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[j][i] = (v[j][i] - mean2) * rstd2 * gamma[i] + beta[i];
                // (past the row's end 0: the padding of the codes)
                if (c + kChunk > cols) {
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) v[j][i] = c + i < cols ? v[j][i] : 0.0f;
                }
                if (own && a.y && c < cols) store_chunk<true>(static_cast<T *>(a.y) + r * a.ldy, c, cols, v[j]);
                if (CODES && own && c < cp * 2) write_chunk(a.codes + r * cp, a.scales + r * sp, (unsigned)(c / kChunk), v[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (own && t == 0 && a.stats) {
            if (a.p.post != DQRM_NORM_NONE) a.stats[r] = mean1, a.stats[a.all_rows + r] = rstd1;
            if (a.p.pre != DQRM_NORM_NONE) a.stats[2 * a.all_rows + r] = mean2, a.stats[3 * a.all_rows + r] = rstd2;
        }
    };
    while (r - threadIdx.x / TPR < a.rows) {
        one_row(0, 0);
        r += step;
        if (r - threadIdx.x / TPR >= a.rows) break;
        one_row(ahead - 1, 1);
        r += step;
    }
}

struct BwdArgs {
    Params p;
    const void *dout, *dy, *u, *out; // dout or null: 0; dy, out where there is N2; u where there is N1 or the vectors' gradients are wanted
    int64_t lddout, lddy, ldu, ldo, rows, cols;
    const float *stats;
    void *du, *dr; // or null
    int64_t lddu, lddr;
    float *partial; // [workgroups][4][cols] of S0 .. S3, or null
};

// The rows of dout, dy, u and out in registers, the next ones on their way; a thread has the same columns in every row of its workgroup's
// slice and keeps their sums, so that all is read once.  Bound by its bytes, four reads and two writes: 32768 x 4096 bfloat16 285 us, 5.7 TB/s,
// 16384 x 8192 296 us, 5.4, 32768 x 512 float 71 us, 5.7; 8192 x 8192 float, a few of whose registers are in memory, 361, 4.5.  Of rows beyond 8192 values a
// thread of 1024 has two chunks, 64 values of sums and as many of the row beside the next row's, where there are 128 registers: the rest is in memory,
// read and written for every row, and that is what bounds it: 10000 x 16384 bfloat16 1490 us, 1.3 TB/s.
template <int DT, int TPR, int CH, int BLOCK, bool SHORT, Gains GAINS>
__global__ __launch_bounds__(BLOCK) void resnorm_bwd_kernel(BwdArgs a)
{
    constexpr bool held = GAINS == Gains::registers;
    using T = elem_t<DT>;
    constexpr int rows_per_block = BLOCK / TPR;
    __shared__ float s_part[2][2][BLOCK / kWaveSize][2]; // (two rows in turn)
    const int t = threadIdx.x % TPR;
    const int cols = (int)a.cols;
    const float inv_n = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * rows_per_block;
    const bool pre = a.p.pre != DQRM_NORM_NONE, post = a.p.post != DQRM_NORM_NONE;
    auto column = [&](int j) { return (j * TPR + t) * kChunk; };
    int64_t r = (int64_t)blockIdx.x * rows_per_block + threadIdx.x / TPR;
    Raw<T> next_dout[CH], next_dy[CH], next_u[CH], next_out[CH];
    float next_mean1 = 0.0f, next_rstd1 = 1.0f, next_mean2 = 0.0f, next_rstd2 = 1.0f;
    auto ask = [&](int64_t at) {
        const int64_t q = min(at, a.rows - 1);
        if (post) next_mean1 = a.stats[q], next_rstd1 = a.stats[a.rows + q];
        if (pre) next_mean2 = a.stats[2 * a.rows + q], next_rstd2 = a.stats[3 * a.rows + q];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (a.dout) next_dout[j] = request<SHORT>(static_cast<const T *>(a.dout) + q * a.lddout, column(j), cols);
            if (a.u) next_u[j] = request<SHORT>(static_cast<const T *>(a.u) + q * a.ldu, column(j), cols);
            if (pre) {
                next_dy[j] = request<SHORT>(static_cast<const T *>(a.dy) + q * a.lddy, column(j), cols);
                next_out[j] = request<SHORT>(static_cast<const T *>(a.out) + q * a.ldo, column(j), cols);
            }
        }
    };
#pragma unroll
    for (int j = 0; j < CH; ++j) next_dout[j] = next_dy[j] = next_u[j] = next_out[j] = Raw<T>{};
    ask(r);
    float s0[CH][kChunk] = {}, s1[CH][kChunk] = {}, s2[CH][kChunk] = {}, s3[CH][kChunk] = {};
    // which: 0 gate gamma1 (without N1 the gate), 1 gamma2
    auto fetch = [&](int which, int c, float(&v)[kChunk]) {
        load_gain(which ? a.p.pre_gamma : a.p.post_gamma, c, cols, 1.0f, v);
        if (!which && a.p.gate) {
            float gate[kChunk];
            load_gain(a.p.gate, c, cols, 1.0f, gate);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] *= gate[i];
        }
    };
    constexpr int in_lds = GAINS == Gains::lds ? TPR * CH * kChunk : 1;
    __shared__ __align__(16) float s_gains[2][in_lds];
    float gains[2][held ? CH : 1][kChunk];
    if constexpr (held) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) fetch(k, column(j), gains[k][j]);
    } else if constexpr (GAINS == Gains::lds) {
        for (int c = threadIdx.x * kChunk; c < in_lds; c += BLOCK * kChunk)
            for (int k = 0; k < 2; ++k) {
                float v[kChunk];
                fetch(k, c, v);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) s_gains[k][c + i] = v[i];
            }
        __syncthreads();
    }
    auto gain_of = [&](int which, int j, float(&v)[kChunk]) {
        int c = column(j);
        asm volatile("" : "+v"(c)); // (a load of this row, as in the forward)
        if constexpr (held) {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = gains[which][j][i];
        } else if constexpr (GAINS == Gains::lds) {
            __builtin_memcpy(v, __builtin_assume_aligned(&s_gains[which][c], 16), sizeof(v));
        } else {
            fetch(which, c, v);
        }
    };
    int turn = 0;
    for (; r - threadIdx.x / TPR < a.rows; r += step, turn ^= 1) {
        const bool own = r < a.rows;
        const float mean1 = next_mean1, rstd1 = next_rstd1, mean2 = next_mean2, rstd2 = next_rstd2;
        float g[CH][kChunk], dy[CH][kChunk], z1[CH][kChunk], z2[CH][kChunk];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            arrived<SHORT>(next_dout[j], column(j), cols, g[j]);
            arrived<SHORT>(next_dy[j], column(j), cols, dy[j]);
            arrived<SHORT>(next_u[j], column(j), cols, z1[j]);
            arrived<SHORT>(next_out[j], column(j), cols, z2[j]);
        }
        ask(r + step);
        if (pre) {
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                float gain[kChunk];
                gain_of(1, j, gain);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    z2[j][i] = (z2[j][i] - mean2) * rstd2;
                    if (column(j) + kChunk > cols) z2[j][i] = column(j) + i < cols ? z2[j][i] : 0.0f;
                    if (own) s2[j][i] += dy[j][i] * z2[j][i], s3[j][i] += dy[j][i];
                    dy[j][i] *= gain[i];
                    s[0] += dy[j][i];
                    s[1] += dy[j][i] * z2[j][i];
                }
            }
            totals<TPR>(s, s_part[turn][0]);
            const float c0 = a.p.pre == DQRM_NORM_LAYER ? s[0] * inv_n : 0.0f, c1 = s[1] * inv_n;
#pragma unroll
            for (int j = 0; j < CH; ++j)
#pragma unroll
                for (int i = 0; i < kChunk; ++i) g[j][i] += rstd2 * (dy[j][i] - c0 - z2[j][i] * c1);
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float gain[kChunk];
            gain_of(0, j, gain);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                z1[j][i] = (z1[j][i] - mean1) * rstd1;
                if (column(j) + kChunk > cols) {
                    z1[j][i] = column(j) + i < cols ? z1[j][i] : 0.0f;
                    g[j][i] = column(j) + i < cols ? g[j][i] : 0.0f;
                }
                if (own) s0[j][i] += g[j][i], s1[j][i] += g[j][i] * z1[j][i];
                dy[j][i] = g[j][i] * gain[i];
                s[0] += dy[j][i];
                s[1] += dy[j][i] * z1[j][i];
            }
        }
        float c0 = 0.0f, c1 = 0.0f, by = 1.0f;
        if (post) {
            totals<TPR>(s, s_part[turn][1]);
            c0 = a.p.post == DQRM_NORM_LAYER ? s[0] * inv_n : 0.0f, c1 = s[1] * inv_n, by = rstd1;
        }
        // (du and dr may be the memory of a matrix that is read: a thread stores the values that it alone has taken from there)
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if (!own || column(j) >= cols) continue;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                dy[j][i] = by * (dy[j][i] - c0 - z1[j][i] * c1);
                g[j][i] *= a.p.res_scale;
            }
            if (a.du) store_chunk<true>(static_cast<T *>(a.du) + r * a.lddu, column(j), cols, dy[j]);
            if (a.dr) store_chunk<true>(static_cast<T *>(a.dr) + r * a.lddr, column(j), cols, g[j]);
        }
    }
    if (!a.partial) return;
    float *out = a.partial + (int64_t)blockIdx.x * 4 * cols;
    auto store_sums = [&](int k, const float(&v)[CH][kChunk]) {
        if constexpr (rows_per_block == 1) {
#pragma unroll
            for (int j = 0; j < CH; ++j)
                if (column(j) < cols) store_chunk(out + (int64_t)k * cols, column(j), cols, v[j]);
        } else {
            // the rows' groups of the workgroup are added in turn
            __shared__ float s_acc[rows_per_block][TPR * kChunk];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kChunk; ++i) s_acc[threadIdx.x / TPR][t * kChunk + i] = v[j][i];
                __syncthreads();
                for (int c = threadIdx.x; c < TPR * kChunk; c += BLOCK) {
                    float sum = s_acc[0][c];
                    for (int w = 1; w < rows_per_block; ++w) sum += s_acc[w][c];
                    const int col = j * TPR * kChunk + c;
                    if (col < cols) out[(int64_t)k * cols + col] = sum;
                }
            }
        }
    };
    store_sums(0, s0);
    store_sums(1, s1);
    store_sums(2, s2);
    store_sums(3, s3);
}

// The workgroups' sums in turn, 16 lanes with every 16th each, and the five vectors' gradients [5][cols] from them: post gamma and beta,
// gate, pre gamma and beta; those of a norm that is not there are 0.  Latency: 256 sums of 4096 columns 7 us, of 512 5.
static __global__ __launch_bounds__(256) void resnorm_join_kernel(const float *partial, int n, int cols, Params p, float *dparams)
{
    __shared__ float s[4][16][17];
    const int c = (int)blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float sum = 0.0f;
        if (c < cols) sum = add_strided(sum, partial + ((int64_t)slice * 4 + k) * cols + c, (int64_t)16 * 4 * cols, (n - slice + 15) / 16);
        s[k][slice][threadIdx.x & 15] = sum;
    }
    __syncthreads();
    if (slice != 0 || c >= cols) return;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[k] = s[k][0][threadIdx.x];
        for (int i = 1; i < 16; ++i) v[k] += s[k][i][threadIdx.x];
    }
    const bool pre = p.pre != DQRM_NORM_NONE, post = p.post != DQRM_NORM_NONE;
    const float gate = p.gate ? p.gate[c] : 1.0f, gamma = p.post_gamma ? p.post_gamma[c] : 1.0f, beta = p.post_beta ? p.post_beta[c] : 0.0f;
    const int64_t C = cols;
    dparams[c] = post ? gate * v[1] : 0.0f;
    dparams[C + c] = post ? gate * v[0] : 0.0f;
    dparams[2 * C + c] = post ? gamma * v[1] + beta * v[0] : v[1];
    dparams[3 * C + c] = pre ? v[2] : 0.0f;
    dparams[4 * C + c] = pre ? v[3] : 0.0f;
}

} // namespace dqrm_resnorm
