// Products of MXFP4 matrices with few rows of A (requests), from codes or from activations as they are (gfx950, wave64).
//
// What such a product costs is W's bytes, read once.  A workgroup has ST strips of 16 rows of W; its eight waves cut k between
// them and read W straight into the operand registers of v_mfma_scale_f32_16x16x128_f8f6f4 (lane l: row l % 16, block l / 16 of 128
// values), no LDS on the way, the next batch of groups in flight while this one is multiplied.  The waves' sums meet in LDS in a fixed
// order.
#pragma once

#include "dqrm_mx_gemm.hpp"
#include "dqrm_norm.hpp"

namespace dqrm_mx {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kFewWaves = 8, kFewBlock = kFewWaves * kWaveSize;
constexpr int kFewChunks = 4; // chunks of 8 activations to a thread, where the product quantises them itself

__device__ __forceinline__ v4f mfma_16x16x128(uint4 a, uint4 b, v4f c, unsigned scale_a, unsigned scale_b)
{
    const v8i va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, kFp4, kFp4, 0, (int)scale_a, 0, (int)scale_b);
}

// Where A's codes come from.
enum FewSource { kFewCodes, kFewPlain, kFewNorm };

struct FewArgs {
    MatmulArgs g; // (a_codes, a_scales: for kFewCodes)
    NormArgs x;   // activations, and the norm's gain and offset: for the others
};

// kFewPlain, kFewNorm: the m <= 8 rows of x to codes and scales in LDS, by 8 / m waves to a row, each thread's values in registers
// (k <= waves of a row * 64 * 4 * 8).  Rows past the last one repeat it.
template <typename T, bool NORM>
__device__ __forceinline__ void quantise_few(const NormArgs &a, uint8_t *codes, uint8_t *scales, float (*s_sum)[2])
{
    const int rows = (int)a.rows;
    const int log_waves = rows <= 1 ? 3 : rows <= 2 ? 2 : rows <= 4 ? 1 : 0; // of a row
    const int wave = threadIdx.x / kWaveSize, waves = 1 << log_waves;
    const int own = wave >> log_waves, r = min(own, rows - 1);
    const int t = threadIdx.x & ((kWaveSize << log_waves) - 1), stride = kWaveSize << log_waves;
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    float x[kFewChunks][kChunk];
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) load_chunk(row, (int64_t)(j * stride + t) * kChunk, a.cols, r + 1 < rows, x[j]);
    if constexpr (NORM) {
        auto row_sum = [&](float v, int k) {
#pragma unroll
            for (int d = kWaveSize / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWaveSize);
            if ((threadIdx.x & (kWaveSize - 1)) == 0) s_sum[wave][k] = v;
            __syncthreads();
            const int first = own << log_waves;
            float sum = s_sum[first][k];
            for (int w = 1; w < waves; ++w) sum += s_sum[first + w][k];
            return sum;
        };
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j)
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v += x[j][i];
        const float mean = row_sum(v, 0) / (float)a.cols;
        v = 0.0f;
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j) {
            const int64_t c = (int64_t)(j * stride + t) * kChunk;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                x[j][i] -= mean;
                if (c + i < a.cols) v += x[j][i] * x[j][i];
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum(v, 1) / (float)a.cols + a.eps);
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j) {
            const int64_t c = (int64_t)(j * stride + t) * kChunk;
            if (c >= a.cols) continue;
            float g[kChunk], b[kChunk];
            load_gain(a.gamma, c, a.cols, 1.0f, g);
            load_gain(a.beta, c, a.cols, 0.0f, b);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) x[j][i] = c + i < a.cols ? x[j][i] * rstd * g[i] + b[i] : 0.0f;
        }
        // (a chunk past the row's end: x - mean must not count)
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j)
            if ((int64_t)(j * stride + t) * kChunk >= a.cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = 0.0f;
            }
    }
    const int64_t pitch = codes_pitch(a.cols), spitch = scales_pitch(a.cols), chunks = pitch / 4;
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) {
        const int chunk = j * stride + t;
        if (chunk < chunks && own < rows) write_chunk(codes + r * pitch, scales + r * spitch, (unsigned)chunk, x[j]);
    }
    __syncthreads();
}

// MT: groups of 16 rows of A.
template <int DT, FewSource SRC, int MT, int ST>
__global__ __launch_bounds__(kFewBlock) void few_kernel(FewArgs a)
{
    using T = elem_t<DT>;
    static_assert(SRC == kFewCodes || MT == 1, "quantise_few has up to 8 rows");
    constexpr int batch = MT * ST > 4 ? 2 : 4; // groups of 128 values that are in flight together
    __shared__ v4f s_acc[kFewWaves][ST][MT][kWaveSize];
    __shared__ float s_sum[kFewWaves][2];
    extern __shared__ __align__(16) uint8_t s_x[]; // codes, then scales, of x
    const MatmulArgs &g = a.g;
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6);
    const int row = lane & 15, block = lane >> 4;
    const int64_t groups = groups_of(g.k), cp = groups * 64, sp = groups * 4;
    const int64_t n0 = (int64_t)blockIdx.x * (ST * 16);
    const int from = (int)(groups * wave / kFewWaves), to = (int)(groups * (wave + 1) / kFewWaves);

    struct Batch {
        uint4 w[ST][batch], x[MT][batch];
        unsigned ws[ST][batch], xs[MT][batch];
    };
    const uint8_t *w_codes[ST], *w_scales[ST];
#pragma unroll
    for (int s = 0; s < ST; ++s) {
        const int64_t n = min(n0 + s * 16 + row, g.n - 1);
        w_codes[s] = g.b_codes + n * cp + block * 16, w_scales[s] = g.b_scales + n * sp + block;
    }
    const uint8_t *x_codes[MT], *x_scales[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t r = min((int64_t)(m * 16 + row), g.m - 1);
        const uint8_t *codes = SRC == kFewCodes ? g.a_codes : s_x, *scales = SRC == kFewCodes ? g.a_scales : s_x + g.m * cp;
        x_codes[m] = codes + r * cp + block * 16, x_scales[m] = scales + r * sp + block;
    }
    // (groups past the wave's last one repeat it: loaded, not multiplied)
    auto load_w = [&](int k, Batch &b) {
#pragma unroll
        for (int i = 0; i < batch; ++i) {
            const int at = min(k + i, to - 1);
#pragma unroll
            for (int s = 0; s < ST; ++s) {
                typedef unsigned u4 __attribute__((ext_vector_type(4)));
                const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(w_codes[s] + (int64_t)at * 64));
                b.w[s][i] = make_uint4(v.x, v.y, v.z, v.w);
                b.ws[s][i] = w_scales[s][(int64_t)at * 4];
            }
        }
    };
    auto load_x = [&](int k, Batch &b) {
#pragma unroll
        for (int i = 0; i < batch; ++i) {
            const int at = min(k + i, to - 1);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                b.x[m][i] = *reinterpret_cast<const uint4 *>(x_codes[m] + (int64_t)at * 64);
                b.xs[m][i] = x_scales[m][(int64_t)at * 4];
            }
        }
    };
    v4f acc[ST][MT] = {};
    auto multiply = [&](int k, const Batch &b) {
#pragma unroll
        for (int i = 0; i < batch; ++i)
            if (k + i < to) {
#pragma unroll
                for (int s = 0; s < ST; ++s)
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[s][m] = mfma_16x16x128(b.w[s][i], b.x[m][i], acc[s][m], b.ws[s][i], b.xs[m][i]);
            }
    };
    Batch now, next;
    if (from < to) load_w(from, now);
    if constexpr (SRC != kFewCodes) quantise_few<T, SRC == kFewNorm>(a.x, s_x, s_x + g.m * cp, s_sum);
    if (from < to) {
        load_x(from, now);
        for (int k = from; k < to; k += batch) {
            if (k + batch < to) {
                load_w(k + batch, next);
                load_x(k + batch, next);
            }
            multiply(k, now);
            now = next;
        }
    }
#pragma unroll
    for (int s = 0; s < ST; ++s)
#pragma unroll
        for (int m = 0; m < MT; ++m) s_acc[wave][s][m][lane] = acc[s][m];
    __syncthreads();
    // accumulator i of lane l: row 4 (l / 16) + i of the strip, row l % 16 of A
    constexpr int outputs = ST * MT * 256;
    for (int o = threadIdx.x; o < outputs; o += kFewBlock) {
        const int in_strip = o % 16, s = o / 16 % ST, r = o / (16 * ST);
        const int64_t n = n0 + s * 16 + in_strip, m = r;
        if (n >= g.n || m >= g.m) continue;
        const int l = (in_strip >> 2) * 16 + (r & 15);
        float v = s_acc[0][s][r >> 4][l][in_strip & 3];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) v += s_acc[w][s][r >> 4][l][in_strip & 3];
        if (g.bias) v += g.bias[n];
        if (g.relu) v = v < 0.0f ? 0.0f : v; // (a NaN stays)
        static_cast<T *>(g.c)[m * g.ldc + n] = (T)v;
    }
}

} // namespace dqrm_mx
