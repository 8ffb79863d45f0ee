// Products of MXFP4 matrices with few rows of A (requests), from codes or from activations as they are (gfx950, wave64).
//
// What such a product costs is W's bytes, read once.  A workgroup has ST strips of 16 rows of W; its four waves take every fourth
// unit of 512 values of k.  A wave's loads go straight into LDS of its own, where no other wave looks (so it waits for its loads, but
// for no barrier): a load has whole lines of 4 rows, while the operands of v_mfma_scale_f32_16x16x128_f8f6f4 (lane l: row l % 16,
// block l / 16 of 128 values) would have halves of 16 rows' lines; what a load costs the address unit is its lines.  The waves' sums
// meet in LDS in a fixed order.
//
// 16 x 8192 x 8192 takes 11 us (36 MB of W, 3.2 TB/s; 16.4 with the operands' own loads): a workgroup has four units to a wave, and
// the first one's latency and the launch are a third of it.  1 x 367 for 512 outputs, quantised within: 3.6 us, all latency.
#pragma once

#include "dqrm_mx_gemm.hpp"
#include "dqrm_norm.hpp"

namespace dqrm_mx {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kFewWaves = 4, kFewBlock = kFewWaves * kWaveSize;
constexpr int kFewChunks = 4; // chunks of 8 activations to a thread, where the product quantises them itself
constexpr int kFewRows = 4;   // rows that it quantises itself, at most
constexpr int kUnitGroups = 4, kUnitBytes = 16 * kUnitGroups * 64, kUnitTile = kUnitBytes + 16 * kUnitGroups * 4; // 16 rows' codes and scales

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

// kFewPlain, kFewNorm: the rows of x (kFewRows at most) to codes and scales in LDS, by as many waves to a row as there are, each
// thread's values in registers (k <= waves of a row * 64 * kFewChunks * 8).
template <typename T, bool NORM>
__device__ __forceinline__ void quantise_few(const NormArgs &a, uint8_t *codes, uint8_t *scales, float (*s_sum)[2])
{
    const int rows = (int)a.rows;
    const int log_waves = rows <= 1 ? 2 : rows <= 2 ? 1 : 0; // of a row
    const int wave = threadIdx.x / kWaveSize, waves = 1 << log_waves;
    const int own = wave >> log_waves, r = min(own, rows - 1);
    const int t = threadIdx.x & ((kWaveSize << log_waves) - 1), stride = kWaveSize << log_waves;
    const T *row = static_cast<const T *>(a.x) + r * a.ldx;
    const int cols = (int)a.cols, pitch = (int)codes_pitch(cols), spitch = (int)scales_pitch(cols);
    auto column = [&](int j) { return (j * stride + t) * kChunk; };
    auto used = [&](int j) { return j * stride * kChunk < cols; }; // by any thread
    Raw<T> raw[kFewChunks];
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j)
        if (used(j)) raw[j] = load_raw(row, column(j), cols);
    float gamma[NORM ? kFewChunks : 1][kChunk], beta[NORM ? kFewChunks : 1][kChunk];
    if constexpr (NORM) {
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j) {
            if (!used(j)) continue;
            // (the last 8 of a row that ends within the chunk are asked for, and moved like the row's own)
            if (a.gamma) values_of<float>(load_raw(a.gamma, column(j), cols), column(j), cols, gamma[j]);
            if (a.beta) values_of<float>(load_raw(a.beta, column(j), cols), column(j), cols, beta[j]);
        }
    }
    float x[kFewChunks][kChunk];
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j)
        if (used(j)) values_of<T>(raw[j], column(j), cols, x[j]);
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
        for (int j = 0; j < kFewChunks; ++j) {
            if (!used(j)) continue;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v += x[j][i];
        }
        const float mean = row_sum(v, 0) / (float)cols;
        v = 0.0f;
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j) {
            if (!used(j)) continue;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) x[j][i] -= mean;
            if (column(j) + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = column(j) + i < cols ? x[j][i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v += x[j][i] * x[j][i];
        }
        const float rstd = 1.0f / sqrtf(row_sum(v, 1) / (float)cols + a.eps);
#pragma unroll
        for (int j = 0; j < kFewChunks; ++j) {
            if (!used(j)) continue;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) x[j][i] = x[j][i] * rstd * (a.gamma ? gamma[j][i] : 1.0f) + (a.beta ? beta[j][i] : 0.0f);
            // (past the row's end 0, also where rstd is infinite or a NaN: the padding of the codes)
            if (column(j) + kChunk > cols) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = column(j) + i < cols ? x[j][i] : 0.0f;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) {
        const int chunk = j * stride + t;
        // (the padding behind a row may begin in a chunk that no value is in)
        if (j * stride < pitch / 4 && chunk < pitch / 4 && own < rows) {
            if (!used(j)) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i) x[j][i] = 0.0f;
            }
            write_chunk(codes + r * pitch, scales + r * spitch, (unsigned)chunk, x[j]);
        }
    }
    __syncthreads();
}

// MT: groups of 16 rows of A; RING: units of a wave that are in flight or in use.
template <int DT, FewSource SRC, int MT, int ST, int RING>
__global__ __launch_bounds__(kFewBlock) void few_kernel(FewArgs a)
{
    using T = elem_t<DT>;
    static_assert(SRC == kFewCodes || MT == 1, "quantise_few has a few rows");
    constexpr int tiles = ST + (SRC == kFewCodes ? MT : 0); // of 16 rows that a unit loads: W's, then A's
    constexpr int loads = 5;                                // of a tile: four of codes, one of scales
    constexpr int ring_bytes = kFewWaves * RING * tiles * kUnitTile, sum_bytes = kFewWaves * ST * MT * kWaveSize * (int)sizeof(v4f);
    __shared__ __align__(1024) uint8_t s_ring[ring_bytes > sum_bytes ? ring_bytes : sum_bytes];
    __shared__ float s_sum[kFewWaves][2];
    extern __shared__ __align__(16) uint8_t s_x[]; // codes, then scales, of x
    const MatmulArgs &g = a.g;
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6);
    const int row = lane & 15, block = lane >> 4;
    const int64_t groups = groups_of(g.k), cp = groups * 64, sp = groups * 4;
    const int64_t n0 = (int64_t)blockIdx.x * (ST * 16);
    const int units = (int)((groups + kUnitGroups - 1) / kUnitGroups);
    const int mine = (units - wave + kFewWaves - 1) / kFewWaves; // the wave's units: wave, wave + 4, ...

    // memory from a tile's first row on; what lies past the matrix reads as zeros
    rsrc_t codes[tiles], scales[tiles];
#pragma unroll
    for (int t = 0; t < tiles; ++t) {
        const int64_t r0 = t < ST ? n0 + t * 16 : (int64_t)(t - ST) * 16;
        const int64_t left = max((t < ST ? g.n : g.m) - r0, (int64_t)0);
        codes[t] = buffer_of((t < ST ? g.b_codes : g.a_codes) + r0 * cp, min(left, (int64_t)16) * cp);
        scales[t] = buffer_of((t < ST ? g.b_scales : g.a_scales) + r0 * sp, min(left, (int64_t)16) * sp);
    }
    // a row's 16 vectors of a unit, vector v of row r in place v ^ r; load j has rows 4 j .. 4 j + 3
    unsigned code_at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) code_at[j] = (unsigned)(j * 4 + block) * (unsigned)cp + (unsigned)((row ^ (j * 4 + block)) * 16);
    const unsigned scale_at = (unsigned)(lane >> 2) * (unsigned)sp + (unsigned)(lane & 3) * 4;
    const unsigned lds0 = uniform(lds_address(s_ring)) + (unsigned)wave * (RING * tiles * kUnitTile);
    // unit i of the wave; one past its last is requested from a buffer without bytes, so that every unit is as many loads
    auto request = [&](int i) {
        const unsigned unit = (unsigned)(wave + i * kFewWaves), to = lds0 + (unsigned)(i % RING) * (tiles * kUnitTile);
        auto here = [&](rsrc_t r) {
            r.z = uniform(i < mine ? r.z : 0u);
            return r;
        };
#pragma unroll
        for (int t = 0; t < tiles; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) load16_to_lds(here(codes[t]), code_at[j] + unit * (kUnitGroups * 64), to + t * kUnitTile + j * 1024);
            load4_to_lds(here(scales[t]), scale_at + unit * (kUnitGroups * 4), to + t * kUnitTile + kUnitBytes);
        }
    };
    auto tile_of = [&](int i, int t) { return s_ring + (wave * RING + i % RING) * (tiles * kUnitTile) + t * kUnitTile; };
#pragma unroll
    for (int i = 0; i < RING; ++i) request(i);
    if constexpr (SRC != kFewCodes) quantise_few<T, SRC == kFewNorm>(a.x, s_x, s_x + g.m * cp, s_sum);

    v4f acc[ST][MT] = {};
    for (int i = 0; i < mine; ++i) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * tiles * loads) : "memory"); // unit i is in LDS
        const int first = (wave + i * kFewWaves) * kUnitGroups;
        uint4 w[ST][kUnitGroups], x[MT][kUnitGroups];
        uint4 ws[ST], xs[MT];
#pragma unroll
        for (int t = 0; t < ST + MT; ++t) {
            if (t < ST || SRC == kFewCodes) {
                const uint8_t *tile = tile_of(i, t);
                const uint4 s = *reinterpret_cast<const uint4 *>(tile + kUnitBytes + row * 16);
                (t < ST ? ws[t < ST ? t : 0] : xs[t < ST ? 0 : t - ST]) = s;
#pragma unroll
                for (int k = 0; k < kUnitGroups; ++k) {
                    const uint4 c = *reinterpret_cast<const uint4 *>(tile + row * 256 + (((k * 4 + block) ^ row) * 16));
                    (t < ST ? w[t < ST ? t : 0][k] : x[t < ST ? 0 : t - ST][k]) = c;
                }
            } else {
                const int64_t r = min((int64_t)row, g.m - 1);
                unsigned d[kUnitGroups];
#pragma unroll
                for (int k = 0; k < kUnitGroups; ++k) {
                    const int64_t at = min((int64_t)(first + k), groups - 1); // (a group past the last one is not multiplied)
                    x[0][k] = *reinterpret_cast<const uint4 *>(s_x + r * cp + at * 64 + block * 16);
                    d[k] = *reinterpret_cast<const unsigned *>(s_x + g.m * cp + r * sp + at * 4);
                }
                xs[0] = make_uint4(d[0], d[1], d[2], d[3]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // the unit is in registers: its memory may be loaded into
        request(i + RING);
#pragma unroll
        for (int k = 0; k < kUnitGroups; ++k) {
            if (first + k >= groups) break;
            auto byte = [&](const uint4 &v) { return (k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w) >> (8 * block); };
#pragma unroll
            for (int s = 0; s < ST; ++s)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[s][m] = mfma_16x16x128(w[s][k], x[m][k], acc[s][m], byte(ws[s]), byte(xs[m]));
        }
    }
    lds_barrier(); // no load is on its way any more
    v4f(*s_acc)[ST][MT][kWaveSize] = reinterpret_cast<v4f(*)[ST][MT][kWaveSize]>(s_ring);
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
