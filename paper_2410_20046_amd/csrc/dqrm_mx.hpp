// MXFP4 matrices: element types, codes and scales, quantisation along rows and columns, dequantisation (gfx950, wave64).
//
// 32 consecutive values of a row share a scale 2^e, e = max(floor(log2(max |v|)) - 2, -127); a value is held as the nearest of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale and a sign (E2M1), ties to the even code, magnitudes beyond 6 as 6.  Multiplying
// by 2^-e is exact, or ends below every code, so a code is one rounding of the value itself.  A block that holds an infinity or
// a NaN gets the NaN scale (255) and zero codes.  Rows are padded to multiples of 128 values: zero codes, zero scale bytes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dqrm.h"
#include "dqrm_fastdiv.hpp"

#pragma clang fp contract(off)

namespace dqrm_mx {

constexpr int kWaveSize = 64;
constexpr int kRowPad = 128;   // values that a row is padded to a multiple of
constexpr int kChunk = 8;      // values that a lane takes at a time; four lanes to a block of 32

__host__ __device__ __forceinline__ int64_t groups_of(int64_t cols) { return (cols + kRowPad - 1) / kRowPad; }
__host__ __device__ __forceinline__ int64_t codes_pitch(int64_t cols) { return groups_of(cols) * (kRowPad / 2); }
__host__ __device__ __forceinline__ int64_t scales_pitch(int64_t cols) { return groups_of(cols) * (kRowPad / 32); }

// ---- element types ---------------------------------------------------------------------------------------------------
// Vectors are loaded and stored at the elements' own alignment: rows of odd widths start anywhere.
template <int DT> struct Elem;
template <> struct Elem<DQRM_F32> { using T = float; };
template <> struct Elem<DQRM_BF16> { using T = __bf16; };
template <> struct Elem<DQRM_F16> { using T = _Float16; };
template <int DT> using elem_t = typename Elem<DT>::T;

template <typename T> struct Vec8 { T v[kChunk]; };

// 16 bytes past the caches, at the elements' alignment
template <typename T, typename V>
__device__ __forceinline__ void store_stream(T *p, const V &v)
{
    static_assert(sizeof(V) == 16);
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    typedef u4 u4_by_2 __attribute__((aligned(2)));
    typedef u4 u4_by_4 __attribute__((aligned(4)));
    u4 w;
    __builtin_memcpy(&w, &v, 16);
    if constexpr (alignof(T) == 2)
        __builtin_nontemporal_store(w, reinterpret_cast<u4_by_2 *>(p));
    else
        __builtin_nontemporal_store(w, reinterpret_cast<u4_by_4 *>(p));
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[kChunk])
{
    Vec8<T> t;
    __builtin_memcpy(&t, p, sizeof(t));
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = (float)t.v[i];
}

// the first n of 8 values, the others 0
template <typename T>
__device__ __forceinline__ void load_first(const T *p, int n, float (&v)[kChunk])
{
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
}

// values c .. c + 7 of a row of `cols`; those past its end are 0.  `inside`: the 8 values lie inside the matrix's memory, so they
// may be loaded as one vector also where some belong to what follows the row.
template <typename T, typename I>
__device__ __forceinline__ void load_chunk(const T *row, I c, I cols, bool inside, float (&v)[kChunk])
{
    if (c + kChunk <= cols) {
        load8(row + c, v);
    } else if (c >= cols) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = 0.0f;
    } else if (inside) {
        load8(row + c, v);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = c + i < cols ? v[i] : 0.0f;
    } else {
        load_first(row + c, (int)(cols - c), v);
    }
}

// A row's chunk as it lies in memory, to be requested long before its use.  Where fewer than 8 values are left, it is the last 8
// of the row (cols >= 8): a load without a branch, which nothing has to wait for.
template <typename T> struct Raw { unsigned w[kChunk * sizeof(T) / 4]; };

template <typename T, typename I>
__device__ __forceinline__ Raw<T> load_raw(const T *row, I c, I cols)
{
    Raw<T> t;
    __builtin_memcpy(&t, row + min(c, cols - (I)kChunk), sizeof(t));
    return t;
}

// ... and its values c .. c + 7; those past the row's end are 0
template <typename T, typename I>
__device__ __forceinline__ void values_of(const Raw<T> &raw, I c, I cols, float (&v)[kChunk])
{
    Vec8<T> t;
    __builtin_memcpy(&t, &raw, sizeof(t));
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = (float)t.v[i];
    const int skip = (int)min(c + (I)kChunk - cols, (I)(2 * kChunk)); // of the 8 belong to the chunk before
    if (skip > 0) {
#pragma unroll
        for (int s = 1; s < 2 * kChunk; s *= 2) {
            if (skip & s || (s == kChunk && skip > kChunk)) { // (8 and more: nothing of the row)
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[i] = i + s < kChunk ? v[i + s < kChunk ? i + s : 0] : 0.0f;
            }
        }
    }
}

// STREAM: past the caches (for outputs that are not read again soon)
template <bool STREAM = false, typename T, typename I>
__device__ __forceinline__ void store_chunk(T *row, I c, I cols, const float (&v)[kChunk])
{
    if (c + kChunk <= cols) {
        Vec8<T> t;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) t.v[i] = (T)v[i];
        if constexpr (STREAM) {
            struct Half { T v[16 / sizeof(T)]; };
#pragma unroll
            for (int i = 0; i < (int)sizeof(t) / 16; ++i) store_stream(row + c + i * (16 / sizeof(T)), reinterpret_cast<const Half *>(&t)[i]);
        } else {
            __builtin_memcpy(row + c, &t, sizeof(t));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (c + i < cols) row[c + i] = (T)v[i];
    }
}

// ---- codes and scales --------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// scale byte of a block from the bits of its largest magnitude (NaNs order above infinities above numbers)
__device__ __forceinline__ unsigned scale_byte(unsigned amax_bits)
{
    const unsigned e = amax_bits >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}

// 2^-e for a scale byte of a finite block (0 .. 252)
__device__ __forceinline__ float inverse_scale(unsigned s) { return __uint_as_float((254u - s) << 23); }
// 2^e; 255 is NaN
__device__ __forceinline__ float scale_value(unsigned s)
{
    return __uint_as_float(s == 255u ? 0x7FC00000u : s == 0u ? 0x00400000u : s << 23);
}

// eight codes, value 0 in the low four bits; the conversion rounds to even and saturates
__device__ __forceinline__ unsigned pack_codes(const float (&v)[kChunk], unsigned s)
{
    const float inv = inverse_scale(s & 0xFFu);
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0] * inv, v[1] * inv, 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2] * inv, v[3] * inv, 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4] * inv, v[5] * inv, 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6] * inv, v[7] * inv, 1.0f, 3);
    return s == 255u ? 0u : r;
}

__device__ __forceinline__ unsigned max8(const float (&v)[kChunk])
{
    unsigned m = abs_bits(v[0]);
#pragma unroll
    for (int i = 1; i < kChunk; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

// the largest over the four lanes of a block
__device__ __forceinline__ unsigned quad_max(unsigned m)
{
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true)); // lanes 1 0 3 2
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true)); // lanes 2 3 0 1
}

// A chunk of a row's codes and, from the first lane of each block, its scale byte.  All four lanes of a block take part.
// chunk: index of the 8 values in the padded row.  (A block of the padding has zeros: its scale byte is 0.)
__device__ __forceinline__ void write_chunk(uint8_t *codes_row, uint8_t *scales_row, unsigned chunk, const float (&v)[kChunk])
{
    const unsigned s = scale_byte(quad_max(max8(v)));
    *reinterpret_cast<unsigned *>(codes_row + (size_t)chunk * 4) = pack_codes(v, s);
    if ((chunk & 3u) == 0u) scales_row[chunk >> 2] = (uint8_t)s;
}

// ---- along rows --------------------------------------------------------------------------------------------------------
struct QuantArgs {
    const void *x, *gate;      // gate: x counts where gate > 0; or null
    int64_t ldx, ldgate, rows, cols;
    uint8_t *codes, *scales;     // along rows, or null
    uint8_t *codes_t, *scales_t; // along columns, or null
    float *partial;              // [row tiles][cols] column sums, or null
    unsigned col_tiles;          // of quant_tile_kernel's grid
};

template <typename T>
__device__ __forceinline__ void load_gated(const QuantArgs &a, int64_t r, int64_t c, float (&v)[kChunk])
{
    // (are there 8 values from this one on before the matrix's memory ends?  Rows may be shorter than that.)
    auto inside = [&](int64_t ld) { return (a.rows - 1 - r) * ld + a.cols >= c + kChunk; };
    load_chunk(static_cast<const T *>(a.x) + r * a.ldx, c, a.cols, inside(a.ldx), v);
    if (a.gate) {
        float g[kChunk];
        load_chunk(static_cast<const T *>(a.gate) + r * a.ldgate, c, a.cols, inside(a.ldgate), g);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = g[i] > 0.0f ? v[i] : 0.0f;
    }
}

// One chunk to a lane, rows' chunks one after another; per_row: chunks of a row, of fewer than 2^31 in all.
template <int DT>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a, dqrm::FastDiv per_row)
{
    using T = elem_t<DT>;
    const unsigned at = blockIdx.x * 256 + threadIdx.x, r = per_row.div(at), chunk = at - r * per_row.d;
    if (r >= a.rows) return; // (whole blocks of 32 values: a row has a multiple of 16 chunks)
    float v[kChunk];
    load_gated<T>(a, r, (int64_t)chunk * kChunk, v);
    write_chunk(a.codes + r * codes_pitch(a.cols), a.scales + r * scales_pitch(a.cols), chunk, v);
}

// ---- along columns, and both ways from one read ----------------------------------------------------------------------------
// A workgroup takes 128 rows by 128 columns.  The chunks that its lanes load are blocks of rows already (four lanes to a block);
// the tile then goes through LDS in its own type, and each wave takes 32 rows of it, two columns to a lane: a block of a column is
// in one lane's registers.
constexpr int kTile = 128;

template <int DT>
__global__ __launch_bounds__(256, DT == DQRM_F32 ? 2 : 4) void quant_tile_kernel(QuantArgs a)
{
    using T = elem_t<DT>;
    struct alignas(2 * sizeof(T)) Pair { T v[2]; };
    constexpr int passes = kTile / 16;
    __shared__ __align__(16) T tile[kTile][kTile];
    __shared__ unsigned s_scale[kTile];
    __shared__ float s_sum[4][kTile];
    const unsigned row_tile = blockIdx.x / a.col_tiles;
    const int64_t r0 = (int64_t)row_tile * kTile, c0 = (int64_t)(blockIdx.x - row_tile * a.col_tiles) * kTile;
    const int tid = threadIdx.x;
    const int lane_chunk = tid & 15;
    const int64_t c = c0 + lane_chunk * kChunk;
    auto finish_chunk = [&](int dr, float (&v)[kChunk]) {
        if (a.codes && r0 + dr < a.rows)
            write_chunk(a.codes + (r0 + dr) * codes_pitch(a.cols), a.scales + (r0 + dr) * scales_pitch(a.cols), (unsigned)(c / kChunk), v);
        Vec8<T> t;
#pragma unroll
        for (int k = 0; k < kChunk; ++k) t.v[k] = (T)v[k];
        __builtin_memcpy(__builtin_assume_aligned(&tile[dr][lane_chunk * kChunk], 16), &t, sizeof(t));
    };
    if (a.cols >= kChunk) {
        // (rows past the last one repeat it and then count as zeros)
        auto row = [&](const void *p, int64_t ld, int i) { return static_cast<const T *>(p) + min(r0 + i * 16 + (tid >> 4), a.rows - 1) * ld; };
        Raw<T> x[passes], gate[passes];
#pragma unroll
        for (int i = 0; i < passes; ++i) x[i] = load_raw(row(a.x, a.ldx, i), c, a.cols);
        if (a.gate) {
#pragma unroll
            for (int i = 0; i < passes; ++i) gate[i] = load_raw(row(a.gate, a.ldgate, i), c, a.cols);
        }
#pragma unroll
        for (int i = 0; i < passes; ++i) {
            const int dr = i * 16 + (tid >> 4);
            float v[kChunk];
            values_of<T>(x[i], c, a.cols, v);
            if (a.gate) {
                float g[kChunk];
                values_of<T>(gate[i], c, a.cols, g);
#pragma unroll
                for (int k = 0; k < kChunk; ++k) v[k] = g[k] > 0.0f ? v[k] : 0.0f;
            }
            if (r0 + dr >= a.rows) {
#pragma unroll
                for (int k = 0; k < kChunk; ++k) v[k] = 0.0f;
            }
            finish_chunk(dr, v);
        }
    } else {
        for (int i = 0; i < passes; ++i) {
            const int dr = i * 16 + (tid >> 4);
            float v[kChunk] = {};
            if (r0 + dr < a.rows) load_gated<T>(a, r0 + dr, c, v);
            finish_chunk(dr, v);
        }
    }
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    uint4 codes[2] = {};
    unsigned scale[2] = {0, 0};
    float sum[2] = {0.0f, 0.0f};
    float v[2][32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        const Pair p = *reinterpret_cast<const Pair *>(&tile[wave * 32 + k][lane * 2]);
        v[0][k] = (float)p.v[0], v[1][k] = (float)p.v[1];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        unsigned m = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) m = max(m, abs_bits(v[j][k]));
        if (a.partial) {
#pragma unroll
            for (int k = 0; k < 32; ++k) sum[j] += v[j][k];
        }
        scale[j] = scale_byte(m);
        unsigned w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float t[kChunk];
#pragma unroll
            for (int k = 0; k < kChunk; ++k) t[k] = v[j][q * kChunk + k];
            w[q] = pack_codes(t, scale[j]);
        }
        codes[j] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads(); // the tile is read; its memory takes the codes: [128 columns][64 bytes]
    uint4 *s_codes = reinterpret_cast<uint4 *>(&tile[0][0]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = lane * 2 + j;
        s_codes[c * 4 + (wave ^ (lane & 3))] = codes[j]; // (columns apart in LDS's banks)
        reinterpret_cast<uint8_t *>(&s_scale[c])[wave] = (uint8_t)scale[j];
        s_sum[wave][c] = sum[j];
    }
    __syncthreads();
    if (a.codes_t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = i * 256 + tid, c = at >> 2;
            if (c0 + c < a.cols)
                store_stream(reinterpret_cast<unsigned *>(a.codes_t + (c0 + c) * codes_pitch(a.rows) + r0 / 2 + (at & 3) * 16), s_codes[at ^ ((c >> 1) & 3)]);
        }
        if (tid < kTile && c0 + tid < a.cols)
            *reinterpret_cast<unsigned *>(a.scales_t + (c0 + tid) * scales_pitch(a.rows) + r0 / 32) = s_scale[tid];
    }
    if (a.partial && tid < kTile && c0 + tid < a.cols)
        a.partial[(int64_t)row_tile * a.cols + c0 + tid] = (s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]);
}

// out[c] = sum over p of partial[p][c] (and a second pair of arrays behind it), in a fixed order: 16 lanes take every 16th each, then
// their sums are added in turn.
__global__ __launch_bounds__(256) void join_columns_kernel(const float *partial, int64_t stride, int n, int64_t cols, float *out0, float *out1)
{
    __shared__ float s[16][17];
    const int64_t c = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
    const int slice = threadIdx.x >> 4;
    const float *p = partial + (blockIdx.y ? cols : 0);
    float sum = 0.0f;
    if (c < cols)
        for (int i = slice; i < n; i += 16) sum += p[(int64_t)i * stride + c];
    s[slice][threadIdx.x & 15] = sum;
    __syncthreads();
    if (slice == 0 && c < cols) {
        float t = s[0][threadIdx.x];
        for (int i = 1; i < 16; ++i) t += s[i][threadIdx.x];
        (blockIdx.y ? out1 : out0)[c] = t;
    }
}

// ---- back to values --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void unpack_codes(unsigned w, float scale, float (&v)[kChunk])
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    v[0] = a.x * scale, v[1] = a.y * scale, v[2] = b.x * scale, v[3] = b.y * scale;
    v[4] = c.x * scale, v[5] = c.y * scale, v[6] = d.x * scale, v[7] = d.y * scale;
}

// per_row: chunks of a row that hold values, of fewer than 2^31 in all
template <int DT>
__global__ __launch_bounds__(256) void dequant_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out, int64_t ldo,
                                                      dqrm::FastDiv per_row)
{
    using T = elem_t<DT>;
    const unsigned at = blockIdx.x * 256 + threadIdx.x, r = per_row.div(at), chunk = at - r * per_row.d;
    if (r >= rows) return;
    const unsigned w = *reinterpret_cast<const unsigned *>(codes + r * codes_pitch(cols) + (size_t)chunk * 4);
    float v[kChunk];
    unpack_codes(w, scale_value(scales[r * scales_pitch(cols) + (chunk >> 2)]), v);
    store_chunk<true>(static_cast<T *>(out) + r * ldo, (int64_t)chunk * kChunk, cols, v);
}

} // namespace dqrm_mx
