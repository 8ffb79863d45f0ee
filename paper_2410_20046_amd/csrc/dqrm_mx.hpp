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
__device__ __forceinline__ void to_float(const Vec8<T> &t, float (&v)[kChunk])
{
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = (float)t.v[i];
}

// Values c .. c + 7 of a row of `cols`; those past its end are 0.  `inside`: the 8 values lie inside the matrix's memory, so they
// may be loaded as one vector also where some belong to what follows the row.
template <typename T, typename I>
__device__ __forceinline__ Vec8<T> load_vec(const T *row, I c, I cols, bool inside)
{
    Vec8<T> t;
    if (c + kChunk <= cols || (inside && c < cols)) {
        __builtin_memcpy(&t, row + c, sizeof(t));
        if (c + kChunk > cols) {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) t.v[i] = c + i < cols ? t.v[i] : (T)0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) t.v[i] = c + i < cols ? row[c + i] : (T)0.0f;
    }
    return t;
}

template <typename T, typename I>
__device__ __forceinline__ void load_chunk(const T *row, I c, I cols, float (&v)[kChunk])
{
    to_float(load_vec(row, c, cols, false), v);
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
template <typename V, typename I>
__device__ __forceinline__ void drop_before(V (&v)[kChunk], I c, I cols)
{
    const int skip = (int)min(c + (I)kChunk - cols, (I)(2 * kChunk)); // of the 8 belong to the chunk before
    if (skip > 0) {
#pragma unroll
        for (int s = 1; s < 2 * kChunk; s *= 2) {
            if (skip & s || (s == kChunk && skip > kChunk)) { // (8 and more: nothing of the row)
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[i] = i + s < kChunk ? v[i + s < kChunk ? i + s : 0] : (V)0.0f;
            }
        }
    }
}

template <typename T, typename I>
__device__ __forceinline__ Vec8<T> vec_of(const Raw<T> &raw, I c, I cols)
{
    Vec8<T> t;
    __builtin_memcpy(&t, &raw, sizeof(t));
    drop_before(t.v, c, cols);
    return t;
}

template <typename T, typename I>
__device__ __forceinline__ void values_of(const Raw<T> &raw, I c, I cols, float (&v)[kChunk])
{
    Vec8<T> t;
    __builtin_memcpy(&t, &raw, sizeof(t));
    to_float(t, v);
    drop_before(v, c, cols);
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

// 2^e; 255 is NaN
__device__ __forceinline__ float scale_value(unsigned s)
{
    return __uint_as_float(s == 255u ? 0x7FC00000u : s == 0u ? 0x00400000u : s << 23);
}

// Eight codes, value 0 in the low four bits.  The conversion divides by the scale, rounds to even and saturates.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned convert8(const float (&v)[kChunk], float scale)
{
    unsigned r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
}
__device__ __forceinline__ unsigned convert8(const __bf16 (&v)[kChunk], float scale)
{
    unsigned r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, bf16x2{v[0], v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16x2{v[2], v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16x2{v[4], v[5]}, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bf16x2{v[6], v[7]}, scale, 3);
}
__device__ __forceinline__ unsigned convert8(const _Float16 (&v)[kChunk], float scale)
{
    unsigned r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, f16x2{v[0], v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, f16x2{v[2], v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, f16x2{v[4], v[5]}, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, f16x2{v[6], v[7]}, scale, 3);
}

template <typename T>
__device__ __forceinline__ unsigned pack_codes(const T (&v)[kChunk], unsigned s)
{
    const unsigned r = convert8(v, __uint_as_float(s << 23)); // (of the scale only the exponent's field counts, 0 being 2^-127)
    return s == 255u ? 0u : r;
}

// bits, as a float's, of the largest magnitude of eight values
__device__ __forceinline__ unsigned max8(const float (&v)[kChunk])
{
    unsigned m = abs_bits(v[0]);
#pragma unroll
    for (int i = 1; i < kChunk; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

// ... of 16-bit types: magnitudes order like their bits, two to a register
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 abs_pair(unsigned w)
{
    u16x2 r;
    w &= 0x7FFF7FFFu;
    __builtin_memcpy(&r, &w, 4);
    return r;
}
template <typename T>
__device__ __forceinline__ unsigned bits_of_16(unsigned short m)
{
    T t;
    __builtin_memcpy(&t, &m, 2);
    return __float_as_uint((float)t);
}
template <typename T>
__device__ __forceinline__ unsigned max8(const T (&v)[kChunk])
{
    unsigned w[4];
    __builtin_memcpy(w, v, 16);
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(abs_pair(w[0]), abs_pair(w[1])), __builtin_elementwise_max(abs_pair(w[2]), abs_pair(w[3])));
    return bits_of_16<T>(m.x > m.y ? m.x : m.y);
}

// the largest over the four lanes of a block
__device__ __forceinline__ unsigned quad_max(unsigned m)
{
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true)); // lanes 1 0 3 2
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true)); // lanes 2 3 0 1
}

// A chunk of a row's codes and, from the first lane of each block, its scale byte.  All four lanes of a block take part.
// chunk: index of the 8 values in the padded row.  (A block of the padding has zeros: its scale byte is 0.)
template <typename T>
__device__ __forceinline__ void write_chunk(uint8_t *codes_row, uint8_t *scales_row, unsigned chunk, const T (&v)[kChunk])
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

// x where gate > 0
template <typename T>
__device__ __forceinline__ void apply_gate(Vec8<T> &v, const Vec8<T> &gate)
{
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v.v[i] = gate.v[i] > (T)0.0f ? v.v[i] : (T)0.0f;
}

template <typename T>
__device__ __forceinline__ Vec8<T> load_gated(const QuantArgs &a, int64_t r, int64_t c)
{
    // (are there 8 values from this one on before the matrix's memory ends?  Rows may be shorter than that.)
    auto inside = [&](int64_t ld) { return (a.rows - 1 - r) * ld + a.cols >= c + kChunk; };
    Vec8<T> v = load_vec(static_cast<const T *>(a.x) + r * a.ldx, c, a.cols, inside(a.ldx));
    if (a.gate) apply_gate(v, load_vec(static_cast<const T *>(a.gate) + r * a.ldgate, c, a.cols, inside(a.ldgate)));
    return v;
}

// One chunk to a lane, rows' chunks one after another; per_row: chunks of a row, of fewer than 2^31 in all.  Bound by its bytes:
// 8192 x 512 float (19 MB) 4.6 us, of which the launch and a read's latency are about 3.
template <int DT>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a, dqrm::FastDiv per_row)
{
    using T = elem_t<DT>;
    const unsigned at = blockIdx.x * 256 + threadIdx.x, r = per_row.div(at), chunk = at - r * per_row.d;
    if (r >= a.rows) return; // (whole blocks of 32 values: a row has a multiple of 16 chunks)
    const Vec8<T> v = load_gated<T>(a, r, (int64_t)chunk * kChunk);
    write_chunk(a.codes + r * codes_pitch(a.cols), a.scales + r * scales_pitch(a.cols), chunk, v.v);
}

// ---- along columns, and both ways from one read ----------------------------------------------------------------------------
// A workgroup takes 128 rows by 128 columns.  The chunks that its lanes load are blocks of rows already (four lanes to a block);
// the tile then goes through LDS in its own type, and each wave takes 32 rows of it, two columns to a lane: a block of a column is
// in one lane's registers.  128 because a line of the columns' codes is 64 bytes of 128 values.  Bound by its bytes, then by the
// columns' stores of half lines: 16384 x 8191 bfloat16 both ways (411 MB) 100 us, 4.1 TB/s, where a copy has 5.1; 8192 x 2048 with a
// gate and column sums 19 us (85 MB).  By columns alone 71 us (340 MB, 4.8 TB/s), of 8192 x 2048 11.5 us (42 MB).  Float, which has half the
// workgroups to a CU: both ways 149 us (679 MB, 4.6 TB/s), by columns 125 (608 MB); 2048 x 2048 6 us.
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
    auto finish_chunk = [&](int dr, const Vec8<T> &v) {
        if (a.codes && r0 + dr < a.rows)
            write_chunk(a.codes + (r0 + dr) * codes_pitch(a.cols), a.scales + (r0 + dr) * scales_pitch(a.cols), (unsigned)(c / kChunk), v.v);
        __builtin_memcpy(__builtin_assume_aligned(&tile[dr][lane_chunk * kChunk], 16), &v, sizeof(v));
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
            Vec8<T> v = vec_of<T>(x[i], c, a.cols);
            if (a.gate) apply_gate(v, vec_of<T>(gate[i], c, a.cols));
            if (r0 + dr >= a.rows) {
#pragma unroll
                for (int k = 0; k < kChunk; ++k) v.v[k] = (T)0.0f;
            }
            finish_chunk(dr, v);
        }
    } else {
        for (int i = 0; i < passes; ++i) {
            const int dr = i * 16 + (tid >> 4);
            Vec8<T> v{};
            if (r0 + dr < a.rows) v = load_gated<T>(a, r0 + dr, c);
            finish_chunk(dr, v);
        }
    }
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    uint4 codes[2];
    unsigned scale[2];
    float sum[2] = {0.0f, 0.0f};
    T v[2][4][kChunk];
    unsigned most[2];
    u16x2 pair_most = {0, 0};
    most[0] = most[1] = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        const Pair p = *reinterpret_cast<const Pair *>(&tile[wave * 32 + k][lane * 2]);
        v[0][k / kChunk][k % kChunk] = p.v[0], v[1][k / kChunk][k % kChunk] = p.v[1];
        if constexpr (sizeof(T) == 2) {
            unsigned w;
            __builtin_memcpy(&w, &p, 4);
            pair_most = __builtin_elementwise_max(pair_most, abs_pair(w));
        } else {
            most[0] = max(most[0], abs_bits(p.v[0])), most[1] = max(most[1], abs_bits(p.v[1]));
        }
    }
    if (a.partial) {
#pragma unroll
        for (int k = 0; k < 32; ++k) sum[0] += (float)v[0][k / kChunk][k % kChunk], sum[1] += (float)v[1][k / kChunk][k % kChunk];
    }
    if constexpr (sizeof(T) == 2) most[0] = bits_of_16<T>(pair_most.x), most[1] = bits_of_16<T>(pair_most.y);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        scale[j] = scale_byte(most[j]);
        codes[j] = make_uint4(pack_codes(v[j][0], scale[j]), pack_codes(v[j][1], scale[j]), pack_codes(v[j][2], scale[j]), pack_codes(v[j][3], scale[j]));
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

// v + p[0] + p[stride] + ... (n of them, in this order), 16 loads at a time on their way: behind the last one it is asked for again, and
// not added.
__device__ __forceinline__ float add_strided(float v, const float *p, int64_t stride, int n)
{
    constexpr int ahead = 16;
    for (int i = 0; i < n; i += ahead) {
        float x[ahead];
#pragma unroll
        for (int j = 0; j < ahead; ++j) x[j] = p[(int64_t)min(i + j, n - 1) * stride];
#pragma unroll
        for (int j = 0; j < ahead; ++j) v = i + j < n ? v + x[j] : v;
    }
    return v;
}

// out[c] = sum over p of partial[p][c], and another such sum from `second` values on, in a fixed order: 16 lanes take every 16th each,
// then their sums are added in turn.  The launch and two reads' latencies: 256 parts of 512 columns twice 2.8 us, of 8190 columns 8.
__global__ __launch_bounds__(256) void join_columns_kernel(const float *partial, int64_t stride, int n, int64_t cols, int64_t second, float *out0,
                                                           float *out1)
{
    __shared__ float s[16][17];
    const int64_t c = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
    const int slice = threadIdx.x >> 4;
    const float *p = partial + (blockIdx.y ? second : 0);
    float sum = 0.0f;
    if (c < cols) sum = add_strided(sum, p + (int64_t)slice * stride + c, 16 * stride, (n - slice + 15) / 16); // (none: n - slice <= 0)
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

// per_row: chunks of a row that hold values, of fewer than 2^31 in all.  Bound by its bytes: 16384 x 8191 bfloat16 (340 MB) 62 us, 5.5 TB/s.
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
