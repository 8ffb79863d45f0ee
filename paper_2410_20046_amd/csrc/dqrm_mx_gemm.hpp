// Products of MXFP4 matrices: C[m][n] = act(sum over k of A[m][k] B[n][k] + bias[n]) (gfx950, wave64).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 codes of a row from each lane, one block with one scale byte: lane l holds row l % 32,
// block l / 32 of the 64 values.  Sums are held in 32 bits.
#pragma once

#include <type_traits>

#include "dqrm_mx.hpp"

namespace dqrm_mx {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
constexpr int kFp4 = 4; // the instruction's number for E2M1 operands

// BYTE: which byte of the scale registers counts
template <int BYTE>
__device__ __forceinline__ v16f mfma_32x32x64(uint4 a, uint4 b, v16f c, unsigned scale_a, unsigned scale_b)
{
    const v8i va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, c, kFp4, kFp4, BYTE, (int)scale_a, BYTE, (int)scale_b);
}

struct MatmulArgs {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    int64_t m, n, k;
    const float *bias; // [n] or null
    int relu;
    void *c;
    int64_t ldc;
    unsigned tiles_m, tiles_n, slices; // of the grid; slices > 1: c is [slices][m][n] of partial sums, bias and relu wait for the join
    unsigned stages_per_slice;
};

constexpr unsigned kParts = 8;              // of the chip, each with a second-level cache
constexpr unsigned kTileRows = 8;
constexpr int kStage = 256;                // values of k that a stage holds of each row: 128 bytes of codes, 8 of scales
constexpr int kStageCodes = kStage / 2, kStageScales = kStage / 32;

// ---- loads from memory straight into LDS -------------------------------------------------------------------------------
// The instructions are written out because the compiler, which cannot tell the stages' halves of LDS apart, would wait for every
// such load before any read of LDS.  They have no output registers; lds_barrier() is what waits for them.
typedef unsigned rsrc_t __attribute__((ext_vector_type(4)));

// `bytes` of memory from p on; what lies past them reads as zeros
__device__ __forceinline__ rsrc_t buffer_of(const uint8_t *p, int64_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    rsrc_t r;
    r.x = __builtin_amdgcn_readfirstlane((unsigned)at), r.y = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32) & 0xFFFFu);
    r.z = __builtin_amdgcn_readfirstlane((unsigned)min(bytes, (int64_t)0xFFFFFFFF)), r.w = 0x00027000u;
    return r;
}

// lane l's 16 (4) bytes at offset + base come to LDS address lds + 16 l (4 l); lds and base are the wave's
__device__ __forceinline__ void load16_to_lds(rsrc_t r, unsigned offset, unsigned base, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(r), "s"(__builtin_amdgcn_readfirstlane(base)) : "memory");
}
__device__ __forceinline__ void load4_to_lds(rsrc_t r, unsigned offset, unsigned base, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(r), "s"(__builtin_amdgcn_readfirstlane(base)) : "memory");
}
// every load of this wave is in LDS and every read of LDS has its data; then every wave's
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// A tile of WM * TM * 32 rows of A by WN * TN * 32 of B: WM by WN waves, each TM by TN accumulators of 32 by 32.
template <int TM_, int TN_, int WM_, int WN_>
struct TileShape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, waves = WM * WN, BM = TM * WM * 32, BN = TN * WN * 32;
    static constexpr int rows = BM + BN;
    static constexpr int code_bytes = rows * kStageCodes, stage_bytes = code_bytes + rows * kStageScales;
};

// Rows m by columns n of a wave's accumulators through LDS to memory: the lane has four neighbouring columns of one row in
// four registers, and stores 16 bytes of a row beside its neighbours'.
template <typename T, typename S>
__device__ __forceinline__ void store_tile(const MatmulArgs &g, T *c, int64_t ldc, const v16f (&acc)[S::TM][S::TN], char *lds, int64_t m0, int64_t n0, bool finish)
{
    constexpr int per = 16 / sizeof(T);             // values of a vector
    constexpr int cols = S::TN * 32, pitch = cols * sizeof(T) + 16;
    const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
    for (int t = 0; t < S::TM; ++t) {
        struct alignas(4 * sizeof(T)) Four { T v[4]; };
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                Four f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = acc[t][j][q * 4 + i];
                    if (finish && g.relu) v = v < 0.0f ? 0.0f : v; // (a NaN stays)
                    f.v[i] = (T)v;
                }
                *reinterpret_cast<Four *>(lds + (lane & 31) * pitch + (j * 32 + q * 8 + half * 4) * sizeof(T)) = f;
            }
        __builtin_amdgcn_wave_barrier();
        constexpr int vectors = cols / per; // of a row
#pragma unroll
        for (int i = 0; i < 32 * vectors / kWaveSize; ++i) {
            const int at = i * kWaveSize + lane, r = at / vectors, v = at % vectors;
            struct alignas(16) Many { T v[per]; };
            const Many x = *reinterpret_cast<const Many *>(lds + r * pitch + v * 16);
            const int64_t m = m0 + t * 32 + r, n = n0 + v * per;
            if (m >= g.m) continue;
            T *to = c + m * ldc + n;
            if (n + per <= g.n) {
                __builtin_memcpy(to, &x, sizeof(x));
            } else {
#pragma unroll
                for (int e = 0; e < per; ++e)
                    if (n + e < g.n) to[e] = x.v[e];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, typename S>
__global__ __launch_bounds__(S::waves *kWaveSize, 1) void matmul_kernel(MatmulArgs g)
{
    constexpr int pitch_out = S::TN * 32 * sizeof(T) + 16;
    constexpr int lds_bytes = 2 * S::stage_bytes > S::waves * 32 * pitch_out ? 2 * S::stage_bytes : S::waves * 32 * pitch_out;
    __shared__ __align__(1024) char lds[lds_bytes];
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned tiles = g.tiles_m * g.tiles_n;
    // Workgroups are dealt to the chip's parts in turn: each part gets a run of tiles, in columns of up to 8 rows of tiles, so
    // that the operands its second-level cache holds are read by several.
    const unsigned part = blockIdx.x % kParts, per_part = gridDim.x / kParts, more = gridDim.x % kParts;
    const unsigned place = part * per_part + min(part, more) + blockIdx.x / kParts;
    const unsigned slice = place / tiles, at = place - slice * tiles;
    const unsigned column = at / (kTileRows * g.tiles_n), in_column = at - column * kTileRows * g.tiles_n;
    const unsigned high = min((unsigned)kTileRows, g.tiles_m - column * kTileRows);
    const unsigned tn = in_column / high, tm = column * kTileRows + in_column - tn * high;
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const int64_t groups = groups_of(g.k), cp = groups * 64, sp = groups * 4;
    const int all = (int)((groups + 1) / 2);
    const int first = (int)(slice * g.stages_per_slice), last = min(all, first + (int)g.stages_per_slice);

    // operand memory from the tile's first row on; what lies past the matrix reads as zeros
    const rsrc_t ra = buffer_of(g.a_codes + m0 * cp, (g.m - m0) * cp), rb = buffer_of(g.b_codes + n0 * cp, (g.n - n0) * cp);
    const rsrc_t rsa = buffer_of(g.a_scales + m0 * sp, (g.m - m0) * sp), rsb = buffer_of(g.b_scales + n0 * sp, (g.n - n0) * sp);
    // codes in LDS: 8 vectors of 16 bytes to a row, vector v of row r in place v ^ (r & 7)
    const unsigned code_at = (unsigned)(lane >> 3) * (unsigned)cp + (unsigned)(((lane & 7) ^ (lane >> 3)) * 16);
    const unsigned scale_at = (unsigned)(lane >> 1) * (unsigned)sp + (unsigned)(lane & 1) * 4;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));

    auto request = [&](int s) {
        constexpr int a_loads = S::BM / 8, b_loads = S::BN / 8, sa_loads = S::BM / 32, s_loads = S::rows / 32;
        const unsigned to = lds0 + (unsigned)((s - first) & 1) * S::stage_bytes;
#pragma unroll
        for (int i = 0; i < a_loads / S::waves; ++i) {
            const unsigned j = (unsigned)(i * S::waves + wave);
            load16_to_lds(ra, code_at, (unsigned)s * kStageCodes + j * 8 * (unsigned)cp, to + j * 1024);
        }
#pragma unroll
        for (int i = 0; i < b_loads / S::waves; ++i) {
            const unsigned j = (unsigned)(i * S::waves + wave);
            load16_to_lds(rb, code_at, (unsigned)s * kStageCodes + j * 8 * (unsigned)cp, to + (a_loads + j) * 1024);
        }
if constexpr (sa_loads % S::waves == 0) {
#pragma unroll
            for (int i = 0; i < sa_loads / S::waves; ++i) {
                const unsigned j = (unsigned)(i * S::waves + wave);
                load4_to_lds(rsa, scale_at, (unsigned)s * kStageScales + j * 32 * (unsigned)sp, to + S::code_bytes + j * 256);
            }
#pragma unroll
            for (int i = 0; i < (s_loads - sa_loads) / S::waves; ++i) {
                const unsigned j = (unsigned)(i * S::waves + wave);
                load4_to_lds(rsb, scale_at, (unsigned)s * kStageScales + j * 32 * (unsigned)sp, to + S::code_bytes + (sa_loads + j) * 256);
            }
        } else {
            static_assert(s_loads == S::waves, "one load of scales to a wave");
            const bool of_a = wave < sa_loads;
            const unsigned j = (unsigned)(of_a ? wave : wave - sa_loads);
            load4_to_lds(of_a ? rsa : rsb, scale_at, (unsigned)s * kStageScales + j * 32 * (unsigned)sp, to + S::code_bytes + wave * 256);
        }
    };

    const int wm = wave / S::WN, wn = wave % S::WN;
    const int row_a = wm * S::TM * 32 + (lane & 31), row_b = S::BM + wn * S::TN * 32 + (lane & 31);
    uint4 a[2][S::TM], b[2][S::TN];
    auto read_codes = [&](int s, int t, int to) {
        const char *now = lds + ((s - first) & 1) * S::stage_bytes;
        const int at = ((2 * t + half) ^ (lane & 7)) * 16;
#pragma unroll
        for (int i = 0; i < S::TM; ++i) a[to][i] = *reinterpret_cast<const uint4 *>(now + (row_a + i * 32) * kStageCodes + at);
#pragma unroll
        for (int i = 0; i < S::TN; ++i) b[to][i] = *reinterpret_cast<const uint4 *>(now + (row_b + i * 32) * kStageCodes + at);
    };
    uint2 sa[S::TM], sb[S::TN];
    auto read_scales = [&](int s) {
        const char *now = lds + ((s - first) & 1) * S::stage_bytes + S::code_bytes;
#pragma unroll
        for (int i = 0; i < S::TM; ++i) sa[i] = *reinterpret_cast<const uint2 *>(now + (row_a + i * 32) * kStageScales);
#pragma unroll
        for (int i = 0; i < S::TN; ++i) sb[i] = *reinterpret_cast<const uint2 *>(now + (row_b + i * 32) * kStageScales);
    };
    // the sums begin with the bias
    const bool finish = g.slices <= 1;
    v16f acc[S::TM][S::TN] = {};
    if (finish && g.bias) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t n = n0 + (wn * S::TN + j) * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
                const float v = n < g.n ? g.bias[n] : 0.0f;
#pragma unroll
                for (int t = 0; t < S::TM; ++t) acc[t][j][i] = v;
            }
    }
    auto compute = [&](int s, auto is_last) {
        // the lane's bytes: block 2 t + half of the stage; past the row's end (the second half of an odd last stage) scales of 0 on
        // both sides give 0
        const bool odd_end = (int64_t)(s + 1) * 2 > groups;
        unsigned ua[2][S::TM], ub[2][S::TN];
#pragma unroll
        for (int i = 0; i < S::TM; ++i) ua[0][i] = sa[i].x >> (8 * half), ua[1][i] = odd_end ? 0u : sa[i].y >> (8 * half);
#pragma unroll
        for (int i = 0; i < S::TN; ++i) ub[0][i] = sb[i].x >> (8 * half), ub[1][i] = odd_end ? 0u : sb[i].y >> (8 * half);
#pragma unroll
        for (int t = 0; t < kStage / 64; ++t) {
            // what the next step needs is requested before this step's products; the compiler would gather all reads of the stage
            // at its beginning, where nothing hides them
            __builtin_amdgcn_sched_barrier(0);
            if (t + 1 < kStage / 64) {
                read_codes(s, t + 1, (t + 1) & 1);
            } else if constexpr (!decltype(is_last)::value) {
                lds_barrier();
                read_scales(s + 1);
                read_codes(s + 1, 0, 0);
                request(s + 2); // (past the last stage: nobody reads it)
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int j = 0; j < S::TN; ++j) {
                    if (t & 1)
                        acc[i][j] = mfma_32x32x64<2>(b[t & 1][j], a[t & 1][i], acc[i][j], ub[t >> 1][j], ua[t >> 1][i]);
                    else
                        acc[i][j] = mfma_32x32x64<0>(b[t & 1][j], a[t & 1][i], acc[i][j], ub[t >> 1][j], ua[t >> 1][i]);
                }
        }
    };
    if (first < last) {
        request(first);
        lds_barrier();
        request(first + 1);
        read_scales(first);
        read_codes(first, 0, 0);
        for (int s = first; s + 1 < last; ++s) compute(s, std::false_type{});
        compute(last - 1, std::true_type{});
    }
    lds_barrier(); // the last stage is read
    T *c = static_cast<T *>(g.c) + (finish ? 0 : (int64_t)slice * g.m * g.n);
    store_tile<T, S>(g, c, finish ? g.ldc : g.n, acc, lds + wave * 32 * pitch_out, m0 + wm * S::TM * 32, n0 + wn * S::TN * 32, finish);
}

// the slices' partial sums in turn, bias, relu, rounding
template <int DT>
__global__ __launch_bounds__(256) void matmul_join_kernel(const float *partial, MatmulArgs g)
{
    using T = elem_t<DT>;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, all = g.m * g.n;
    if (at >= all) return;
    const int count = (int)min((int64_t)4, all - at);
    float v[4] = {};
    for (unsigned s = 0; s < g.slices; ++s) {
        const float *p = partial + (int64_t)s * all + at;
        if (count == 4) {
            float4 x;
            __builtin_memcpy(&x, p, 16);
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        } else {
            for (int i = 0; i < count; ++i) v[i] += p[i];
        }
    }
    int64_t m = at / g.n, n = at - m * g.n;
    for (int i = 0; i < count; ++i) {
        float x = v[i] + (g.bias ? g.bias[n] : 0.0f);
        if (g.relu) x = x < 0.0f ? 0.0f : x;
        static_cast<T *>(g.c)[m * g.ldc + n] = (T)x;
        if (++n == g.n) n = 0, ++m;
    }
}

} // namespace dqrm_mx
