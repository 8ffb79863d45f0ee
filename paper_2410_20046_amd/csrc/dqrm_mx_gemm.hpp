// Products of MXFP4 matrices: C[m][n] = act(sum over k of A[m][k] B[n][k] + bias[n]) (gfx950, wave64).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 codes of a row from each lane, one block with one scale byte: lane l holds row l % 32,
// block l / 32 of the 64 values.  Sums are held in 32 bits.
//
// What bounds them: from registers alone the instruction reaches 9.6 PFLOP/s with one code throughout and 6.2 with random ones, at which
// the card lowers its clock.  16384 x 8192 x 8192 takes 490 to 515 us, 4.3 to 4.5 PFLOP/s: tiles of 256 (6 operands read from LDS for 8
// products, two barriers to a stage of 256 values of k) keep the matrix cores at work for 67 % of the time and LDS for 41 %.  Tiles of 128 (4
// operands for 4 products, or 3 for 2) have one barrier to a stage and few products between two of them: 2048 x 2048 x 8192, 27 us, matrix
// cores 36 %, LDS 40 %; no unit is at its limit, what is left is waiting.  Short sums are bound by the launch, the first loads' latency and the output's stores: 8192 x 512 x 415 in float, 8 us.
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

constexpr unsigned kParts = 8;     // of the chip, each with a second-level cache
constexpr unsigned kTileRows = 4;
constexpr int kStage = 256; // values of k that a stage holds of each row: 128 bytes of codes
constexpr int kStageCodes = kStage / 2;
// Scales come for two stages at a time, 16 bytes of a row: what a load costs is its lines, and a row's scales of one stage are 8 bytes
// of a line.  A's of a pair of stages are requested with the stage before the pair, B's with the pair's first one.
constexpr int kPairScales = 2 * kStage / 32;

// ---- loads from memory straight into LDS -------------------------------------------------------------------------------
// The instructions are written out because the compiler, which cannot tell the stages' halves of LDS apart, would wait for every
// such load before any read of LDS.  They have no output registers; lds_barrier() is what waits for them.
typedef unsigned rsrc_t __attribute__((ext_vector_type(4)));

// a value that all lanes hold, in a scalar register
__device__ __forceinline__ unsigned uniform(unsigned v) { return __builtin_amdgcn_readfirstlane(v); }

// `bytes` of memory from p on; what lies past them reads as zeros
__device__ __forceinline__ rsrc_t buffer_of(const uint8_t *p, int64_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    rsrc_t r;
    r.x = uniform((unsigned)at), r.y = uniform((unsigned)(at >> 32) & 0xFFFFu);
    r.z = uniform((unsigned)min(bytes, (int64_t)0xFFFFFFFF)), r.w = 0x00027000u;
    return r;
}

// Lane l's 16 (4) bytes at `offset` come to LDS address lds + 16 l (4 l); lds is the wave's.  All of the offset is in the vector register:
// that is what the bounds check looks at (an offset from a scalar register is not part of it).
__device__ __forceinline__ void load16_to_lds(rsrc_t r, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform(lds)), "v"(offset), "s"(r) : "memory");
}
__device__ __forceinline__ void load4_to_lds(rsrc_t r, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(uniform(lds)), "v"(offset), "s"(r) : "memory");
}
// every load of this wave is in LDS and every read of LDS has its data; then every wave's
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// every wave has what it has read from LDS
__device__ __forceinline__ void read_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// every wave's loads are in LDS but for its last N
template <int N>
__device__ __forceinline__ void loaded_barrier() { asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory"); }
// both
template <int N>
__device__ __forceinline__ void loaded_and_read_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// A tile of WM * TM * 32 rows of A by WN * TN * 32 of B: WM by WN waves, each TM by TN accumulators of 32 by 32; memory for `ring`
// stages of k in LDS.
template <int TM_, int TN_, int WM_, int WN_, int RING_>
struct TileShape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, ring = RING_, waves = WM * WN, BM = TM * WM * 32, BN = TN * WN * 32;
    static constexpr int rows = BM + BN;
    static constexpr int per_simd = TM * TN > 8 ? 1 : 2; // waves that the accumulators leave room for
    static_assert(BM == BN, "A's and B's scales are as many loads");
    static constexpr int pairs = ring / 2 + 2; // of stages whose scales are in LDS: from the one in use to the one that is loaded
    static constexpr int stage_bytes = rows * kStageCodes, pair_bytes = rows * kPairScales, lds_bytes = ring * stage_bytes + pairs * pair_bytes;
    // loads of a wave in a stage: vectors of A's and of B's codes, scales
    static constexpr int a_loads = BM / 8 / waves, b_loads = BN / 8 / waves, scale_loads = BM / 16 / waves, loads = a_loads + b_loads + scale_loads;
    // Order of a stage's instructions, in places behind each of a step's products.  Reads of LDS: the operands of steps 1 and 2 in step
    // 0, those of step 3 in the first half of step 1, so that a stage's memory is free early; behind place `freed` of step 1 every wave
    // has read the stage, and the loads of the stage `ring` later go into its memory, spread evenly over the rest.  In the last step,
    // behind place `arrived`, the next stage is there, and the operands of its step 0 are read.
    static constexpr int steps = kStage / 64, products = TM * TN, free_step = 1, freed = products * 3 / 4 - (products > 1), arrived = products / 4 - (products > 3);
    // A wave with few products in a step has no time to hide reads of LDS behind them: it reads a whole stage ahead.
    static constexpr bool stage_ahead = products <= 4;
    static constexpr int load_places = (steps - free_step) * products - freed;
    static constexpr int load_place(int q) { return q * load_places / loads; }
    static constexpr int loads_before_arrival()
    {
        int n = 0;
        for (int q = 0; q < loads; ++q) n += load_place(q) <= (steps - 1 - free_step) * products - freed + arrived;
        return n + (ring - 2) * loads; // (and those of the stages in between)
    }
    static constexpr int read_place(int r) { return r * products / (TM + TN) / 2; } // in half a step
};

// Rows m by columns n of a wave's accumulators through LDS to memory: the lane has four neighbouring columns of one row in
// four registers, and stores 16 bytes of a row beside its neighbours'.
template <typename T, typename S>
struct StoreTile {
    static constexpr int per = 16 / sizeof(T);                       // values of a vector
    static constexpr int cols = S::TN * 32, pitch = cols * sizeof(T) + 16;
    static constexpr int vectors = cols / per, rows_each = kWaveSize / vectors; // of a row; rows that a wave stores at a time
    static constexpr int block_bytes = 32 * pitch;                   // 32 rows of a wave's accumulators
    static constexpr int fit = S::lds_bytes / (S::waves * block_bytes);
    static constexpr int together = fit >= S::TM ? S::TM : fit > 0 ? fit : 1; // such blocks that are in LDS together
    static constexpr int wave_bytes = together * block_bytes;
    static_assert(S::TM % together == 0);

    static __device__ __forceinline__ void run(const MatmulArgs &g, T *c, int64_t ldc, v16f (&acc)[S::TM][S::TN], char *lds, int64_t m0, int64_t n0, bool relu)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        if (relu) {
#pragma unroll
            for (int t = 0; t < S::TM; ++t)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[t][j][i] = acc[t][j][i] < 0.0f ? 0.0f : acc[t][j][i]; // (a NaN stays)
        }
        char *write = lds + (lane & 31) * pitch + half * 4 * sizeof(T);
        const int r = lane / vectors, v = lane % vectors;
        const char *read = lds + r * pitch + v * 16;
        const int64_t m = m0 + r, n = n0 + v * per;
        T *to = c + m * ldc + n;
        const bool inside = m0 + S::TM * 32 <= g.m && n0 + cols <= g.n; // of the whole wave
        // whole lines go past the caches; parts of lines meet their other parts there
        const bool lines = (ldc * sizeof(T)) % 128 == 0 && reinterpret_cast<uintptr_t>(c) % 128 == 0;
#pragma unroll
        for (int first = 0; first < S::TM; first += together) {
#pragma unroll
            for (int t = 0; t < together; ++t)
#pragma unroll
                for (int j = 0; j < S::TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        struct alignas(4 * sizeof(T)) Four { T v[4]; } f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) f.v[i] = (T)acc[first + t][j][q * 4 + i];
                        *reinterpret_cast<Four *>(write + t * block_bytes + (j * 32 + q * 8) * sizeof(T)) = f;
                    }
            __builtin_amdgcn_wave_barrier();
            struct alignas(16) Many { T v[per]; };
            if (inside && lines) {
#pragma unroll
                for (int i = 0; i < together * 32 / rows_each; ++i)
                    store_stream(to + (int64_t)(first * 32 + i * rows_each) * ldc, *reinterpret_cast<const Many *>(read + i * rows_each * pitch));
            } else if (inside) {
#pragma unroll
                for (int i = 0; i < together * 32 / rows_each; ++i)
                    __builtin_memcpy(to + (int64_t)(first * 32 + i * rows_each) * ldc, read + i * rows_each * pitch, 16);
            } else {
                for (int i = 0; i < together * 32 / rows_each; ++i) {
                    const Many x = *reinterpret_cast<const Many *>(read + i * rows_each * pitch);
                    if (m + first * 32 + i * rows_each >= g.m) break;
                    T *at = to + (int64_t)(first * 32 + i * rows_each) * ldc;
                    if (n + per <= g.n) {
                        __builtin_memcpy(at, &x, 16);
                    } else {
                        for (int e = 0; e < per; ++e)
                            if (n + e < g.n) at[e] = x.v[e];
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

template <typename T, typename S>
__global__ __launch_bounds__(S::waves *kWaveSize, S::per_simd) void matmul_kernel(MatmulArgs g)
{
    constexpr int out_bytes = S::waves * StoreTile<T, S>::wave_bytes, lds_bytes = S::lds_bytes > out_bytes ? S::lds_bytes : out_bytes;
    __shared__ __align__(1024) char lds[lds_bytes];
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = (int)uniform(threadIdx.x >> 6);
    const unsigned tiles = g.tiles_m * g.tiles_n;
    // Workgroups are dealt to the chip's parts in turn: each part gets a run of tiles, in columns of up to 4 rows of tiles, so
    // that the operands its second-level cache holds are read by several.
    const unsigned part = blockIdx.x % kParts, per_part = gridDim.x / kParts, more = gridDim.x % kParts;
    const unsigned place = part * per_part + min(part, more) + blockIdx.x / kParts;
    const unsigned slice = uniform(place / tiles), at = place - slice * tiles;
    const unsigned column = uniform(at / (kTileRows * g.tiles_n)), in_column = at - column * kTileRows * g.tiles_n;
    const unsigned high = min((unsigned)kTileRows, g.tiles_m - column * kTileRows);
    const unsigned tn = uniform(in_column / high), tm = column * kTileRows + in_column - tn * high;
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const int64_t groups = groups_of(g.k), cp = groups * 64, sp = groups * 4;
    const int all = (int)((groups + 1) / 2);
    const int first = (int)(slice * g.stages_per_slice), last = min(all, first + (int)g.stages_per_slice);

    // operand memory from the tile's first row on; what lies past the matrix reads as zeros
    const rsrc_t ra = buffer_of(g.a_codes + m0 * cp, (g.m - m0) * cp), rb = buffer_of(g.b_codes + n0 * cp, (g.n - n0) * cp);
    const rsrc_t rsa = buffer_of(g.a_scales + m0 * sp, (g.m - m0) * sp), rsb = buffer_of(g.b_scales + n0 * sp, (g.n - n0) * sp);
    // Codes in LDS: 8 vectors of 16 bytes to a row, vector v of row r in place v ^ (r / 2 % 8): the 16 rows that are read together
    // lie in different banks.  (A load has 8 rows from an 8-fold on, an odd one in odd waves.)
    static_assert(S::waves % 2 == 0);
    const unsigned code_at = (unsigned)(lane >> 3) * (unsigned)cp + (unsigned)(((lane & 7) ^ ((lane >> 4) + 4 * (wave & 1))) * 16);
    const unsigned scale_at = (unsigned)(lane >> 2) * (unsigned)sp + (unsigned)(lane & 3) * 4;
    const unsigned lds0 = uniform(lds_address(lds));

    // what is past `last` is requested from a buffer without bytes, so that every stage is as many loads
    auto until_last = [&](rsrc_t r, int s) {
        r.z = uniform(s < last ? r.z : 0u);
        return r;
    };
    const unsigned lds_scales = lds0 + S::ring * S::stage_bytes;
    // load k of the S::scale_loads that a wave has of A's or B's scales of a pair of stages
    auto request_scales = [&](int pair, bool of_a, int k) {
        const unsigned j = (unsigned)(k * S::waves + wave);
        load4_to_lds(until_last(of_a ? rsa : rsb, 2 * pair), scale_at + (unsigned)pair * kPairScales + j * 16 * (unsigned)sp,
                     lds_scales + (unsigned)(pair % S::pairs) * S::pair_bytes + (of_a ? 0 : S::BM * kPairScales) + j * 256);
    };
    // load q of the S::loads that a wave has with stage s
    auto request = [&](int s, int q) {
        if (q < S::a_loads + S::b_loads) {
            const bool of_a = q < S::a_loads;
            const unsigned j = (unsigned)((of_a ? q : q - S::a_loads) * S::waves + wave);
            load16_to_lds(until_last(of_a ? ra : rb, s), code_at + (unsigned)s * kStageCodes + j * 8 * (unsigned)cp,
                          lds0 + (unsigned)((s - first) & (S::ring - 1)) * S::stage_bytes + (of_a ? 0 : S::BM * kStageCodes) + j * 1024);
        } else {
            request_scales((s + 1) >> 1, s & 1, q - S::a_loads - S::b_loads);
        }
    };

    const int wm = wave / S::WN, wn = wave % S::WN;
    const int row_a = wm * S::TM * 32 + (lane & 31), row_b = S::BM + wn * S::TN * 32 + (lane & 31);
    constexpr int steps = S::steps, reads = S::TM + S::TN;
    constexpr int sets = S::stage_ahead ? 2 * steps : steps; // of operands in registers
    uint4 a[sets][S::TM], b[sets][S::TN];
    // operand r of step t, A's rows, then B's, into a set
    auto read_codes = [&](int s, int t, int r, int set) {
        const char *now = lds + ((s - first) & (S::ring - 1)) * S::stage_bytes;
        const int at = ((2 * t + half) ^ ((lane >> 1) & 7)) * 16;
        if (r < S::TM)
            a[set][r] = *reinterpret_cast<const uint4 *>(now + (row_a + r * 32) * kStageCodes + at);
        else
            b[set][r - S::TM] = *reinterpret_cast<const uint4 *>(now + (row_b + (r - S::TM) * 32) * kStageCodes + at);
    };
    uint2 raw_scales[reads];
    auto read_scales = [&](int s, int r) {
        const char *now = lds + S::ring * S::stage_bytes + (s >> 1) % S::pairs * S::pair_bytes + (s & 1) * (kPairScales / 2);
        const int row = r < S::TM ? row_a + r * 32 : row_b + (r - S::TM) * 32;
        raw_scales[r] = *reinterpret_cast<const uint2 *>(now + row * kPairScales);
    };
    // The lane's bytes: block 2 t + half of the stage.  Past the row's end (the second half of an odd last stage) scales of 0 on both
    // sides give 0.
    unsigned scales[reads][2];
    auto take_scales = [&](int s) {
        const bool odd_end = (int64_t)(s + 1) * 2 > groups;
#pragma unroll
        for (int r = 0; r < reads; ++r) scales[r][0] = raw_scales[r].x >> (8 * half), scales[r][1] = odd_end ? 0u : raw_scales[r].y >> (8 * half);
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
                const float v = g.bias[min(n, g.n - 1)]; // (a column past the last one is not stored)
#pragma unroll
                for (int t = 0; t < S::TM; ++t) acc[t][j][i] = v;
            }
    }
    auto multiply = [&](int t, int p, int set) {
        const int i = p / S::TN, j = p % S::TN;
        if (t & 1)
            acc[i][j] = mfma_32x32x64<2>(b[set][j], a[set][i], acc[i][j], scales[S::TM + j][t >> 1], scales[i][t >> 1]);
        else
            acc[i][j] = mfma_32x32x64<0>(b[set][j], a[set][i], acc[i][j], scales[S::TM + j][t >> 1], scales[i][t >> 1]);
    };
    // (sched_barrier: the compiler keeps this order; left to itself it gathers the reads where nothing hides them)
    auto compute = [&](int s, auto is_last) {
        constexpr bool more = !decltype(is_last)::value;
        take_scales(s);
#pragma unroll
        for (int t = 0; t < steps; ++t) {
#pragma unroll
            for (int p = 0; p < S::products; ++p) {
                multiply(t, p, t);
                __builtin_amdgcn_sched_barrier(0);
                if (t < 2) {
#pragma unroll
                    for (int r = 0; r < reads; ++r) {
                        if (S::read_place(r) == p) read_codes(s, t == 0 ? 1 : 3, r, t == 0 ? 1 : 3);
                        if (t == 0 && S::read_place(r) + S::products / 2 == p) read_codes(s, 2, r, 2);
                    }
                }
                if constexpr (more) {
                    if (t == S::free_step && p == S::freed) read_barrier();
                    const int place = (t - S::free_step) * S::products + p - S::freed; // (negative before)
#pragma unroll
                    for (int q = 0; q < S::loads; ++q)
                        if (S::load_place(q) == place) request(s + S::ring, q);
                    if (t == steps - 1 && p == S::arrived) {
                        loaded_barrier<S::loads_before_arrival()>();
#pragma unroll
                        for (int r = 0; r < reads; ++r) read_scales(s + 1, r);
                    }
                    if (t == steps - 1 && p >= S::arrived) {
                        constexpr int left = S::products - S::arrived;
#pragma unroll
                        for (int r = 0; r < reads; ++r)
                            if (r * left / reads == p - S::arrived) read_codes(s + 1, 0, r, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // stage_ahead: stage s from the sets of its parity, stage s + 1 into the others
    auto compute_ahead = [&](int s, auto parity, auto is_last) {
        constexpr int now = decltype(parity)::value * steps, next = steps - now;
        constexpr bool more = !decltype(is_last)::value;
        take_scales(s);
        if constexpr (more) loaded_and_read_barrier<(S::ring - 2) * S::loads>(); // stage s is in registers everywhere, stage s + 1 in LDS
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < steps; ++t) {
#pragma unroll
            for (int p = 0; p < S::products; ++p) {
                multiply(t, p, now + t);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (more) {
                    constexpr int all = steps * S::products;
                    const int place = t * S::products + p;
                    if (place == 0) {
#pragma unroll
                        for (int r = 0; r < reads; ++r) read_scales(s + 1, r);
                    }
#pragma unroll
                    for (int k = 0; k < steps * reads; ++k)
                        if (k * all / (steps * reads) == place) read_codes(s + 1, k / reads, k % reads, next + k / reads);
#pragma unroll
                    for (int q = 0; q < S::loads; ++q)
                        if (q * all / S::loads == place) request(s + S::ring, q);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    if (first < last) { // (first is even)
#pragma unroll
        for (int k = 0; k < S::scale_loads; ++k) request_scales(first >> 1, true, k);
#pragma unroll
        for (int k = 0; k < S::ring; ++k) {
#pragma unroll
            for (int q = 0; q < S::loads; ++q) request(first + k, q);
        }
        loaded_barrier<(S::ring - 1) * S::loads>();
#pragma unroll
        for (int r = 0; r < reads; ++r) read_scales(first, r);
#pragma unroll
        for (int k = 0; k < (S::stage_ahead ? steps : 1) * reads; ++k) read_codes(first, k / reads, k % reads, k / reads);
        const std::integral_constant<int, 0> even;
        const std::integral_constant<int, 1> odd;
        if constexpr (S::stage_ahead) {
            int s = first;
            for (; s + 2 < last; s += 2) {
                compute_ahead(s, even, std::false_type{});
                compute_ahead(s + 1, odd, std::false_type{});
            }
            if (s + 1 < last) {
                compute_ahead(s, even, std::false_type{});
                compute_ahead(s + 1, odd, std::true_type{});
            } else {
                compute_ahead(s, even, std::true_type{});
            }
        } else {
            for (int s = first; s + 1 < last; ++s) compute(s, std::false_type{});
            compute(last - 1, std::true_type{});
        }
    }
    lds_barrier(); // the last stage is read
    T *c = static_cast<T *>(g.c) + (finish ? 0 : (int64_t)slice * g.m * g.n);
    StoreTile<T, S>::run(g, c, finish ? g.ldc : g.n, acc, lds + wave * StoreTile<T, S>::wave_bytes, m0 + wm * S::TM * 32, n0 + wn * S::TN * 32, finish && g.relu);
}

// the slices' partial sums in turn, bias, relu, rounding: bound by the partial sums' bytes (16 of 512 x 367, 12 MB: 4.6 us)
template <int DT>
__global__ __launch_bounds__(256) void matmul_join_kernel(const float *partial, MatmulArgs g)
{
    using T = elem_t<DT>;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, all = g.m * g.n;
    if (at >= all) return;
    const unsigned m = (unsigned)(at / g.n), n = (unsigned)(at - m * g.n);
    float v = g.bias ? g.bias[n] : 0.0f;
    constexpr int ahead = 8; // loads in flight
    unsigned s = 0;
    for (; s + ahead <= g.slices; s += ahead) {
        float x[ahead];
#pragma unroll
        for (int i = 0; i < ahead; ++i) x[i] = partial[(int64_t)(s + i) * all + at];
#pragma unroll
        for (int i = 0; i < ahead; ++i) v += x[i];
    }
    for (; s < g.slices; ++s) v += partial[(int64_t)s * all + at];
    if (g.relu) v = v < 0.0f ? 0.0f : v; // (a NaN stays)
    static_cast<T *>(g.c)[m * g.ldc + n] = (T)v;
}

} // namespace dqrm_mx
