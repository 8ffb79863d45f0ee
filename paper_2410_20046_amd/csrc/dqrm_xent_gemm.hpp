// Products of 16-bit matrices for the softmax cross entropy: sums over k of A[m][k] B[n][k] in tiles (gfx950, wave64).
//
// v_mfma_f32_32x32x16 takes 8 values of k from each lane: lane l holds row l % 32, values 8 (l / 32) .. + 7 of 16.  An operand lies in memory with
// its k along the rows, whose 16-byte vectors are what a lane needs, or with k as the rows (a gradient's products sum over samples or
// classes): then it is read from LDS by the transposing read, which gives a lane 4 values of a column.  fp32 operands are three bfloat16
// planes, whose sum they are exactly; the six largest of the planes' nine products are six stages of the sum, the smallest first.
#pragma once

#include "dqrm_mx_gemm.hpp"

namespace dqrm_xent {

using namespace dqrm_mx;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short short4_t __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ v16f mfma_32x32x16(uint4 a, uint4 b, v16f c)
{
    if constexpr (std::is_same_v<T, __bf16>) {
        bf16x8 x, y;
        __builtin_memcpy(&x, &a, 16), __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
    } else {
        f16x8 x, y;
        __builtin_memcpy(&x, &a, 16), __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
    }
}

// An operand in memory: [rows][cols] of 16-bit values, 16-byte aligned, cols and the pitch (in bytes) multiples of 8 values; three planes of it
// for fp32, `plane` bytes apart.  Or in blocks of 64 by 64 values, 8 KB each, a row of blocks behind the other (cols and rows multiples of 64; the
// pitch is a row's of blocks over 64): what a tile's stage takes of it then are whole blocks, whichever way it is read, where rows of a large
// pitch give 128 or 512 bytes here and there.
struct Operand {
    const char *p;
    int64_t plane, pitch, rows, cols;
    const uint64_t *live; // or null; k as the rows: bit r % 64 of word r / 64 is 0 where row r counts as zeros, whatever it holds
};

struct Products {
    Operand a, b;
    int64_t m, n;                         // of the result
    unsigned stages;                      // of k, of one pair of planes
    unsigned pairs;                       // of planes: 1 or kPlanePairs
    unsigned tiles_m, tiles_n, slices, stages_per_slice;
};

constexpr int kDepth = 64;              // values of k in a stage: 128 bytes of each row
constexpr int kBlock = 64, kBlockBytes = kBlock * kBlock * 2;
constexpr int kStageRow = kDepth * 2;
constexpr unsigned kPlanePairs = 6;
constexpr unsigned kNowhere = 0xFFFFFFF0u; // an offset past every buffer: reads as zeros

// planes of A and B of a pair, two bits each, the smallest products first
__device__ __forceinline__ unsigned plane_a(unsigned pairs, unsigned pair) { return pairs == 1 ? 0u : (0x52u >> (2 * pair)) & 3u; }
__device__ __forceinline__ unsigned plane_b(unsigned pairs, unsigned pair) { return pairs == 1 ? 0u : (0x118u >> (2 * pair)) & 3u; }

__device__ __forceinline__ rsrc_t memory_at(const char *p, int64_t bytes)
{
    return buffer_of(reinterpret_cast<const uint8_t *>(p), min(max(bytes, (int64_t)0), (int64_t)0xFFFF0000));
}

// WM by WN waves, each with TM by TN accumulators of 32 by 32; LDS for `ring` stages.
// ROTATE: a tile begins its sum somewhere else than its neighbours (see multiply_tile).
template <int TM_, int TN_, int WM_, int WN_, int RING_, bool ROTATE_ = false>
struct Tile {
    static constexpr bool rotate = ROTATE_;
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, ring = RING_, waves = WM * WN, threads = waves * kWaveSize, BM = TM * WM * 32, BN = TN * WN * 32;
    static constexpr int stage_bytes = (BM + BN) * kStageRow, lds_bytes = ring * stage_bytes;
    static constexpr int per_simd = TM * TN > 8 ? 1 : 2; // waves that the accumulators leave room for
    static constexpr int a_loads = BM / 8 / waves, b_loads = BN / 8 / waves, loads = a_loads + b_loads; // of a wave in a stage
    // Order of a stage's instructions, in places behind each of a step's products: reads of the operands of steps 1 and 2 in step 0, of step 3
    // in the first half of step 1; behind place `freed` of step 1 every wave has read the stage, and the loads of the stage `ring` later go
    // into its memory, spread over the rest.  In the last step, behind place `arrived`, the next stage is there, and the operands of its
    // step 0 are read.
    static constexpr int steps = kDepth / 16, products = TM * TN, free_step = 1, freed = products * 3 / 4 - (products > 1), arrived = products / 4 - (products > 3);
    static constexpr int load_places = (steps - free_step) * products - freed;
    static constexpr int load_place(int q) { return q * load_places / loads; }
    static constexpr int loads_before_arrival()
    {
        int n = 0;
        for (int q = 0; q < loads; ++q) n += load_place(q) <= (steps - 1 - free_step) * products - freed + arrived;
        return n + (ring - 2) * loads; // (and those of the stages in between)
    }
    static constexpr int read_place(int r) { return r * products / (TM + TN) / 2; } // in half a step
    static_assert(waves % 2 == 0 && BM % (8 * waves) == 0 && BN % (8 * waves) == 0);
};

// A tile's place in the grid.  Workgroups are dealt to the chip's parts in turn: each part gets a run of tiles, in columns of up to 4 rows
// of tiles, so that the operands its second-level cache holds are read by several.
struct Place {
    unsigned slice, tm, tn;
};
__device__ __forceinline__ Place place_of(const Products &g)
{
    const unsigned tiles = g.tiles_m * g.tiles_n;
    const unsigned part = blockIdx.x % kParts, per_part = gridDim.x / kParts, more = gridDim.x % kParts;
    const unsigned place = part * per_part + min(part, more) + blockIdx.x / kParts;
    Place p;
    p.slice = uniform(place / tiles);
    const unsigned at = place - p.slice * tiles;
    const unsigned column = uniform(at / (kTileRows * g.tiles_n)), in_column = at - column * kTileRows * g.tiles_n;
    const unsigned high = min((unsigned)kTileRows, g.tiles_m - column * kTileRows);
    p.tn = uniform(in_column / high), p.tm = column * kTileRows + in_column - p.tn * high;
    return p;
}

// How an operand's stage comes to LDS and from there to registers.  BY_K: k as the rows.
//   rows along k:  [W rows][8 vectors of 16 bytes], vector v of row r in place v ^ (r / 2 % 8): the 16 rows that are read together lie in
//                  different banks.
//   BY_K:          [64 of k][W / 8 vectors], the groups of 4 vectors (32 values) of row r exchanged by r: the 4 rows that half a wave
//                  reads together do.
template <int W, int WAVES, bool BY_K, bool BLOCKS>
struct Carrier {
    static_assert(!BLOCKS || W % kBlock == 0);
    static constexpr int vectors = W / 8, groups = vectors / 4, turns = groups < 8 ? groups : 8;
    static constexpr int rows_per_load = BY_K ? 64 / vectors : 8; // that a wave's load of 1024 bytes covers

    // lane's part of a load's offset, and what says whether it lies inside
    unsigned at, row, vector;
    __device__ __forceinline__ Carrier(const Operand &o, int lane, int wave)
    {
        if constexpr (BY_K) {
            row = (unsigned)lane / vectors;
            const unsigned place = (unsigned)lane % vectors, r = (unsigned)wave * rows_per_load + row; // (loads of a wave are a multiple of 8 rows apart)
            vector = (place & 3u) | (((place >> 2) ^ (r & (turns - 1))) << 2);
        } else {
            row = (unsigned)lane >> 3;
            vector = ((unsigned)lane & 7u) ^ (((unsigned)lane >> 4) + 4u * ((unsigned)wave & 1u));
        }
        if constexpr (BLOCKS)
            at = (vector / 8u) * (BY_K ? kBlockBytes : 0) + row * (kBlock * 2) + vector % 8u * 16u;
        else
            at = row * (unsigned)o.pitch + vector * 16u;
    }
    // the wave's part of the stage at k0 (values), of the rows or columns from `first` on
    __device__ __forceinline__ static rsrc_t memory(const Operand &o, unsigned plane, int64_t first, int64_t k0)
    {
        const char *p = o.p + plane * o.plane;
        if constexpr (BLOCKS) {
            const int64_t from = BY_K ? k0 * o.pitch + first / kBlock * kBlockBytes : first * o.pitch + k0 / kBlock * kBlockBytes;
            return memory_at(p + from, o.rows * o.pitch - from);
        } else if constexpr (BY_K)
            return memory_at(p + k0 * o.pitch + first * 2, (o.rows - k0 - 1) * o.pitch + (o.cols - first) * 2);
        else
            return memory_at(p + first * o.pitch, (o.rows - first - 1) * o.pitch + o.cols * 2);
    }
    // load j of the stage
    __device__ __forceinline__ unsigned offset(const Operand &o, unsigned j, unsigned k0, uint64_t live) const
    {
        const unsigned r = j * rows_per_load;
        if constexpr (BLOCKS && BY_K)
            return at + r * (kBlock * 2);
        else if constexpr (BLOCKS) // (a load's 8 rows are of one block)
            return at + r / kBlock * (kBlock * (unsigned)o.pitch) + r % kBlock * (kBlock * 2);
        else if constexpr (BY_K)
            return (live >> (r + row)) & 1 ? at + r * (unsigned)o.pitch : kNowhere;
        else
            return k0 * 2 + vector * 16 < (unsigned)o.cols * 2 ? at + k0 * 2 + r * (unsigned)o.pitch : kNowhere;
    }
    // the lane's 8 values of k of block `block` (32 rows or columns) in step t
    __device__ __forceinline__ static uint4 read(const char *stage, int block, int t, int lane)
    {
        const int half = lane >> 5;
        if constexpr (BY_K) {
            const int j = lane & 15, k = 8 * half + (j >> 2); // (of the step's 16; the second read has k + 4)
            uint4 v;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int group = block ^ (((j >> 2) + 4 * i) & (turns - 1));
                const char *at = stage + (16 * t + k + 4 * i) * W * 2 + group * 64 + ((lane >> 4) & 1) * 32 + (j & 3) * 8;
                const short4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)(uintptr_t)lds_address(at));
                __builtin_memcpy(reinterpret_cast<char *>(&v) + 8 * i, &x, 8);
            }
            return v;
        } else {
            return *reinterpret_cast<const uint4 *>(stage + (block * 32 + (lane & 31)) * kStageRow + (((2 * t + half) ^ ((lane >> 1) & 7)) * 16));
        }
    }
};

// The sums of stages [first, last) for the tile at (m0, n0): accumulator [t][j] of a lane has row lane % 32 of block t, and columns
// 8 (i / 4) + 4 (lane / 32) + i % 4 of block j.  Ends with a barrier: LDS is free.
// S::rotate: the stages are taken in turn from one on that depends on the tile.  Rows whose pitch is a power of two lie in the same few of the
// memory's channels at any one k; tiles that stream different rows at the same pace would all be there at once.
template <typename T, typename S, bool A_BY_K, bool B_BY_K, bool A_BLOCKS>
__device__ __forceinline__ void multiply_tile(const Products &g, char *lds, int64_t m0, int64_t n0, int first, int last, unsigned turn, v16f (&acc)[S::TM][S::TN])
{
    using CA = Carrier<S::BM, S::waves, A_BY_K, A_BLOCKS>;
    using CB = Carrier<S::BN, S::waves, B_BY_K, false>;
    const int lane = threadIdx.x & 63;
    const int wave = (int)uniform(threadIdx.x >> 6);
    const unsigned lds0 = uniform(lds_address(lds));
    const CA ca(g.a, lane, wave);
    const CB cb(g.b, lane, wave);
    // the stage that is requested
    rsrc_t ra, rb;
    unsigned k0 = 0, into = 0;
    uint64_t live_a = ~0ull, live_b = ~0ull;
    const int shift = S::rotate && last > first ? (int)uniform(turn * 5u % (unsigned)(last - first)) : 0;
    auto aim = [&](int at) {
        const bool there = at < last;
        int s = at + shift;
        if (S::rotate && s >= last) s -= last - first;
        // (the planes' products of the same values of k follow each other: a plane that is needed again is still in a cache)
        const unsigned stage = g.pairs == 1 ? (unsigned)s : uniform((unsigned)s / kPlanePairs), pair = g.pairs == 1 ? 0u : (unsigned)s - stage * kPlanePairs;
        k0 = stage * kDepth;
        ra = CA::memory(g.a, plane_a(g.pairs, pair), m0, k0), rb = CB::memory(g.b, plane_b(g.pairs, pair), n0, k0);
        // (what is past `last` is requested from a buffer without bytes, so that every stage is as many loads)
        if (!there) ra.z = 0u, rb.z = 0u;
        if (A_BY_K && g.a.live && there) live_a = g.a.live[stage];
        if (B_BY_K && g.b.live && there) live_b = g.b.live[stage];
        into = lds0 + (unsigned)((at - first) & (S::ring - 1)) * S::stage_bytes;
    };
    auto request = [&](int q) {
        const bool of_a = q < S::a_loads;
        const unsigned j = (unsigned)((of_a ? q : q - S::a_loads) * S::waves + wave);
        load16_to_lds(of_a ? ra : rb, of_a ? ca.offset(g.a, j, k0, live_a) : cb.offset(g.b, j, k0, live_b), into + (of_a ? 0u : S::BM * kStageRow) + j * 1024);
    };
    const int wm = wave / S::WN, wn = wave % S::WN;
    constexpr int steps = S::steps, reads = S::TM + S::TN;
    uint4 a[steps][S::TM], b[steps][S::TN];
    // operand r of step t, A's blocks, then B's
    auto read = [&](int s, int t, int r) {
        const char *now = lds + ((s - first) & (S::ring - 1)) * S::stage_bytes;
        if (r < S::TM)
            a[t][r] = CA::read(now, wm * S::TM + r, t, lane);
        else
            b[t][r - S::TM] = CB::read(now + S::BM * kStageRow, wn * S::TN + r - S::TM, t, lane);
    };
#pragma unroll
    for (int t = 0; t < S::TM; ++t)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[t][j] = v16f{};
    // (sched_barrier: the compiler keeps this order; left to itself it gathers the reads where nothing hides them)
    auto compute = [&](int s, auto is_last) {
        constexpr bool more = !decltype(is_last)::value;
        if constexpr (more) aim(s + S::ring);
#pragma unroll
        for (int t = 0; t < steps; ++t) {
#pragma unroll
            for (int p = 0; p < S::products; ++p) {
                acc[p / S::TN][p % S::TN] = mfma_32x32x16<T>(b[t][p % S::TN], a[t][p / S::TN], acc[p / S::TN][p % S::TN]);
                __builtin_amdgcn_sched_barrier(0);
                if (t < 2) {
#pragma unroll
                    for (int r = 0; r < reads; ++r) {
                        if (S::read_place(r) == p) read(s, t == 0 ? 1 : 3, r);
                        if (t == 0 && S::read_place(r) + S::products / 2 == p) read(s, 2, r);
                    }
                }
                if constexpr (more) {
                    if (t == S::free_step && p == S::freed) read_barrier();
                    const int place = (t - S::free_step) * S::products + p - S::freed; // (negative before)
#pragma unroll
                    for (int q = 0; q < S::loads; ++q)
                        if (S::load_place(q) == place) request(q);
                    if (t == steps - 1 && p == S::arrived) loaded_barrier<S::loads_before_arrival()>();
                    if (t == steps - 1 && p >= S::arrived) {
                        constexpr int left = S::products - S::arrived;
#pragma unroll
                        for (int r = 0; r < reads; ++r)
                            if (r * left / reads == p - S::arrived) read(s + 1, 0, r);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    if (first < last) {
#pragma unroll
        for (int k = 0; k < S::ring; ++k) {
            aim(first + k);
#pragma unroll
            for (int q = 0; q < S::loads; ++q) request(q);
        }
        loaded_barrier<(S::ring - 1) * S::loads>();
#pragma unroll
        for (int r = 0; r < reads; ++r) read(first, 0, r);
        for (int s = first; s + 1 < last; ++s) compute(s, std::false_type{});
        compute(last - 1, std::true_type{});
    }
    lds_barrier(); // the last stage is read
}

// A wave's accumulators through LDS to memory, 16 bytes of a row beside its neighbours'.
enum class To {
    rows,   // of the result
    sums,   // the same (float), added to what is there
    blocks, // 16-bit values in blocks of 64 by 64: ldc is a row's of blocks over 64, n a multiple of 64, m of 64
};
template <typename T, typename S, To TO>
struct TileOut {
    static constexpr bool ADD = TO == To::sums;
    static constexpr int per = 16 / sizeof(T);
    static constexpr int cols = S::TN * 32, pitch = cols * sizeof(T) + 16;
    static constexpr int vectors = cols / per, rows_each = kWaveSize / vectors; // of a row; rows that a wave stores at a time
    static constexpr int block_bytes = 32 * pitch, fit = S::lds_bytes / (S::waves * block_bytes);
    static constexpr int together = fit >= S::TM ? S::TM : fit >= 2 && S::TM % 2 == 0 ? 2 : 1; // blocks that are in LDS together
    static constexpr int wave_bytes = together * block_bytes;
    static_assert(fit >= 1 && vectors <= kWaveSize);

    // c: the result's first value; rows and columns of it up to m and n
    static __device__ __forceinline__ void run(T *c, int64_t ldc, const v16f (&acc)[S::TM][S::TN], char *lds, int64_t m0, int64_t n0, int64_t m, int64_t n,
                                               float by)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        char *write = lds + (lane & 31) * pitch + half * 4 * sizeof(T);
        const int r = lane / vectors, v = lane % vectors;
        const char *read = lds + r * pitch + v * 16;
        const int64_t row = m0 + r, col = n0 + v * per;
        T *to = c + row * ldc + col;
        // (blocks: a wave's blocks of 32 rows begin at the first or the 33rd row of one, and a row's vectors lie in 1 or 2 of them)
        if constexpr (TO == To::blocks) to = c + row / kBlock * kBlock * ldc + col / kBlock * (kBlock * kBlock) + row % kBlock * kBlock + col % kBlock;
        auto row_at = [&](int i) -> T * { // i rows on, i a multiple of rows_each
            if constexpr (TO == To::blocks) {
                const int64_t at = row + i;
                return to + (at / kBlock - row / kBlock) * kBlock * ldc + (at % kBlock - row % kBlock) * kBlock;
            } else {
                return to + (int64_t)i * ldc;
            }
        };
        const bool inside = m0 + S::TM * 32 <= m && n0 + cols <= n; // of the whole wave
        struct alignas(16) Many { T v[per]; };
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
                        for (int i = 0; i < 4; ++i) f.v[i] = (T)(acc[first + t][j][q * 4 + i] * by);
                        *reinterpret_cast<Four *>(write + t * block_bytes + (j * 32 + q * 8) * sizeof(T)) = f;
                    }
            __builtin_amdgcn_wave_barrier();
            if (inside) {
#pragma unroll 4
                for (int i = 0; i < together * 32 / rows_each; ++i) {
                    Many x = *reinterpret_cast<const Many *>(read + i * rows_each * pitch);
                    T *at = row_at(first * 32 + i * rows_each);
                    if constexpr (ADD) {
                        Many old;
                        __builtin_memcpy(&old, at, 16);
#pragma unroll
                        for (int e = 0; e < per; ++e) x.v[e] += old.v[e];
                    }
                    __builtin_memcpy(at, &x, 16);
                }
            } else {
                for (int i = 0; i < together * 32 / rows_each; ++i) {
                    const Many x = *reinterpret_cast<const Many *>(read + i * rows_each * pitch);
                    if (row + first * 32 + i * rows_each >= m) break;
                    T *at = row_at(first * 32 + i * rows_each);
                    for (int e = 0; e < per; ++e)
                        if (col + e < n) at[e] = ADD ? (T)(at[e] + x.v[e]) : x.v[e];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

} // namespace dqrm_xent
