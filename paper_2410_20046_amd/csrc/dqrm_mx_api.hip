// C ABI of layer norm and of MXFP4 linear layers: host-side validation and kernel dispatch.
// Every entry point validates on the host first and enqueues nothing on error.
#include "dqrm_checks.hpp"
#include "dqrm_mx.hpp"
#include "dqrm_mx_gemm.hpp"
#include "dqrm_norm.hpp"
#include "dqrm_mx_few.hpp"

namespace {

using namespace dqrm_mx;
using namespace dqrm_host;

__global__ __launch_bounds__(256) void zero_kernel(float *p, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

void fill_zero(float *p, int64_t n, hipStream_t st)
{
    if (p && n > 0) hipLaunchKernelGGL(zero_kernel, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, p, n);
}

void join_columns(const float *partial, int64_t stride, int n, int64_t cols, float *out0, float *out1, hipStream_t st)
{
    const int64_t step = kMaxBlocks * 16; // columns of a launch
    for (int64_t c0 = 0; c0 < cols; c0 += step) {
        const int64_t some = std::min(step, cols - c0);
        hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)ceil_div(some, 16), out1 ? 2 : 1), dim3(256), 0, st, partial + c0, stride, n, some, cols,
                           out0 + c0, out1 ? out1 + c0 : nullptr);
    }
}

// ---- quantisation ------------------------------------------------------------------------------------------------------
size_t quant_workspace(int64_t rows, int64_t cols) { return align_up((size_t)(ceil_div(rows, kTile) * cols) * sizeof(float), 256); }

void launch_quant_rows(int32_t dtype, QuantArgs a, hipStream_t st)
{
    const int64_t per_row = groups_of(a.cols) * (kRowPad / kChunk);
    const int64_t step = std::max<int64_t>(1, kMaxBlocks * 256 / per_row), rows = a.rows;
    const size_t es = size_of(dtype);
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
        QuantArgs b = a;
        b.rows = std::min(step, rows - r0);
        b.x = static_cast<const char *>(a.x) + r0 * a.ldx * es;
        if (a.gate) b.gate = static_cast<const char *>(a.gate) + r0 * a.ldgate * es;
        b.codes += r0 * codes_pitch(a.cols), b.scales += r0 * scales_pitch(a.cols);
        with_type(dtype, [&](auto t) {
            hipLaunchKernelGGL(quant_rows_kernel<decltype(t)::value>, dim3((unsigned)ceil_div(b.rows * per_row, 256)), dim3(256), 0, st, b,
                               dqrm::FastDiv::make((unsigned)per_row));
        });
    }
}

// ---- layer norm ----------------------------------------------------------------------------------------------------------
// Rows of 8 to 16384 values stay in registers; others are read more than once (shorter ones have no vector of 8).
bool norm_in_registers(int64_t cols) { return cols >= kChunk && cols <= 16384; }

// threads of such another row, a workgroup's; a launch takes as many rows as have 2^31 threads together
template <typename F>
void with_norm_long_block(int64_t cols, F f)
{
    cols < kChunk ? f(std::integral_constant<int, kWaveSize>{}) : f(std::integral_constant<int, 1024>{});
}

int64_t norm_long_rows(int64_t cols)
{
    int64_t rows = 0;
    with_norm_long_block(cols, [&](auto block) { rows = ((int64_t)1 << 31) / decltype(block)::value; });
    return rows;
}

// How a row that stays in registers is laid over threads: f(shape) for the narrowest one that holds it.
template <int TPR_, int CH_, int BLOCK_>
struct NormShape {
    static constexpr int TPR = TPR_, CH = CH_, BLOCK = BLOCK_, cols = TPR * CH * kChunk, rows = BLOCK / TPR;
};

template <typename... S, typename F>
void with_first_that_holds(int64_t cols, F f)
{
    (void)((cols <= S::cols ? (f(S{}), true) : false) || ...);
}

// 16-bit types with this many values: shapes of which a row leaves few threads without values.  Those have more chunks to a
// thread or more rows to a workgroup, whose latency few rows don't hide, and 32-bit rows have bytes enough.  Forward, the shapes below
// for many values and the others: 8000 x 8200 52 and 79 us, 32000 x 1200 31 and 49, 100000 x 300 30 and 38, 500 x 300 4.9 and 3.5; in float
// 32000 x 1200 62 and 50.
constexpr int64_t kNormMany = 1 << 22;

template <int DT, typename F>
void with_norm_fwd_shape(int64_t rows, int64_t cols, F f)
{
    if constexpr (DT != DQRM_F32) {
        if (rows * cols >= kNormMany)
            return with_first_that_holds<NormShape<16, 1, 256>, NormShape<16, 2, 256>, NormShape<16, 3, 256>, NormShape<64, 1, 256>, NormShape<64, 2, 256>,
                                         NormShape<64, 3, 256>, NormShape<128, 2, 256>, NormShape<128, 3, 256>, NormShape<256, 2, 256>,
                                         NormShape<256, 3, 256>, NormShape<512, 2, 512>, NormShape<512, 3, 512>, NormShape<1024, 2, 1024>>(cols, f);
    }
    // A row to a CU at most: its latency counts, which is less the more threads it has (from a graph, with codes: 16 x 700 bfloat16 3.4 us, with two
    // chunks to a thread 4.1; 200 x 2500 3.7 and 4.3; 16 x 6000 4.05 and 4.3)
    if (rows <= num_cus())
        return with_first_that_holds<NormShape<16, 1, 256>, NormShape<64, 1, 256>, NormShape<128, 1, 256>, NormShape<256, 1, 256>, NormShape<512, 1, 512>,
                                     NormShape<1024, 1, 1024>, NormShape<1024, 2, 1024>>(cols, f);
    with_first_that_holds<NormShape<16, 1, 256>, NormShape<64, 1, 256>, NormShape<64, 2, 256>, NormShape<256, 1, 256>, NormShape<256, 2, 256>,
                          NormShape<512, 2, 512>, NormShape<1024, 2, 1024>>(cols, f);
}

// (16001 x 8190 bfloat16: 512 threads with two chunks 141 us, 1024 with one 166; 64000 x 2047: 128 threads with two chunks 150 us, 256 with
// one 201; 8000 x 8200: 512 threads with three chunks 78 us, 1024 with two 126; 8000 x 16000: 512 with four, though some of the compiler's
// registers are in memory then, 153 us, 1024 with two, and the next row not ahead, 197.  The shapes for many values and the others: 16000 x
// 4100 79 and 106 us, 16000 x 1200 26 and 32, 4000 x 300 9.5 and 7.9; in float 16000 x 4100 168 and 156)
template <int DT, typename F>
void with_norm_bwd_shape(int64_t rows, int64_t cols, F f)
{
    if constexpr (DT != DQRM_F32) {
        if (rows * cols >= kNormMany)
            return with_first_that_holds<NormShape<16, 1, 1024>, NormShape<16, 2, 512>, NormShape<16, 3, 512>, NormShape<64, 1, 1024>, NormShape<64, 2, 512>,
                                         NormShape<64, 3, 512>, NormShape<128, 2, 512>, NormShape<128, 3, 512>, NormShape<256, 2, 512>,
                                         NormShape<256, 3, 512>, NormShape<512, 2, 512>, NormShape<512, 3, 512>, NormShape<512, 4, 512>>(cols, f);
    }
    with_first_that_holds<NormShape<16, 1, 1024>, NormShape<64, 1, 1024>, NormShape<64, 2, 512>, NormShape<128, 2, 512>, NormShape<256, 2, 512>,
                          NormShape<512, 2, 512>, NormShape<512, 3, 512>, NormShape<512, 4, 512>>(cols, f);
}

void launch_norm_fwd(int32_t dtype, const NormArgs &a, hipStream_t st)
{
    const bool in_registers = norm_in_registers(a.cols);
    const int64_t step = in_registers ? kMaxBlocks : norm_long_rows(a.cols);
    const size_t es = size_of(dtype);
    for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
        NormArgs b = a;
        b.rows = std::min(step, a.rows - r0);
        b.x = static_cast<const char *>(a.x) + r0 * a.ldx * es;
        if (a.y) b.y = static_cast<char *>(a.y) + r0 * a.ldy * es;
        if (a.mean) b.mean += r0;
        if (a.rstd) b.rstd += r0;
        if (a.codes) b.codes += r0 * codes_pitch(a.cols), b.scales += r0 * scales_pitch(a.cols);
        with_type(dtype, [&](auto t) {
            constexpr int DT = decltype(t)::value;
            if (!in_registers) {
                with_norm_long_block(a.cols, [&](auto block) {
                    constexpr int BLOCK = decltype(block)::value;
                    hipLaunchKernelGGL((norm_fwd_long_kernel<DT, BLOCK>), dim3((unsigned)b.rows), dim3(BLOCK), 0, st, b);
                });
                return;
            }
            with_norm_fwd_shape<DT>(a.rows, a.cols, [&](auto shape) {
                using S = decltype(shape);
                // as many workgroups as the chip holds: each keeps its columns' gain and offset for all of its rows
                const int64_t most = (int64_t)num_cus() * (4 * 4 * kWaveSize / S::BLOCK);
                hipLaunchKernelGGL((norm_fwd_kernel<DT, S::TPR, S::CH, S::BLOCK>), dim3((unsigned)std::min(ceil_div(b.rows, S::rows), most)), dim3(S::BLOCK),
                                   0, st, b);
            });
        });
    }
}

// Workgroups, each with a slice of the rows and a pair of partial sums of every column.  Where two would do, one takes their rows in
// turn and there is nothing to join (from a graph: 16 x 512 3.96 instead of 5.88 us, two turns of 32 x 512 5.07 and 5.91; four turns of
// 64 x 512 7.27 and 5.91).
constexpr int64_t kNormAlone = 2;

int norm_bwd_blocks(int32_t dtype, int64_t rows, int64_t cols)
{
    if (rows < 1 || cols < 1) return 0;
    // (a short row's columns are one thread's)
    if (!norm_in_registers(cols)) return (int)std::min<int64_t>(ceil_div(rows, 32), cols < kChunk ? 1024 : 64);
    int64_t n = 0;
    // (one to a CU: twice as many write and join twice the partial sums, 145 instead of 141 us for 16001 x 8190)
    with_type(dtype, [&](auto t) {
        with_norm_bwd_shape<decltype(t)::value>(rows, cols, [&](auto shape) { n = std::min<int64_t>(ceil_div(rows, decltype(shape)::rows), num_cus()); });
    });
    return n <= kNormAlone ? 1 : (int)n;
}

// (of any type)
size_t norm_bwd_workspace(int64_t rows, int64_t cols)
{
    const int blocks = std::max(norm_bwd_blocks(DQRM_F32, rows, cols), norm_bwd_blocks(DQRM_BF16, rows, cols));
    return align_up((size_t)blocks * 2 * (size_t)cols * sizeof(float), 256);
}

// ---- products --------------------------------------------------------------------------------------------------------------

using Tile256 = TileShape<4, 2, 2, 4, 2>;
using Tile128 = TileShape<2, 1, 2, 4, 4>;
using TilePair = TileShape<2, 2, 2, 2, 2>; // two to a CU
using Tile64 = TileShape<1, 1, 2, 2, 2>;

enum class Tiles { few, by64, by128, by128_pair, by256 }; // few: few_kernel

int side_of(Tiles t) { return t == Tiles::by256 ? 256 : t == Tiles::by64 ? 64 : 128; }

struct MatmulPlan {
    Tiles tiles;
    unsigned slices; // of k
    unsigned stages_per_slice;
};

// Few rows of A, and strips of W enough to keep the chip's memory busy or k short: W straight from memory.  Against tiles, of which
// k can be cut: 64 x 4096 x 8192 11.8 and 14.9 us, 64 x 8192 x 8192 16.6 and 19.6, 16 x 2048 x 2048 3.4 and 6.8, 16 x 512 x 32768 8.5 and 9.1;
// 16 x 512 x 65536 21.8 and 15.3, 64 x 256 x 16384 12.2 and 8.4, 64 x 4096 x 32768 31.2 and 27.4.  More than 32 rows are a fixed cost that
// a short k doesn't cover: 64 x 2048 x 512 3.9 and 3.2, 64 x 8192 x 512 5.7 and 3.8, 64 x 2048 x 2048 5.0 and 6.8.
bool is_few(int64_t m, int64_t n, int64_t k)
{
    if (m > 32) return m <= 64 && (n >= 4096 ? k > 1024 && k <= 16384 : k > 768 && k <= 8192);
    return n >= 4096 || k <= (m <= 16 ? 32768 : 8192);
}

// Time of a product's tiles, to choose among them: us, from how many of them there are to a CU and the stages of k that each has.
// Sides of 64: four workgroups to a CU.  128: two that have the least to read from LDS and hide each other's waits (by128_pair), or
// one whose loads are further ahead, for long sums of few tiles (by128).  256: one; the least to load of all.  Where
// workgroups don't fill the CUs the rest run faster (less to load, a higher clock).  The coefficients are from 112 products, m 100 to
// 65536, n 13 to 4096 and k 256 to 65536, each with every side and up to 12 numbers of slices: the plan that it takes is 0.8 % slower
// than the fastest one measured, geometric mean, 18 % at most.  64, 128, 128 in pairs and 256, best slices of each:
// 4096 x 2048 x 4096 39.8, 29.6, 23.9 and 27.3 us; 4096 x 4096 x 4096 77.8, 58.0, 46.0 and 39.2; 8192 x 512 x 16384 91.6, 56.1, 69.1 and
// 69.1; without pairs 1024 x 1024 x 1024 5.1, 6.5 and 10.1; 1024 x 1024 x 16384 26.9 (3 slices), 24.1 (3) and 31.4 (10).
double matmul_us(Tiles shape, double per_cu, double stages)
{
    const double rounds = std::ceil(per_cu), part = std::min(per_cu, 1.0);
    switch (shape) {
    case Tiles::by128: return 1.57 + 2.94 * rounds + stages * (per_cu > 1 ? 0.72 * rounds : 0.72 * part + 0.50 * (1 - part));
    case Tiles::by128_pair:
        return 2.35 + 1.12 * per_cu +
               stages * (per_cu > 2 ? 1.20 * std::ceil(per_cu / 2) : per_cu > 1 ? 0.98 + 0.22 * (per_cu - 1) : 0.98 * part + 0.85 * (1 - part));
    case Tiles::by256: return 8.72 + 0.21 * rounds + stages * (per_cu > 1 ? 1.77 * rounds : 1.77 * part + 1.06 * (1 - part));
    default: return 2.11 + 0.55 * per_cu + stages * std::max(0.60, 0.28 * per_cu);
    }
}

MatmulPlan matmul_plan(int64_t m, int64_t n, int64_t k)
{
    if (is_few(m, n, k)) return MatmulPlan{Tiles::few, 1, 0};
    const int64_t cus = num_cus(), stages = std::max<int64_t>(1, ceil_div(groups_of(k), 2));
    MatmulPlan best{};
    double least = 0;
    for (Tiles shape : {Tiles::by64, Tiles::by128, Tiles::by128_pair, Tiles::by256})
        for (int slices : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32}) {
            const int64_t side = side_of(shape), tiles = std::max<int64_t>(1, ceil_div(m, side) * ceil_div(n, side));
            if ((side < 256 && tiles > kMaxBlocks) || (slices > 1 && (tiles * slices > 4 * cus || stages < 2 * slices))) break;
            MatmulPlan p{shape, 1, (unsigned)stages};
            if (slices > 1) {
                p.stages_per_slice = (unsigned)ceil_div(ceil_div(stages, slices), 2) * 2; // (a slice begins with a pair of stages' scales)
                p.slices = (unsigned)ceil_div(stages, p.stages_per_slice);
            }
            double us = matmul_us(shape, (double)(tiles * p.slices) / (double)cus, p.stages_per_slice);
            if (p.slices > 1) us += 3.3 + 0.46e-6 * sizeof(float) * p.slices * (double)m * (double)n; // partial sums: another launch, their bytes
            if (best.slices == 0 || us < least) best = p, least = us;
        }
    return best;
}

size_t matmul_workspace(int64_t m, int64_t n, int64_t k)
{
    const MatmulPlan p = matmul_plan(m, n, k);
    return p.slices > 1 ? align_up((size_t)p.slices * (size_t)m * (size_t)n * sizeof(float), 256) : 0;
}

// ... for any number of rows up to m.  Fewer rows may need more, where their tiles are so few that k is cut.  Within a run of rows that
// all sides of tiles see alike the estimates grow by the partial sums alone, so more rows have the plan of the first one or one with fewer
// slices: its slices for the run's last row are enough for the run.  (Some microseconds; 0.23 ms for 200000 rows and n = 100.)
size_t matmul_workspace_up_to(int64_t m, int64_t n, int64_t k)
{
    size_t most = 0;
    for (int64_t first = 1, last = 16; first <= m; first = last + 1, last = last < 64 ? last * 2 : last + 64) {
        if (ceil_div(first, 256) * ceil_div(n, 256) * 2 > 4 * num_cus()) break; // not cut any more
        const MatmulPlan p = matmul_plan(first, n, k);
        if (p.slices > 1) most = std::max(most, (size_t)p.slices * (size_t)std::min(last, m) * (size_t)n * sizeof(float));
    }
    return align_up(most, 256);
}

template <typename T>
void launch_tiles(const MatmulPlan &p, MatmulArgs g, hipStream_t st)
{
    const auto go = [&](auto shape) {
        using S = decltype(shape);
        g.tiles_m = (unsigned)ceil_div(g.m, S::BM), g.tiles_n = (unsigned)ceil_div(g.n, S::BN);
        hipLaunchKernelGGL((matmul_kernel<T, S>), dim3(g.tiles_m * g.tiles_n * g.slices), dim3(S::waves * kWaveSize), 0, st, g);
    };
    switch (p.tiles) {
    case Tiles::by256: return go(Tile256{});
    case Tiles::by128: return go(Tile128{});
    case Tiles::by128_pair: return go(TilePair{});
    default: return go(Tile64{});
    }
}

constexpr int64_t kMaxInner = 1 << 24; // a tile's rows of codes are addressed with 32 bits

// Whether a product of this shape can be launched: asked before anything is.  (Where tiles of 128 or 64 are too many, the plan has none.)
int32_t check_product(int64_t m, int64_t n, int64_t k)
{
    if (k > kMaxInner) return DQRM_ERR_UNSUPPORTED;
    return is_few(m, n, k) || ceil_div(m, 256) * ceil_div(n, 256) <= kMaxBlocks ? DQRM_OK : DQRM_ERR_UNSUPPORTED;
}

template <int DT, FewSource SRC, int MT>
void launch_few(const FewArgs &a, hipStream_t st)
{
    const int64_t strips = ceil_div(a.g.n, 16);
    const size_t lds = SRC == kFewCodes ? 0 : (size_t)(a.g.m * (codes_pitch(a.g.k) + scales_pitch(a.g.k)));
    const auto go = [&](auto st_, auto ring) {
        constexpr int ST = decltype(st_)::value, RING = decltype(ring)::value;
        for (int64_t n0 = 0; n0 < a.g.n; n0 += kMaxBlocks * 16) { // (W's rows of one launch)
            FewArgs b = a;
            b.g.n = std::min(kMaxBlocks * 16, a.g.n - n0);
            b.g.b_codes += n0 * codes_pitch(a.g.k), b.g.b_scales += n0 * scales_pitch(a.g.k);
            b.g.c = static_cast<elem_t<DT> *>(a.g.c) + n0;
            if (a.g.bias) b.g.bias += n0;
            hipLaunchKernelGGL((few_kernel<DT, SRC, MT, ST, RING>), dim3((unsigned)ceil_div(b.g.n, 16 * ST)), dim3(kFewBlock), lds, st, b);
        }
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    // Two strips to a workgroup where there are many, so that A is read half as often (16 rows, 32768 x 2048: 15.1 -> 10.7 us; 64
    // rows, 8192 x 8192: 21 -> 16 us), one strip where there are fewer (16 rows, 4096 x 4096: 5.0 -> 4.2 us).  A second unit in flight
    // pays where a workgroup's LDS is small (16 rows, 8192 x 8192: 12.0 -> 11.6 us; 32 rows: 13.7 -> 15.7 us).
    if (strips >= num_cus() * (MT > 2 ? 2 : 4))
        go(two, one);
    else if constexpr (MT == 1)
        go(one, two);
    else
        go(one, one);
}

int32_t launch_matmul(int32_t dtype, MatmulArgs g, void *workspace, hipStream_t st)
{
    const MatmulPlan p = matmul_plan(g.m, g.n, g.k);
    if (p.tiles == Tiles::few) {
        FewArgs a{};
        a.g = g;
        with_type(dtype, [&](auto t) {
            constexpr int DT = decltype(t)::value;
            if (g.m <= 16)
                launch_few<DT, kFewCodes, 1>(a, st);
            else if (g.m <= 32)
                launch_few<DT, kFewCodes, 2>(a, st);
            else
                launch_few<DT, kFewCodes, 4>(a, st);
        });
        DQRM_HIP_CHECK(hipGetLastError());
        return DQRM_OK;
    }
    g.slices = p.slices, g.stages_per_slice = p.stages_per_slice;
    if (p.slices > 1) {
        MatmulArgs part = g;
        part.c = workspace;
        launch_tiles<float>(p, part, st);
        const unsigned blocks = (unsigned)ceil_div(g.m * g.n, 256);
        with_type(dtype, [&](auto t) {
            hipLaunchKernelGGL(matmul_join_kernel<decltype(t)::value>, dim3(blocks), dim3(256), 0, st, static_cast<const float *>(workspace), g);
        });
    } else {
        with_type(dtype, [&](auto t) { launch_tiles<elem_t<decltype(t)::value>>(p, g, st); });
    }
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

// Whether the product quantises the activations itself, every workgroup all of them: saves a launch where they are few (with a norm,
// from a graph, against two launches: 1 x 367 for 512 outputs 5.3 and 5.8 us, 1 x 8192 for 8192 14.7 and 15.2, 2 x 4096 for 4096 8.4 and
// 8.4; 4 x 4096 11.0 and 8.6).
bool linear_in_one(int64_t m, int64_t n, int64_t k)
{
    const int64_t waves = m <= 1 ? 4 : m <= 2 ? 2 : 1;
    return m <= kFewRows && m * k <= 8192 && k >= kChunk && k <= waves * kWaveSize * kFewChunks * kChunk && is_few(m, n, k);
}

struct LinearWs {
    size_t scales, matmul, total;
};

LinearWs linear_ws(int64_t m, int64_t k, size_t matmul)
{
    LinearWs w;
    w.scales = align_up((size_t)(m * codes_pitch(k)), 256);
    w.matmul = w.scales + align_up((size_t)(m * scales_pitch(k)), 256);
    w.total = w.matmul + matmul;
    return w;
}

} // namespace

extern "C" {

size_t dqrm_mxfp4_quant_workspace_bytes(int64_t rows, int64_t cols)
{
    return check_shape(DQRM_F32, rows, cols) == DQRM_OK ? quant_workspace(rows, cols) : 0;
}

int32_t dqrm_mxfp4_quant(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, const void *gate, int64_t ldgate,
                         const dqrm_mxfp4_t *by_rows, const dqrm_mxfp4_t *by_cols, float *col_sums, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    DQRM_CHECK(check_shape(dtype, rows, cols));
    if (!by_rows && !by_cols && !col_sums && rows > 0 && cols > 0) return DQRM_ERR_INVALID_ARG; // (an empty output may be null)
    DQRM_CHECK(check_matrix(x, ldx, dtype, rows, cols));
    if (gate) DQRM_CHECK(check_matrix(gate, ldgate, dtype, rows, cols));
    if (by_rows) DQRM_CHECK(check_mx(by_rows, rows, cols));
    if (by_cols) DQRM_CHECK(check_mx(by_cols, cols, rows));
    if (col_sums && !aligned(col_sums, 4)) return DQRM_ERR_INVALID_ARG;
    if (col_sums) DQRM_CHECK(check_workspace(workspace, workspace_bytes, quant_workspace(rows, cols)));
    const int64_t row_tiles = ceil_div(rows, kTile), col_tiles = ceil_div(cols, kTile);
    const bool tiles = by_cols || col_sums;
    if (tiles && row_tiles * col_tiles > 2 * kMaxBlocks) return DQRM_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows == 0 || cols == 0) {
        fill_zero(col_sums, cols, st);
        DQRM_HIP_CHECK(hipGetLastError());
        return DQRM_OK;
    }
    QuantArgs a{};
    a.x = x, a.gate = gate, a.ldx = ldx, a.ldgate = ldgate, a.rows = rows, a.cols = cols;
    if (by_rows) a.codes = by_rows->codes, a.scales = by_rows->scales;
    if (by_cols) a.codes_t = by_cols->codes, a.scales_t = by_cols->scales;
    // (one row of tiles has the columns' sums themselves)
    a.partial = !col_sums ? nullptr : row_tiles > 1 ? static_cast<float *>(workspace) : col_sums;
    a.col_tiles = (unsigned)col_tiles;
    if (!tiles) {
        launch_quant_rows(dtype, a, st);
    } else {
        with_type(dtype, [&](auto t) {
            hipLaunchKernelGGL(quant_tile_kernel<decltype(t)::value>, dim3((unsigned)(row_tiles * col_tiles)), dim3(256), 0, st, a);
        });
        if (col_sums && row_tiles > 1) join_columns(a.partial, cols, (int)row_tiles, cols, col_sums, nullptr, st);
    }
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

int32_t dqrm_mxfp4_dequant(const dqrm_mxfp4_t *q, int32_t dtype, void *out, int64_t ldo, void *stream)
{
    if (!q) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_shape(dtype, q->rows, q->cols));
    DQRM_CHECK(check_mx(q, q->rows, q->cols));
    DQRM_CHECK(check_matrix(out, ldo, dtype, q->rows, q->cols));
    if (q->rows == 0 || q->cols == 0) return DQRM_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t per_row = ceil_div(q->cols, kChunk), step = std::max<int64_t>(1, kMaxBlocks * 256 / per_row);
    for (int64_t r0 = 0; r0 < q->rows; r0 += step) {
        const int64_t rows = std::min(step, q->rows - r0);
        with_type(dtype, [&](auto t) {
            hipLaunchKernelGGL(dequant_kernel<decltype(t)::value>, dim3((unsigned)ceil_div(rows * per_row, 256)), dim3(256), 0, st,
                               q->codes + r0 * codes_pitch(q->cols), q->scales + r0 * scales_pitch(q->cols), rows, q->cols,
                               static_cast<char *>(out) + r0 * ldo * size_of(dtype), ldo, dqrm::FastDiv::make((unsigned)per_row));
        });
    }
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

size_t dqrm_mxfp4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (check_shape(DQRM_F32, m, n) != DQRM_OK || check_shape(DQRM_F32, m, k) != DQRM_OK) return 0;
    return matmul_workspace_up_to(m, n, k);
}

int32_t dqrm_mxfp4_matmul(const dqrm_mxfp4_t *a, const dqrm_mxfp4_t *b, const float *bias, int32_t relu, int32_t dtype, void *out,
                          int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a || !b || a->cols != b->cols) return DQRM_ERR_INVALID_ARG;
    const int64_t m = a->rows, n = b->rows, k = a->cols;
    DQRM_CHECK(check_shape(dtype, m, n));
    DQRM_CHECK(check_shape(dtype, m, k));
    DQRM_CHECK(check_mx(a, m, k));
    DQRM_CHECK(check_mx(b, n, k));
    if (bias && !aligned(bias, 4)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_matrix(out, ldo, dtype, m, n));
    DQRM_CHECK(check_workspace(workspace, workspace_bytes, matmul_workspace(m, n, k)));
    DQRM_CHECK(check_product(m, n, k));
    if (m == 0 || n == 0) return DQRM_OK;
    const MatmulArgs g{a->codes, a->scales, b->codes, b->scales, m, n, k, bias, relu != 0, out, ldo};
    return launch_matmul(dtype, g, workspace, static_cast<hipStream_t>(stream));
}

size_t dqrm_mxfp4_linear_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (check_shape(DQRM_F32, m, n) != DQRM_OK || check_shape(DQRM_F32, m, k) != DQRM_OK) return 0;
    return linear_ws(m, k, matmul_workspace_up_to(m, n, k)).total;
}

int32_t dqrm_mxfp4_linear(int32_t dtype, int64_t m, const void *x, int64_t ldx, int32_t norm, const float *gamma, const float *beta,
                          float eps, const dqrm_mxfp4_t *w, const float *bias, int32_t relu, void *out, int64_t ldo, void *workspace,
                          size_t workspace_bytes, void *stream)
{
    if (!w) return DQRM_ERR_INVALID_ARG;
    const int64_t n = w->rows, k = w->cols;
    DQRM_CHECK(check_shape(dtype, m, n));
    DQRM_CHECK(check_shape(dtype, m, k));
    DQRM_CHECK(check_matrix(x, ldx, dtype, m, k));
    DQRM_CHECK(check_mx(w, n, k));
    if ((gamma && !aligned(gamma, 4)) || (beta && !aligned(beta, 4)) || (bias && !aligned(bias, 4))) return DQRM_ERR_INVALID_ARG;
    if (!norm && (gamma || beta)) return DQRM_ERR_INVALID_ARG;
    if (norm && !(eps >= 0.0f)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_matrix(out, ldo, dtype, m, n));
    const LinearWs L = linear_ws(m, k, matmul_workspace(m, n, k));
    DQRM_CHECK(check_workspace(workspace, workspace_bytes, L.total));
    DQRM_CHECK(check_product(m, n, k));
    if (m == 0 || n == 0) return DQRM_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    uint8_t *codes = ws, *scales = ws + L.scales;
    if (linear_in_one(m, n, k)) {
        FewArgs a{};
        a.g = MatmulArgs{nullptr, nullptr, w->codes, w->scales, m, n, k, bias, relu != 0, out, ldo};
        a.x.x = x, a.x.ldx = ldx, a.x.rows = m, a.x.cols = k, a.x.gamma = gamma, a.x.beta = beta, a.x.eps = eps;
        with_type(dtype, [&](auto t) {
            constexpr int DT = decltype(t)::value;
            if (norm)
                launch_few<DT, kFewNorm, 1>(a, st);
            else
                launch_few<DT, kFewPlain, 1>(a, st);
        });
        DQRM_HIP_CHECK(hipGetLastError());
        return DQRM_OK;
    }
    if (k > 0) {
        if (norm) {
            NormArgs a{};
            a.x = x, a.ldx = ldx, a.rows = m, a.cols = k, a.gamma = gamma, a.beta = beta, a.eps = eps, a.codes = codes, a.scales = scales;
            launch_norm_fwd(dtype, a, st);
        } else {
            QuantArgs a{};
            a.x = x, a.ldx = ldx, a.rows = m, a.cols = k, a.codes = codes, a.scales = scales;
            launch_quant_rows(dtype, a, st);
        }
    }
    const MatmulArgs g{codes, scales, w->codes, w->scales, m, n, k, bias, relu != 0, out, ldo};
    return launch_matmul(dtype, g, ws + L.matmul, st);
}

int32_t dqrm_layernorm_fwd(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, const float *gamma, const float *beta,
                           float eps, void *y, int64_t ldy, float *mean, float *rstd, const dqrm_mxfp4_t *q, void *stream)
{
    DQRM_CHECK(check_shape(dtype, rows, cols));
    if (cols < 1 || !(eps >= 0.0f)) return DQRM_ERR_INVALID_ARG;
    if (!y && !mean && !rstd && !q && rows > 0) return DQRM_ERR_INVALID_ARG; // (an empty output may be null)
    DQRM_CHECK(check_matrix(x, ldx, dtype, rows, cols));
    if (y) DQRM_CHECK(check_matrix(y, ldy, dtype, rows, cols));
    if (q) DQRM_CHECK(check_mx(q, rows, cols));
    for (const float *p : {gamma, beta, (const float *)mean, (const float *)rstd})
        if (p && !aligned(p, 4)) return DQRM_ERR_INVALID_ARG;
    if (rows == 0) return DQRM_OK;
    NormArgs a{};
    a.x = x, a.ldx = ldx, a.rows = rows, a.cols = cols, a.gamma = gamma, a.beta = beta, a.eps = eps;
    a.y = y, a.ldy = ldy, a.mean = mean, a.rstd = rstd;
    if (q) a.codes = q->codes, a.scales = q->scales;
    launch_norm_fwd(dtype, a, static_cast<hipStream_t>(stream));
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

size_t dqrm_layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols)
{
    return check_shape(DQRM_F32, rows, cols) == DQRM_OK ? norm_bwd_workspace(rows, cols) : 0;
}

int32_t dqrm_layernorm_bwd(int32_t dtype, int64_t rows, int64_t cols, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                           const float *mean, const float *rstd, const float *gamma, void *dx, int64_t lddx, float *dgamma,
                           float *dbeta, void *workspace, size_t workspace_bytes, void *stream)
{
    DQRM_CHECK(check_shape(dtype, rows, cols));
    if (cols < 1 || (!dgamma) != (!dbeta) || (!dx && !dgamma && rows > 0)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_matrix(dy, lddy, dtype, rows, cols));
    DQRM_CHECK(check_matrix(x, ldx, dtype, rows, cols));
    if (dx) DQRM_CHECK(check_matrix(dx, lddx, dtype, rows, cols));
    if (rows > 0 && (!mean || !rstd)) return DQRM_ERR_INVALID_ARG;
    for (const float *p : {mean, rstd, gamma, (const float *)dgamma, (const float *)dbeta})
        if (p && !aligned(p, 4)) return DQRM_ERR_INVALID_ARG;
    if (dgamma) DQRM_CHECK(check_workspace(workspace, workspace_bytes, norm_bwd_workspace(rows, cols)));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows == 0) {
        fill_zero(dgamma, cols, st);
        fill_zero(dbeta, cols, st);
        DQRM_HIP_CHECK(hipGetLastError());
        return DQRM_OK;
    }
    const int blocks = norm_bwd_blocks(dtype, rows, cols);
    float *partial = static_cast<float *>(workspace);
    NormBwdArgs a{dy, x, lddy, ldx, rows, cols, mean, rstd, gamma, dx, lddx, nullptr, nullptr, 0};
    if (dgamma && blocks > 1)
        a.sum_gamma = partial, a.sum_beta = partial + cols, a.block_stride = 2 * cols;
    else if (dgamma)
        a.sum_gamma = dgamma, a.sum_beta = dbeta;
    with_type(dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (norm_in_registers(cols)) {
            with_norm_bwd_shape<DT>(rows, cols, [&](auto shape) {
                using S = decltype(shape);
                hipLaunchKernelGGL((norm_bwd_kernel<DT, S::TPR, S::CH, S::BLOCK>), dim3((unsigned)blocks), dim3(S::BLOCK), 0, st, a);
            });
            return;
        }
        // (the columns' sums first: dx may be dy's or x's own memory)
        if (dgamma) {
            const dim3 grid((unsigned)ceil_div(cols, 256 * kChunk), (unsigned)blocks);
            if (cols < kChunk)
                hipLaunchKernelGGL((norm_bwd_columns_kernel<DT, true>), grid, dim3(256), 0, st, a, ceil_div(rows, blocks));
            else
                hipLaunchKernelGGL((norm_bwd_columns_kernel<DT, false>), grid, dim3(256), 0, st, a, ceil_div(rows, blocks));
        }
        const size_t es = size_of(dtype);
        const int64_t step = norm_long_rows(cols);
        for (int64_t r0 = 0; dx && r0 < rows; r0 += step) {
            NormBwdArgs b = a;
            b.rows = std::min(step, rows - r0);
            b.dy = static_cast<const char *>(dy) + r0 * lddy * es, b.x = static_cast<const char *>(x) + r0 * ldx * es;
            b.dx = static_cast<char *>(dx) + r0 * lddx * es, b.mean = mean + r0, b.rstd = rstd + r0;
            with_norm_long_block(cols, [&](auto block) {
                constexpr int BLOCK = decltype(block)::value;
                hipLaunchKernelGGL((norm_bwd_long_kernel<DT, BLOCK>), dim3((unsigned)b.rows), dim3(BLOCK), 0, st, b);
            });
        }
    });
    if (dgamma && blocks > 1) join_columns(partial, 2 * cols, blocks, cols, dgamma, dbeta, st);
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

} // extern "C"
