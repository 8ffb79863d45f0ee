// C ABI of the softmax cross entropy over many classes: host-side validation and kernel dispatch.
// Every entry point validates on the host first and enqueues nothing on error.
#include "dqrm_checks.hpp"
#include "dqrm_xent.hpp"
#include "dqrm_xent_narrow.hpp"

namespace {

using namespace dqrm_host;
using namespace dqrm_xent;

constexpr int64_t kMostTiles = 1 << 22;  // of 256 by 256, of any of the products
constexpr int64_t kMostStride = 1 << 22; // values: a tile's offsets stay below 2^32 bytes
constexpr int64_t kMostClasses = 1 << 22; // of a piece, for the same reason
// What a piece of the classes may take of the workspace: its gradients d, and its rows of w where they are laid out anew.  Smaller pieces stay in the
// chip's last-level cache, larger ones are fewer sums to add up, but all of it is the caller's memory (64, 256, 512 and 1024 MB, forward and backward:
// 8192 rows, 131072 classes, width 4096, bf16 32.1, 30.4, 29.8 and 29.3 ms; 200003 classes, width 256, 256, 512 and 1024 MB: fp32 24.0, 22.2 and
// 20.9, bf16 6.5, 6.1 and 5.9).
constexpr int64_t kPieceBytes = 512LL << 20;
constexpr int kMostSlices = 64;
constexpr int64_t kFewBlocks = 1024;  // workgroups that share the classes where there are a few rows
constexpr int64_t kRowsAlone = 16384; // rows that one workgroup looks through for the gradients' unit
constexpr int64_t kSliceTiles = 512; // tiles times slices

using TileBig = Tile<4, 4, 2, 2, 2>; // 256 by 256, one to a CU
using TileMid = Tile<2, 2, 2, 2, 2>; // 128 by 128, two to a CU
using TileFew = Tile<2, 2, 1, 4, 2, true>; // 64 by 256: few rows

enum class Shape { big, mid, few };

int64_t up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }
int planes_of(int32_t dtype) { return dtype == DQRM_F32 ? 3 : 1; }
int pairs_of(int32_t dtype) { return dtype == DQRM_F32 ? (int)kPlanePairs : 1; }
int rows_of(Shape s) { return s == Shape::mid ? 128 : s == Shape::few ? 64 : 256; }
int cols_of(Shape s) { return s == Shape::mid ? 128 : 256; }
int per_cu(Shape s) { return s == Shape::big ? 1 : 2; }

template <typename F>
void with_shape(Shape s, F f)
{
    if (s == Shape::big)
        f(TileBig{});
    else if (s == Shape::mid)
        f(TileMid{});
    else
        f(TileFew{});
}

// bfloat16 also stands for fp32's planes
template <typename F>
void with_operands(int32_t dtype, F f)
{
    if (dtype == DQRM_F16)
        f((_Float16)0.0f);
    else
        f((__bf16)0.0f);
}

// Sums of few stages: two smaller tiles to a CU, of which one's exponentials and stores go beside the other's products (8192 rows, 200003 classes
// in bf16: forward and backward, width 128 4.9 ms with tiles of 256, 4.5 so, width 256 6.4 and 6.1; from 16 stages on no difference).
constexpr int64_t kShortSum = 8;

// (a launch has fewer than 2^32 threads, 256 to a tile: of the largest products' tiles of 256 there are up to kMostTiles, of 128 four times as many)
bool is_short(int64_t m, int64_t n, int64_t stages)
{
    return stages <= kShortSum && ceil_div(m, rows_of(Shape::mid)) * ceil_div(n, cols_of(Shape::mid)) < (int64_t)1 << 24;
}

Shape logits_shape(int64_t m, int64_t n, int64_t stages)
{
    if (m <= 64) return Shape::few;
    if (is_short(m, n, stages)) return Shape::mid;
    return ceil_div(m, 256) * ceil_div(n, 256) >= num_cus() ? Shape::big : Shape::mid;
}

// a gradient's product [m][n]
Shape out_shape(int64_t m, int64_t n, int64_t stages)
{
    if (m <= 64) return Shape::few;
    if (is_short(m, n, stages)) return Shape::mid; // (131072 classes, width 2048, 64 rows, bf16: forward and backward 563 us, with tiles of 256 580)
    return m > 128 && n > 128 ? Shape::big : Shape::mid;
}

struct Sliced {
    Shape shape;
    unsigned slices, stages_per_slice;
};

// few tiles: the sum in slices, joined afterwards
Sliced out_plan(int64_t m, int64_t n, int64_t stages)
{
    Sliced p{out_shape(m, n, stages), 1, (unsigned)std::max<int64_t>(stages, 1)};
    const int64_t tiles = ceil_div(m, rows_of(p.shape)) * ceil_div(n, cols_of(p.shape));
    const int64_t room = (int64_t)num_cus() * per_cu(p.shape);
    if (tiles < 1 || tiles * 2 > room) return p;
    const int64_t slices = std::min<int64_t>({room / tiles, ceil_div(stages, 4), kMostSlices, kSliceTiles / tiles});
    if (slices < 2) return p;
    p.stages_per_slice = (unsigned)ceil_div(stages, slices);
    p.slices = (unsigned)ceil_div(stages, p.stages_per_slice);
    return p;
}

int64_t slices_room(int64_t m, int64_t n, int64_t stages)
{
    return std::min(kSliceTiles * 256 * 256, m * n * std::min<int64_t>(kMostSlices, ceil_div(stages, 4))) * (int64_t)sizeof(float);
}

// classes of a piece, a multiple of 256
int64_t most_classes(int64_t classes, int64_t width, int planes)
{
    const int64_t fit = kPieceBytes / (std::max<int64_t>(up(width, kDepth), kDepth) * 2 * planes);
    return std::min(up(std::max<int64_t>(classes, 1), 256), std::max<int64_t>(256, std::min(fit, kMostClasses) / 256 * 256));
}

int64_t piece_classes(int64_t rows, int64_t classes, int64_t width, int planes, bool with_d)
{
    int64_t most = most_classes(classes, width, planes);
    if (with_d) most = std::min(most, std::max<int64_t>(256, kPieceBytes / (std::max<int64_t>(up(rows, kBlock), 1) * 2 * planes) / 256 * 256));
    return up(ceil_div(classes, ceil_div(classes, most)), 256);
}

size_t bytes(int64_t n) { return align_up((size_t)n, 256); }

// Widths up to 64, more than 64 rows: without d.  Workgroups of 128 rows of x or w, slices of the others.  (Forward and backward, with the tiles of
// the other widths and so: 8192 rows, 200003 classes, width 64 in fp32 10.3 and 5.1 ms, in bf16 4.0 and 1.75; 8192 x 1000 x 64 in fp32 110 and
// 89 us; 100 x 1000000 x 16 in fp32 1976 and 666.  In bf16 64 rows of 200003 classes took 102 and 128 us: up to 64 rows the other kernels are used.)
constexpr int64_t kNarrowSums = 256LL << 20; // bytes of their sums, if a slice is less
constexpr int64_t kNarrowSlices = 256;
bool is_narrow(int64_t m, int64_t k) { return m > 64 && k > 0 && k <= kDepth; }
int64_t most_narrow_slices(int64_t rows, int64_t k) { return std::max<int64_t>(1, std::min<int64_t>(kNarrowSlices, kNarrowSums / (up(rows, 128) * k * 4))); }

// the slices with which the last workgroup ends first, each with some stages' time before and after its own (three workgroups to a CU)
Sliced narrow_plan(int64_t rows, int64_t others, int64_t k)
{
    const int64_t tiles = ceil_div(rows, 128), stages = ceil_div(others, 64), room = num_cus() * 3;
    Sliced p{Shape::mid, 1, (unsigned)stages};
    const int64_t most = std::min(most_narrow_slices(rows, k), ceil_div(stages, 2));
    int64_t least = std::numeric_limits<int64_t>::max();
    for (int64_t n = 1, each; n <= most; n = each > 1 ? ceil_div(stages, each - 1) : most + 1) { // (the fewest slices of each length)
        each = ceil_div(stages, n);
        const int64_t time = ceil_div(tiles * n, room) * (each + 4) + n / 32;
        if (time < least) least = time, p.stages_per_slice = (unsigned)each, p.slices = (unsigned)ceil_div(stages, each);
    }
    return p;
}
size_t narrow_sums(int64_t rows, int64_t others, int64_t k) { return (size_t)narrow_plan(rows, others, k).slices * (size_t)(rows * k * 4); }
// ... and the most that any plan for so many rows or fewer takes, without a look at them
size_t most_narrow_sums(int64_t rows, int64_t k) { return std::max(rows * k * 4, std::min(kNarrowSums, kNarrowSlices * rows * k * 4)); }

// Few tiles of long sums: in slices, joined by what follows.  (Forward and backward, in one piece by tiles or strips and so: 233 rows, 27 classes, width
// 5541 in fp32 504 and 96 us, bf16 128 and 65; 1024 x 1024 x 8192 945 and 521, 235 and 185; 300 x 300 x 384 in fp32 109 and 94; but 64 x 16000 x
// 2048 in fp32, 63 tiles of few rows, 326 and 376.)
constexpr int64_t kSumsTiles = 64, kSumsTilesOfFew = 32, kSumsStages = 32;
Sliced sums_plan(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    const int64_t stages = ceil_div(k, kDepth) * pairs_of(dtype);
    Sliced p{m <= 64 ? Shape::few : Shape::mid, 1, (unsigned)std::max<int64_t>(stages, 1)};
    const int64_t tiles = ceil_div(m, rows_of(p.shape)) * ceil_div(v, cols_of(p.shape));
    if (tiles < 1 || tiles > (p.shape == Shape::few ? kSumsTilesOfFew : kSumsTiles) || stages < kSumsStages || piece_classes(m, v, k, planes_of(dtype), true) < v) return p;
    const int64_t slices = std::min<int64_t>({kSliceTiles / tiles, ceil_div(stages, 4), kMostSlices});
    p.stages_per_slice = (unsigned)ceil_div(stages, slices), p.slices = (unsigned)ceil_div(stages, p.stages_per_slice);
    return p;
}
size_t sums_space(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    const Sliced p = sums_plan(m, v, k, dtype);
    return p.slices > 1 ? bytes(p.slices * m * v * 4) : 0;
}
// ... the most that any number of rows up to m takes: there are fewer slices the more tiles there are, so it is one that fills its tiles
size_t most_sums_space(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    if (ceil_div(k, kDepth) * pairs_of(dtype) < kSumsStages) return 0;
    size_t most = 0;
    for (int64_t rows = std::min<int64_t>(m, 64);; rows = std::min(m, up(rows + 1, 128))) {
        most = std::max(most, sums_space(rows, v, k, dtype));
        if (rows == m || rows > kSumsTiles * 128) return most;
    }
}

// the regions of the workspace
struct Space {
    char *at;
    size_t used = 0;
    void *take(size_t n)
    {
        void *p = at + used;
        used += n;
        return p;
    }
};

// rows of x laid out anew: as an operand of the tiles, or up to 64 of them by the steps of the strips' products (32 or 64 rows then)
size_t x_space(int64_t m, int64_t k, int32_t dtype)
{
    return bytes(std::max<int64_t>(m, m <= 32 ? 32 : 64) * up(std::max<int64_t>(k, 1), kDepth) * 2 * planes_of(dtype));
}

struct FwdSpace {
    size_t parts, at, x, w, logits;
    size_t total() const { return parts + at + x + w + logits; }
};

FwdSpace fwd_space(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    const int pl = planes_of(dtype);
    FwdSpace s{};
    s.parts = bytes(std::max(ceil_div(v, 128), std::min(v, kFewBlocks)) * m * 8); // (of the narrowest tiles, and of few rows' workgroups)
    s.at = bytes(m * 4);
    s.x = x_space(m, k, dtype);
    s.w = bytes(most_classes(v, k, pl) * up(k, kDepth) * 2 * pl);
    s.logits = sums_space(m, v, k, dtype);
    return s;
}

// widths up to 64: classes of the pieces
struct NarrowPieces {
    int64_t whole, last;
};
NarrowPieces narrow_pieces(int64_t m, int64_t v, int64_t k, int planes)
{
    const int64_t step = v > 0 ? piece_classes(m, v, k, planes, false) : 1;
    return {std::min(step, v), v > 0 ? v - (v - 1) / step * step : 0};
}

struct BwdSpace {
    size_t live, classes, most, unit, x, strip, w, logits, d, sums, dx, dw;
    size_t total() const { return live + classes + most + unit + x + strip + w + logits + d + sums + dx + dw; }
};

BwdSpace bwd_space(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    const int pl = planes_of(dtype), pairs = pairs_of(dtype);
    const int64_t most = most_classes(v, k, pl);
    // (a piece has at most `most` classes, and at most 256 or those whose d fits)
    const int64_t rows = up(m, kBlock), d = std::max(rows * 256, std::min(rows * most, kPieceBytes / (2 * pl)));
    BwdSpace s{};
    s.live = bytes(ceil_div(m, 64) * 8), s.classes = bytes(ceil_div(v, 64) * 8), s.most = 1024, s.unit = 256;
    s.x = x_space(m, k, dtype), s.strip = m <= 64 ? s.x : x_space(64, k, dtype), s.w = bytes(most * up(k, kDepth) * 2 * pl);
    s.logits = sums_space(m, v, k, dtype);
    if (is_narrow(m, k)) {
        const NarrowPieces p = narrow_pieces(m, v, k, pl);
        const size_t dw = std::max(narrow_sums(p.whole, m, k), narrow_sums(p.last, m, k));
        s.dx = bytes(narrow_sums(m, p.whole, k)), s.dw = bytes(dw), s.sums = bytes(dw / k);
        return s;
    }
    s.d = bytes(d * 2 * pl);
    s.sums = bytes((d / 64 + most) * 4);
    s.dx = bytes(std::max(m * k * 4, slices_room(m, k, most / kDepth * pairs)));
    s.dw = bytes(slices_room(most, k, ceil_div(m, kDepth) * pairs));
    return s;
}

// what is enough for any number of rows up to m
size_t most_bwd_space(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    BwdSpace s = bwd_space(m, v, k, dtype);
    s.logits = most_sums_space(m, v, k, dtype);
    if (!is_narrow(m, k)) return s.total();
    // Fewer rows may have more slices of dx's sums, or dw's: by the tiles or stages that the rows are, up to so many of them
    constexpr int64_t kTried = 256;
    const NarrowPieces p = narrow_pieces(m, v, k, planes_of(dtype));
    for (int64_t tiles = 1; tiles <= std::min(ceil_div(m, 128), kTried); ++tiles) s.dx = std::max(s.dx, bytes(narrow_sums(std::min(m, tiles * 128), p.whole, k)));
    size_t dw = 0;
    for (int64_t stages = 2; stages <= std::min(ceil_div(m, 64), kTried * 2); ++stages)
        dw = std::max({dw, narrow_sums(p.whole, stages * 64, k), narrow_sums(p.last, stages * 64, k)});
    if (m > kTried * 128) s.dx = std::max(s.dx, bytes(most_narrow_sums(m, k))), dw = std::max(dw, most_narrow_sums(p.whole, k));
    s.dw = std::max(s.dw, bytes(dw)), s.sums = std::max(s.sums, bytes(dw / k));
    return std::max(s.total(), bwd_space(64, v, k, dtype).total()); // (up to 64 rows other kernels are used)
}

struct Call {
    int32_t dtype;
    int64_t m, v, k;
    const void *x, *w;
    int64_t ldx, ldw;
    const float *bias;
    float scale;
    const int64_t *targets;
};

int32_t check_call(const Call &c)
{
    DQRM_CHECK(check_shape(c.dtype, c.m, c.v));
    DQRM_CHECK(check_shape(c.dtype, c.m, c.k));
    if (c.v < 1 && c.m > 0) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_matrix(c.x, c.ldx, c.dtype, c.m, c.k));
    DQRM_CHECK(check_matrix(c.w, c.ldw, c.dtype, c.v, c.k));
    if (!std::isfinite(c.scale) || (c.bias && !aligned(c.bias, 4))) return DQRM_ERR_INVALID_ARG;
    if (c.m > 0 && (!c.targets || !aligned(c.targets, 8))) return DQRM_ERR_INVALID_ARG;
    if ((c.m > 1 && c.ldx > kMostStride) || (c.v > 1 && c.ldw > kMostStride) || c.k > kMostStride) return DQRM_ERR_UNSUPPORTED;
    const int64_t tm = ceil_div(c.m, 256), tv = ceil_div(c.v, 256), tk = ceil_div(c.k, 256);
    if (tm * tv > kMostTiles || tm * tk > kMostTiles || tv * tk > kMostTiles) return DQRM_ERR_UNSUPPORTED;
    return DQRM_OK;
}

bool sizes_are_known(int64_t m, int64_t v, int64_t k, int32_t dtype)
{
    if (check_shape(dtype, m, v) != DQRM_OK || check_shape(dtype, m, k) != DQRM_OK || k > kMostStride) return false;
    const int64_t tm = ceil_div(m, 256), tv = ceil_div(v, 256), tk = ceil_div(k, 256);
    return tm * tv <= kMostTiles && tm * tk <= kMostTiles && tv * tk <= kMostTiles;
}

// can the products read the matrix where it is?
bool as_it_is(const void *p, int64_t ld, int32_t dtype, int64_t rows, int64_t cols)
{
    return dtype != DQRM_F32 && aligned(p, 16) && cols % kChunk == 0 && (rows <= 1 || ld % kChunk == 0);
}

// The matrix as an operand, laid out in `space` first if it has to be.
Operand operand(int32_t dtype, const void *p, int64_t ld, int64_t rows, int64_t cols, void *space, hipStream_t st)
{
    if (rows == 0 || cols == 0) return Operand{nullptr, 0, 0, rows, cols, nullptr};
    if (as_it_is(p, ld, dtype, rows, cols)) return Operand{static_cast<const char *>(p), 0, (rows > 1 ? ld : cols) * 2, rows, cols, nullptr};
    const int64_t padded = up(cols, kDepth), pitch = padded * 2, per_row = padded / kChunk, step = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
    const Operand o{static_cast<const char *>(space), rows * pitch, pitch, rows, padded, nullptr};
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
        PackArgs a{static_cast<const char *>(p) + r0 * ld * (int64_t)size_of(dtype), ld, std::min(step, rows - r0), cols, static_cast<char *>(space) + r0 * pitch,
                   o.plane, pitch};
        with_type(dtype, [&](auto t) {
            hipLaunchKernelGGL(xent_pack_kernel<decltype(t)::value>, dim3((unsigned)ceil_div(a.rows * per_row, 256)), dim3(256), 0, st, a,
                               dqrm::FastDiv::make((unsigned)per_row));
        });
    }
    return o;
}

Products products(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int pairs, Shape shape)
{
    Products g{};
    g.a = a, g.b = b, g.m = m, g.n = n, g.stages = (unsigned)ceil_div(k, kDepth), g.pairs = (unsigned)pairs;
    g.tiles_m = (unsigned)ceil_div(m, rows_of(shape)), g.tiles_n = (unsigned)ceil_div(n, cols_of(shape)), g.slices = 1;
    g.stages_per_slice = g.stages * g.pairs;
    return g;
}

// rows of w as an operand
Operand classes_of(const Call &c, int64_t first, int64_t n, void *space, hipStream_t st)
{
    return operand(c.dtype, static_cast<const char *>(c.w) + first * c.ldw * (int64_t)size_of(c.dtype), c.ldw, n, c.k, space, st);
}

Classifier classifier(const Call &c, const Products &g, int64_t first)
{
    return Classifier{g, c.bias ? c.bias + first : nullptr, c.scale * kLog2e, c.targets, first};
}

// Up to 4 rows of fp32, and of what the tiles can't read where it is, by the kernel that reads w as it is, as long as its LDS holds them.  (More rows
// by strips: 200003 classes of width 1021 in fp32, 2, 4, 8 and 16 rows 161, 176, 231 and 457 us, by strips 220 for each; bf16 143, 165, 222 and
// 434, by strips 140.)
constexpr int64_t kFewRows = 4;
constexpr int64_t kFewLds = 64 << 10;

int few_lanes(int64_t k)
{
    int lanes = 1;
    while (lanes < kWaveSize && lanes * kChunk < k) lanes *= 2;
    return lanes;
}

int64_t few_padded(int64_t k) { return up(std::max<int64_t>(k, 1), few_lanes(k) * kChunk); }

int few_held(int64_t m) { return m <= 2 ? (int)m : 4; }

bool is_few(const Call &c)
{
    return c.m <= kFewRows && few_held(c.m) * few_padded(c.k) * 4 <= kFewLds && !as_it_is(c.w, c.ldw, c.dtype, c.v, c.k);
}

void launch_few(const Call &c, float2 *parts, float *at, float *loss, float *lse, hipStream_t st)
{
    const int lanes = few_lanes(c.k), at_once = 256 / lanes * (c.m <= 2 ? 4 : 2);
    // (four workgroups to a CU, and no fewer classes than a group takes at a time)
    const int64_t per_block = up(ceil_div(c.v, std::min<int64_t>(ceil_div(c.v, at_once), kFewBlocks)), at_once), blocks = ceil_div(c.v, per_block);
    const FewArgs a{static_cast<const char *>(c.x), c.w, c.ldx, c.ldw, c.m, c.v, c.k, c.bias, c.scale * kLog2e, c.targets, per_block, lanes,
                    (int)few_padded(c.k), parts, at, c.m};
    with_type(c.dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        const auto go = [&](auto rows) {
            constexpr int M = decltype(rows)::value;
            hipLaunchKernelGGL((xent_rows_fwd_kernel<DT, M>), dim3((unsigned)blocks), dim3(256), (size_t)M * a.padded * sizeof(float), st, a);
        };
        if (c.m == 1)
            go(std::integral_constant<int, 1>{});
        else if (c.m == 2)
            go(std::integral_constant<int, 2>{});
        else
            go(std::integral_constant<int, 4>{});
    });
    launch_xent_join(parts, blocks, c.m, at, c.targets, c.v, loss, lse, st);
}

// Up to 64 rows, by strips of the classes.
int64_t strips_of(int64_t n) { return up(n, kBlock) / 32; }
int strip_blocks(int64_t rows) { return rows <= 32 ? 1 : 2; }
int64_t strip_chunks(int64_t k) { return std::max<int64_t>(1, ceil_div(k, kDepth)); }
size_t strip_space(int64_t rows, int64_t k, int32_t dtype) { return (size_t)(strip_chunks(k) * 4 * planes_of(dtype) * strip_blocks(rows)) * 1024; }

// as many workgroups as the registers let run at once
int strip_grid(const Call &c, int64_t strips)
{
    const int64_t per_cu = strip_blocks(c.m) == 2 ? 2 : c.dtype == DQRM_F32 ? 3 : 4;
    return (int)std::min<int64_t>({ceil_div(strips, 4), num_cus() * per_cu, kFewBlocks});
}

bool is_strips(const Call &c)
{
    return c.m <= 64 && !as_it_is(c.w, c.ldw, c.dtype, c.v, c.k) && sums_plan(c.m, c.v, c.k, c.dtype).slices == 1;
}

StripArgs strip_args(const Call &c, int64_t first, int64_t n, const void *x)
{
    StripArgs a{};
    a.w = static_cast<const char *>(c.w) + first * c.ldw * (int64_t)size_of(c.dtype), a.ldw = c.ldw, a.classes = n, a.first = first;
    a.width = (int)c.k, a.rows = (int)c.m, a.chunks = (int)ceil_div(c.k, kDepth), a.strips = (int)strips_of(n);
    a.x = static_cast<const uint4 *>(x), a.bias = c.bias ? c.bias + first : nullptr, a.scale2 = c.scale * kLog2e, a.targets = c.targets;
    return a;
}

void launch_strip_pack(const Call &c, void *out, hipStream_t st)
{
    const int blocks = strip_blocks(c.m), vectors = (int)strip_chunks(c.k) * 4 * blocks * 64;
    with_type(c.dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        hipLaunchKernelGGL(xent_strip_pack_kernel<DT>, dim3((unsigned)ceil_div(vectors, 256)), dim3(256), 0, st, static_cast<const elem_t<DT> *>(c.x), c.ldx, (int)c.m,
                           (int)c.k, blocks, vectors, static_cast<uint4 *>(out));
    });
}

template <bool GRAD>
void launch_strips(const Call &c, const StripArgs &a, hipStream_t st)
{
    with_type(c.dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (strip_blocks(c.m) == 1)
            hipLaunchKernelGGL((xent_strip_kernel<DT, 1, GRAD>), dim3((unsigned)strip_grid(c, a.strips)), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((xent_strip_kernel<DT, 2, GRAD>), dim3((unsigned)strip_grid(c, a.strips)), dim3(256), 0, st, a);
    });
}

void launch_strip_dx(const Call &c, const StripDxArgs &a, int slices, hipStream_t st)
{
    with_type(c.dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (strip_blocks(c.m) == 1)
            hipLaunchKernelGGL((xent_strip_dx_kernel<DT, 1>), dim3((unsigned)(slices * a.columns)), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((xent_strip_dx_kernel<DT, 2>), dim3((unsigned)(slices * a.columns)), dim3(256), 0, st, a);
    });
}

template <Narrow WHAT>
void launch_narrow(const Call &c, const NarrowArgs &a, unsigned slices, hipStream_t st)
{
    with_type(c.dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        const dim3 grid(a.tiles * slices);
        if (c.k <= 16)
            hipLaunchKernelGGL((xent_narrow_kernel<DT, 1, WHAT>), grid, dim3(256), 0, st, a);
        else if (c.k <= 32)
            hipLaunchKernelGGL((xent_narrow_kernel<DT, 2, WHAT>), grid, dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((xent_narrow_kernel<DT, 4, WHAT>), grid, dim3(256), 0, st, a);
    });
}

// the logits' sums in slices, and what of the arguments of those that read them is the same
SumsArgs launch_sums(const Call &c, const Operand &x, const Operand &w, const Sliced &p, float *sums, hipStream_t st)
{
    Products g = products(x, w, c.m, c.v, c.k, pairs_of(c.dtype), p.shape);
    g.slices = p.slices, g.stages_per_slice = p.stages_per_slice;
    with_operands(c.dtype, [&](auto zero) {
        using T = decltype(zero);
        const dim3 grid(g.tiles_m * g.tiles_n * g.slices);
        if (p.shape == Shape::few)
            hipLaunchKernelGGL((xent_sums_kernel<T, TileFew>), grid, dim3(TileFew::threads), 0, st, g, sums);
        else
            hipLaunchKernelGGL((xent_sums_kernel<T, TileMid>), grid, dim3(TileMid::threads), 0, st, g, sums);
    });
    SumsArgs a{};
    a.sums = sums, a.slices = (int)p.slices, a.classes = (int)c.v, a.rows = c.m, a.bias = c.bias, a.scale2 = c.scale * kLog2e, a.targets = c.targets;
    return a;
}

void launch_fwd(const Call &c, float *loss, float *lse, void *workspace, hipStream_t st)
{
    const int pairs = pairs_of(c.dtype);
    const FwdSpace need = fwd_space(c.m, c.v, c.k, c.dtype);
    Space ws{static_cast<char *>(workspace)};
    FwdArgs a{};
    a.parts = static_cast<float2 *>(ws.take(need.parts)), a.at = static_cast<float *>(ws.take(need.at));
    void *x_space = ws.take(need.x), *w_space = ws.take(need.w);
    float *logits_space = static_cast<float *>(ws.take(need.logits));
    if (is_few(c)) return launch_few(c, a.parts, a.at, loss, lse, st);
    if (is_strips(c)) {
        launch_strip_pack(c, x_space, st);
        StripArgs strips = strip_args(c, 0, c.v, x_space);
        strips.parts = a.parts, strips.at = a.at;
        launch_strips<false>(c, strips, st);
        return launch_xent_join(a.parts, strip_grid(c, strips.strips), c.m, a.at, c.targets, c.v, loss, lse, st);
    }
    const Operand x = operand(c.dtype, c.x, c.ldx, c.m, c.k, x_space, st);
    if (is_narrow(c.m, c.k)) {
        const int64_t step = piece_classes(c.m, c.v, c.k, planes_of(c.dtype), false);
        int64_t slices = 0;
        for (int64_t first = 0; first < c.v; first += step) {
            const int64_t n = std::min(step, c.v - first);
            const Sliced p = narrow_plan(c.m, n, c.k);
            NarrowArgs b{};
            b.x = x, b.w = classes_of(c, first, n, w_space, st), b.rows = c.m, b.classes = n, b.width = (int)c.k;
            b.bias = c.bias ? c.bias + first : nullptr, b.scale2 = c.scale * kLog2e, b.targets = c.targets, b.first = first;
            b.tiles = (unsigned)ceil_div(c.m, 128), b.stages = (unsigned)ceil_div(n, 64), b.per_slice = p.stages_per_slice;
            b.parts = a.parts + slices * c.m, b.at = a.at;
            launch_narrow<Narrow::loss>(c, b, p.slices, st);
            slices += p.slices;
        }
        return launch_xent_join(a.parts, slices, c.m, a.at, c.targets, c.v, loss, lse, st);
    }
    if (const Sliced p = sums_plan(c.m, c.v, c.k, c.dtype); p.slices > 1) {
        SumsArgs s = launch_sums(c, x, classes_of(c, 0, c.v, w_space, st), p, logits_space, st);
        s.parts = a.parts, s.at = a.at;
        const int64_t parts = ceil_div(c.v, kSumsClasses);
        hipLaunchKernelGGL(xent_sums_loss_kernel, dim3((unsigned)c.m, (unsigned)parts), dim3(256), 0, st, s);
        return launch_xent_join(a.parts, parts, c.m, a.at, c.targets, c.v, loss, lse, st);
    }
    const Shape shape = logits_shape(c.m, c.v, ceil_div(c.k, kDepth) * pairs);
    const int64_t step = as_it_is(c.w, c.ldw, c.dtype, c.v, c.k) ? c.v : piece_classes(c.m, c.v, c.k, planes_of(c.dtype), false);
    for (int64_t first = 0; first < c.v; first += step) {
        const int64_t n = std::min(step, c.v - first);
        const Products g = products(x, classes_of(c, first, n, w_space, st), c.m, n, c.k, pairs, shape);
        a.c = classifier(c, g, first), a.first_tile = (unsigned)(first / cols_of(shape));
        with_operands(c.dtype, [&](auto zero) {
            with_shape(shape, [&](auto tile) {
                using S = decltype(tile);
                hipLaunchKernelGGL((xent_fwd_kernel<decltype(zero), S>), dim3(g.tiles_m * g.tiles_n), dim3(S::threads), 0, st, a);
            });
        });
    }
    launch_xent_join(a.parts, ceil_div(c.v, cols_of(shape)), c.m, a.at, c.targets, c.v, loss, lse, st);
}

// sums [slices][m][n] to the result
void launch_out_join(int32_t dtype, const float *sums, unsigned slices, int64_t m, int64_t n, void *c, int64_t ldc, float scale, const float *by, hipStream_t st)
{
    const int64_t step = std::max<int64_t>(1, ((int64_t)1 << 30) / n);
    for (int64_t r0 = 0; r0 < m; r0 += step) {
        const int64_t some = std::min(step, m - r0);
        with_type(dtype, [&](auto t) {
            using TO = elem_t<decltype(t)::value>;
            hipLaunchKernelGGL(xent_out_join_kernel<TO>, dim3((unsigned)ceil_div(some * n, 256)), dim3(256), 0, st, sums + r0 * n, slices, m * n, (unsigned)some,
                               dqrm::FastDiv::make((unsigned)n), static_cast<TO *>(c) + r0 * ldc, ldc, scale, by);
        });
    }
}

template <bool A_BY_K>
void launch_out(int32_t dtype, Shape shape, const OutArgs &a, bool sums, bool add, hipStream_t st)
{
    const dim3 grid(a.g.tiles_m * a.g.tiles_n * a.g.slices);
    with_operands(dtype, [&](auto zero) {
        using T = decltype(zero);
        with_shape(shape, [&](auto tile) {
            using S = decltype(tile);
            if (add) {
                if constexpr (!A_BY_K) hipLaunchKernelGGL((xent_out_kernel<T, float, S, A_BY_K, true>), grid, dim3(S::threads), 0, st, a);
            } else if (sums || dtype == DQRM_F32)
                hipLaunchKernelGGL((xent_out_kernel<T, float, S, A_BY_K, false>), grid, dim3(S::threads), 0, st, a);
            else
                hipLaunchKernelGGL((xent_out_kernel<T, T, S, A_BY_K, false>), grid, dim3(S::threads), 0, st, a);
        });
    });
}

void launch_bwd(const Call &c, const float *lse, const float *grad, void *dx, int64_t lddx, void *dw, int64_t lddw, float *dbias, void *workspace, hipStream_t st)
{
    const int planes = planes_of(c.dtype), pairs = pairs_of(c.dtype);
    const BwdSpace need = bwd_space(c.m, c.v, c.k, c.dtype);
    Space ws{static_cast<char *>(workspace)};
    uint64_t *live = static_cast<uint64_t *>(ws.take(need.live)), *live_classes = static_cast<uint64_t *>(ws.take(need.classes));
    unsigned *most = static_cast<unsigned *>(ws.take(need.most));
    float *unit = static_cast<float *>(ws.take(need.unit));
    void *x_space = ws.take(need.x), *strip_space = ws.take(need.strip), *w_space = ws.take(need.w);
    float *logits_space = static_cast<float *>(ws.take(need.logits));
    char *d = static_cast<char *>(ws.take(need.d));
    float *sums = static_cast<float *>(ws.take(need.sums)), *dx_sums = static_cast<float *>(ws.take(need.dx)), *dw_sums = static_cast<float *>(ws.take(need.dw));

    const int row_blocks = c.m <= kRowsAlone ? 1 : (int)std::min<int64_t>(ceil_div(c.m, 1024), 256);
    hipLaunchKernelGGL(xent_rows_kernel, dim3((unsigned)row_blocks), dim3(1024), 0, st, c.targets, c.v, lse, grad, c.m, live, most, unit);
    if (row_blocks > 1) hipLaunchKernelGGL(xent_unit_kernel, dim3(1), dim3(1024), 0, st, most, row_blocks, unit);
    // d is held in units of the largest |grad|, in fp16 times 2^14
    const float by = c.dtype == DQRM_F16 ? 16384.0f : 1.0f, scale = c.scale / by;
    if (c.bias && dx) hipLaunchKernelGGL(xent_classes_kernel, dim3((unsigned)ceil_div(c.v, 256)), dim3(256), 0, st, c.bias, c.v, live_classes);

    const Operand x = operand(c.dtype, c.x, c.ldx, c.m, c.k, x_space, st);
    const bool narrow = is_narrow(c.m, c.k);
    const int64_t step = piece_classes(c.m, c.v, c.k, planes, !narrow);
    const bool one = step >= c.v;
    const bool strips = is_strips(c);
    const Sliced in_slices = sums_plan(c.m, c.v, c.k, c.dtype);
    if (strips) launch_strip_pack(c, strip_space, st);
    const int64_t columns = ceil_div(c.k, kBlock), blocks = ceil_div(std::min(step, c.v), kBlock);
    Sliced dx_plan = out_plan(c.m, c.k, blocks * pairs);
    if (strips) { // (of blocks of classes; four waves to a workgroup, six workgroups to a CU)
        const int64_t slices = std::min<int64_t>({std::max<int64_t>(1, num_cus() * 6 / std::max<int64_t>(columns, 1)), ceil_div(blocks, 4), kMostSlices});
        dx_plan.stages_per_slice = (unsigned)ceil_div(blocks, slices), dx_plan.slices = (unsigned)ceil_div(blocks, dx_plan.stages_per_slice);
    }
    if (narrow) dx_plan = narrow_plan(c.m, std::min(step, c.v), c.k);
    for (int64_t first = 0; first < c.v; first += step) {
        const int64_t n = std::min(step, c.v - first);
        if (narrow) {
            NarrowArgs a{};
            a.x = x, a.w = classes_of(c, first, n, w_space, st), a.rows = c.m, a.classes = n, a.width = (int)c.k;
            a.x.live = live, a.w.live = c.bias && dx ? live_classes + first / 64 : nullptr;
            a.bias = c.bias ? c.bias + first : nullptr, a.scale2 = c.scale * kLog2e, a.targets = c.targets, a.first = first;
            a.lse = lse, a.grad = grad, a.most = unit, a.by = by;
            if (dx) {
                a.tiles = (unsigned)ceil_div(c.m, 128), a.stages = (unsigned)ceil_div(n, 64), a.per_slice = dx_plan.stages_per_slice, a.sums = dx_sums, a.add = first > 0;
                launch_narrow<Narrow::dx>(c, a, dx_plan.slices, st);
            }
            if (dw || dbias) {
                const Sliced p = narrow_plan(n, c.m, c.k);
                a.tiles = (unsigned)ceil_div(n, 128), a.stages = (unsigned)ceil_div(c.m, 64), a.per_slice = p.stages_per_slice, a.sums = dw_sums, a.add = false;
                a.dbias = dbias ? sums : nullptr;
                launch_narrow<Narrow::dw>(c, a, p.slices, st);
                if (dw)
                    launch_out_join(c.dtype, dw_sums, p.slices, n, c.k, static_cast<char *>(dw) + first * lddw * (int64_t)size_of(c.dtype), lddw, scale, unit, st);
                if (dbias) hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)ceil_div(n, 16)), dim3(256), 0, st, sums, n, (int)p.slices, n, n, dbias + first, nullptr);
            }
            continue;
        }
        const Operand w = strips ? Operand{} : classes_of(c, first, n, w_space, st);
        const Shape shape = logits_shape(c.m, n, ceil_div(c.k, kDepth) * pairs);
        GradArgs a{};
        const Products g = products(x, w, c.m, n, c.k, pairs, shape);
        a.c = classifier(c, g, first), a.lse = lse, a.grad = grad, a.live = live, a.most = unit, a.by = by;
        a.rows = up(c.m, kBlock), a.cols = up(n, kBlock), a.plane = a.rows * a.cols * 2, a.planes = planes, a.d = d, a.sums = dbias ? sums : nullptr;
        if (strips && c.m > 0) {
            StripArgs b = strip_args(c, first, n, strip_space);
            b.lse = lse, b.grad = grad, b.most = unit, b.live = live, b.by = by, b.d = d, b.plane = a.plane, b.dbias = dbias ? dbias + first : nullptr;
            launch_strips<true>(c, b, st);
        } else if (in_slices.slices > 1) {
            SumsArgs b = launch_sums(c, x, w, in_slices, logits_space, st);
            // (added up where the first one is, a value to a thread: a block of d has few threads)
            launch_out_join(DQRM_F32, logits_space, in_slices.slices, c.m, n, logits_space, n, 1.0f, nullptr, st);
            b.slices = 1;
            b.lse = lse, b.grad = grad, b.most = unit, b.live = live, b.by = by, b.d = d, b.plane = a.plane, b.pitch = a.cols * 2, b.dbias = a.sums;
            const dim3 grid((unsigned)(a.cols / kBlock), (unsigned)(a.rows / kBlock));
            with_type(c.dtype, [&](auto t) { hipLaunchKernelGGL(xent_sums_grad_kernel<decltype(t)::value>, grid, dim3(256), 0, st, b); });
        } else if (g.tiles_m > 0)
            with_operands(c.dtype, [&](auto zero) {
                with_shape(shape, [&](auto tile) {
                    using S = decltype(tile);
                    hipLaunchKernelGGL((xent_grad_kernel<decltype(zero), S>), dim3(g.tiles_m * g.tiles_n), dim3(S::threads), 0, st, a);
                });
            });
        if (dbias && !(strips && c.m > 0)) hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)ceil_div(n, 16)), dim3(256), 0, st, sums, n,
                               in_slices.slices > 1 ? (int)(a.rows / kBlock) : (int)g.tiles_m, n, n, dbias + first, nullptr);
        if (c.k == 0) continue;
        const Operand dm{d, a.plane, a.cols * 2, a.rows, a.cols, nullptr};
        if (dx && c.m > 0 && strips) {
            StripDxArgs b{};
            b.w = static_cast<const char *>(c.w) + first * c.ldw * (int64_t)size_of(c.dtype), b.ldw = c.ldw, b.classes = n, b.width = (int)c.k, b.rows = (int)c.m;
            b.columns = (int)columns, b.d = d, b.plane = a.plane, b.live = c.bias ? live_classes + first / 64 : nullptr, b.blocks = (int)ceil_div(n, kBlock);
            b.per_slice = (int)dx_plan.stages_per_slice, b.sums = dx_sums, b.add = first > 0;
            launch_strip_dx(c, b, (int)dx_plan.slices, st);
        } else if (dx && c.m > 0) {
            Operand by = w;
            by.live = c.bias ? live_classes + first / 64 : nullptr;
            OutArgs o{products(dm, by, c.m, c.k, n, pairs, dx_plan.shape), dx, lddx, scale, unit};
            o.g.slices = dx_plan.slices, o.g.stages_per_slice = dx_plan.stages_per_slice;
            const bool in_sums = !one || dx_plan.slices > 1;
            if (in_sums) o.c = dx_sums, o.ldc = c.k, o.scale = 1.0f, o.by = nullptr;
            launch_out<false>(c.dtype, dx_plan.shape, o, in_sums, first > 0, st);
        }
        if (dw) {
            Operand by = x;
            by.live = live;
            const Sliced p = out_plan(n, c.k, ceil_div(c.m, kDepth) * pairs);
            char *to = static_cast<char *>(dw) + first * lddw * (int64_t)size_of(c.dtype);
            OutArgs o{products(dm, by, n, c.k, c.m, pairs, p.shape), to, lddw, scale, unit};
            o.g.slices = p.slices, o.g.stages_per_slice = p.stages_per_slice;
            if (p.slices > 1) o.c = dw_sums, o.ldc = c.k, o.scale = 1.0f, o.by = nullptr;
            launch_out<true>(c.dtype, p.shape, o, p.slices > 1, false, st);
            if (p.slices > 1) launch_out_join(c.dtype, dw_sums, p.slices, n, c.k, to, lddw, scale, unit, st);
        }
    }
    if (dx && c.m > 0 && c.k > 0 && (!one || dx_plan.slices > 1 || strips || narrow))
        launch_out_join(c.dtype, dx_sums, dx_plan.slices, c.m, c.k, dx, lddx, scale, unit, st);
}

} // namespace

extern "C" {

size_t dqrm_softmax_xent_fwd_workspace_bytes(int64_t rows, int64_t classes, int64_t width, int32_t dtype)
{
    if (!sizes_are_known(rows, classes, width, dtype)) return 0;
    FwdSpace s = fwd_space(rows, classes, width, dtype);
    s.logits = most_sums_space(rows, classes, width, dtype); // (for fewer rows too)
    return s.total();
}

int32_t dqrm_softmax_xent_fwd(int32_t dtype, int64_t rows, int64_t classes, int64_t width, const void *x, int64_t ldx, const void *w, int64_t ldw,
                              const float *bias, float scale, const int64_t *targets, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                              void *stream)
{
    const Call c{dtype, rows, classes, width, x, w, ldx, ldw, bias, scale, targets};
    DQRM_CHECK(check_call(c));
    if (rows > 0 && (!loss || !lse || !aligned(loss, 4) || !aligned(lse, 4))) return DQRM_ERR_INVALID_ARG;
    if (rows == 0) return DQRM_OK;
    DQRM_CHECK(check_workspace(workspace, workspace_bytes, fwd_space(rows, classes, width, dtype).total()));
    launch_fwd(c, loss, lse, workspace, static_cast<hipStream_t>(stream));
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

size_t dqrm_softmax_xent_bwd_workspace_bytes(int64_t rows, int64_t classes, int64_t width, int32_t dtype)
{
    return sizes_are_known(rows, classes, width, dtype) ? most_bwd_space(rows, classes, width, dtype) : 0;
}

int32_t dqrm_softmax_xent_bwd(int32_t dtype, int64_t rows, int64_t classes, int64_t width, const void *x, int64_t ldx, const void *w, int64_t ldw,
                              const float *bias, float scale, const int64_t *targets, const float *lse, const float *grad, void *dx, int64_t lddx, void *dw,
                              int64_t lddw, float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    const Call c{dtype, rows, classes, width, x, w, ldx, ldw, bias, scale, targets};
    DQRM_CHECK(check_call(c));
    if (!dx && !dw && !dbias && rows > 0 && width > 0) return DQRM_ERR_INVALID_ARG; // (an empty output may be null)
    if (rows > 0 && (!lse || !grad || !aligned(lse, 4) || !aligned(grad, 4))) return DQRM_ERR_INVALID_ARG;
    if (dx) DQRM_CHECK(check_matrix(dx, lddx, dtype, rows, width));
    if (dw) DQRM_CHECK(check_matrix(dw, lddw, dtype, classes, width));
    if (dbias && !aligned(dbias, 4)) return DQRM_ERR_INVALID_ARG;
    if (classes == 0) return DQRM_OK;
    DQRM_CHECK(check_workspace(workspace, workspace_bytes, bwd_space(rows, classes, width, dtype).total()));
    launch_bwd(c, lse, grad, dx, lddx, dw, lddw, dbias, workspace, static_cast<hipStream_t>(stream));
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

} // extern "C"
