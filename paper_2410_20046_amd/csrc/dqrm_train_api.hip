// C ABI of the gradients' norm and of residual norms: host-side validation and kernel dispatch.
// Every entry point validates on the host first and enqueues nothing on error.
#include "dqrm_checks.hpp"
#include "dqrm_grad.hpp"
#include "dqrm_resnorm.hpp"

#include <cstdlib>

namespace {

using namespace dqrm_host;

// ---- the norm of all gradients -----------------------------------------------------------------------------------------------
using dqrm_grad::Batch;
using dqrm_grad::Item;
using dqrm_mx::kChunk;

constexpr int32_t kMostTensors = 65536;
// Pieces of the tensors of a launch, on average: a few workgroups to a CU.  A piece has at least four rounds of vectors.
constexpr int64_t kPieces = 2048, kLeastPiece = dqrm_grad::kThreads * dqrm_grad::kAhead;
// Up to so many parts every workgroup of the scaling joins them for itself; more are joined by a launch of their own.
constexpr unsigned kJoinedByAll = 2 * kPieces;

bool empty(const dqrm_grad_t &g) { return g.rows == 0 || g.cols == 0; }

// a tensor whose rows lie one behind the other is one row, unless only some of them are there
Item item_of(const dqrm_grad_t &g)
{
    Item t{};
    t.data = static_cast<const char *>(g.data), t.out = static_cast<char *>(g.out ? g.out : g.data);
    t.count = g.count, t.rows = g.rows, t.cols = g.cols, t.ld = g.ld, t.ld_out = g.out ? g.ld_out : g.ld, t.dtype = g.dtype;
    if (!g.count && (g.rows == 1 || (t.ld == g.cols && t.ld_out == g.cols))) t.cols = g.rows * g.cols, t.rows = 1, t.ld = t.ld_out = t.cols;
    return t;
}

int64_t vectors_of(const Item &t) { return t.rows * ceil_div(t.cols, kChunk); }

int32_t check_grads(const dqrm_grad_t *g, int32_t n)
{
    if (n < 0 || (n > 0 && !g)) return DQRM_ERR_INVALID_ARG;
    if (n > kMostTensors) return DQRM_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int32_t i = 0; i < n; ++i) {
        DQRM_CHECK(check_shape(g[i].dtype, g[i].rows, 0));
        // (a flat buffer is one row of any length)
        if (g[i].cols < 0) return DQRM_ERR_INVALID_ARG;
        if (g[i].cols > (int64_t)1 << 40 || (g[i].rows > 0 && g[i].cols > ((int64_t)1 << 44) / g[i].rows)) return DQRM_ERR_UNSUPPORTED;
        DQRM_CHECK(check_matrix(g[i].data, g[i].ld, g[i].dtype, g[i].rows, g[i].cols));
        if (g[i].out) DQRM_CHECK(check_matrix(g[i].out, g[i].ld_out, g[i].dtype, g[i].rows, g[i].cols));
        if (g[i].count && !aligned(g[i].count, 4)) return DQRM_ERR_INVALID_ARG;
        all += g[i].rows * g[i].cols;
        if (all > (int64_t)1 << 44) return DQRM_ERR_UNSUPPORTED;
    }
    return DQRM_OK;
}

// Memory of a tensor: rows of `width` bytes every `pitch`, or one block.
struct Region {
    uintptr_t from, to;
    int64_t rows, width, pitch;
    bool written;
};

Region region_of(const void *p, const dqrm_grad_t &g, int64_t ld, bool written)
{
    const int64_t size = (int64_t)size_of(g.dtype);
    const bool block = g.rows == 1 || ld == g.cols; // (a single row's stride may be anything)
    Region r{reinterpret_cast<uintptr_t>(p), 0, block ? 1 : g.rows, (block ? g.rows : 1) * g.cols * size, 0, written};
    r.pitch = block ? r.width : ld * size;
    r.to = r.from + (uintptr_t)((r.rows - 1) * r.pitch + r.width);
    return r;
}

// does [from, to) meet a row? (it begins in or behind the first one)
bool meets(const Region &r, uintptr_t from, uintptr_t to)
{
    if (from >= r.to) return false;
    const int64_t at = (int64_t)(from - r.from), row = at < r.pitch ? 0 : at / r.pitch, in = at - row * r.pitch;
    return in < r.width || (row + 1 < r.rows && (int64_t)(to - from) > r.pitch - in);
}

// b begins in or behind a.  Rows of one pitch lie to each other as the first ones do; of others each is looked at, of the shorter tensor.
bool overlap(const Region &a, const Region &b)
{
    if (a.pitch == b.pitch || b.rows == 1) return meets(a, b.from, b.from + (uintptr_t)b.width);
    for (int64_t r = 0; r < a.rows && a.rows <= b.rows; ++r) {
        const uintptr_t from = a.from + (uintptr_t)(r * a.pitch), to = from + (uintptr_t)a.width;
        if (to > b.from && meets(b, std::max(from, b.from), to)) return true;
    }
    for (int64_t r = 0; r < b.rows && a.rows > b.rows; ++r) {
        const uintptr_t from = b.from + (uintptr_t)(r * b.pitch);
        if (meets(a, from, from + (uintptr_t)b.width)) return true;
    }
    return false;
}

// What is written must be nothing else's memory: no other tensor's, nor the tensor's own input with another stride or shifted.  (Rows may lie in
// another's gaps.)  Regions in the order of their first bytes, each against those before it that have not ended.
int32_t check_apart(const dqrm_grad_t *g, int32_t n)
{
    if (n < 1) return DQRM_OK;
    Region *s = static_cast<Region *>(std::malloc((sizeof(Region) * 2 + sizeof(int32_t) * 2) * (size_t)n));
    if (!s) return DQRM_ERR_UNSUPPORTED;
    int32_t *open = reinterpret_cast<int32_t *>(s + 2 * (size_t)n);
    int32_t some = 0, opened = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (empty(g[i])) continue;
        const bool in_place = !g[i].out || (g[i].out == g[i].data && (g[i].ld_out == g[i].ld || g[i].rows == 1));
        s[some++] = in_place ? region_of(g[i].data, g[i], g[i].ld, true) : region_of(g[i].out, g[i], g[i].ld_out, true);
        if (!in_place) s[some++] = region_of(g[i].data, g[i], g[i].ld, false);
    }
    std::sort(s, s + some, [](const Region &a, const Region &b) { return a.from < b.from; });
    bool bad = false;
    for (int32_t i = 0; i < some && !bad; ++i) {
        int32_t left = 0;
        for (int32_t k = 0; k < opened; ++k) {
            const Region &a = s[open[k]];
            if (a.to <= s[i].from) continue;
            bad |= (a.written || s[i].written) && overlap(a, s[i]);
            open[left++] = open[k];
        }
        open[left++] = i, opened = left;
    }
    std::free(s);
    return bad ? DQRM_ERR_INVALID_ARG : DQRM_OK;
}

struct GradPlan {
    int64_t per_piece;
    unsigned pieces;
};

GradPlan grad_plan(const dqrm_grad_t *g, int32_t n)
{
    int64_t all = 0;
    for (int32_t i = 0; i < n; ++i)
        if (!empty(g[i])) all += vectors_of(item_of(g[i]));
    const int64_t pieces = kPieces * std::max<int64_t>(1, ceil_div(n, dqrm_grad::kItems));
    GradPlan p{std::max(kLeastPiece, ceil_div(ceil_div(all, pieces), kLeastPiece) * kLeastPiece), 0};
    for (int32_t i = 0; i < n; ++i)
        if (!empty(g[i])) p.pieces += (unsigned)ceil_div(vectors_of(item_of(g[i])), p.per_piece);
    return p;
}

size_t grad_workspace(const GradPlan &p) { return align_up((size_t)p.pieces * sizeof(double), 256); }

// f(batch, its first tensor's number, whether it is the last one) for the tensors in turn; empty ones stay in: their norm is 0
template <typename F>
void for_batches(const dqrm_grad_t *g, int32_t n, const GradPlan &p, F f)
{
    unsigned next = 0;
    for (int32_t i = 0; i < n || i == 0; i += dqrm_grad::kItems) {
        Batch b{};
        b.items = std::min(dqrm_grad::kItems, n - i), b.first = next, b.all = p.pieces, b.per_piece = p.per_piece;
        for (int32_t k = 0; k < b.items; ++k) {
            if (!empty(g[i + k])) b.item[k] = item_of(g[i + k]);
            b.item[k].first = next;
            if (!empty(g[i + k])) next += (unsigned)ceil_div(vectors_of(b.item[k]), p.per_piece);
        }
        b.pieces = next - b.first;
        f(b, i, i + dqrm_grad::kItems >= n);
    }
}

template <typename F>
void with_kind(int32_t kind, F f)
{
    if (kind == DQRM_GRAD_NORM_2)
        f(std::integral_constant<int, DQRM_GRAD_NORM_2>{});
    else
        f(std::integral_constant<int, DQRM_GRAD_NORM_MAX>{});
}

int32_t check_norm_call(const dqrm_grad_t *g, int32_t n, int32_t kind, const float *norm, const float *norms, GradPlan &p, const void *ws, size_t ws_bytes)
{
    if (kind != DQRM_GRAD_NORM_2 && kind != DQRM_GRAD_NORM_MAX) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_grads(g, n));
    if (!norm || !aligned(norm, 4) || (norms && !aligned(norms, 4))) return DQRM_ERR_INVALID_ARG;
    p = grad_plan(g, n);
    return check_workspace(ws, ws_bytes, grad_workspace(p));
}

void launch_parts(const dqrm_grad_t *g, int32_t n, int32_t kind, const GradPlan &p, double *parts, hipStream_t st)
{
    for_batches(g, n, p, [&](const Batch &b, int32_t, bool) {
        if (!b.pieces) return;
        with_kind(kind, [&](auto k) {
            hipLaunchKernelGGL(dqrm_grad::grad_part_kernel<decltype(k)::value>, dim3(b.pieces), dim3(dqrm_grad::kThreads), 0, st, b, parts);
        });
    });
}

void launch_joins(const dqrm_grad_t *g, int32_t n, int32_t kind, const GradPlan &p, const double *parts, float *norm, float *norms, hipStream_t st)
{
    for_batches(g, n, p, [&](const Batch &b, int32_t first, bool last) {
        const unsigned grid = (norms ? (unsigned)b.items : 0u) + (last && norm ? 1u : 0u);
        if (!grid) return;
        with_kind(kind, [&](auto k) {
            hipLaunchKernelGGL(dqrm_grad::grad_join_kernel<decltype(k)::value>, dim3(grid), dim3(dqrm_grad::kThreads), 0, st, b, parts, norms, (int)first, norm);
        });
    });
}

void launch_scale(const dqrm_grad_t *g, int32_t n, int32_t kind, const GradPlan &p, const double *parts, const float *given, float *norm, float *norms,
                  float max_norm, hipStream_t st)
{
    for_batches(g, n, p, [&](const Batch &b, int32_t, bool) {
        if (!b.pieces) return;
        with_kind(kind, [&](auto k) {
            hipLaunchKernelGGL(dqrm_grad::grad_scale_kernel<decltype(k)::value>, dim3(b.pieces), dim3(dqrm_grad::kThreads), 0, st, b, parts, given, norm,
                               norms, max_norm);
        });
    });
}

// ---- residual norms ----------------------------------------------------------------------------------------------------------
namespace rn = dqrm_resnorm;

constexpr int64_t kMostNormCols = 16384;

// threads and chunks of 8 values to a row; rows of fewer than 8
template <int TPR_, int CH_, int BLOCK_, rn::Gains GAINS_ = rn::Gains::registers, bool SHORT_ = false>
struct RowShape {
    static constexpr int TPR = TPR_, CH = CH_, BLOCK = BLOCK_, cols = TPR * CH * kChunk, rows = BLOCK / TPR;
    static constexpr rn::Gains GAINS = GAINS_;
    static constexpr bool SHORT = SHORT_;
};

template <typename... S, typename F>
void with_first_that_holds(int64_t cols, F f)
{
    (void)((cols <= S::cols ? (f(S{}), true) : false) || ...);
}

// Many rows without codes: several chunks to a thread, and the columns' vectors in LDS; else a chunk to a thread: a row's latency counts.  Both ways, us,
// the second one what is taken of few rows: bf16 65536 x 1024 105 and 111, 32768 x 3000 221 and 232, 16384 x 6000 230 and 244, of 4096 and 8192 columns
// 229 and 221, 246 and 244; fp32 16384 x 2048 101 and 109, 32768 x 1024 106 and 107, 8192 x 6000 175 and 203, 8192 x 8192 226 and 247.  With codes bf16
// 65536 x 1024 164 and 141, 32768 x 4096 388 and 324, 16384 x 8192 336 and 266, fp32 16384 x 2048 103 either way, 8192 x 8192 263 and 271.
template <int DT, bool CODES, typename F>
void with_resnorm_fwd_shape(int64_t rows, int64_t cols, F f)
{
    using rn::Gains;
    if (cols < kChunk) return f(RowShape<16, 1, 256, Gains::registers, true>{});
    if constexpr (!CODES) {
        if (rows >= (int64_t)num_cus() * 16) {
            if constexpr (DT == DQRM_F32)
                return with_first_that_holds<RowShape<16, 1, 256>, RowShape<64, 1, 256>, RowShape<64, 2, 256>, RowShape<128, 2, 512, Gains::lds>,
                                             RowShape<512, 1, 512>, RowShape<512, 2, 1024, Gains::lds>, RowShape<1024, 2, 1024, Gains::memory>>(cols, f);
            else
                return with_first_that_holds<RowShape<16, 1, 256>, RowShape<64, 1, 256>, RowShape<64, 2, 256>, RowShape<256, 1, 256>,
                                             RowShape<128, 4, 256, Gains::lds>, RowShape<512, 2, 1024, Gains::lds>, RowShape<1024, 2, 1024, Gains::memory>>(cols, f);
        }
    }
    with_first_that_holds<RowShape<16, 1, 256>, RowShape<64, 1, 256>, RowShape<128, 1, 256>, RowShape<256, 1, 256>, RowShape<512, 1, 512>,
                          RowShape<1024, 1, 1024>, RowShape<1024, 2, 1024, Gains::memory>>(cols, f);
}

// (1024 threads and the columns' vectors in LDS, and 512 threads with two chunks, us: fp32 8192 x 8192 371 and 422, 8192 x 6000 265 and 364; bf16 4000 x
// 8192 88 and 86, 16384 x 8192 307 and 310, but 16384 x 6000 234 and 257.  Rows beyond 8192 values: 10000 x 16384 bf16 1510 us, of fp32 2210.)
template <int DT, typename F>
void with_resnorm_bwd_shape(int64_t cols, F f)
{
    using rn::Gains;
    if (cols < kChunk) return f(RowShape<16, 1, 512, Gains::registers, true>{});
    using Wide = std::conditional_t<DT == DQRM_F32, RowShape<1024, 1, 1024, Gains::lds>, RowShape<512, 2, 512>>;
    with_first_that_holds<RowShape<16, 1, 512>, RowShape<64, 1, 512>, RowShape<128, 1, 512>, RowShape<256, 1, 512>, RowShape<512, 1, 512>, Wide,
                          RowShape<1024, 2, 1024, Gains::memory>>(cols, f);
}

int resnorm_bwd_blocks(int64_t rows, int64_t cols)
{
    int64_t n = 0; // (every type's shapes have as many rows to a workgroup)
    if (rows > 0 && cols > 0) with_resnorm_bwd_shape<DQRM_F32>(cols, [&](auto shape) { n = std::min<int64_t>(ceil_div(rows, decltype(shape)::rows), num_cus()); });
    return (int)n;
}

size_t resnorm_bwd_workspace(int64_t rows, int64_t cols) { return align_up((size_t)resnorm_bwd_blocks(rows, cols) * 4 * (size_t)cols * sizeof(float), 256); }

int32_t check_resnorm(const dqrm_residual_norm_t *n, int32_t dtype, int64_t rows, int64_t cols)
{
    DQRM_CHECK(check_shape(dtype, rows, cols));
    if (!n || cols < 1) return DQRM_ERR_INVALID_ARG;
    if (cols > kMostNormCols) return DQRM_ERR_UNSUPPORTED;
    for (int32_t kind : {n->post, n->pre})
        if (kind != DQRM_NORM_NONE && kind != DQRM_NORM_LAYER && kind != DQRM_NORM_RMS) return DQRM_ERR_INVALID_ARG;
    if (!(n->post_eps >= 0.0f) || !(n->pre_eps >= 0.0f)) return DQRM_ERR_INVALID_ARG;
    if ((n->post == DQRM_NORM_NONE && (n->post_gamma || n->post_beta)) || (n->pre == DQRM_NORM_NONE && (n->pre_gamma || n->pre_beta))) return DQRM_ERR_INVALID_ARG;
    for (const float *p : {n->post_gamma, n->post_beta, n->gate, n->pre_gamma, n->pre_beta})
        if (p && !aligned(p, 4)) return DQRM_ERR_INVALID_ARG;
    return DQRM_OK;
}

rn::Params params_of(const dqrm_residual_norm_t &n)
{
    return rn::Params{n.post, n.pre, n.post_gamma, n.post_beta, n.gate, n.pre_gamma, n.pre_beta, n.res_scale, n.post_eps, n.pre_eps};
}

} // namespace

extern "C" {

size_t dqrm_grad_workspace_bytes(const dqrm_grad_t *grads, int32_t n)
{
    return check_grads(grads, n) == DQRM_OK ? grad_workspace(grad_plan(grads, n)) : 0;
}

int32_t dqrm_grad_norm(const dqrm_grad_t *grads, int32_t n, int32_t kind, float *norm, float *norms, void *workspace, size_t workspace_bytes, void *stream)
{
    GradPlan p{};
    DQRM_CHECK(check_norm_call(grads, n, kind, norm, norms, p, workspace, workspace_bytes));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *parts = static_cast<double *>(workspace);
    launch_parts(grads, n, kind, p, parts, st);
    launch_joins(grads, n, kind, p, parts, norm, norms, st);
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

int32_t dqrm_grad_scale(const dqrm_grad_t *grads, int32_t n, const float *norm, float max_norm, void *stream)
{
    DQRM_CHECK(check_grads(grads, n));
    if (!norm || !aligned(norm, 4) || !(max_norm >= 0.0f)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_apart(grads, n));
    launch_scale(grads, n, DQRM_GRAD_NORM_2, grad_plan(grads, n), nullptr, norm, nullptr, nullptr, max_norm, static_cast<hipStream_t>(stream));
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

int32_t dqrm_grad_clip(const dqrm_grad_t *grads, int32_t n, int32_t kind, float max_norm, float *norm, float *norms, void *workspace, size_t workspace_bytes,
                       void *stream)
{
    GradPlan p{};
    DQRM_CHECK(check_norm_call(grads, n, kind, norm, norms, p, workspace, workspace_bytes));
    if (!(max_norm >= 0.0f)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_apart(grads, n));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *parts = static_cast<double *>(workspace);
    launch_parts(grads, n, kind, p, parts, st);
    if (n <= dqrm_grad::kItems && p.pieces > 0 && p.pieces <= kJoinedByAll) { // (one launch: it joins the parts as well)
        launch_scale(grads, n, kind, p, parts, nullptr, norm, norms, max_norm, st);
    } else {
        launch_joins(grads, n, kind, p, parts, norm, norms, st);
        launch_scale(grads, n, kind, p, nullptr, norm, nullptr, nullptr, max_norm, st);
    }
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

int32_t dqrm_residual_norm_fwd(int32_t dtype, int64_t rows, int64_t cols, const dqrm_residual_norm_t *norm, const void *u, int64_t ldu, const void *r,
                               int64_t ldr, void *out, int64_t ldo, void *y, int64_t ldy, float *stats, const dqrm_mxfp4_t *q, void *stream)
{
    DQRM_CHECK(check_resnorm(norm, dtype, rows, cols));
    if (norm->pre == DQRM_NORM_NONE && (y || q)) return DQRM_ERR_INVALID_ARG;
    DQRM_CHECK(check_matrix(u, ldu, dtype, rows, cols));
    DQRM_CHECK(check_matrix(r, ldr, dtype, rows, cols));
    DQRM_CHECK(check_matrix(out, ldo, dtype, rows, cols));
    if (y) DQRM_CHECK(check_matrix(y, ldy, dtype, rows, cols));
    if (q) DQRM_CHECK(check_mx(q, rows, cols));
    if (stats && !aligned(stats, 4)) return DQRM_ERR_INVALID_ARG;
    if (rows == 0) return DQRM_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const size_t es = size_of(dtype);
    for (int64_t r0 = 0; r0 < rows; r0 += kMaxBlocks) {
        rn::FwdArgs a{};
        a.p = params_of(*norm), a.rows = std::min(kMaxBlocks, rows - r0), a.cols = cols, a.all_rows = rows;
        a.u = static_cast<const char *>(u) + r0 * ldu * es, a.ldu = ldu, a.r = static_cast<const char *>(r) + r0 * ldr * es, a.ldr = ldr;
        a.out = static_cast<char *>(out) + r0 * ldo * es, a.ldo = ldo;
        if (y) a.y = static_cast<char *>(y) + r0 * ldy * es, a.ldy = ldy;
        if (stats) a.stats = stats + r0;
        if (q) a.codes = q->codes + r0 * dqrm_mx::codes_pitch(cols), a.scales = q->scales + r0 * dqrm_mx::scales_pitch(cols);
        with_type(dtype, [&](auto t) {
            const auto go = [&](auto codes) {
                constexpr bool CODES = decltype(codes)::value;
                with_resnorm_fwd_shape<decltype(t)::value, CODES>(rows, cols, [&](auto shape) {
                    using S = decltype(shape);
                    // as many workgroups as the chip holds: each keeps the columns' vectors for all of its rows
                    const int64_t most = (int64_t)num_cus() * std::max(1, 1024 / S::BLOCK);
                    hipLaunchKernelGGL((rn::resnorm_fwd_kernel<decltype(t)::value, S::TPR, S::CH, S::BLOCK, S::SHORT, S::GAINS, CODES>),
                                       dim3((unsigned)std::min(ceil_div(a.rows, S::rows), most)), dim3(S::BLOCK), 0, st, a);
                });
            };
            if (q)
                go(std::true_type{});
            else
                go(std::false_type{});
        });
    }
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

size_t dqrm_residual_norm_bwd_workspace_bytes(int64_t rows, int64_t cols)
{
    return check_shape(DQRM_F32, rows, cols) == DQRM_OK && cols <= kMostNormCols ? resnorm_bwd_workspace(rows, cols) : 0;
}

int32_t dqrm_residual_norm_bwd(int32_t dtype, int64_t rows, int64_t cols, const dqrm_residual_norm_t *norm, const void *dout, int64_t lddout, const void *dy,
                               int64_t lddy, const void *u, int64_t ldu, const void *out, int64_t ldo, const float *stats, void *du, int64_t lddu, void *dr,
                               int64_t lddr, float *dparams, void *workspace, size_t workspace_bytes, void *stream)
{
    DQRM_CHECK(check_resnorm(norm, dtype, rows, cols));
    const bool pre = norm->pre != DQRM_NORM_NONE, post = norm->post != DQRM_NORM_NONE;
    if ((!dout && !pre && rows > 0) || (!du && !dr && !dparams && rows > 0)) return DQRM_ERR_INVALID_ARG;
    if (dout) DQRM_CHECK(check_matrix(dout, lddout, dtype, rows, cols));
    if (pre) {
        DQRM_CHECK(check_matrix(dy, lddy, dtype, rows, cols));
        DQRM_CHECK(check_matrix(out, ldo, dtype, rows, cols));
    }
    const bool needs_u = post || dparams;
    if (needs_u) DQRM_CHECK(check_matrix(u, ldu, dtype, rows, cols));
    if (du) DQRM_CHECK(check_matrix(du, lddu, dtype, rows, cols));
    if (dr) DQRM_CHECK(check_matrix(dr, lddr, dtype, rows, cols));
    if (((pre || post) && rows > 0 && !stats) || (stats && !aligned(stats, 4)) || (dparams && !aligned(dparams, 4))) return DQRM_ERR_INVALID_ARG;
    if (dparams) DQRM_CHECK(check_workspace(workspace, workspace_bytes, resnorm_bwd_workspace(rows, cols)));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int blocks = resnorm_bwd_blocks(rows, cols);
    rn::BwdArgs a{};
    a.p = params_of(*norm), a.rows = rows, a.cols = cols, a.stats = stats;
    a.dout = dout, a.lddout = lddout;
    if (pre) a.dy = dy, a.lddy = lddy, a.out = out, a.ldo = ldo;
    if (needs_u) a.u = u, a.ldu = ldu;
    a.du = du, a.lddu = lddu, a.dr = dr, a.lddr = lddr;
    a.partial = dparams ? static_cast<float *>(workspace) : nullptr;
    if (blocks > 0)
        with_type(dtype, [&](auto t) {
            with_resnorm_bwd_shape<decltype(t)::value>(cols, [&](auto shape) {
                using S = decltype(shape);
                hipLaunchKernelGGL((rn::resnorm_bwd_kernel<decltype(t)::value, S::TPR, S::CH, S::BLOCK, S::SHORT, S::GAINS>), dim3((unsigned)blocks), dim3(S::BLOCK), 0, st,
                                   a);
            });
        });
    if (dparams) // (without rows: zeros)
        hipLaunchKernelGGL(rn::resnorm_join_kernel, dim3((unsigned)ceil_div(cols, 16)), dim3(256), 0, st, a.partial, blocks, (int)cols, a.p, dparams);
    DQRM_HIP_CHECK(hipGetLastError());
    return DQRM_OK;
}

} // extern "C"
