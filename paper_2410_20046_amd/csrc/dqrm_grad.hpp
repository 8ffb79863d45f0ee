// The norm of many gradient tensors together, and the tensors scaled by it (gfx950, wave64).
//
//   n = sqrt(sum v^2) or max |v| over all values of all tensors; v <- v (max_norm / n) where n > max_norm and n is finite
//
// Squares and their sums are held in 64 bits: no gradient overflows them, and a sum over 10^9 values loses nothing that counts.  The
// tensors are cut into pieces of equal size, a workgroup to each; a piece's sum is a place in the workspace, and whoever needs the norm
// adds the places in a fixed order: no atomics.
#pragma once

#include "dqrm_mx.hpp"

namespace dqrm_grad {

using namespace dqrm_mx;

// A tensor as rows of values.  (Contiguous ones are a single row.)
struct Item {
    const char *data;
    char *out;            // where the scaled values go
    const int32_t *count; // rows that are there, or null: all
    int64_t rows, cols, ld, ld_out;
    unsigned first; // piece, of all tensors' pieces
    int32_t dtype;
};
constexpr int kItems = 48; // of a launch: its arguments have to stay below 4 KB

struct Batch {
    Item item[kItems];
    int items;
    unsigned first, pieces; // of this launch
    unsigned all;           // pieces of all tensors
    int64_t per_piece;      // vectors of 8 values
};

constexpr int kThreads = 256;
constexpr int kAhead = 4; // vectors of a thread that are on their way together

__device__ __forceinline__ int item_of(const Batch &b, unsigned piece)
{
    int lo = 0, hi = b.items - 1;
    while (lo < hi) { // the last item that begins at or before the piece
        const int mid = (lo + hi + 1) / 2;
        if (b.item[mid].first <= piece)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ int64_t rows_of(const Item &t)
{
    if (!t.count) return t.rows;
    const int64_t n = *t.count;
    return n < 0 ? 0 : min(n, t.rows);
}

// The thread's vectors of vectors [v0, v1) of a tensor, kAhead of them at a time: f(rows, columns, how many)
template <typename F>
__device__ __forceinline__ void for_vectors(int64_t rows_of_tensor, int64_t v0, int64_t v1, int64_t per_row, F f)
{
    int64_t v = v0 + threadIdx.x, r = 0, c = v, down = 0, right = kThreads;
    if (v >= v1) return;
    if (rows_of_tensor > 1) { // (a single row needs no divisions: they are most of a small tensor's time)
        r = v / per_row, c = v - r * per_row;
        down = kThreads / per_row, right = kThreads - down * per_row;
    }
    while (v < v1) {
        int64_t rows[kAhead], cols[kAhead];
        int n = 0;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (v < v1) {
                n = i + 1;
                rows[i] = r, cols[i] = c * kChunk;
            } else { // (the last one again)
                rows[i] = rows[i ? i - 1 : 0], cols[i] = cols[i ? i - 1 : 0];
            }
            v += kThreads, r += down, c += right;
            if (c >= per_row) c -= per_row, ++r;
        }
        f(rows, cols, n);
    }
}

// A vector of a row: those with 8 values and more load the last 8 where fewer are left
template <typename T, bool SHORT>
__device__ __forceinline__ void load_values(const T *row, int64_t c, int64_t cols, Raw<T> &raw)
{
    if constexpr (SHORT) {
        const Vec8<T> t = load_vec(row, c, cols, false);
        __builtin_memcpy(&raw, &t, sizeof(t));
    } else {
        raw = load_raw(row, c, cols);
    }
}
template <typename T, bool SHORT>
__device__ __forceinline__ void take_values(const Raw<T> &raw, int64_t c, int64_t cols, float (&v)[kChunk])
{
    if constexpr (SHORT) {
        Vec8<T> t;
        __builtin_memcpy(&t, &raw, sizeof(t));
        to_float(t, v);
    } else {
        values_of(raw, c, cols, v);
    }
}

// a vector to where it is copied to, bit for bit (a float that is a signalling NaN would not stay one)
template <typename T, bool SHORT>
__device__ __forceinline__ void copy_values(const Raw<T> &raw, int64_t c, int64_t cols, T *row)
{
    struct Bits { std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> v[kChunk]; } t;
    __builtin_memcpy(&t, &raw, sizeof(t));
    if constexpr (!SHORT) drop_before(t.v, c, cols);
    if (c + kChunk <= cols) {
        __builtin_memcpy(row + c, &t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (c + i < cols) __builtin_memcpy(row + c + i, &t.v[i], sizeof(T));
    }
}

// the tensor's type, and whether its rows are shorter than a vector
template <typename F>
__device__ __forceinline__ void with_item(const Item &t, F f)
{
    const auto typed = [&](auto zero) {
        if (t.cols < kChunk)
            f(zero, std::true_type{});
        else
            f(zero, std::false_type{});
    };
    if (t.dtype == DQRM_F32)
        typed(0.0f);
    else if (t.dtype == DQRM_BF16)
        typed((__bf16)0.0f);
    else
        typed((_Float16)0.0f);
}

template <int KIND>
__device__ __forceinline__ double join(double a, double b)
{
    if constexpr (KIND == DQRM_GRAD_NORM_2)
        return a + b;
    else
        return (a > b || a != a) ? a : b; // (a NaN stays)
}

// over the workgroup; every thread gets it
template <int KIND>
__device__ __forceinline__ double join_all(double v, double *s)
{
#pragma unroll
    for (int d = kWaveSize / 2; d >= 1; d >>= 1) v = join<KIND>(v, __shfl_xor(v, d, kWaveSize));
    if ((threadIdx.x & (kWaveSize - 1)) == 0) s[threadIdx.x / kWaveSize] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWaveSize; ++w) v = join<KIND>(v, s[w]);
    return v;
}

// parts [first, first + n) joined: in the same order wherever it is done
template <int KIND>
__device__ __forceinline__ double join_parts(const double *parts, unsigned first, unsigned n, double *s)
{
    double v = 0.0;
    constexpr unsigned ahead = 8; // loads in flight (a part past the last one is the last one again, and not added)
    for (unsigned i = threadIdx.x; i < n; i += kThreads * ahead) {
        double x[ahead];
#pragma unroll
        for (unsigned k = 0; k < ahead; ++k) x[k] = parts[first + min(i + k * kThreads, n - 1)];
#pragma unroll
        for (unsigned k = 0; k < ahead; ++k)
            if (i + k * kThreads < n) v = join<KIND>(v, x[k]);
    }
    return join_all<KIND>(v, s);
}

template <int KIND>
__device__ __forceinline__ float norm_of(double v)
{
    return (float)(KIND == DQRM_GRAD_NORM_2 ? sqrt(v) : v);
}

// A piece's sum of squares, or its largest magnitude.  Bound by its bytes: 1.07 G values in 400 tensors, 2.5 GB, nine launches of 61 us, 4.6 TB/s.
template <int KIND>
__global__ __launch_bounds__(kThreads) void grad_part_kernel(Batch b, double *parts)
{
    __shared__ double s[kThreads / kWaveSize];
    const unsigned piece = b.first + blockIdx.x;
    const Item &t = b.item[item_of(b, piece)];
    const int64_t per_row = (t.cols + kChunk - 1) / kChunk, v0 = (int64_t)(piece - t.first) * b.per_piece;
    const int64_t v1 = min(v0 + b.per_piece, rows_of(t) * per_row);
    double sum = 0.0;
    unsigned most = 0;
    with_item(t, [&](auto zero, auto is_short) {
        using T = decltype(zero);
        constexpr bool SHORT = decltype(is_short)::value;
        const T *data = reinterpret_cast<const T *>(t.data);
        for_vectors(t.rows, v0, v1, per_row, [&](const int64_t(&r)[kAhead], const int64_t(&c)[kAhead], int n) {
            Raw<T> raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load_values<T, SHORT>(data + r[i] * t.ld, c[i], t.cols, raw[i]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                float v[kChunk];
                take_values<T, SHORT>(raw[i], c[i], t.cols, v);
                if (i >= n) break;
#pragma unroll
                for (int k = 0; k < kChunk; ++k) {
                    if constexpr (KIND == DQRM_GRAD_NORM_2)
                        sum = fma((double)v[k], (double)v[k], sum);
                    else
                        most = max(most, abs_bits(v[k])); // (NaNs order above infinities above numbers)
                }
            }
        });
    });
    if constexpr (KIND != DQRM_GRAD_NORM_2) sum = (double)__uint_as_float(most);
    sum = join_all<KIND>(sum, s);
    if (threadIdx.x == 0) parts[piece] = sum;
}

__device__ __forceinline__ unsigned pieces_of(const Batch &b, int item)
{
    return (item + 1 < b.items ? b.item[item + 1].first : b.first + b.pieces) - b.item[item].first;
}

// A workgroup to each tensor's norm, and one to the norm of all.
template <int KIND>
__global__ __launch_bounds__(kThreads) void grad_join_kernel(Batch b, const double *parts, float *norms, int first_norm, float *norm)
{
    __shared__ double s[kThreads / kWaveSize];
    const int at = (int)blockIdx.x;
    const bool one = norms && at < b.items;
    const double v = join_parts<KIND>(parts, one ? b.item[at].first : 0u, one ? pieces_of(b, at) : b.all, s);
    if (threadIdx.x == 0) (one ? norms[first_norm + at] : *norm) = norm_of<KIND>(v);
}

// The values times max_norm / norm.  The norm is the joined parts', or given; a workgroup of a tensor that stays as it is ends there.  With
// parts, each tensor's norm is written beside (`norms`) by the workgroup of its first piece, an empty one's by the first of all.  Bound by its bytes, a
// read and a write: 2.5 GB of tensors nine times 125-131 us, 4.4 TB/s.
template <int KIND>
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Batch b, const double *parts, const float *given, float *norm, float *norms, float max_norm)
{
    __shared__ double s[2][kThreads / kWaveSize];
    const unsigned piece = b.first + blockIdx.x;
    const int item = item_of(b, piece);
    const Item &t = b.item[item];
    float total;
    if (parts) {
        total = norm_of<KIND>(join_parts<KIND>(parts, 0, b.all, s[0]));
        if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = total;
        if (norms) {
            if (blockIdx.x == 0 && (int)threadIdx.x < b.items && pieces_of(b, threadIdx.x) == 0) norms[threadIdx.x] = 0.0f;
            if (piece == t.first) {
                const double v = join_parts<KIND>(parts, t.first, pieces_of(b, item), s[1]);
                if (threadIdx.x == 0) norms[item] = norm_of<KIND>(v);
            }
        }
    } else {
        total = *given;
    }
    const bool scaled = total > max_norm && total < __builtin_inff(); // (not with a NaN)
    const float by = max_norm / total;
    if (!scaled && t.out == t.data) return;
    const int64_t per_row = (t.cols + kChunk - 1) / kChunk, v0 = (int64_t)(piece - t.first) * b.per_piece;
    const int64_t v1 = min(v0 + b.per_piece, rows_of(t) * per_row);
    with_item(t, [&](auto zero, auto is_short) {
        using T = decltype(zero);
        constexpr bool SHORT = decltype(is_short)::value;
        const T *data = reinterpret_cast<const T *>(t.data);
        T *out = reinterpret_cast<T *>(t.out);
        for_vectors(t.rows, v0, v1, per_row, [&](const int64_t(&r)[kAhead], const int64_t(&c)[kAhead], int n) {
            Raw<T> raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load_values<T, SHORT>(data + r[i] * t.ld, c[i], t.cols, raw[i]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (!scaled) {
                    if (i < n) copy_values<T, SHORT>(raw[i], c[i], t.cols, out + r[i] * t.ld_out);
                    continue;
                }
                float v[kChunk];
                take_values<T, SHORT>(raw[i], c[i], t.cols, v);
                if (i >= n) break;
#pragma unroll
                for (int k = 0; k < kChunk; ++k) v[k] *= by;
                store_chunk(out + r[i] * t.ld_out, c[i], t.cols, v);
            }
        });
    });
}

} // namespace dqrm_grad
