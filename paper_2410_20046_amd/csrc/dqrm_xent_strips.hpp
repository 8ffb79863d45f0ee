// Softmax cross entropy of up to 64 rows whose classes the tiles can't read where they are (fp32, or 16 bits at any alignment): w straight from memory
// into registers, each of its values once for the logits and once for dx (gfx950, wave64).
//
// Logits: a wave takes strips of 32 classes.  Of 16 values of a class's row, the 8 from 8 (l / 32) on are lane l's, of class l % 32: a step of the
// products, of which 4 read a line of each row in turn.  x lies in the order that goes with it.  fp32 is split into its three bfloat16 planes in
// registers.  dx: lane l has the column l % 32 of 8 classes in a step, a line of 32 columns to each half of the wave.
#pragma once

#include "dqrm_xent.hpp"

namespace dqrm_xent {

using v4u = unsigned __attribute__((ext_vector_type(4)));

template <int DT> struct Planes {
    using T = std::conditional_t<DT == DQRM_F16, _Float16, __bf16>; // of the products
    static constexpr int n = DT == DQRM_F32 ? 3 : 1, pairs = DT == DQRM_F32 ? (int)kPlanePairs : 1;
};

// eight values as operands of the products; ANY: also such as would round to infinity
template <int DT, bool ANY = true>
__device__ __forceinline__ void planes_of(const elem_t<DT> (&v)[kChunk], uint4 (&p)[Planes<DT>::n])
{
    if constexpr (DT == DQRM_F32) {
        struct alignas(16) Eight { __bf16 v[kChunk]; } e[3];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            __bf16 s[3];
            split<ANY>(v[i], s);
            e[0].v[i] = s[0], e[1].v[i] = s[1], e[2].v[i] = s[2];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) __builtin_memcpy(&p[k], &e[k], 16);
    } else {
        __builtin_memcpy(&p[0], &v, 16);
    }
}

// sum over the pairs of planes of a and b, the smallest first
template <int DT>
__device__ __forceinline__ v16f multiply_planes(const uint4 (&b)[Planes<DT>::n], const uint4 (&a)[Planes<DT>::n], v16f c)
{
#pragma unroll
    for (int k = 0; k < Planes<DT>::pairs; ++k)
        c = mfma_32x32x16<typename Planes<DT>::T>(b[Planes<DT>::n == 1 ? 0 : (0x118 >> (2 * k)) & 3], a[Planes<DT>::n == 1 ? 0 : (0x52 >> (2 * k)) & 3], c);
    return c;
}

// x in the order of the products: [chunk of 64 values][step][plane][block of 32 rows][lane] vectors of 16 bytes, zeros past rows and width.
template <int DT>
__global__ __launch_bounds__(256) void xent_strip_pack_kernel(const elem_t<DT> *x, int64_t ldx, int rows, int width, int blocks, int vectors, uint4 *out)
{
    constexpr int planes = Planes<DT>::n;
    const int at = blockIdx.x * 256 + threadIdx.x; // of [chunk][step][block][lane]
    if (at >= vectors) return;
    const int lane = at & 63, block = (at >> 6) % blocks, step = ((at >> 6) / blocks) & 3, chunk = (at >> 6) / blocks >> 2;
    const int r = block * 32 + (lane & 31), c = chunk * 64 + step * 16 + (lane >> 5) * kChunk;
    Vec8<elem_t<DT>> v{};
    if (r < rows) v = load_vec(x + r * ldx, c, width, false);
    uint4 p[planes];
    planes_of<DT>(v.v, p);
#pragma unroll
    for (int k = 0; k < planes; ++k) out[(((chunk * 4 + step) * planes + k) * blocks + block) * 64 + lane] = p[k];
}

// (what the logits' helpers ask of a tile)
template <int MB> struct StripTile {
    static constexpr int TM = MB, TN = 1;
};

struct StripArgs {
    const void *w;
    int64_t ldw, classes, first; // of this piece, its first one
    int width, rows, chunks, strips;
    const uint4 *x; // as xent_strip_pack_kernel lays it out
    const float *bias;
    float scale2;
    const int64_t *targets;
    // forward
    float2 *parts; // [workgroups][rows]
    float *at;
    // backward
    const float *lse, *grad, *most;
    const uint64_t *live;
    float by;
    char *d; // in blocks of 64 by 64: a row of blocks, their 64 rows all written
    int64_t plane;
    float *dbias; // of the piece, or null
};

// The logits of strips of 32 classes by MB blocks of 32 rows, and forward their maxima and sums, backward d.  The next 64 values of the strip (or the next
// strip's first) are on their way while these are multiplied; x, which all waves need, comes through LDS and is asked for before w, so that nobody
// awaits w for it (with x from memory in each wave: 640 us where it is 490 now).  457731 classes of width 1172 in fp32, 2.15 GB, forward: 9 rows
// 490 us, 4.4 TB/s, 59 rows 647; 200003 of width 1021 in bfloat16, 0.41 GB: 141 and 165.  The splitting in planes and the products share the time with
// the loads, and a lane's 16 bytes at a time with the lines that they are of.
template <int DT, int MB, bool GRAD>
__global__ __launch_bounds__(256) void xent_strip_kernel(StripArgs a)
{
    using T = elem_t<DT>;
    using Q = typename Planes<DT>::T;
    constexpr int planes = Planes<DT>::n;
    using S = StripTile<MB>;
    constexpr int vectors = 4 * planes * MB * 64; // of x to 64 values
    constexpr int mine = vectors / 256;
    __shared__ __align__(16) uint4 s_x[2][vectors];
    __shared__ float2 s_part[4][MB * 32];
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = (int)uniform(threadIdx.x >> 6);
    const int stride = (int)gridDim.x * 4;
    int64_t target[MB];
    RowLse lse[MB];
    float grad[MB], best[MB], sum[MB];
    bool live[MB];
    const float most = GRAD ? *a.most : 1.0f;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int r = b * 32 + (lane & 31);
        target[b] = r < a.rows ? a.targets[r] : -1;
        best[b] = -__builtin_inff(), sum[b] = 0.0f;
        if constexpr (GRAD) {
            live[b] = r < a.rows && (a.live[0] >> r) & 1;
            lse[b] = lse_of(live[b] ? a.lse[r] : 0.0f), grad[b] = live[b] ? a.grad[r] / most * lse[b].factor : 0.0f;
            if (!live[b]) target[b] = -1;
        }
    }
    Vec8<T> next[4];
    auto ask = [&](int strip, int chunk) {
        const int64_t r = min((int64_t)strip * 32 + (lane & 31), a.classes - 1);
        const T *row = static_cast<const T *>(a.w) + r * a.ldw;
        const int c = chunk * 64 + half * kChunk;
        if (chunk * 64 + 64 <= a.width) {
#pragma unroll
            for (int s = 0; s < 4; ++s) __builtin_memcpy(&next[s], row + c + s * 16, sizeof(next[s]));
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) next[s] = load_vec(row, c + s * 16, a.width, false);
        }
    };
    v4u x_next[mine];
    auto ask_x = [&](int chunk) {
#pragma unroll
        for (int i = 0; i < mine; ++i) x_next[i] = reinterpret_cast<const v4u *>(a.x)[(int64_t)chunk * vectors + i * 256 + (int)threadIdx.x];
    };
    auto put_x = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < mine; ++i) reinterpret_cast<v4u *>(s_x[buffer])[i * 256 + (int)threadIdx.x] = x_next[i];
    };
    int buffer = 0;
    ask_x(0);
    put_x(0);
    ask((int)blockIdx.x * 4 + wave, 0);
    __syncthreads();
    for (int four = (int)blockIdx.x * 4; four < a.strips; four += stride) { // (past the last strip, the last class is read)
        const int strip = four + wave;
        v16f acc[MB][1];
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[b][0] = v16f{};
        for (int chunk = 0; chunk < a.chunks; ++chunk) {
            Vec8<T> w[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = next[s];
            const bool more = chunk + 1 < a.chunks;
            ask_x(more ? chunk + 1 : 0); // (before w, whose arrival it need not await)
            ask(more ? strip : strip + stride, more ? chunk + 1 : 0);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                uint4 p[planes];
                planes_of<DT>(w[s].v, p);
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    uint4 x[planes];
#pragma unroll
                    for (int k = 0; k < planes; ++k) x[k] = s_x[buffer][((s * planes + k) * MB + b) * 64 + lane];
                    acc[b][0] = multiply_planes<DT>(p, x, acc[b][0]);
                }
            }
            buffer ^= 1;
            put_x(buffer); // (which the products before the last barrier read)
            __syncthreads();
        }
        if (strip >= a.strips) continue;
        const int64_t n0 = (int64_t)strip * 32;
        Classifier c{};
        c.g.n = a.classes, c.bias = a.bias, c.scale2 = a.scale2;
        logits<S, !GRAD>(c, acc, n0);
        int at[MB];
#pragma unroll
        for (int b = 0; b < MB; ++b) at[b] = place_of_target<S>(target[b], a.first + n0);
        if constexpr (!GRAD) {
            at_target<S>(at, [&](int b, int, int i) { a.at[b * 32 + (lane & 31)] = acc[b][0][i]; });
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                float top = best[b];
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, acc[b][0][i]);
                const float base = top == -__builtin_inff() ? 0.0f : top;
                sum[b] *= power2(best[b] - base);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[b] += power2(acc[b][0][i] - base);
                best[b] = top;
            }
        } else {
            float total[16] = {};
#pragma unroll
            for (int b = 0; b < MB; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float v = power2(acc[b][0][i] - lse[b].lse2);
                    v = (at[b] == (i >> 2) * 8 + half * 4 + (i & 3) ? v - lse[b].inverse : v) * grad[b];
                    acc[b][0][i] = live[b] ? v : 0.0f;
                    total[i] += acc[b][0][i];
                }
            }
            if (a.dbias) {
                const float all = sum_over_rows(total);
                const int i = (lane >> 1) & 15;
                const int64_t n = n0 + (i >> 2) * 8 + half * 4 + (i & 3);
                if (!(lane & 1) && n < a.classes) a.dbias[n] = all * most;
            }
            char *to = a.d + (n0 / kBlock) * kBlockBytes + (lane & 31) * (kBlock * 2) + (n0 % kBlock + half * 4) * 2;
#pragma unroll
            for (int k = 0; k < planes; ++k)
#pragma unroll
                for (int b = 0; b < 2; ++b) // (of a block's 64 rows those past MB blocks of 32 are zeros)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        struct alignas(8) Four { Q v[4]; } f{};
                        if (b < MB) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float v = acc[b < MB ? b : 0][0][q * 4 + i];
                                f.v[i] = (Q)(v * a.by);
                                if (k + 1 < planes) acc[b < MB ? b : 0][0][q * 4 + i] = v - (float)f.v[i]; // (by is 1 then)
                            }
                        }
                        *reinterpret_cast<Four *>(to + k * a.plane + b * 32 * (kBlock * 2) + q * 16) = f;
                    }
        }
    }
    if constexpr (!GRAD) {
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            float2 p = make_float2(best[b], sum[b]);
            p = join_parts(p, make_float2(__shfl_xor(p.x, 32, kWaveSize), __shfl_xor(p.y, 32, kWaveSize)));
            if (lane < 32) s_part[wave][b * 32 + lane] = p;
        }
        __syncthreads();
        if ((int)threadIdx.x < a.rows) {
            float2 p = s_part[0][threadIdx.x];
            for (int w = 1; w < 4; ++w) p = join_parts(p, s_part[w][threadIdx.x]);
            a.parts[(int64_t)blockIdx.x * a.rows + threadIdx.x] = p;
        }
    }
}

struct StripDxArgs {
    const void *w;
    int64_t ldw, classes;
    int width, rows, columns; // blocks of 64 columns
    const char *d;
    int64_t plane;
    const uint64_t *live; // classes that are not taken out, or null
    int blocks, per_slice; // of 64 classes: in all, of a workgroup
    float *sums;          // [slices][rows][width]
    bool add;
};

// dx's sums over a slice of the classes, 64 columns to a workgroup, whose waves take every fourth 64 classes and then add up.  (65536 classes of width 1172
// in fp32, 0.31 GB: 9 rows 115 us, 59 rows 184.  With the next step's loads on their way the registers are twice as many and the waves half.)
template <int DT, int MB>
__global__ __launch_bounds__(256) void xent_strip_dx_kernel(StripDxArgs a)
{
    using T = elem_t<DT>;
    constexpr int planes = Planes<DT>::n;
    __shared__ float s_sum[MB * 32][64 + 1];
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = (int)uniform(threadIdx.x >> 6);
    const int slice = (int)(blockIdx.x / a.columns), column = (int)blockIdx.x - slice * a.columns;
    const int last = min((slice + 1) * a.per_slice, a.blocks);
    v16f acc[MB][2];
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[b][0] = acc[b][1] = v16f{};
    int c[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) c[j] = min(column * 64 + j * 32 + (lane & 31), a.width - 1); // (a column past the last one is not stored)
    for (int block = slice * a.per_slice + wave; block < last; block += 4) {
        const uint64_t live = a.live ? a.live[block] : ~0ull;
        const bool whole = (int64_t)(block + 1) * 64 <= a.classes;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = 16 * s + 8 * half; // of the block's classes
            T v[2][kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const int64_t r = (int64_t)block * 64 + at + i;
                const T *row = static_cast<const T *>(a.w) + (whole ? r : min(r, a.classes - 1)) * a.ldw;
#pragma unroll
                for (int j = 0; j < 2; ++j) v[j][i] = row[c[j]];
            }
            if (a.live || !whole) {
#pragma unroll
                for (int i = 0; i < kChunk; ++i)
                    if (!((live >> (at + i)) & 1) || (int64_t)block * 64 + at + i >= a.classes) v[0][i] = v[1][i] = (T)0.0f;
            }
            uint4 p[2][planes];
#pragma unroll
            for (int j = 0; j < 2; ++j) planes_of<DT>(v[j], p[j]);
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                uint4 d[planes];
#pragma unroll
                for (int k = 0; k < planes; ++k)
                    d[k] = *reinterpret_cast<const uint4 *>(a.d + k * a.plane + (int64_t)block * kBlockBytes + (b * 32 + (lane & 31)) * (kBlock * 2) + at * 2);
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[b][j] = multiply_planes<DT>(p[j], d, acc[b][j]);
            }
        }
    }
    // the waves in turn
    for (int w = 0; w < 4; ++w) {
        if (wave == w) {
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float &s = s_sum[b * 32 + (lane & 31)][j * 32 + (i >> 2) * 8 + half * 4 + (i & 3)];
                        s = w == 0 ? acc[b][j][i] : s + acc[b][j][i];
                    }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < MB * 32 * 64; i += 256) {
        const int r = i >> 6, col = column * 64 + (i & 63);
        if (r < a.rows && col < a.width) {
            float *to = a.sums + ((int64_t)slice * a.rows + r) * a.width + col;
            *to = a.add ? *to + s_sum[r][i & 63] : s_sum[r][i & 63];
        }
    }
}

} // namespace dqrm_xent
