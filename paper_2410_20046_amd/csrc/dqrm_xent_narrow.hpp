// Softmax cross entropy for widths up to 64: its gradients without d in memory (gfx950, wave64).
//
// A sum over 64 values takes less time than d takes to memory and back: so the logits are computed twice, once beside each gradient.
// A wave holds 32 rows of x (for the loss and dx) or of w (for dw) in registers; the other matrix comes through LDS, 64 of its rows at a time.  Lane l has
// the logits of its row l % 32 with 16 of 32 others; what d needs becomes the operand of the second product where it is, since the
// order in which that sum takes the others is free: in a step of 16, lane l has those at 4 (l / 32) and at 8 + 4 (l / 32), and the
// transposing read gives the other operand in the same order.
#pragma once

#include "dqrm_xent_strips.hpp"

namespace dqrm_xent {

struct NarrowArgs {
    Operand x, w; // with the rows that have a gradient; with the classes that are not taken out, or null
    int64_t rows, classes;
    int width;
    const float *bias;
    float scale2;
    const int64_t *targets;
    int64_t first; // class of the piece
    unsigned tiles, stages, per_slice;
    // loss
    float2 *parts; // [slices][rows]
    float *at;
    // gradients
    const float *lse, *grad, *most;
    float by; // d is held times this
    float *sums; // [slices][rows or classes][width]
    bool add;
    float *dbias; // dw: [slices][classes], or null
};

// Bound by the matrix instructions and the vector ones beside them: 8192 rows, 200003 classes, width 64 in fp32 (six products), loss 1.06-1.13 ms, 1.1-1.2
// PFLOP/s, dx and dw 1.9-2.0 each, 1.3 PFLOP/s with the logits, where a large library product has 1.46.  d in memory would be 29 GB of traffic.  In bf16
// vector instructions bound it (an exponential takes as long as four others): 0.47-0.49, 0.59 and 0.67 ms, 3-6 % of the loss for the look for
// infinities.  Three workgroups to a CU, as LDS has it for three planes; the loop over the two blocks is not unrolled: its operands' addresses and
// reads would take the registers of a wave.
enum class Narrow { loss, dx, dw };

template <int DT, int KS, Narrow WHAT>
__global__ __launch_bounds__(256, 3) void xent_narrow_kernel(NarrowArgs a)
{
    using Q = typename Planes<DT>::T;
    using C = Carrier<64, 4, false, false>;
    constexpr bool LOSS = WHAT == Narrow::loss, DW = WHAT == Narrow::dw;
    constexpr int planes = Planes<DT>::n, CB = (KS + 1) / 2, plane_bytes = 64 * kStageRow, stage_bytes = planes * plane_bytes;
    __shared__ __align__(1024) char lds[2 * stage_bytes];
    __shared__ __align__(16) float s_a[2][64], s_b[2][64]; // of the 64 others: bias; lse and gradient
    __shared__ __align__(16) float s_one[2][64];           // ... and what a target's place is less
    __shared__ __align__(16) int s_target[2][64];
    const int lane = threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6), half = lane >> 5;
    const Operand &held = DW ? a.w : a.x, &others = DW ? a.x : a.w;
    const int64_t held_rows = DW ? a.classes : a.rows;
    // (each of the chip's parts gets a run of tiles, which read the same others)
    const unsigned part = blockIdx.x % kParts, per_part = gridDim.x / kParts, more = gridDim.x % kParts;
    const unsigned place = part * per_part + min(part, more) + blockIdx.x / kParts;
    const unsigned slice = uniform(place / a.tiles), tile = uniform(place - slice * a.tiles);
    const unsigned first = slice * a.per_slice, last = min(a.stages, first + a.per_slice);
    const int64_t row = (int64_t)tile * 128 + wave * 32 + (lane & 31);
    const bool inside = row < held_rows;
    const float most = LOSS ? 1.0f : *a.most;

    const bool there = inside && !(DW && a.bias && taken_out(a.bias[row]));
    uint4 mine[KS][planes];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int k = 0; k < planes; ++k)
            mine[s][k] = there && s * 16 + half * 8 < held.cols ? *reinterpret_cast<const uint4 *>(held.p + k * held.plane + row * held.pitch + s * 32 + half * 16)
                                                                 : make_uint4(0, 0, 0, 0);
    // of the lane's row: loss: target; dx: lse, gradient and target; dw: bias
    float lse2 = 0.0f, one = 1.0f, grad = 0.0f, bias2 = -__builtin_inff();
    int64_t target = -1;
    if constexpr (DW) {
        if (inside) bias2 = a.bias ? a.bias[row] * kLog2e : 0.0f;
    } else if constexpr (LOSS) {
        if (inside) target = a.targets[row] - a.first;
    } else if (inside && (a.x.live[row >> 6] >> (row & 63)) & 1) {
        const RowLse lse = lse_of(a.lse[row]);
        lse2 = lse.lse2, one = lse.inverse, grad = a.grad[row] / most * lse.factor, target = a.targets[row] - a.first;
    }
    const C carrier(others, lane, wave);
    const unsigned lds0 = uniform(lds_address(lds));
    auto request = [&](unsigned stage, int buffer) {
        const uint64_t live = others.live ? others.live[stage] : ~0ull;
#pragma unroll
        for (int k = 0; k < planes; ++k) {
            const rsrc_t r = C::memory(others, (unsigned)k, (int64_t)stage * 64, 0);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const unsigned j = (unsigned)(q * 4 + wave);
                const bool wanted = carrier.vector < 2 * KS && (live >> (j * 8 + carrier.row)) & 1;
                load16_to_lds(r, wanted ? carrier.offset(others, j, 0, 0) : kNowhere, lds0 + (unsigned)(buffer * stage_bytes + k * plane_bytes) + j * 1024);
            }
        }
    };
    // what goes with the others, by the first wave: asked for with their stage, made of it when that is computed
    float side_a = 0.0f, side_b = 0.0f;
    int side_target = -1;
    auto ask_side = [&](unsigned stage) {
        if (threadIdx.x >= 64) return;
        const int64_t r = (int64_t)stage * 64 + lane;
        if constexpr (DW) {
            const bool live = r < a.rows && (a.x.live[stage] >> lane) & 1;
            const int64_t t = live ? a.targets[r] - a.first : -1;
            side_a = live ? a.lse[r] : 0.0f, side_b = live ? a.grad[r] : 0.0f, side_target = t >= 0 && t < a.classes ? (int)t : -1;
        } else {
            side_a = r >= a.classes ? -__builtin_inff() : a.bias ? a.bias[r] : 0.0f;
        }
    };
    auto put_side = [&](int buffer) {
        if (threadIdx.x >= 64) return;
        if constexpr (DW) {
            const RowLse lse = lse_of(side_a);
            s_a[buffer][lane] = lse.lse2, s_b[buffer][lane] = side_b / most * lse.factor, s_one[buffer][lane] = lse.inverse, s_target[buffer][lane] = side_target;
        } else {
            s_a[buffer][lane] = side_a * kLog2e;
        }
    };
    // the lane's place in a transposing read of 8 rows by 32 columns c and half i of a step: row 4 half + j / 4 (j: lane % 16) of them, the vector of its 4
    // columns where the row's number exchanges it (i exchanges the halves of the row)
    const unsigned across = lds0 + (unsigned)((4 * half + ((lane & 15) >> 2)) * kStageRow + ((((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) ^ (2 * half + ((lane >> 3) & 1))) * 16 +
                                              (lane & 1) * 8);
    v16f out[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) out[c] = v16f{};
    float column = 0.0f;                        // dw: sum of the row's d
    float best = -__builtin_inff(), sum = 0.0f; // loss: of the row's logits
    int buffer = 0;
    if (first < last) {
        ask_side(first);
        request(first, 0);
        put_side(0);
    }
    for (unsigned s = first; s < last; ++s, buffer ^= 1) {
        lds_barrier();
        if (s + 1 < last) {
            ask_side(s + 1);
            request(s + 1, buffer ^ 1);
        }
        const char *now = lds + buffer * stage_bytes;
#pragma unroll 1
        for (int block = 0; block < 2; ++block) {
            v16f acc{};
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                uint4 o[planes];
#pragma unroll
                for (int k = 0; k < planes; ++k) o[k] = C::read(now + k * plane_bytes, block, t, lane);
                acc = multiply_planes<DT>(o, mine[t], acc);
            }
            // what is rare is looked for once: a target among the block's logits, a class that is taken out, an infinity.  (Gradients need not look for those: their
            // operands are zeros.)
            const int64_t at = target - ((int64_t)s * 64 + block * 32);
            int place_of = at >= 0 && at < 32 ? (int)at : -1;
            bool some_out = false;
            if constexpr (LOSS) some_out = __any(s_a[buffer][block * 32 + (lane & 31)] == -__builtin_inff());
            if constexpr (DW) place_of = s_target[buffer][block * 32 + (lane & 31)] - (int)(row - (lane & 31)); // (of a row among the wave's classes)
            const bool hit = __any(place_of >= 0 && place_of < 32);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(&s_a[buffer][block * 32 + q * 8 + half * 4]);
                const float side[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float l = __builtin_fmaf(acc[q * 4 + i], a.scale2, DW ? bias2 : side[i]);
                    acc[q * 4 + i] = LOSS ? l : power2(l - (DW ? side[i] : lse2));
                }
            }
            if constexpr (LOSS) {
                float least = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) least = fminf(least, acc[i]);
                if (some_out || __any(least == -__builtin_inff())) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float b = s_a[buffer][block * 32 + (i >> 2) * 8 + half * 4 + (i & 3)];
                        acc[i] = b == -__builtin_inff() ? b : no_infinity(acc[i]);
                    }
                }
            }
            if constexpr (LOSS) {
                if (hit) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (place_of == (i >> 2) * 8 + half * 4 + (i & 3)) a.at[row] = acc[i];
                }
                float top = best;
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, acc[i]);
                const float base = top == -__builtin_inff() ? 0.0f : top;
                float part = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) part += power2(acc[i] - base);
                sum = sum * power2(best - base) + part, best = top;
                continue;
            }
            if (hit) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int from = q * 8 + half * 4;
                    int4 t{};
                    float4 o = make_float4(one, one, one, one);
                    if constexpr (DW) {
                        t = *reinterpret_cast<const int4 *>(&s_target[buffer][block * 32 + from]);
                        o = *reinterpret_cast<const float4 *>(&s_one[buffer][block * 32 + from]);
                    }
                    const int targets[4] = {t.x, t.y, t.z, t.w};
                    const float ones[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[q * 4 + i] -= (DW ? targets[i] == (int)row : place_of == from + i) ? ones[i] : 0.0f;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float4 v{};
                if constexpr (DW) v = *reinterpret_cast<const float4 *>(&s_b[buffer][block * 32 + q * 8 + half * 4]);
                const float side[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (a row without a gradient, whatever its logits are: dx of such a row is not what the sums are)
                    if constexpr (DW) {
                        acc[q * 4 + i] = side[i] == 0.0f ? 0.0f : acc[q * 4 + i] * side[i];
                        column += acc[q * 4 + i];
                    } else {
                        acc[q * 4 + i] *= grad;
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint4 d[planes];
                if constexpr (DT == DQRM_F32) {
                    float v[kChunk];
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) v[i] = acc[8 * t + i];
                    planes_of<DT, false>(v, d);
                } else {
                    Q v[kChunk];
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) v[i] = (Q)(acc[8 * t + i] * a.by);
                    __builtin_memcpy(&d[0], &v, 16);
                }
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    uint4 o[planes];
#pragma unroll
                    for (int k = 0; k < planes; ++k) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const unsigned from = across + (unsigned)(buffer * stage_bytes + k * plane_bytes + (block * 32 + 16 * t + 8 * i) * kStageRow + (c ^ i) * 64);
                            const short4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)(uintptr_t)from);
                            __builtin_memcpy(reinterpret_cast<char *>(&o[k]) + 8 * i, &x, 8);
                        }
                    }
                    out[c] = multiply_planes<DT>(o, d, out[c]);
                }
            }
        }
        if (s + 1 < last) put_side(buffer ^ 1); // (which nobody has read since the barrier)
    }
    if constexpr (LOSS) {
        const float2 all = join_parts(make_float2(best, sum), make_float2(__shfl_xor(best, 32, kWaveSize), __shfl_xor(sum, 32, kWaveSize)));
        if (inside && lane < 32) a.parts[(int64_t)slice * a.rows + row] = all;
        return;
    }
    if (inside) {
        float *to = a.sums + ((int64_t)slice * held_rows + row) * a.width;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = c * 32 + q * 8 + half * 4;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = !DW && grad == 0.0f ? 0.0f : out[c][q * 4 + i];
                if (!a.add && col + 4 <= a.width) {
                    __builtin_memcpy(to + col, v, sizeof(v));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col + i < a.width) to[col + i] = a.add ? to[col + i] + v[i] : v[i];
                }
            }
    }
    if constexpr (DW) {
        column += __shfl_xor(column, 32, kWaveSize);
        if (a.dbias && inside && lane < 32) a.dbias[(int64_t)slice * a.classes + row] = column * most;
    }
}

} // namespace dqrm_xent
