#pragma once

#include <hip/hip_runtime.h>

namespace dqrm {

// unsigned division of numbers below 2^31 by a fixed divisor (host-side set-up)
struct FastDiv {
    unsigned magic, shift, d;
    __host__ static FastDiv make(unsigned divisor)
    {
        FastDiv f;
        unsigned l = 0;
        while ((1u << l) < divisor) ++l;
        // ceil(2^(31 + l) / d) < 2^32 for d >= 2; exact quotients for every dividend below 2^31
        const unsigned long long p = 1ull << (31 + l);
        f.magic = divisor > 1 ? (unsigned)((p + divisor - 1) / divisor) : 0u;
        f.shift = l > 0 ? l - 1 : 0;
        f.d = divisor;
        return f;
    }
    __device__ __forceinline__ unsigned div(unsigned x) const { return d > 1 ? __umulhi(x, magic) >> shift : x; }
};

} // namespace dqrm
