// n / d for n < 2^31 and a d that the host knows: (mulhi(n, mul) + n) >> shift, mul = ceil(2^(32 + shift) / d) - 2^32.
#pragma once
#include <hip/hip_runtime.h>

struct Divisor {
    unsigned d = 1, mul = 1, shift = 0;
    Divisor() = default;
    explicit Divisor(unsigned x) : d(x), shift(0)
    {
        while ((1ull << shift) < x) ++shift;
        mul = (unsigned)(((1ull << 32) * ((1ull << shift) - x)) / x + 1);
    }
    __host__ __device__ __attribute__((always_inline)) unsigned operator()(unsigned n) const
    {
        return ((unsigned)(((unsigned long long)n * mul) >> 32) + n) >> shift;
    }
};
