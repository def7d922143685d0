// Products of 16 query vectors with 16 keys by one wavefront, straight from memory: shared by the kernels for few rows.
//
// S^T[key][vector] = K Q^T: lane (g, l), g = lane / 16, holds row l of either.  A lane then has keys 4 g + e of ONE vector, l, and P as it stands is an operand of
// O^T[column][vector] = V^T P^T, whose other operand it makes of rows 4 g + e of V.
#pragma once
#include "hexi_blocks.h"
#include "hexi_f32_common.h"

namespace {

// Operands and products by element type: ROW loads of 16 bytes to a row of q or k per lane; a lane's PIECE of neighbouring columns of a row of v.
template <class T, int D> struct Ops;
template <int D> struct Ops<float, D> {
    static constexpr int ROW = D / 16, PIECE = 4, NC = D / 16;     // (D = 128: the piece is twice 4 columns, 64 apart)
    f32x4 k[ROW], v[4][D / 64];
    // columns 16 i + 4 g .. + 3 of a row
    static __device__ __forceinline__ void row(f32x4 (&x)[ROW], const float* p, int g)
    {
#pragma unroll
        for (int i = 0; i < ROW; ++i) x[i] = *reinterpret_cast<const f32x4*>(p + 16 * i + 4 * g);
    }
    __device__ __forceinline__ void values(int e, const float* p, int l)
    {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) v[e][i] = *reinterpret_cast<const f32x4*>(p + 64 * i + 4 * l);
    }
    __device__ __forceinline__ f32x4 scores(const f32x4 (&q)[ROW]) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROW; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q[i][e], s, 0, 0, 0);
        return s;
    }
    // acc[c] += ...; l: sum of p as it is multiplied
    __device__ __forceinline__ void sums(f32x4 (&acc)[NC], const f32x4& p, float& l) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            l += p[e];
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][c / 4][c % 4], p[e], acc[c], 0, 0, 0);
        }
    }
    // column of row r of product c (r = 4 g + register)
    static __device__ __forceinline__ int column(int c, int r) { return 64 * (c / 4) + 4 * r + c % 4; }
};
template <int D> struct Ops<uint16_t, D> {
    static constexpr int ROW = D / 32, PIECE = D / 16, NC = D / 16;
    bf16x8 k[ROW];
    uint32_t v[4][PIECE / 2];
    static __device__ __forceinline__ void row(bf16x8 (&x)[ROW], const uint16_t* p, int g)
    {
#pragma unroll
        for (int i = 0; i < ROW; ++i) x[i] = *reinterpret_cast<const bf16x8*>(p + 32 * i + 8 * g);
    }
    __device__ __forceinline__ void values(int e, const uint16_t* p, int l)
    {
        if constexpr (PIECE == 8) {
            const uint4 x = *reinterpret_cast<const uint4*>(p + 8 * l);
            v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(p + 4 * l);
            v[e][0] = x.x; v[e][1] = x.y;
        }
    }
    __device__ __forceinline__ f32x4 scores(const bf16x8 (&q)[ROW]) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROW; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q[i], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void sums(f32x4 (&acc)[NC], const f32x4& p, float& l) const
    {
        const bf16x4 b = {(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) l += (float)b[e];
        products(acc, __builtin_bit_cast(s16x4, b));
    }
    // with weights of 16 bits, the rounded ones and what rounding left of them
    __device__ __forceinline__ void sums_fine(f32x4 (&acc)[NC], const f32x4& p, float& l) const
    {
        const bf16x4 b = {(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
        const bf16x4 rest = {(__bf16)(p[0] - (float)b[0]), (__bf16)(p[1] - (float)b[1]), (__bf16)(p[2] - (float)b[2]), (__bf16)(p[3] - (float)b[3])};
#pragma unroll
        for (int e = 0; e < 4; ++e) l += (float)b[e] + (float)rest[e];
        products(acc, __builtin_bit_cast(s16x4, b));
        products(acc, __builtin_bit_cast(s16x4, rest));
    }
    __device__ __forceinline__ void products(f32x4 (&acc)[NC], const s16x4& pb) const
    {
#pragma unroll
        for (int i = 0; i < PIECE / 2; ++i) {      // columns 2 i (low halves) and 2 i + 1 (high ones) of the four rows
            const uint2 lo = {__builtin_amdgcn_perm(v[1][i], v[0][i], 0x05040100), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x05040100)};
            const uint2 hi = {__builtin_amdgcn_perm(v[1][i], v[0][i], 0x07060302), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x07060302)};
            acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, lo), pb, acc[2 * i], 0, 0, 0);
            acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, hi), pb, acc[2 * i + 1], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ int column(int c, int r) { return PIECE * r + c; }
};

__device__ __forceinline__ float over_groups(float x, bool maximum)      // over lanes l, l + 16, l + 32, l + 48
{
    const float y = __shfl_xor(x, 16, 64);
    x = maximum ? fmaxf(x, y) : x + y;
    const float z = __shfl_xor(x, 32, 64);
    return maximum ? fmaxf(x, z) : x + z;
}

}  // namespace
