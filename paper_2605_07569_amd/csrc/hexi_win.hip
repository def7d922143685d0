// Attention under a sliding window with sink tokens: dispatch, and the kernels that follow the definition.
#include "hexi_window_plain.h"
#include <type_traits>

namespace {

template <class T, int D> __global__ void __launch_bounds__(256) win_fwd_kernel(const WinFwdArgs a)
{
    win_plain::fwd_unit<T, D>(a, (int)blockIdx.x % a.g.nq, (int)blockIdx.x / a.g.nq * win_plain::ROWS);
}
template <class T, int D> __global__ void __launch_bounds__(256) win_bwd_kernel(const WinBwdArgs a, const int n_dkdv)
{
    if ((int)blockIdx.x < n_dkdv) win_plain::dkdv_unit<T, D>(a, (int)blockIdx.x % a.g.nkv, (int)blockIdx.x / a.g.nkv * win_plain::ROWS);
    else win_plain::dq_unit<T, D>(a, ((int)blockIdx.x - n_dkdv) % a.g.nq, ((int)blockIdx.x - n_dkdv) / a.g.nq * win_plain::ROWS);
}

// f(element type, head_dim)
template <class F> void with_type(int dtype, int d, F f)
{
    if (dtype == HEXI_F32) { if (d == 128) f(float{}, std::integral_constant<int, 128>{}); else f(float{}, std::integral_constant<int, 64>{}); }
    else if (d == 128) f(uint16_t{}, std::integral_constant<int, 128>{});
    else f(uint16_t{}, std::integral_constant<int, 64>{});
}

}  // namespace

hipError_t hexi_launch_win_fwd(const WinFwdArgs& a, int dtype, hipStream_t s)
{
    if (dtype == HEXI_BF16) return hexi_launch_win_fwd_quad_bf16(a, s);
    const unsigned grid = (unsigned)((a.g.lq + win_plain::ROWS - 1) / win_plain::ROWS) * (unsigned)a.g.nq;
    with_type(dtype, a.g.d, [&](auto t, auto d) { win_fwd_kernel<decltype(t), decltype(d)::value><<<grid, 256, 0, s>>>(a); });
    return hipGetLastError();
}

hipError_t hexi_launch_win_bwd(const WinBwdArgs& a, int dtype, hipStream_t s)
{
    if (dtype == HEXI_BF16) return hexi_launch_win_bwd_quad_bf16(a, s);
    const int n_dkdv = a.want_dkdv ? (a.g.lc + win_plain::ROWS - 1) / win_plain::ROWS * a.g.nkv : 0;
    const int n_dq = a.want_dq ? (a.g.lq + win_plain::ROWS - 1) / win_plain::ROWS * a.g.nq : 0;
    with_type(dtype, a.g.d, [&](auto t, auto d) { win_bwd_kernel<decltype(t), decltype(d)::value><<<(unsigned)(n_dkdv + n_dq), 256, 0, s>>>(a, n_dkdv); });
    return hipGetLastError();
}

namespace {

// Delta of one (row, head): D / 8 lanes, 8 columns each.
template <class T, int D>
__global__ void __launch_bounds__(256) delta_bf16_o_kernel(long long lq, int nq, const uint16_t* __restrict__ o, const T* __restrict__ d_o,
                                                           long long stride_tok, long long stride_head, float* __restrict__ delta)
{
    constexpr int LANES = D / 8;
    const long long rh = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int c = threadIdx.x % LANES * 8;
    const bool valid = rh < lq * nq;
    const long long row = valid ? rh / nq : 0;
    const int h = valid ? (int)(rh - row * nq) : 0;
    float acc = 0.f;
    if (valid) {
        float x[8], y[8];
        win_plain::load_cols(o + rh * D + c, x);
        win_plain::load_cols(d_o + row * stride_tok + h * stride_head + c, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc = fmaf(x[i], y[i], acc);
    }
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) acc += __shfl_xor(acc, off, 64);
    if (valid && c == 0) delta[(long long)h * lq + row] = acc;
}

}  // namespace

hipError_t hexi_launch_delta_bf16_o(long long lq, int nq, int d, const void* o, const void* d_o, int dtype,
                                    long long stride_tok, long long stride_head, float* delta, hipStream_t s)
{
    const unsigned grid = (unsigned)((lq * nq * (d / 8) + 255) / 256);
    with_type(dtype, d, [&](auto t, auto dd) {
        delta_bf16_o_kernel<decltype(t), decltype(dd)::value><<<grid, 256, 0, s>>>(lq, nq, (const uint16_t*)o, (const decltype(t)*)d_o, stride_tok, stride_head, delta);
    });
    return hipGetLastError();
}
