// Attention under a sliding window with sink tokens: the fp32 kernels (units of hexi_f32_units.h on windowed runs of keys and rows), dispatch, and Delta from a
// bf16 o.  The bf16 kernels are those of hexi_bf16_quad.h and hexi_bf16_fwd.hip.
#include "hexi_f32_units.h"
#include <type_traits>

namespace {

template <int D, bool SPLIT, bool TWO> using Cfg = rows16::F32Cfg<D, SPLIT, TWO>;

template <int D, bool SPLIT, bool TWO>
__global__ void __launch_bounds__((64 * Cfg<D, SPLIT, TWO>::NW), TWO ? 4 : 1) win_fwd_f32_kernel(const WinFwdArgs a)
{
    using C = Cfg<D, SPLIT, TWO>;
    __shared__ __attribute__((aligned(1024))) rows16::FwdSmem<C> sm;
    const int tile = __builtin_amdgcn_readfirstlane(blockIdx.x / (unsigned)a.g.nq);
    rows16::fwd_unit<C, true>(a, (int)blockIdx.x - tile * a.g.nq, tile, sm, (int)blockIdx.y);
}

// Workgroups [0, n_dkdv) are dK / dV units, the others dQ units.
template <int D, bool SPLIT, bool TWO>
__global__ void __launch_bounds__((64 * Cfg<D, SPLIT, TWO>::NW), TWO ? 4 : SPLIT ? 1 : 2) win_bwd_f32_kernel(const WinBwdArgs a, const unsigned n_dkdv)
{
    using C = Cfg<D, SPLIT, TWO>;
    __shared__ __attribute__((aligned(1024))) union { rows16::DkdvSmem<C> dkdv; rows16::DqSmem<C> dq; } sm;
    if (blockIdx.x < n_dkdv) {
        const WinUnit unit(a, C::ROWS, (int)blockIdx.x);
        rows16::dkdv_unit<C, true>(a, unit.kvh, unit.tile, sm.dkdv, 0, a.g.nq, false, &unit);
    } else {
        const unsigned unit = blockIdx.x - n_dkdv;
        const int tile = __builtin_amdgcn_readfirstlane(unit / (unsigned)a.g.nq);
        rows16::dq_unit<C, true>(a, (int)unit - tile * a.g.nq, a.q_tile(tile), sm.dq);
    }
}

// f(configuration)
template <class F> hipError_t with_cfg(int d, bool split, F f)
{
    if (d == 128) { if (split) f(Cfg<128, true, false>{}); else f(Cfg<128, false, false>{}); }
    else if (split) f(Cfg<64, true, true>{});
    else f(Cfg<64, false, false>{});
    return hipGetLastError();
}

}  // namespace

static hipError_t launch_fwd(const WinFwdArgs& a, int dtype, hipStream_t s)
{
    if (a.few) return hexi_launch_win_few(a, dtype, s);
    if (dtype == HEXI_BF16) {
        if (a.n_splits == 1 && hexi_win_fwd_large(a.g, a.window, a.n_sink)) return hexi_launch_win_fwd_large_bf16(a, s);
        return (a.n_splits > 1 ? a.rows32 != 0 : hexi_win_fwd_rows32(a.g, a.window, a.n_sink)) ? hexi_launch_win_fwd_split_bf16(a, s) : hexi_launch_win_fwd_quad_bf16(a, s);
    }
    const AttnGeom& g = a.g;
    const bool split = a.n_splits > 1 || hexi_win_f32_split(0, g, a.window, a.n_sink);      // (runs of keys that are split further are 16-row units')
    return with_cfg(g.d, split, [&](auto cfg) {
        using C = decltype(cfg);
        const unsigned grid = (unsigned)((a.g.lq + C::ROWS - 1) / C::ROWS) * (unsigned)a.g.nq;
        win_fwd_f32_kernel<C::D, C::SPLIT, C::TWO><<<dim3(grid, (unsigned)a.n_splits), 64 * C::NW, 0, s>>>(a);
    });
}

hipError_t hexi_launch_win_fwd(const WinFwdArgs& a, int dtype, hipStream_t s)
{
    const hipError_t e = launch_fwd(a, dtype, s);
    return e != hipSuccess || a.n_splits == 1 ? e : hexi_launch_win_join(a, s);
}

namespace {

// A thread adds four columns of a key's dV or dK over the parts, in their order; 128 / (D / 4) keys a workgroup.
template <class T, int D> __global__ void __launch_bounds__(256) win_parts_kernel(const WinBwdArgs a, const int keys)
{
    constexpr int D4 = D / 4, R = 128 / D4;
    const AttnGeom& g = a.g;
    const int groups = keys / R, tid = threadIdx.x;
    const int tk = (int)blockIdx.x / groups, first = ((int)blockIdx.x - tk * groups) * R, tile = tk / g.nkv, kvh = tk - tile * g.nkv;
    const bool sink = tile < a.sink_tiles;
    const int n = sink ? a.n_sink_parts : a.n_parts;
    const long long units = sink ? (long long)tile * n : (a.n_sink_parts > 1 ? (long long)a.sink_tiles * a.n_sink_parts : 0) + (long long)(tile - a.sink_tiles) * n;
    const int which = tid / 128, r = first + tid % 128 / D4, c = 4 * (tid % D4), key = tile * keys + r;
    const float* p = a.part + (((units * g.nkv + kvh) * 2 + which) * keys + r) * D + c;
    const long long step = 2ll * g.nkv * keys * D;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < n; ++i) x += *reinterpret_cast<const f32x4*>(p + i * step);
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) z = fmaf(x[e], 0.f, z);
    if (__syncthreads_or(z != 0.f && key < g.lc)) {      // (keys a row does not see have P = 0, and 0 x inf is NaN)
        win_plain::dkdv_unit<T, D>(a, kvh, tile * keys + first, R);
        return;
    }
    if (key >= g.lc) return;
    float* const out = which ? a.dk : a.dv;
    const long long at = ((long long)key * g.nkv + kvh) * D + c;
    if (a.accumulate) x += *reinterpret_cast<const f32x4*>(out + at);
    win_plain::store4(out, at, a.out_bf16, x[0], x[1], x[2], x[3]);
}

}  // namespace

WinBwdArgs hexi_win_tiles_of(const WinBwdArgs& a, int keys)
{
    WinBwdArgs b = a;
    b.sink_tiles = a.n_sink_parts > 1 ? (seg_rows_le(a.g.ks, a.n_sink - 1) + keys - 1) / keys : 0;
    if (b.sink_tiles == 0) b.n_sink_parts = 1;
    // Rows (keys) in the middle see (are seen by) no fewer than those at the ends, so the ends say where the longest units are: of a step in front of the shard the last keys and
    // the first rows, without an end to the window the first keys and the last rows.
    const AttnGeom& g = a.g;
    auto rows_of = [&](int key) { const WinRows w = win_rows_of_key(g.qs, seg_pos_of_row(g.ks, key), a.window, a.n_sink); return w.end - w.first; };
    auto keys_of = [&](int row) { const WinKeys w = win_keys_of_row(g.ks, seg_pos_of_row(g.qs, row), a.window, a.n_sink); return w.sink + w.hi - w.lo; };
    const int other = b.sink_tiles * keys < g.lc ? b.sink_tiles * keys : g.lc - 1;      // the first key that is not in a tile of sinks
    b.keys_down = rows_of(g.lc - 1) > rows_of(other);
    b.rows_down = keys_of(g.lq - 1) > keys_of(0);
    int first = 0, end = g.lq;
    if (!a.out_bf16) {
        const int p0 = g.ks.start[0], p1 = seg_pos_of_row(g.ks, g.lc - 1);
        first = seg_rows_le(g.qs, p0 - 1);
        if (p0 >= a.n_sink && p1 < 0x7fffffff - a.window) end = seg_rows_le(g.qs, p1 + a.window - 1);
    }
    b.first_q_tile = first / keys;
    b.n_q_tiles = a.want_dq && end > first ? (end + keys - 1) / keys - b.first_q_tile : 0;
    return b;
}

hipError_t hexi_launch_win_parts(const WinBwdArgs& a, int dtype, int keys, hipStream_t s)
{
    const int tiles = a.n_parts > 1 ? (a.g.lc + keys - 1) / keys : a.sink_tiles;
    if (tiles == 0) return hipSuccess;
    const unsigned grid = (unsigned)tiles * (unsigned)a.g.nkv * (unsigned)(keys * a.g.d / 512);
    if (dtype == HEXI_BF16) {
        if (a.g.d == 128) win_parts_kernel<uint16_t, 128><<<grid, 256, 0, s>>>(a, keys);
        else win_parts_kernel<uint16_t, 64><<<grid, 256, 0, s>>>(a, keys);
    } else if (a.g.d == 128) win_parts_kernel<float, 128><<<grid, 256, 0, s>>>(a, keys);
    else win_parts_kernel<float, 64><<<grid, 256, 0, s>>>(a, keys);
    return hipGetLastError();
}

hipError_t hexi_launch_win_bwd(const WinBwdArgs& a, int dtype, hipStream_t s)
{
    if (dtype == HEXI_BF16)
        return hexi_win_bwd_split(a.g, a.window, a.n_sink, a.want_dq, a.want_dkdv) ? hexi_launch_win_bwd_split_bf16(a, s) : hexi_launch_win_bwd_quad_bf16(a, s);
    const AttnGeom& g = a.g;
    hipError_t joined = hipSuccess;
    auto launch = [&](bool split, bool dkdv, bool dq) {
        return with_cfg(g.d, split, [&](auto cfg) {
            using C = decltype(cfg);
            const WinBwdArgs b = hexi_win_tiles_of(a, C::ROWS);
            const unsigned n_dkdv = dkdv ? (unsigned)hexi_win_dkdv_units(b, (g.lc + C::ROWS - 1) / C::ROWS) : 0u;
            const unsigned n_dq = dq ? (unsigned)b.n_q_tiles * (unsigned)g.nq : 0u;
            if (n_dkdv + n_dq > 0) win_bwd_f32_kernel<C::D, C::SPLIT, C::TWO><<<n_dkdv + n_dq, 64 * C::NW, 0, s>>>(b, n_dkdv);
            if (dkdv) joined = hexi_launch_win_parts(b, dtype, C::ROWS, s);
        });
    };
    // (halves of one shape in one launch: they fill each other's last round)
    const bool kv_split = hexi_win_f32_split(2, g, a.window, a.n_sink), q_split = hexi_win_f32_split(1, g, a.window, a.n_sink);
    hipError_t e = hipSuccess;
    if (a.want_dkdv && a.want_dq && kv_split == q_split) e = launch(kv_split, true, true);
    else {
        if (a.want_dkdv) e = launch(kv_split, true, false);
        if (e == hipSuccess && a.want_dq) e = launch(q_split, false, true);
    }
    return e == hipSuccess ? joined : e;
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

// f(element type, head_dim)
template <class F> void with_type(int dtype, int d, F f)
{
    if (dtype == HEXI_F32) { if (d == 128) f(float{}, std::integral_constant<int, 128>{}); else f(float{}, std::integral_constant<int, 64>{}); }
    else if (d == 128) f(uint16_t{}, std::integral_constant<int, 128>{});
    else f(uint16_t{}, std::integral_constant<int, 64>{});
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
