// The launchers of windowed attention in 64-row bf16 workgroups (hexi_bf16_quad.h).
#include "hexi_bf16_quad.h"

hipError_t hexi_launch_win_fwd_quad_bf16(const WinFwdArgs& a, hipStream_t s)
{
    QuadRest rest;
    rest.tiles = (a.g.lq + ROWS - 1) / ROWS;
    const dim3 grid((unsigned)a.g.nq * (unsigned)rest.tiles, (unsigned)a.n_splits);
    if (a.g.d == 128) fwd_quad_bf16_kernel<128, true><<<grid, 256, 0, s>>>(a, rest);
    else fwd_quad_bf16_kernel<64, true><<<grid, 256, 0, s>>>(a, rest);
    return hipGetLastError();
}

hipError_t hexi_launch_win_bwd_quad_bf16(const WinBwdArgs& whole, hipStream_t s)
{
    const WinBwdArgs a = hexi_win_tiles_of(whole, ROWS);
    const int n_q_tiles = a.n_q_tiles;
    HeadRuns runs;
    hexi_head_run_of_each_kv(a.g.kv_of_q, a.g.nq, a.g.nkv, &runs);
    const unsigned n_dkdv = a.want_dkdv ? (unsigned)hexi_win_dkdv_units(a, (a.g.lc + ROWS - 1) / ROWS) : 0u;
    const unsigned grid = n_dkdv + (unsigned)n_q_tiles * (unsigned)a.g.nq;
    if (grid == 0) return hipSuccess;
    if (a.g.d == 128) bwd_quad_bf16_kernel<128, false, true><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    else bwd_quad_bf16_kernel<64, false, true><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || !a.want_dkdv ? e : hexi_launch_win_parts(a, HEXI_BF16, ROWS, s);
}
