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

hipError_t hexi_launch_win_bwd_quad_bf16(const WinBwdArgs& a, hipStream_t s)
{
    const int n_q_tiles = a.want_dq ? (a.g.lq + ROWS - 1) / ROWS : 0;
    HeadRuns runs;
    hexi_head_run_of_each_kv(a.g.kv_of_q, a.g.nq, a.g.nkv, &runs);
    const unsigned n_dkdv = a.want_dkdv ? (unsigned)((a.g.lc + ROWS - 1) / ROWS) * (unsigned)a.g.nkv : 0u;
    const unsigned grid = n_dkdv + (unsigned)n_q_tiles * (unsigned)a.g.nq;
    if (a.g.d == 128) bwd_quad_bf16_kernel<128, false, true><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    else bwd_quad_bf16_kernel<64, false, true><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    return hipGetLastError();
}
