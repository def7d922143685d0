// The launchers of the bf16 ring step in 64-row workgroups (hexi_bf16_quad.h).
#include "hexi_bf16_quad.h"

hipError_t hexi_launch_fwd_quad_bf16(const FwdArgs& a, QuadRest rest, hipStream_t s)
{
    if (rest.tiles == 0) rest.tiles = (a.g.lq + ROWS - 1) / ROWS;
    const dim3 grid((unsigned)a.g.nq, (unsigned)rest.tiles);
    if (a.g.d == 128) fwd_quad_bf16_kernel<128, false><<<grid, 256, 0, s>>>(a, rest);
    else if (a.g.d == 64) fwd_quad_bf16_kernel<64, false><<<grid, 256, 0, s>>>(a, rest);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

// dq, dkdv: which halves; runs: the head runs of the dK / dV workgroups
hipError_t hexi_launch_bwd_quad_bf16(const BwdArgs& a, bool dq, const HeadRuns& runs, bool shared, hipStream_t s)
{
    const int n_q_tiles = dq ? (a.g.lq + ROWS - 1) / ROWS : 0;
    const int n_keys = shared ? hexi_keys_seen(a.g) : a.g.lc;
    const unsigned n_dkdv = (unsigned)((n_keys + ROWS - 1) / ROWS) * (unsigned)runs.n;
    const unsigned grid = n_dkdv + (unsigned)n_q_tiles * (unsigned)a.g.nq;
    if (grid == 0) return hipSuccess;
    if (a.g.d == 128) {
        if (shared) bwd_quad_bf16_kernel<128, true, false><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
        else bwd_quad_bf16_kernel<128, false, false><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    } else if (a.g.d == 64) {
        if (shared) bwd_quad_bf16_kernel<64, true, false><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
        else bwd_quad_bf16_kernel<64, false, false><<<grid, 256, 0, s>>>(a, runs, n_dkdv, n_q_tiles);
    } else return hipErrorInvalidValue;
    return hipGetLastError();
}
