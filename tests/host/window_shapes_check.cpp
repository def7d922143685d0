// Which kernels a windowed call takes, by the rules that the launchers use (csrc/hexi_window.h).  One call a line:
//   dtype nq nkv head_dim  window n_sink  q range  kv range   (dtype: 0 bf16, 1 fp32; ranges as read_segs reads them)
// prints, in words with the number of splits or parts behind a colon, the forward's units, dQ's and dK / dV's.
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include "read_segs.h"
#include "hexi_window.h"

int main()
{
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream is(line);
        AttnGeom g = {};
        int dtype, window, n_sink;
        is >> dtype >> g.nq >> g.nkv >> g.d >> window >> n_sink;
        g.qs = read_segs(is);
        g.ks = read_segs(is);
        g.lq = g.qs.total;
        g.lc = g.ks.total;
        const bool bf16 = dtype == HEXI_BF16;
        const WinFwdPlan f = hexi_win_fwd_plan(dtype, g.d, g.nq, g.nkv, g.lq, g.lc, window, n_sink);
        const WinBwdPlan b = hexi_win_bwd_plan(dtype, g.nq, g.nkv, g.lq, g.lc, window, n_sink);
        int fwd, dq, dkdv;      // rows of a unit; 0: few rows
        if (f.few) fwd = 0;
        else if (!bf16) fwd = f.n_splits > 1 || hexi_win_f32_split(0, g, window, n_sink) ? 16 : 64;
        else if (f.n_splits > 1) fwd = f.rows32 ? 32 : 64;
        else fwd = hexi_win_fwd_large(g, window, n_sink) ? 256 : hexi_win_fwd_rows32(g, window, n_sink) ? 32 : 64;
        if (bf16) dq = dkdv = hexi_win_bwd_split(g, window, n_sink, true, true) ? 32 : 64;
        else {
            dq = hexi_win_f32_split(1, g, window, n_sink) ? 16 : 64;
            dkdv = hexi_win_f32_split(2, g, window, n_sink) ? 16 : 64;
        }
        std::printf("fwd%d:%d dq%d dkdv%d:%d\n", fwd, f.n_splits, dq, dkdv, b.n_sink_parts > b.n_parts ? b.n_sink_parts : b.n_parts);
    }
    return 0;
}
