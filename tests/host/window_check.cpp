// Host-side check of the window geometry that the kernels use (csrc/hexi_window.h).  One command a line:
//   window n_sink  q range  kv range   (ranges as read_segs reads them)
// prints for every q row "sink:lo:hi", "|", then for every key "first:end".  Or
//   large nq nkv head_dim  window n_sink  q range  kv range
// prints whether a bf16 forward call takes 256-row workgroups, whether a backward call of everything takes 32-row ones, ":" and into how many parts that
// divides the rows of a tile of sinks, ":" and of another one.
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
        int window, n_sink;
        if (line.rfind("large", 0) == 0) {
            std::string cmd;
            AttnGeom g = {};
            is >> cmd >> g.nq >> g.nkv >> g.d >> window >> n_sink;
            g.qs = read_segs(is);
            g.ks = read_segs(is);
            g.lq = g.qs.total;
            g.lc = g.ks.total;
            const WinBwdPlan plan = hexi_win_bwd_plan(HEXI_BF16, g.nq, g.nkv, g.lq, g.lc, window, n_sink);
            std::printf("%d%d:%d:%d\n", (int)hexi_win_fwd_large(g, window, n_sink), (int)hexi_win_bwd_split(g, window, n_sink, true, true), plan.n_sink_parts, plan.n_parts);
            continue;
        }
        is >> window >> n_sink;
        const SegTable qs = read_segs(is), ks = read_segs(is);
        for (int r = 0; r < qs.total; ++r) {
            const WinKeys w = win_keys_of_row(ks, seg_pos_of_row(qs, r), window, n_sink);
            std::printf("%d:%d:%d ", w.sink, w.lo, w.hi);
        }
        std::printf("|");
        for (int c = 0; c < ks.total; ++c) {
            const WinRows w = win_rows_of_key(qs, seg_pos_of_row(ks, c), window, n_sink);
            std::printf(" %d:%d", w.first, w.end);
        }
        std::printf("\n");
    }
    return 0;
}
