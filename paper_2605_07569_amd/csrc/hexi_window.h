// Attention under a sliding window with sink tokens: geometry shared by the host and the kernels, and argument blocks.
//
// Positions ascend with the packed row index, so what a row sees of a chunk is two runs of keys, [0, sink) and [lo, hi): the keys
// before its own position that are sinks, and those inside its window.  What a key is seen by is one run of rows (a sink: all rows
// from its own position on; another key: the window - 1 rows' positions behind it).
#pragma once
#include "hexi_internal.h"

struct WinFwdArgs : FwdArgs {
    int window, n_sink;     // both clamped to 2^31 - 1
    int out_bf16;           // o is bf16, overwritten
};
struct WinBwdArgs : BwdArgs {
    int window, n_sink;
    int out_bf16;           // dq, dk, dv are bf16, overwritten
};

// Keys that a row at position p sees: [0, sink) and [lo, hi), sink <= lo <= hi (sink = lo where the sinks reach the window).
struct WinKeys { int sink, lo, hi; };
__host__ __device__ inline WinKeys win_keys_of_row(const SegTable& ks, int p, int window, int n_sink)
{
    WinKeys w;
    w.hi = seg_rows_le(ks, p);
    w.lo = p < window ? 0 : seg_rows_le(ks, p - window);
    const int s = seg_rows_le(ks, n_sink - 1);
    w.sink = s < w.lo ? s : w.lo;                 // (lo <= hi: sinks past the row's own position are not seen)
    return w;
}

// Rows that see a key at position p: [first, end).
struct WinRows { int first, end; };
__host__ __device__ inline WinRows win_rows_of_key(const SegTable& qs, int p, int window, int n_sink)
{
    WinRows w;
    w.first = seg_rows_le(qs, p - 1);
    const unsigned last = (unsigned)p + (unsigned)(window - 1);      // at most 2^32 - 3
    w.end = p < n_sink || last > 0x7ffffffeu ? qs.total : seg_rows_le(qs, (int)last);
    return w;
}

// Launchers.
hipError_t hexi_launch_win_fwd(const WinFwdArgs& a, int dtype, hipStream_t s);
hipError_t hexi_launch_win_bwd(const WinBwdArgs& a, int dtype, hipStream_t s);
// Delta = rowsum(dO o) of a bf16 o
hipError_t hexi_launch_delta_bf16_o(long long lq, int nq, int d, const void* o, const void* d_o, int dtype,
                                    long long stride_tok, long long stride_head, float* delta, hipStream_t s);
