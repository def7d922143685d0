// Attention under a sliding window with sink tokens: geometry shared by the host and the kernels, and argument blocks.
//
// Positions ascend with the packed row index, so what a row sees of a chunk is two runs of keys, [0, sink) and [lo, hi): the keys
// before its own position that are sinks, and those inside its window.  What a key is seen by is one run of rows (a sink: all rows
// from its own position on; another key: the window - 1 rows' positions behind it).
#pragma once
#include <cmath>
#include "hexi_internal.h"

struct WinFwdArgs : FwdArgs {
    int window, n_sink;     // both clamped to 2^31 - 1
    int out_bf16;           // o is bf16, overwritten
    // Splits of a unit's run of blocks, one workgroup each; with more than one their normalised results go to part_o [splits][lq][nq][d] and part_lse
    // [splits][nq][lq], and a second launch joins them.
    int few;                // the units are those of few rows
    int rows32;             // (bf16, with more than one split) the units have 32 rows, not 64
    int n_splits;
    float *part_o, *part_lse;
    // where a split writes
    __device__ float* out_o(int split) const { return n_splits > 1 ? part_o + (long long)split * g.lq * g.nq * g.d : o; }
    __device__ float* out_lse(int split) const { return n_splits > 1 ? part_lse + (long long)split * g.nq * g.lq : lse; }
    __device__ bool merges() const { return n_splits == 1 && accumulate; }
    __device__ bool rounds() const { return n_splits == 1 && out_bf16; }
};
struct WinBwdArgs : BwdArgs {
    int window, n_sink;
    int out_bf16;           // dq, dk, dv are bf16, overwritten
    // The rows that see a tile of keys in parts, a dK / dV unit each: n_sink_parts for the first sink_tiles tiles, which hold the sinks that all later rows see, n_parts for the
    // others.  The sums of a tile that has more than one go to part [part][2][keys of a tile][d], dV and dK, and a second launch adds them up.
    int sink_tiles, n_sink_parts, n_parts;
    float* part;
    // the longest units first: tiles of keys (of rows) from the last one on
    int keys_down, rows_down;
    int first_q_tile, n_q_tiles;      // tiles of rows that are launched: those that see no key may be left out where dq stays as it is
    __host__ __device__ int q_tile(int i) const { return first_q_tile + (rows_down ? n_q_tiles - 1 - i : i); }
};
inline int hexi_win_dkdv_units(const WinBwdArgs& a, int tiles) { return (a.sink_tiles * a.n_sink_parts + (tiles - a.sink_tiles) * a.n_parts) * a.g.nkv; }
#ifdef __HIP__
// A dK / dV unit, by its workgroup: kv heads side by side, then parts, then tiles.
struct WinUnit {
    int tile, kvh, part, n_parts;
    long long slot;         // of its sums, where it is one of several parts
    __device__ __forceinline__ WinUnit(const WinBwdArgs& a, int keys, int block)      // keys: of a tile
    {
        const int sinks = a.sink_tiles * a.n_sink_parts * a.g.nkv;
        const bool sink = block < sinks;
        const int b = sink ? block : block - sinks;
        n_parts = sink ? a.n_sink_parts : a.n_parts;
        const int ts = __builtin_amdgcn_readfirstlane(b / a.g.nkv);
        kvh = b - ts * a.g.nkv;
        const int t = __builtin_amdgcn_readfirstlane(ts / n_parts);
        part = ts - t * n_parts;
        const int tiles = __builtin_amdgcn_readfirstlane((a.g.lc + keys - 1) / keys);
        tile = sink ? t : a.keys_down ? tiles - 1 - t : t + a.sink_tiles;
        slot = sink ? block : (a.n_sink_parts > 1 ? sinks : 0) + ((long long)(tile - a.sink_tiles) * n_parts + part) * a.g.nkv + kvh;
    }
    // first of n blocks of rows that part i takes
    __device__ __forceinline__ int first_of(int n, int i) const
    {
        if (n_parts == 1) return i * n;
        const int each = __builtin_amdgcn_readfirstlane(n / n_parts), rest = n - each * n_parts;
        return i * each + (i < rest ? i : rest);
    }
};
#else
struct WinUnit;
#endif

// Argument blocks of kernels that serve both: WIN, under a window.
template <bool WIN> struct WinOr { using Fwd = FwdArgs; using Bwd = BwdArgs; };
template <> struct WinOr<true> { using Fwd = WinFwdArgs; using Bwd = WinBwdArgs; };
template <bool WIN> using FwdArgsOf = typename WinOr<WIN>::Fwd;
template <bool WIN> using BwdArgsOf = typename WinOr<WIN>::Bwd;

// Keys that a row at position p sees: [0, sink) and [lo, hi), sink <= lo <= hi.  Where the sinks reach the window they are one run, sink = lo = 0: along
// a shard these rows come first, and sink, lo and hi never fall.
struct WinKeys { int sink, lo, hi; };
__host__ __device__ __attribute__((always_inline)) inline WinKeys win_keys_of_row(const SegTable& ks, int p, int window, int n_sink)
{
    WinKeys w;
    w.hi = seg_rows_le(ks, p);
    w.lo = p < window ? 0 : seg_rows_le(ks, p - window);
    const int s = seg_rows_le(ks, n_sink - 1);
    w.sink = s < w.lo ? s : 0;                    // (lo <= hi: sinks past the row's own position are not seen)
    if (s >= w.lo) w.lo = 0;
    return w;
}

#ifdef __HIP__
// Bits 0 .. n - 1; n below 0 counts as 0, above 32 as 32.
__device__ __forceinline__ uint32_t win_low_bits(int n) { return n <= 0 ? 0u : 0xffffffffu >> (n < 32 ? 32 - n : 0); }
// Bit i: index at + i lies in [lo, hi).
__device__ __forceinline__ uint32_t win_bits(int lo, int hi, int at) { return win_low_bits(hi - at) & ~win_low_bits(lo - at); }
__device__ __forceinline__ uint32_t win_bits(const WinKeys& w, int at) { return win_bits(w.lo, w.hi, at) | win_low_bits(w.sink - at); }
// All ones where bit i of the mask is set, zero where not: two instructions to a masked value (a comparison of positions took six: 1000 clocks of a masked 32-key
// block of two row blocks, in which a step at head_dim 64 takes 2000).
template <int I> __device__ __forceinline__ uint32_t win_bit(uint32_t bits) { return (uint32_t)__builtin_amdgcn_sbfe((int)bits, I, 1); }
template <int I> __device__ __forceinline__ float win_or(uint32_t bits, float x, float other)      // x where bit I is set
{
    const uint32_t m = win_bit<I>(bits);
    return __uint_as_float((__float_as_uint(x) & m) | (__float_as_uint(other) & ~m));
}
#endif

// What a run of rows sees of the chunk in blocks of B keys, from the keys of its first and last rows: the blocks that hold a key some row sees, numbered
// 0 .. n_blocks - 1 in order (those of the sinks, then those of the windows), and which of them every row sees in full.
template <int B> struct WinSpan {
    int n_sink_blocks, skip;          // block i of the run is block i of the chunk, or i + skip behind the sinks'
    int n_blocks;
    int n_whole;                      // blocks of the run before one that the chunk's end cuts
    int full_sink, full_lo, full_hi;  // keys that every row sees: [0, full_sink) and [full_lo, full_hi)
    WinSpan() = default;
    __host__ __device__ __attribute__((always_inline)) WinSpan(const WinKeys& first, const WinKeys& last, int lc)
    {
        const int b0 = first.lo / B, b1 = (last.hi + B - 1) / B, s = (last.sink + B - 1) / B;
        n_sink_blocks = s < b0 ? s : b0;
        skip = b0 - n_sink_blocks;
        n_blocks = n_sink_blocks + (b1 > b0 ? b1 - b0 : 0);
        n_whole = n_blocks - (b1 > b0 && b1 > lc / B ? 1 : 0);
        full_sink = first.sink;
        full_lo = last.lo;
        full_hi = first.hi;
    }
    __host__ __device__ __attribute__((always_inline)) int block(int i) const { return i < n_sink_blocks ? i : i + skip; }
    // blocks [i0, i1) of the run of a split
    __host__ __device__ __attribute__((always_inline)) int split_start(int split, int n_splits) const
    {
        if (n_splits == 1) return split * n_blocks;
        const int each = n_blocks / n_splits, rest = n_blocks - each * n_splits;
        return split * each + (split < rest ? split : rest);
    }
    // whether every row sees all of the chunk's block b
    __host__ __device__ __attribute__((always_inline)) bool full(int b) const { return (B * b >= full_lo && B * b + B <= full_hi) || B * b + B <= full_sink; }
};

// Rows that see a key at position p: [first, end).
struct WinRows { int first, end; };
__host__ __device__ __attribute__((always_inline)) inline WinRows win_rows_of_key(const SegTable& qs, int p, int window, int n_sink)
{
    WinRows w;
    w.first = seg_rows_le(qs, p - 1);
    const unsigned last = (unsigned)p + (unsigned)(window - 1);      // at most 2^32 - 3
    w.end = p < n_sink || last > 0x7ffffffeu ? qs.total : seg_rows_le(qs, (int)last);
    return w;
}

// What a run of keys is seen by, from its first and last: rows [first, end) see some of them, rows [full, full_end) all.  Ends ascend with the keys but for
// sinks, which all rows behind them see; they come first.  (A run of both kinds counts as seen in full by no row.)
struct WinRowSpan {
    int first, end, full, full_end;
    __host__ __device__ WinRowSpan(const WinRows& w0, const WinRows& w1, bool first_is_sink, bool last_is_sink, int lq)
    {
        first = w0.first;
        end = first_is_sink ? lq : w1.end;
        full = w1.first;
        full_end = last_is_sink ? lq : first_is_sink ? 0 : w0.end;
    }
};

#define HEXI_WIN_MAX_SPLITS 256
#define HEXI_WIN_FEW_VECTORS 512
#define HEXI_WIN_FEW_ROWS 8
#define HEXI_WIN_FEW_GROUPS 160      // of 16 vectors: 32 whole ones, and one that is not whole for each of 128 heads

// What a bf16 forward call takes in units of 64 rows (0) or 32 (1), each in n splits, us: a base, a unit's fixed part and its steps of 128 (256) keys, the longer of a unit and
// all units' share of 256 CUs with a part of one, and the join.  Fitted to 2300 timings of 500 random calls (half within 5 %); the choice by it is on average 1 % slower than
// the best of them.  64 rows / 32 rows, and in how many splits, 128 columns: 8/1 heads of 775 rows, window 87 10.6 / 6.9, 12/3 of 2158, 3425 75 / 98, 6/2 of 21, 5494 43 / 32, in 8
// 16.8 / 13.7, in 16 14.5 / 12.1; 64 columns: 16/4 of 278, 4423 28.6 / 21.0, in 4 23.8 / 30.2, 32/8 of 4144, 283 42 / 88.
inline double hexi_win_fwd_us(int rows32, int d, long long lq, int nq, double share, double keys, int n)
{
    struct Fit { double base, fixed, step, rest, join, join_values; };      // join_values: per 10^6 partial results
    static const Fit fits[2][2] = {{{4.4, 2.1, 0.65, 0.30, 3.3, 3.5}, {1.2, 3.8, 0.94, 0.33, 3.4, 5.0}}, {{0.9, 7.2, 0.90, 0.46, 3.0, 2.6}, {1.0, 4.8, 1.40, 0.38, 3.3, 3.6}}};
    const Fit& f = fits[d == 128][rows32];
    const int rows = rows32 ? 32 : 64, step = rows32 ? 256 : 128;
    const double unit = f.fixed + f.step * (keys + (lq < rows ? lq : rows) + 30) / (step * n), even = share * ((lq + rows - 1) / rows) * nq * n / 256.0 * unit + f.rest * unit;
    return f.base + (unit > even ? unit : even) + (n > 1 ? f.join + f.join_values * 1e-6 * n * lq * nq * d : 0.0);
}

// How a forward call is cut, by the descriptor, the window and the lengths alone, so that its workspace can be asked for without the ranges.
struct WinFwdPlan { int few, n_splits, rows32; };
// Few rows whose q heads share kv heads take workgroups of 16 query vectors (hexi_win_few.hip), two a CU in all, in one split up to two blocks of 64 keys; but bf16 rows of more
// than two blocks and at most eight, for which one unit without a join is faster.  us, bf16, 32-row units / these, 128 columns, one row of 8/1 heads, 60 keys 6.0 / 5.1,
// 250 6.8 / 7.9, 1000 10.1 / 8.7, 4096 10.7 / 9.2; 32/8, 4096 19.3 / 10.9; 64/8, 32000 150 / 30; 8 rows of 8/4, 500 8.2 / 9.5, 4096 10.6 / 11.5; 32/8, 30000 76 / 46; heads of
// their own, 64-row units / these, one row of 24/24, 4096 18.7 / 18.7, 128/128, 500 11.8 / 14.8.  fp32, 16-row units / these: 32/8, 4096 29.6 / 18.2, 8/1, 400 13.9 / 10.0, 190
// 9.6 / 10.0, 24/24, 4096 25.6 / 28.3.
// Otherwise bf16 units are split by hexi_win_fwd_us, where a wavefront is left with a block at least; fp32 ones as far as fills the chip with workgroups, if that takes at least
// eight steps off a unit (a step is 0.8 us, joining the results 3 to 4).
inline WinFwdPlan hexi_win_fwd_plan(int dtype, int d, int nq, int nkv, long long lq, long long lc, long long window, long long n_sink)
{
    const long long sinks = n_sink < lc ? n_sink : lc, seen = window < lc ? (window + sinks < lc ? window + sinks : lc) : lc;      // keys of a row
    auto keys_of = [&](long long rows) { return seen + (lq < rows ? lq : rows) < lc ? seen + (lq < rows ? lq : rows) : lc; };
    WinFwdPlan plan = {0, 1, 0};
    const long long blocks = (keys_of(lq) + 63) / 64;
    if (lq <= HEXI_WIN_FEW_ROWS && lq * nq <= HEXI_WIN_FEW_VECTORS && lq * nq <= 32 * nkv && nq >= 2 * nkv && (dtype != HEXI_BF16 || blocks <= 2 || blocks > 8)) {
        const long long groups = nkv * ((lq * nq + 16 * nkv - 1) / (16 * nkv));
        long long n = 512 / groups;
        n = blocks <= 2 ? 1 : n < blocks ? n : blocks;
        plan.few = 1;
        plan.n_splits = n < 1 ? 1 : n < HEXI_WIN_MAX_SPLITS ? (int)n : HEXI_WIN_MAX_SPLITS;
        return plan;
    }
    if (dtype == HEXI_BF16) {
        double best = 0.0;
        for (int r = 0; r < 2; ++r) {
            const long long rows = r ? 32 : 64, step = r ? 256 : 128, units = (lq + rows - 1) / rows * nq;
            for (int n = 1; n == 1 || (n <= HEXI_WIN_MAX_SPLITS && units * n <= 512 && step * n < keys_of(rows) + step); n *= 2) {
                const double us = hexi_win_fwd_us(r, d, lq, nq, 1.0, (double)seen, n);
                if (best == 0.0 || us < best) { best = us; plan.n_splits = n; plan.rows32 = r; }
            }
        }
        return plan;
    }
    const long long units = (lq + 15) / 16 * nq, steps = (keys_of(16) + 127) / 128;
    if (units > 128) return plan;
    long long n = 256 / units;
    n = n < steps ? n : steps;
    if (n > 1 && steps - (steps + n - 1) / n >= 8) plan.n_splits = (int)n;
    return plan;
}
inline size_t hexi_win_fwd_workspace(int n_splits, int nq, long long lq, int d)
{
    return n_splits > 1 ? (size_t)n_splits * (size_t)lq * (size_t)nq * (size_t)(d + 1) * sizeof(float) : 0;
}

// Parts of the rows of a tile of sinks and of another one in the backward, by the descriptor, the window and the lengths alone.  A part is left with `least` rows of all heads, and a
// tile is cut if that takes as many off its chain: 1024 rows of bf16 or 256 of fp32 are about 8 us, the join 4.  Sinks, which all later rows see, are cut to the other tiles' length or
// to 0.7 of what a CU has of all units (a unit's start and end counted as `least` rows, dQ's rows as 0.6), whichever is more; other tiles, where they are fewer than half the CUs, to what
// a CU has of them.  us, in one / in parts: bf16, 3/1 heads of 1269 rows, window 121, a sink 36 / 20; fp32, 6/3 of 498, 37, four sinks 53 / 33, 2/1 of 3798, 432, 128 sinks 266 / 104, 4/1
// of 2766 and the step in front of them, 1086, a sink 537 / 100.
struct WinBwdPlan { int n_sink_parts, n_parts; };
inline WinBwdPlan hexi_win_bwd_plan(int dtype, int nq, int nkv, long long lq, long long lc, long long window, long long n_sink)
{
    const long long least = dtype == HEXI_BF16 ? 1024 : 256, sinks = n_sink < lc ? n_sink : lc;
    const long long all = lq * nq / nkv, chain = (window < lq ? window : lq) * nq / nkv;      // rows of all heads that a sink's tile walks, another's
    auto parts_of = [&](long long rows, long long target, long long keys) {
        const long long units = (keys + 31) / 32 * nkv;
        target = target > least ? target : least;
        if (rows - target < least || units > 256) return 1;
        const long long n = (rows + target - 1) / target, most = units > 16 ? 512 / units : 32;
        return (int)(n < most ? n : most);
    };
    WinBwdPlan plan = {1, 1};
    const long long units = (lc + 31) / 32 * nkv;
    const double keys = (double)(window < lc ? window : lc) + sinks;
    const double even = 0.7 * (units * (double)(chain + least) + 0.6 * ((lq + 31) / 32 * nq) * ((keys < lc ? keys : lc) + least)) / 256.0;
    if (units <= 128) plan.n_parts = parts_of(chain, chain * units / 256, lc);
    if (sinks > 0) plan.n_sink_parts = parts_of(all, chain / plan.n_parts > even ? chain / plan.n_parts : (long long)even, sinks);
    return plan;
}
inline size_t hexi_win_bwd_workspace(const WinBwdPlan& plan, int nkv, int d, long long lc, long long n_sink)
{
    const long long sinks = n_sink < lc ? n_sink : lc;
    const long long keys = (plan.n_sink_parts > 1 ? plan.n_sink_parts * (sinks + 63) : 0) + (plan.n_parts > 1 ? plan.n_parts * (lc + 63) : 0);
    return (size_t)keys * (size_t)nkv * (size_t)d * 2 * sizeof(float);
}

// What the rows of a shard see of a chunk, and what sees its keys, from 16 of each: the share that sees (is seen by) anything, and the keys (rows) of one that does, on average and at most.
struct WinLoad { double share, mean, most; };
template <class F> inline WinLoad hexi_win_load(int n, F count)
{
    int some = 0, most = 0;
    double sum = 0.0;
    for (int i = 0; i < 16; ++i) {
        const int c = count((int)((long long)n * (2 * i + 1) / 32));
        some += c > 0;
        most = c > most ? c : most;
        sum += c;
    }
    return {some / 16.0, some ? sum / some : 0.0, (double)most};
}
inline WinLoad hexi_win_row_load(const AttnGeom& g, int window, int n_sink)
{
    return hexi_win_load(g.lq, [&](int row) { const WinKeys w = win_keys_of_row(g.ks, seg_pos_of_row(g.qs, row), window, n_sink); return w.sink + w.hi - w.lo; });
}
inline WinLoad hexi_win_key_load(const AttnGeom& g, int window, int n_sink)
{
    return hexi_win_load(g.lc, [&](int key) { const WinRows w = win_rows_of_key(g.qs, seg_pos_of_row(g.ks, key), window, n_sink); return w.end > w.first ? w.end - w.first : 0; });
}

// Whether a bf16 forward call takes 256-row workgroups (head_dim 128 alone; at 64 they are slower everywhere).  Fitted to 45 random calls (half within 4 %, the choice 1 %
// slower than the better one), us: rounds of 256 workgroups times a start and end and their key tiles, 17.7 + 1.53 a tile of 64 keys, against rounds of 64-row ones, 6.9 + 0.98 a
// step of 128.  64 rows / 256 rows: 16 heads of 3729 rows, window 4873 202 / 167; 24 of 13495, 2972 592 / 514; 8 of 16384, 4096 312 / 269; 32 of 18703, 1190 598 / 518; 8 of 8513,
// 2018 (272 workgroups of 256) 117 / 140; 6 of 11340, 4680 218 / 263.
inline bool hexi_win_fwd_large(const AttnGeom& g, int window, int n_sink)
{
    if (g.d != 128) return false;
    const WinLoad load = hexi_win_row_load(g, window, n_sink);
    if (load.share == 0.0) return false;
    const double large = load.share * ((g.lq + 255) / 256) * g.nq, small = load.share * ((g.lq + 63) / 64) * g.nq;
    const double t_large = ceil(large / 256.0) * (17.7 + 1.53 / 64.0 * (load.mean + 255 + 63));
    const double t_small = (small / 256.0 + 0.41) * (6.9 + 0.98 / 128.0 * (load.mean + 63 + 31));
    return t_large < t_small;
}

// Whether the units of a bf16 forward call that is not split have 32 rows.
inline bool hexi_win_fwd_rows32(const AttnGeom& g, int window, int n_sink)
{
    const WinLoad load = hexi_win_row_load(g, window, n_sink);
    return hexi_win_fwd_us(1, g.d, g.lq, g.nq, load.share, load.mean, 1) < hexi_win_fwd_us(0, g.d, g.lq, g.nq, load.share, load.mean, 1);
}

// Whether a bf16 backward call takes 32-row (32-key) workgroups of eight wavefronts, or 64-row ones of four.  Fitted to 900 random calls (half within 6 %), us: a base, a unit's
// fixed part and its steps of 256 (128) streamed rows, and the longer of the longest unit and all units' share of 256 CUs with a part of the longest one.  The choice is on
// average 0.7 % slower than the better one.  64 rows / 32 rows, backward of all three, window 296, 4/4 heads of 241 rows 14.0 / 9.0 (128 columns), 850, 8/2 of 193 22.1 / 13.3, 1469,
// 12/3 of 1505 85.8 / 82.4, 404, 8/1 of 7646 91 / 108; 64 columns, 163, 8/1 of 1863 27 / 16, 27, 12/3 of 3862 29 / 36.
inline bool hexi_win_bwd_split(const AttnGeom& g, int window, int n_sink, bool dq, bool dkdv)
{
    struct Fit { double base, q_fixed, q_step, k_fixed, k_step, rest; };
    static const Fit fits[2][2] = {{{1.1, 5.6, 0.75, 6.4, 1.07, 0.33}, {1.3, 3.7, 0.84, 4.7, 1.17, 0.36}}, {{0.3, 8.5, 1.14, 9.4, 1.67, 0.40}, {1.0, 4.8, 1.34, 6.3, 1.92, 0.43}}};
    const WinLoad keys = hexi_win_row_load(g, window, n_sink), rows = hexi_win_key_load(g, window, n_sink);
    auto us = [&](int split) {
        const Fit& f = fits[g.d == 128][split];
        const int n = split ? 32 : 64, step = split ? 256 : 128;
        const double q = f.q_fixed + f.q_step * (keys.mean + n + 30) / step, k = f.k_fixed + f.k_step * (rows.mean + n + 30) * g.nq / g.nkv / step;
        const double sum = (dq ? keys.share * ((g.lq + n - 1) / n) * g.nq * q : 0.0) + (dkdv ? rows.share * ((g.lc + n - 1) / n) * g.nkv * k : 0.0);
        const double q_most = f.q_fixed + f.q_step * (keys.most + n + 30) / step, k_most = f.k_fixed + f.k_step * (rows.most + n + 30) * g.nq / g.nkv / step;
        const double longest = dq && (!dkdv || q_most > k_most) ? q_most : k_most, even = sum / 256.0 + f.rest * (dq && (!dkdv || q > k) ? q : k);
        return f.base + (longest > even ? longest : even);
    };
    return us(1) < us(0);
}

// Whether the fp32 units of a windowed call take 16 rows (or keys), streamed rows split over eight wavefronts, or 64 that share tiles: PART 0 forward, 1 dQ, 2 dK/dV.
// Fitted to 189 random calls (90 % within 15 %), us: a base, and for every round of 256 workgroups a fixed part and a step, 32 streamed rows in the 64-row shape and 128 in
// the other; more 64-row units than CUs share one and take at least 1.6 rounds at head_dim 128.  The choice is on average under 1 % slower than the better one.  64 rows / 16 rows:
// forward, 128 columns, 16 heads of 3667, window 26 54 / 104, 4 of 4173, 1581 254 / 190; dQ, 64 columns, 24 of 6094, 83 89 / 156; dK/dV, 8 kv heads, 8000, 821 476 / 642,
// 8/4 of 1707, 1274 393 / 184.
inline bool hexi_win_f32_split(int part, const AttnGeom& g, int window, int n_sink)
{
    struct Fit { double base, fixed, step; };
    static const Fit fits[2][3][2] = {{{{8.0, 1.0, 1.60}, {4.8, 2.5, 1.47}}, {{6.6, 1.9, 2.03}, {4.9, 3.4, 1.73}}, {{4.2, 3.4, 3.16}, {6.8, 4.7, 2.42}}},
                                      {{{3.0, 7.4, 2.66}, {1.2, 7.4, 2.79}}, {{0.7, 11.1, 3.51}, {0.7, 9.8, 3.48}}, {{5.7, 4.4, 5.23}, {1.7, 13.6, 4.76}}}};
    const WinLoad load = part == 2 ? hexi_win_key_load(g, window, n_sink) : hexi_win_row_load(g, window, n_sink);
    auto us = [&](int shape) {
        const Fit& f = fits[g.d == 128][part][shape];
        const int rows = shape ? 16 : 64;
        const double units = load.share * (part == 2 ? (double)((g.lc + rows - 1) / rows) * g.nkv : (double)((g.lq + rows - 1) / rows) * g.nq);
        const double chain = (load.mean + rows - 1) * (part == 2 ? (double)g.nq / g.nkv : 1.0) / (shape ? 128.0 : 32.0);
        double rounds = units > 256.0 ? units / 256.0 : 1.0;
        if (!shape && g.d == 128 && units > 256.0 && rounds < 1.6) rounds = 1.6;
        const double longest = f.fixed + f.step * (load.most + rows - 1) * (part == 2 ? (double)g.nq / g.nkv : 1.0) / (shape ? 128.0 : 32.0), even = rounds * (f.fixed + f.step * chain);
        return f.base + (longest > even ? longest : even);
    };
    return us(1) <= us(0);
}

// One run of q heads to every kv head, in head order; empty for a kv head that no q head reads.
inline void hexi_head_run_of_each_kv(const signed char* kv_of_q, int nq, int nkv, HeadRuns* runs)
{
    int last[HEXI_MAX_HEADS];
    runs->n = nkv;
    for (int kh = 0; kh < nkv; ++kh) { runs->first[kh] = 0; runs->len[kh] = 0; last[kh] = -1; }
    for (int h = 0; h < nq; ++h) {
        const int kh = kv_of_q[h];
        runs->next[h] = -1;
        if (last[kh] < 0) runs->first[kh] = (signed char)h;
        else runs->next[last[kh]] = (signed char)h;
        ++runs->len[kh];
        last[kh] = h;
    }
}

// Launchers.
hipError_t hexi_launch_win_fwd(const WinFwdArgs& a, int dtype, hipStream_t s);
hipError_t hexi_launch_win_bwd(const WinBwdArgs& a, int dtype, hipStream_t s);
WinBwdArgs hexi_win_tiles_of(const WinBwdArgs& a, int keys);      // in hexi_win.hip: the arguments for tiles of so many keys, and the parts of such tiles added up
hipError_t hexi_launch_win_parts(const WinBwdArgs& a, int dtype, int keys, hipStream_t s);
hipError_t hexi_launch_win_few(const WinFwdArgs& a, int dtype, hipStream_t s);      // in hexi_win_few.hip
hipError_t hexi_launch_win_join(const WinFwdArgs& a, hipStream_t s);
hipError_t hexi_launch_win_fwd_large_bf16(const WinFwdArgs& a, hipStream_t s);      // in hexi_bf16_fwd.hip: 256-row workgroups
hipError_t hexi_launch_win_fwd_quad_bf16(const WinFwdArgs& a, hipStream_t s);      // in hexi_bf16_quad_win.hip
hipError_t hexi_launch_win_fwd_split_bf16(const WinFwdArgs& a, hipStream_t s);      // in hexi_bf16_split.hip
hipError_t hexi_launch_win_bwd_quad_bf16(const WinBwdArgs& a, hipStream_t s);
hipError_t hexi_launch_win_bwd_split_bf16(const WinBwdArgs& a, hipStream_t s);      // in hexi_bf16_split.hip
// Delta = rowsum(dO o) of a bf16 o
hipError_t hexi_launch_delta_bf16_o(long long lq, int nq, int d, const void* o, const void* d_o, int dtype,
                                    long long stride_tok, long long stride_head, float* delta, hipStream_t s);
