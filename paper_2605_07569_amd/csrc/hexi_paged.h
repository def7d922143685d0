// Paged key / value caches: geometry shared by the host and the kernels, argument blocks, launch rules.
//
// A request's keys lie on pages of `page` tokens; its row of the block table says which.  What the lengths are only the device knows, so everything that follows from them
// (which rows, which keys, how the work is cut) is worked out in the kernels, and nothing that is read there (lengths, page ids, slots) leads outside a tensor, whatever it holds.
#pragma once
#include "hexi_divisor.h"
#include "hexi_internal.h"
#include "hexi_window.h"

struct PagedGeom {
    const int *table, *row_start, *kv_len, *q_start, *kv_start;      // device; q_start and kv_start may be null
    long long stride_page, stride_head, stride_tok;                  // of the cache, in elements
    long long q_stride_tok, q_stride_head;
    int columns, n_requests, n_rows, max_rows;
    int n_pages;
    Divisor by_page;
    int window, n_sink;               // window: 2^31 - 1 without one
    int nq, n_runs, most;             // most: heads of the run that has most
    float scale;
    // The q heads sorted by the kv head that they read: run i, heads head[first[i]] .. head[first[i + 1] - 1], reads kv head kvh[i].
    unsigned char kvh[HEXI_MAX_HEADS], head[HEXI_MAX_HEADS], first[HEXI_MAX_HEADS + 1];
};

inline void hexi_paged_runs(const signed char* kv_of_q, int nq, int nkv, PagedGeom* g)
{
    int n = 0, at = 0;
    g->nq = nq;
    g->most = 0;
    for (int kh = 0; kh < nkv; ++kh) {
        const int from = at;
        for (int h = 0; h < nq; ++h)
            if (kv_of_q[h] == kh) g->head[at++] = (unsigned char)h;
        if (at == from) continue;
        g->kvh[n] = (unsigned char)kh;
        g->first[n++] = (unsigned char)from;
        g->most = at - from > g->most ? at - from : g->most;
    }
    g->first[n] = (unsigned char)at;
    g->n_runs = n;
}

__host__ __device__ __attribute__((always_inline)) inline int paged_clamp(long long x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : (int)x; }

// Rows and keys of a request.  Row i of it sees keys up to at + i, less where a window ends; sinks: keys of this cache that stay visible.
struct PagedRequest { int row0, rows, kv, sinks; long long at; };
__host__ __device__ __attribute__((always_inline)) inline PagedRequest paged_request(const PagedGeom& g, int r)
{
    PagedRequest q;
    const int kv_start = g.kv_start ? g.kv_start[r] : 0, end = paged_clamp(g.row_start[r + 1], 0, g.n_rows);
    q.row0 = paged_clamp(g.row_start[r], 0, end);
    const int rows = end - q.row0;
    q.rows = rows < g.max_rows ? rows : g.max_rows;
    q.kv = paged_clamp(g.kv_len[r], 0, g.columns * (int)g.by_page.d);
    q.at = g.q_start ? (long long)g.q_start[r] - kv_start : (long long)q.kv - rows;
    q.sinks = paged_clamp((long long)g.n_sink - kv_start, 0, q.kv);
    return q;
}
// As win_keys_of_row(): sink, lo and hi never fall along a request's rows.
__host__ __device__ __attribute__((always_inline)) inline WinKeys paged_keys_of_row(const PagedGeom& g, const PagedRequest& q, int row)
{
    WinKeys w;
    const long long p = q.at + row;
    w.hi = paged_clamp(p + 1, 0, q.kv);
    w.lo = paged_clamp(p + 1 - g.window, 0, q.kv);
    w.sink = q.sinks < w.lo ? q.sinks : 0;
    if (q.sinks >= w.lo) w.lo = 0;
    return w;
}

// Page id and row of a key; id -1 where the table's entry is no page of the cache (its keys are not seen).
struct PagedPlace { int id, row; };
__host__ __device__ __attribute__((always_inline)) inline PagedPlace paged_place(const PagedGeom& g, const int* table_row, int key)
{
    const unsigned column = g.by_page((unsigned)key);
    PagedPlace p;
    p.id = (int)column < g.columns ? table_row[column] : -1;
    if ((unsigned)p.id >= (unsigned)g.n_pages) p.id = -1;
    p.row = key - (int)(column * g.by_page.d);
    return p;
}

// What a plan does with one request's pages.
struct PagedAsk { long long cached, added, want; int held, keep; };
__host__ __device__ __attribute__((always_inline)) inline PagedAsk paged_ask(int cached, int added, int held, int page, int columns)
{
    PagedAsk a;
    a.cached = cached > 0 ? cached : 0;
    a.added = added > 0 ? added : 0;
    a.want = (a.cached + a.added + page - 1) / page;
    a.held = paged_clamp(held, 0, columns);
    a.keep = a.want < a.held ? (int)a.want : a.held;
    return a;
}

struct PagedPlanArgs {
    const int *cached, *added;
    int *table, *held, *free_list, *n_free, *row_start, *kv_len, *pos, *slot;
    int n_requests, columns, n_pages, n_rows;
    Divisor by_page;
};

struct PagedWriteArgs {
    const int* slot;
    const void* x[2];      // new keys, new values
    void* y[2];            // caches
    long long n_rows, n_slots, x_stride_tok, x_stride_head, stride_page, stride_head, stride_tok;
    int n_heads, d;
    Divisor by_page, by_row, by_head;      // pieces of a row, of a head
};

// Attention.  The work is the tiles of all requests (query vectors of one head run, row by row) times the 64-key blocks that the request's rows see, one behind the other; every
// workgroup takes an equal range of it.  A range that ends inside a tile leaves a partial result: part_o [2 ranges][vectors][d], normalised, and part_lse; piece 2 w + 1 is that of a tile
// which range w starts, 2 w that of one which it goes on with.  tiles[w]: the tile that range w starts and does not end, for the joining launch.
struct PagedTile { int pieces, run, row0, rows, v0, pad[3]; };      // pieces: 0 where there is no such tile; v0: first vector
struct PagedArgs {
    PagedGeom g;
    const void *q, *k, *v;
    void* o;
    float* lse;               // may be null
    int out_bf16;
    int n_ranges, min_blocks; // a range has at least so many blocks
    int* n_active;            // ranges that there is work for
    PagedTile* tiles;
    float *part_o, *part_lse;
};

// How a call is launched.
struct PagedShape {
    int vectors;              // of a tile: 16 or 32
    int ranges;               // workgroups, a multiple of 8
    int min_blocks;
    bool splits;              // a tile can be cut: a second launch joins
};
inline PagedShape hexi_paged_shape(int dtype, int d, int n_runs, int most, long long n_requests, long long n_rows, long long max_rows, long long max_keys)
{
    PagedShape s;
    const long long most_vectors = max_rows * most;
    s.vectors = most_vectors > 16 ? 32 : 16;
    s.min_blocks = 2;
    const long long blocks = (max_keys + 63) / 64 + 1, tiles = n_runs * ((n_rows * most + s.vectors - 1) / s.vectors + (n_requests < n_rows ? n_requests : n_rows));
    const int full = 512;
    long long n = tiles > full ? full : tiles * blocks / s.min_blocks + 1;
    n = n > full ? full : n;
    s.ranges = (int)((n + 7) / 8 * 8);
    s.splits = blocks > s.min_blocks;
    (void)d;
    return s;
}
inline size_t hexi_paged_workspace(const PagedShape& s, int d)
{
    return 256 + (size_t)s.ranges * sizeof(PagedTile) + (size_t)2 * (size_t)s.ranges * (size_t)s.vectors * (size_t)(d + 1) * 4;
}

hipError_t hexi_launch_paged_plan(const PagedPlanArgs& a, hipStream_t s);
hipError_t hexi_launch_paged_write(const PagedWriteArgs& a, int x_dtype, int y_dtype, hipStream_t s);
hipError_t hexi_launch_paged_attn(const PagedArgs& a, const PagedShape& shape, int dtype, int d, hipStream_t s);
