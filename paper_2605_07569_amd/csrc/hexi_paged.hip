// Pages handed out and taken back for the requests' lengths, and the writes into a paged cache.
#include "hexi_paged.h"
#include "hexi_mfma.h"

namespace {

// ---- plan ----
//
// Sums over the requests in front (pages that go back, pages that are asked for, rows) say where everything goes, so one workgroup forms them, a few requests to a thread,
// and the flat lists of pages and rows are then shared out over all threads, each of which finds its request by halving.
// What bounds it: latency, of the reads that follow each other (lengths, then pages, then the free list) and of the barriers between them.

constexpr int PT = 1024;      // threads

// Exclusive sum over the workgroup, and the total.
__device__ __forceinline__ long long sum_before(long long x, long long* of_wave, long long* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long s = x;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const long long y = __shfl_up(s, off, 64);
        if (lane >= off) s += y;
    }
    if (lane == 63) of_wave[wave] = s;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < PT / 64; ++w) {
        if (w < wave) before += of_wave[w];
        all += of_wave[w];
    }
    __syncthreads();
    *total = all;
    return before + s - x;
}

// Last r in [0, n) with first[r] <= i (first[0] = 0, ascending).
__device__ __forceinline__ int owner_of(const int* first, int n, int i)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

// Position and slot of row t; `first`: the requests' first rows.
__device__ __forceinline__ void place_row(const PagedPlanArgs& a, const int* first, int total, int t)
{
    int pos = 0, slot = -1;
    if (t < total) {
        const int r = owner_of(first, a.n_requests, t), cached = a.cached[r];
        const long long p = (long long)(cached > 0 ? cached : 0) + (t - first[r]);
        pos = p < 0x7fffffffLL ? (int)p : 0x7fffffff;
        if (p < a.kv_len[r]) {
            const unsigned column = a.by_page((unsigned)pos);
            const int id = a.table[(long long)r * a.columns + column];
            if ((unsigned)id < (unsigned)a.n_pages) slot = id * (int)a.by_page.d + (pos - (int)(column * a.by_page.d));
        }
    }
    a.pos[t] = pos;
    a.slot[t] = slot;
}

__global__ void __launch_bounds__(PT) paged_plan_kernel(const PagedPlanArgs a, const int rows_here)
{
    extern __shared__ int first[];      // [n_requests]
    __shared__ long long of_wave[PT / 64];
    const int tid = threadIdx.x, n = a.n_requests, page = (int)a.by_page.d;
    const int each = (n + PT - 1) / PT, r0 = tid * each < n ? tid * each : n, r1 = r0 + each < n ? r0 + each : n;
    auto ask = [&](int r) { return paged_ask(a.cached[r], a.added[r], a.held[r], page, a.columns); };
    const int had = paged_clamp(a.n_free[0], 0, a.n_pages);
    // pages that go back
    long long mine[2] = {0, 0}, total_back, total, rows;
    for (int r = r0; r < r1; ++r) {
        const PagedAsk q = ask(r);
        mine[0] += q.held - q.keep;
        mine[1] += q.want - q.keep;
    }
    long long before = sum_before(mine[0], of_wave, &total_back);
    const int n_back = paged_clamp(total_back, 0, a.n_pages - had);
    if (total_back > 0) {
        for (int r = r0; r < r1; ++r) {
            const PagedAsk q = ask(r);
            first[r] = paged_clamp(before, 0, 0x7fffffff);
            before += q.held - q.keep;
        }
        __syncthreads();
        for (int i = tid; i < n_back; i += PT) {
            const int r = owner_of(first, n, i);
            a.free_list[had + i] = a.table[(long long)r * a.columns + ask(r).keep + (i - first[r])];
        }
        __syncthreads();
    }
    // pages that are asked for: to the requests whose needs, and those in front of them, the list can meet
    const int top = had + n_back;
    long long asked = sum_before(mine[1], of_wave, &total), added = 0, got = 0;
    for (int r = r0; r < r1; ++r) added += a.added[r] > 0 ? a.added[r] : 0;
    long long row = sum_before(added, of_wave, &rows);
    {
        long long need_to = asked, row_to = row;
        for (int r = r0; r < r1; ++r) {
            const PagedAsk q = ask(r);
            need_to += q.want - q.keep;
            row_to += q.added;
            const bool granted = need_to <= top && q.want <= a.columns && row_to <= a.n_rows;
            got += granted ? q.want - q.keep : 0;
        }
    }
    long long given, at = sum_before(got, of_wave, &given);
    for (int r = r0; r < r1; ++r) {
        const PagedAsk q = ask(r);
        asked += q.want - q.keep;
        const long long row_to = row + q.added;
        const bool granted = asked <= top && q.want <= a.columns && row_to <= a.n_rows;
        first[r] = (int)at;           // at most `top`
        at += granted ? q.want - q.keep : 0;
        a.row_start[r] = paged_clamp(row, 0, 0x7fffffff);
        const long long kept = (long long)q.keep * page;
        a.kv_len[r] = paged_clamp(granted ? q.cached + q.added : q.cached < kept ? q.cached : kept, 0, 0x7fffffff);
        a.held[r] = granted ? (int)q.want : q.keep;
        row = row_to;
    }
    if (tid == 0) {
        a.row_start[n] = paged_clamp(rows, 0, 0x7fffffff);
        a.n_free[0] = top - (int)given;
    }
    __syncthreads();
    for (int j = tid; j < (int)given; j += PT) {
        const int r = owner_of(first, n, j), end = r + 1 < n ? first[r + 1] : (int)given;
        a.table[(long long)r * a.columns + a.held[r] - (end - j)] = a.free_list[top - 1 - j];
    }
    if (!rows_here) return;
    __syncthreads();
    for (int r = tid; r < n; r += PT) first[r] = a.row_start[r];
    __syncthreads();
    for (int t = tid; t < a.n_rows; t += PT) place_row(a, first, paged_clamp(rows, 0, 0x7fffffff), t);
}

// Positions and slots of many rows: as the plan's last part, by the whole chip.
__global__ void __launch_bounds__(256) paged_rows_kernel(const PagedPlanArgs a)
{
    extern __shared__ int first[];
    for (int r = threadIdx.x; r < a.n_requests; r += 256) first[r] = a.row_start[r];
    const int total = a.row_start[a.n_requests];
    __syncthreads();
    for (int t = blockIdx.x * 256 + threadIdx.x; t < a.n_rows; t += gridDim.x * 256) place_row(a, first, total, t);
}

// ---- writes ----
//
// A thread takes pieces of eight columns of a row; neighbouring threads neighbouring pieces, heads and rows.  What bounds it: HBM.
template <class X, class Y> __global__ void __launch_bounds__(256) paged_write_kernel(const PagedWriteArgs a, const unsigned pieces)
{
    const unsigned step = gridDim.x * 256;
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < pieces; i += step) {
        const unsigned row = a.by_row(i), in_row = i - row * a.by_row.d, h = a.by_head(in_row);
        const int c = 8 * (int)(in_row - h * a.by_head.d), slot = a.slot[row];
        if (slot < 0 || slot >= a.n_slots) continue;
        const unsigned p = a.by_page((unsigned)slot);
        const long long from = row * a.x_stride_tok + h * a.x_stride_head + c, to = p * a.stride_page + h * a.stride_head + (slot - p * a.by_page.d) * a.stride_tok + c;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const X* x = static_cast<const X*>(a.x[t]) + from;
            Y* y = static_cast<Y*>(a.y[t]) + to;
            if constexpr (sizeof(X) == sizeof(Y)) {
#pragma unroll
                for (int e = 0; e < (int)sizeof(X) / 2; ++e) reinterpret_cast<uint4*>(y)[e] = reinterpret_cast<const uint4*>(x)[e];
            } else {
                const float4 lo = reinterpret_cast<const float4*>(x)[0], hi = reinterpret_cast<const float4*>(x)[1];
                *reinterpret_cast<bf16x8*>(y) = pack_bf16x8(lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w);
            }
        }
    }
}

}  // namespace

hipError_t hexi_launch_paged_plan(const PagedPlanArgs& a, hipStream_t s)
{
    const size_t lds = (size_t)a.n_requests * sizeof(int);
    const bool rows_here = a.n_rows <= 2048;
    paged_plan_kernel<<<1, PT, lds, s>>>(a, rows_here);
    if (!rows_here) {
        const unsigned grid = (unsigned)((a.n_rows + 255) / 256);
        paged_rows_kernel<<<grid < 1024u ? grid : 1024u, 256, lds, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t hexi_launch_paged_write(const PagedWriteArgs& a, int x_dtype, int y_dtype, hipStream_t s)
{
    const unsigned pieces = (unsigned)(a.n_rows * a.n_heads * (a.d / 8));      // below 2^31
    if (pieces == 0) return hipSuccess;
    const unsigned all = (pieces + 255) / 256, grid = all < 4096u ? all : 4096u;
    if (y_dtype == HEXI_F32) paged_write_kernel<float, float><<<grid, 256, 0, s>>>(a, pieces);
    else if (x_dtype == HEXI_F32) paged_write_kernel<float, uint16_t><<<grid, 256, 0, s>>>(a, pieces);
    else paged_write_kernel<uint16_t, uint16_t><<<grid, 256, 0, s>>>(a, pieces);
    return hipGetLastError();
}
