// Attention of new tokens over a paged cache: 16 or 32 query vectors to a tile, and the join of tiles that several workgroups share.
//
// The query vectors of a request and a kv head are its rows' q heads that read it, row by row.  A workgroup's four wavefronts split every 64-key block of a tile, 16 keys each, which lie on
// one page; operands come straight from memory, the next block's while this one is multiplied (hexi_few.h has the products).  Every wavefront keeps a softmax of its own; LDS joins the four at a tile's end.
// What bounds it: few vectors a key, so the reads of K and V.
#include "hexi_few.h"
#include "hexi_paged.h"
#include "hexi_window_plain.h"

namespace {

constexpr int KEYS = 64, NW = 4;

// A tile of a request.
struct Tile {
    PagedRequest q;
    WinSpan<KEYS> span;       // of all rows of the request
    int r, run, count, v0, vectors;      // count: heads of the run; vectors: of the tile, 0 or less: none
};

// ---- element by element ----
// A tile's vectors, eight lanes each, walk the keys of blocks [b0, b1) of the request's run that they see, one by one: what a vector does not see is not read into it.
template <class T, int D> __device__ __forceinline__ void plain_tile(const PagedArgs& a, const Tile& t, const int b0, const int b1, float* part_o, float* part_lse)
{
    constexpr int N = D / win_plain::LANES;
    const PagedGeom& g = a.g;
    const int col = (int)threadIdx.x % win_plain::LANES * N;
    const int* table = g.table + (long long)t.r * g.columns;
    for (int i = (int)threadIdx.x / win_plain::LANES; i < t.vectors; i += (int)blockDim.x / win_plain::LANES) {
        const int row = (t.v0 + i) / t.count, h = g.head[g.first[t.run] + (t.v0 + i) - row * t.count];
        const WinKeys w = paged_keys_of_row(g, t.q, row);
        const long long head = (long long)g.kvh[t.run] * g.stride_head + col;
        float q[N], acc[N];
        win_plain::load_cols(static_cast<const T*>(a.q) + (long long)(t.q.row0 + row) * g.q_stride_tok + (long long)h * g.q_stride_head + col, q);
#pragma unroll
        for (int c = 0; c < N; ++c) acc[c] = 0.f;
        float m = -INFINITY, l = 0.f;
        for (int b = b0; b < b1; ++b) {
            const int k0 = KEYS * t.span.block(b);
            for (int j = k0; j < k0 + KEYS && j < w.hi; ++j) {
                if (j >= w.sink && j < w.lo) continue;
                const PagedPlace p = paged_place(g, table, j);
                if (p.id < 0) continue;
                const long long at = (long long)p.id * g.stride_page + (long long)p.row * g.stride_tok + head;
                float x[N];
                win_plain::load_cols(static_cast<const T*>(a.k) + at, x);
                const float s = win_plain::dot(q, x) * g.scale;
                win_plain::load_cols(static_cast<const T*>(a.v) + at, x);
                if (s > m) {
                    const float alpha = expf(m - s);   // (m = -inf: 0)
                    m = s;
                    l *= alpha;
#pragma unroll
                    for (int c = 0; c < N; ++c) acc[c] *= alpha;
                }
                const float p_j = s == -INFINITY ? 0.f : expf(s - m);
                l += p_j;
#pragma unroll
                for (int c = 0; c < N; ++c) acc[c] = fmaf(p_j, x[c], acc[c]);
            }
        }
        const float lse = l == 0.f ? -INFINITY : m + logf(l), r = l == 0.f ? 0.f : 1.0f / l;
        if (part_o) {
            if (col == 0) part_lse[i] = lse;
#pragma unroll
            for (int c = 0; c < N; c += 4) win_plain::store4(part_o, i * D + col + c, false, r * acc[c], r * acc[c + 1], r * acc[c + 2], r * acc[c + 3]);
        } else {
            if (col == 0 && a.lse) a.lse[(long long)h * g.n_rows + t.q.row0 + row] = lse;
            const long long at = ((long long)(t.q.row0 + row) * g.nq + h) * D + col;
#pragma unroll
            for (int c = 0; c < N; c += 4) win_plain::store4(a.o, at + c, a.out_bf16, r * acc[c], r * acc[c + 1], r * acc[c + 2], r * acc[c + 3]);
        }
    }
}

// ---- work ----

struct Work { PagedRequest q; WinSpan<KEYS> span; int tiles, blocks; };     // of one head run
template <int NV> __device__ __forceinline__ Work work_of(const PagedGeom& g, int r)
{
    Work w;
    w.q = paged_request(g, r);
    w.tiles = w.blocks = 0;
    if (w.q.rows > 0) {
        w.span = WinSpan<KEYS>(paged_keys_of_row(g, w.q, 0), paged_keys_of_row(g, w.q, w.q.rows - 1), w.q.kv);
        w.tiles = (w.q.rows * g.most + NV - 1) / NV;
        w.blocks = w.span.n_blocks > 0 ? w.span.n_blocks : 1;      // (a tile that sees nothing is written too)
    }
    return w;
}

template <class T, int D, int NG>
__global__ void __launch_bounds__(64 * NW) paged_few_kernel(const PagedArgs a)
{
    using O = Ops<T, D>;
    constexpr int NV = 16 * NG;
    __shared__ __attribute__((aligned(16))) float acc_of[NW][NV][D + 4];
    __shared__ float stat[3][NW][NV];             // reference, sum of P, sum of P as it was multiplied
    __shared__ long long of_wave[NW], found[2];
    const PagedGeom& g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, l16 = lane & 15;

    // The ranges: sums over the requests, a few to a thread.
    const int each = (g.n_requests + 64 * NW - 1) / (64 * NW), r0 = tid * each < g.n_requests ? tid * each : g.n_requests, r1 = r0 + each < g.n_requests ? r0 + each : g.n_requests;
    long long mine = 0;
    for (int r = r0; r < r1; ++r) {
        const Work w = work_of<NV>(g, r);
        mine += (long long)w.tiles * w.blocks * g.n_runs;
    }
    long long before = mine;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const long long y = __shfl_up(before, off, 64);
        if (lane >= off) before += y;
    }
    if (lane == 63) of_wave[wave] = before;
    __syncthreads();
    before -= mine;
    long long total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) before += of_wave[w];
        total += of_wave[w];
    }
    long long range = (total + a.n_ranges - 1) / a.n_ranges;
    range = range < a.min_blocks ? a.min_blocks : range;
    const int active = (int)((total + range - 1) / range), per_xcd = (active + 7) / 8;
    if (blockIdx.x == 0 && tid == 0) *a.n_active = active;
    const int slot = (int)blockIdx.x >> 3, me = ((int)blockIdx.x & 7) * per_xcd + slot;
    if (slot >= per_xcd || me >= active) return;
    const long long start = me * range, end = start + range < total ? start + range : total;
    if (start >= before && start < before + mine) {
        long long at = before;
        for (int r = r0; r < r1; ++r) {
            const Work w = work_of<NV>(g, r);
            const long long n = (long long)w.tiles * w.blocks * g.n_runs;
            if (start < at + n) { found[0] = r; found[1] = at; break; }
            at += n;
        }
    }
    __syncthreads();
    int r = __builtin_amdgcn_readfirstlane((int)found[0]);
    long long first = found[1];                   // work in front of request r
    const float c_hi = g.scale * LOG2E_HI, c_lo = fmaf(g.scale, LOG2E_HI, -c_hi) + g.scale * LOG2E_LO;
    PagedTile open = {0, 0, 0, 0, 0, {0, 0, 0}};
    bool alone = true;                            // no wavefront is behind in a tile's end

    for (long long at = start; at < end;) {
        Work w = work_of<NV>(g, r);
        const long long n = (long long)w.tiles * w.blocks * g.n_runs;
        if (at >= first + n) { first += n; ++r; continue; }
        // the tile that `at` lies in, and which of its blocks are this range's
        Tile t;
        const long long in = (at - first) / w.blocks;
        const int b0 = __builtin_amdgcn_readfirstlane((int)(at - first - in * w.blocks));
        const long long tile_at = at - b0, tile_end = tile_at + w.blocks;
        const int b1 = __builtin_amdgcn_readfirstlane((int)((tile_end < end ? tile_end : end) - tile_at));
        const bool starts = b0 == 0, ends = b1 == w.blocks;
        at = tile_at + b1;
        t.r = r;
        t.q = w.q;
        t.span = w.span;
        t.run = __builtin_amdgcn_readfirstlane((int)(in / w.tiles));
        t.count = g.first[t.run + 1] - g.first[t.run];
        t.v0 = __builtin_amdgcn_readfirstlane((int)(in - (long long)t.run * w.tiles)) * NV;
        t.vectors = w.q.rows * t.count - t.v0;
        if (t.vectors > NV) t.vectors = NV;
        if (t.vectors <= 0) continue;
        const bool part = !(starts && ends);
        if (starts && part) open = {(int)((tile_end - 1) / range) - me + 1, t.run, t.q.row0, t.q.rows, t.v0, {0, 0, 0}};
        const long long piece = 2 * (long long)me + (starts ? 1 : 0);
        float* const part_o = part ? a.part_o + piece * NV * D : nullptr;
        float* const part_lse = part ? a.part_lse + piece * NV : nullptr;

        // what the tile's own rows see: keys [0, last], and blocks of the run in front of and behind which there is nothing
        const int row_a = t.v0 / t.count, row_b = (t.v0 + t.vectors - 1) / t.count;
        const WinKeys keys_a = paged_keys_of_row(g, t.q, row_a), keys_b = paged_keys_of_row(g, t.q, row_b);
        const int last = __builtin_amdgcn_readfirstlane(keys_b.hi > keys_b.sink ? keys_b.hi : keys_b.sink) - 1;      // -1: nothing
        int lane_row[NG], lane_head[NG];
        WinKeys keys[NG];
        decltype(O::k) q[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int v = 16 * i + l16 < t.vectors ? t.v0 + 16 * i + l16 : t.v0;      // (of no vector: the first one again)
            lane_row[i] = v / t.count;
            lane_head[i] = g.head[g.first[t.run] + v - lane_row[i] * t.count];
            keys[i] = paged_keys_of_row(g, t.q, lane_row[i]);
            O::row(q[i], static_cast<const T*>(a.q) + (long long)(t.q.row0 + lane_row[i]) * g.q_stride_tok + (long long)lane_head[i] * g.q_stride_head, grp);
            if (16 * i + l16 >= t.vectors) keys[i] = WinKeys{0, 0, 0};
        }
        (void)keys_a;

        const int* table = g.table + (long long)r * g.columns;
        const long long head = (long long)g.kvh[t.run] * g.stride_head;
        int ids = -1, page_rows = 0;              // lane i: page and row of this wavefront's first key in block `listed` + i
        int listed = 0;
        auto list = [&](int b) {
            listed = b;
            const int key = KEYS * t.span.block(b + lane) + 16 * wave;
            const PagedPlace p = paged_place(g, table, key < last ? key : last & ~15);
            ids = p.id;
            page_rows = p.row;
        };
        struct Block { O ops; int key; bool seen; };
        auto load = [&](Block& x, int b) {
            if (b - listed >= 64) list(b);
            const int key = KEYS * t.span.block(b) + 16 * wave;
            const int id = __builtin_amdgcn_readlane(ids, b - listed), row = __builtin_amdgcn_readlane(page_rows, b - listed);
            x.key = key;
            x.seen = id >= 0;
            const int from = key < last ? key : last & ~15, most = last - from;      // keys past the last one that is seen: that one again
            const long long at = (long long)(id < 0 ? 0 : id) * g.stride_page + (long long)row * g.stride_tok + head;
            const T* k = static_cast<const T*>(a.k) + at;
            const T* v = static_cast<const T*>(a.v) + at;
            O::row(x.ops.k, k + (l16 < most ? l16 : most) * (int)g.stride_tok, grp);
#pragma unroll
            for (int e = 0; e < 4; ++e) x.ops.values(e, v + (4 * grp + e < most ? 4 * grp + e : most) * (int)g.stride_tok, l16);
        };
        float m[NG], l[NG], l_used[NG];
        f32x4 acc[NG][O::NC];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            m[i] = -INFINITY; l[i] = l_used[i] = 0.f;
#pragma unroll
            for (int c = 0; c < O::NC; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        auto use = [&](Block& x) {
            const int key = x.key + 4 * grp;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                f32x4 s = x.ops.scores(q[i]);     // register e: key 4 grp + e of the wavefront's 16
                bool seen[4];
                float mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    seen[e] = x.seen && (key + e < keys[i].sink || (key + e >= keys[i].lo && key + e < keys[i].hi));
                    if (seen[e]) mx = fmaxf(mx, s[e]);
                }
                mx = fmaxf(m[i], over_groups(mx, true));
                const float y = m[i] - mx, alpha = mx == -INFINITY ? 1.f : fast_exp2(fmaf(y, c_hi, y == -INFINITY ? 0.f : y * c_lo));
                m[i] = mx;
                l[i] *= alpha;
                l_used[i] *= alpha;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = s[e] - mx;
                    s[e] = !seen[e] || s[e] == -INFINITY ? 0.f : fast_exp2(fmaf(d, c_hi, d == -INFINITY ? 0.f : d * c_lo));
                    l[i] += s[e];
                }
#pragma unroll
                for (int c = 0; c < O::NC; ++c) acc[i][c] *= alpha;
                x.ops.sums(acc[i], s, l_used[i]);
            }
        };
        if (last >= 0) {
            Block x, y;
            int b = b0;
            list(b);
            load(x, b);
            for (; b + 1 < b1; b += 2) {
                load(y, b + 1);
                __builtin_amdgcn_sched_barrier(0);
                use(x);
                if (b + 2 < b1) load(x, b + 2);
                __builtin_amdgcn_sched_barrier(0);
                use(y);
            }
            if (b < b1) use(x);
        }

        // the four wavefronts' results joined
        if (!alone) __syncthreads();              // the last tile's have been read
        alone = false;
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            l[i] = over_groups(l[i], false);
            l_used[i] = over_groups(l_used[i], false);
            if (grp == 0) { stat[0][wave][16 * i + l16] = m[i]; stat[1][wave][16 * i + l16] = l[i]; stat[2][wave][16 * i + l16] = l_used[i]; }
#pragma unroll
            for (int c = 0; c < O::NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z = fmaf(acc[i][c][e], 0.f, z);
                    acc_of[wave][16 * i + l16][O::column(c, 4 * grp + e)] = acc[i][c][e];
                }
        }
        // (a key that a vector does not see has P = 0, and 0 x inf is NaN: what is not finite is done again element by element)
        if (__syncthreads_or(z != 0.f)) {
            plain_tile<T, D>(a, t, b0, b1, part_o, part_lse);
            continue;
        }
        for (int p = tid; p < NV * D / 4; p += 64 * NW) {       // four columns of a vector
            const int i = p / (D / 4), c = 4 * (p % (D / 4));
            if (i >= t.vectors) break;
            float mm = -INFINITY, sum = 0.f, used = 0.f;
#pragma unroll
            for (int x = 0; x < NW; ++x) mm = fmaxf(mm, stat[0][x][i]);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < NW; ++x) {
                // (d is -inf too where the two are finite and far apart: 0, whatever the sign of c_lo)
                const float d = stat[0][x][i] - mm, e = stat[0][x][i] == -INFINITY ? 0.f : fast_exp2(fmaf(d, c_hi, d == -INFINITY ? 0.f : d * c_lo));
                sum += e * stat[1][x][i];
                used += e * stat[2][x][i];
                o += e * *reinterpret_cast<const f32x4*>(&acc_of[x][i][c]);
            }
            const float lse = sum == 0.f ? -INFINITY : fmaf(mm, g.scale, logf(sum));
            o *= used == 0.f ? 0.f : 1.0f / used;
            if (part) {
                if (c == 0) part_lse[i] = lse;
                win_plain::store4(part_o, i * D + c, false, o[0], o[1], o[2], o[3]);
            } else {
                const int row = (t.v0 + i) / t.count, h = g.head[g.first[t.run] + t.v0 + i - row * t.count];
                if (c == 0 && a.lse) a.lse[(long long)h * g.n_rows + t.q.row0 + row] = lse;
                win_plain::store4(a.o, ((long long)(t.q.row0 + row) * g.nq + h) * D + c, a.out_bf16, o[0], o[1], o[2], o[3]);
            }
        }
    }
    if (tid == 0) a.tiles[me] = open;
}

// The pieces of a tile joined, as hexi_attn_merge_lse joins two.  Workgroup (w, y): the tile that range w starts and does not end, every gridDim.y-th vector of it.
template <int D> __global__ void __launch_bounds__(256) paged_join_kernel(const PagedArgs a, const int nv)
{
    constexpr int D4 = D / 4, G = 256 / D4, MAX = 1024;
    __shared__ float weight[MAX], reduced[4];
    __shared__ __attribute__((aligned(16))) float sum[G][D];
    const PagedGeom& g = a.g;
    const int w = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int active = *a.n_active;
    const PagedTile t = a.tiles[w];
    if (w >= active || t.pieces == 0) return;
    const int count = g.first[t.run + 1] - g.first[t.run], left = t.rows * count - t.v0, vectors = left < nv ? left : nv;
    auto piece_of = [&](int i) { return i == 0 ? 2 * w + 1 : 2 * (w + i); };
    for (int i = blockIdx.y; i < vectors; i += gridDim.y) {
        float m = -INFINITY;
        for (int p = tid; p < t.pieces; p += 256) {
            const float x = a.part_lse[(long long)piece_of(p) * nv + i];
            weight[p] = x;
            m = fmaxf(m, x);
        }
#pragma unroll
        for (int off = 1; off < 64; off *= 2) m = fmaxf(m, __shfl_xor(m, off, 64));
        if (lane == 0) reduced[wave] = m;
        __syncthreads();
        m = fmaxf(fmaxf(reduced[0], reduced[1]), fmaxf(reduced[2], reduced[3]));
        if (m == -INFINITY) m = 0.f;              // no weight at all, or NaN alone
        float total = 0.f;
        for (int p = 0; p < t.pieces; ++p) total += expf(weight[p] - m);
        const int c = 4 * (tid % D4), p0 = tid / D4;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = p0; p < t.pieces; p += G) o += expf(weight[p] - m) * *reinterpret_cast<const f32x4*>(a.part_o + ((long long)piece_of(p) * nv + i) * D + c);
        *reinterpret_cast<f32x4*>(&sum[p0][c]) = o;
        __syncthreads();
        if (tid < D4) {
            o = *reinterpret_cast<const f32x4*>(&sum[0][c]);
#pragma unroll
            for (int x = 1; x < G; ++x) o += *reinterpret_cast<const f32x4*>(&sum[x][c]);
            o *= total == 0.f ? 0.f : 1.0f / total;
            const int row = (t.v0 + i) / count, h = g.head[g.first[t.run] + t.v0 + i - row * count];
            if (tid == 0 && a.lse) a.lse[(long long)h * g.n_rows + t.row0 + row] = total == 0.f ? -INFINITY : m + logf(total);
            win_plain::store4(a.o, ((long long)(t.row0 + row) * g.nq + h) * D + c, a.out_bf16, o[0], o[1], o[2], o[3]);
        }
        __syncthreads();
    }
}

template <class T, int D> void launch_few(const PagedArgs& a, const PagedShape& shape, hipStream_t s)
{
    if (shape.vectors == 16) paged_few_kernel<T, D, 1><<<a.n_ranges, 64 * NW, 0, s>>>(a);
    else paged_few_kernel<T, D, 2><<<a.n_ranges, 64 * NW, 0, s>>>(a);
    if (shape.splits) paged_join_kernel<D><<<dim3((unsigned)a.n_ranges, 4u), 256, 0, s>>>(a, shape.vectors);
}

}  // namespace

hipError_t hexi_launch_paged_attn(const PagedArgs& a, const PagedShape& shape, int dtype, int d, hipStream_t s)
{
    if (dtype == HEXI_F32) {
        if (d == 128) launch_few<float, 128>(a, shape, s); else launch_few<float, 64>(a, shape, s);
    } else if (d == 128) launch_few<uint16_t, 128>(a, shape, s);
    else launch_few<uint16_t, 64>(a, shape, s);
    return hipGetLastError();
}
