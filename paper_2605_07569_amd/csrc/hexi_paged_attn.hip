// Attention of new tokens over a paged cache: tiles of 16 or 32 query vectors, and the join of tiles that several workgroups share.
//
// A workgroup's four wavefronts split every 64-key block of a tile, 16 keys each, which lie on one page; operands come straight from memory, the next block's while this one is multiplied
// (hexi_few.h has the products).  Every wavefront keeps a softmax of its own; LDS joins the four at a tile's end.
// P as an operand: bf16 where results are bf16 (FINE off: a weight is off by at most 2^-8 of itself, less than the result's own rounding in all), two bf16 values where they are fp32 (2^-16: partial
// results of a context on several devices); the sum that normalises is that of the weights as they are multiplied.
// What bounds it: few vectors a key, so the reads of K and V.
#include "hexi_few.h"
#include "hexi_paged_tiles.h"

namespace {

constexpr int NW = 4;

template <class T, int D, int NG, bool FINE>
__global__ void __launch_bounds__(64 * NW, sizeof(T) == 4 && D * NG == 256 ? 1 : 2) paged_few_kernel(const PagedArgs a)
{
    using O = Ops<T, D>;
    constexpr int NV = 16 * NG;
    __shared__ __attribute__((aligned(16))) float acc_of[NW][NV][D + 4];
    __shared__ float stat[3][NW][NV];             // reference, sum of P, sum of P as it was multiplied
    __shared__ typename PagedWalk<64 * NW>::Shared shared;
    const PagedGeom& g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, l16 = lane & 15;
    PagedWalk<64 * NW> walk(a, shared);
    if (!walk.any) return;
    const float c_hi = g.scale * LOG2E_HI, c_lo = fmaf(g.scale, LOG2E_HI, -c_hi) + g.scale * LOG2E_LO;
    PagedTile open = {0, 0, 0, 0, 0, {0, 0, 0}};
    Tile t;
    for (bool again = false; walk.next(t, open); again = true) {
        // the lane's vectors; of one that is none the first one's row again, which sees no key
        WinKeys keys[NG];
        decltype(O::k) q[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const bool real = 16 * i + l16 < t.vectors;
            const int v = real ? 16 * i + l16 : 0, row = t.row_of(v);
            keys[i] = paged_keys_of_row(g, t.q, row);
            O::row(q[i], static_cast<const T*>(a.q) + (long long)(t.q.row0 + row) * g.q_stride_tok + (long long)t.head_of(g, v, row) * g.q_stride_head, grp);
            if (!real) keys[i] = WinKeys{0, 0, 0};
        }
        const int* table = g.table + (long long)t.r * g.columns;
        const long long head = (long long)t.kv_head(g) * g.stride_head;
        const int last = t.last;
        int ids = -1, page_rows = 0, listed = 0;  // lane i: page and row of this wavefront's first key in block `listed` + i
        auto list = [&](int b) {
            listed = b;
            const int key = PAGED_KEYS * t.span.block(b + lane) + 16 * wave;
            const PagedPlace p = paged_place(g, table, key < last ? key : last & ~15);
            ids = p.id;
            page_rows = p.row;
        };
        struct Block { O ops; int key; bool seen; };
        auto load = [&](Block& x, int b) {
            if (b - listed >= 64) list(b);
            const int key = PAGED_KEYS * t.span.block(b) + 16 * wave;
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
                if constexpr (FINE) x.ops.sums_fine(acc[i], s, l_used[i]);
                else x.ops.sums(acc[i], s, l_used[i]);
            }
        };
        if (t.b0 < t.b1) {
            Block x, y;
            int b = t.b0;
            list(b);
            load(x, b);
            for (; b + 1 < t.b1; b += 2) {
                load(y, b + 1);
                __builtin_amdgcn_sched_barrier(0);
                use(x);
                if (b + 2 < t.b1) load(x, b + 2);
                __builtin_amdgcn_sched_barrier(0);
                use(y);
            }
            if (b < t.b1) use(x);
        }

        // the four wavefronts' results joined
        if (again) __syncthreads();               // the last tile's have been read
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
            plain_tile<T, D>(t);
            continue;
        }
        const PagedArgs& a = paged_args();
        const PagedGeom& g = a.g;
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
            if (t.piece >= 0) {
                const long long at = t.piece * NV + i;
                if (c == 0) a.part_lse[at] = lse;
                win_plain::store4(a.part_o, at * D + c, false, o[0], o[1], o[2], o[3]);
            } else {
                const int row = t.row_of(i), h = t.head_of(g, i, row);
                if (c == 0 && a.lse) a.lse[(long long)h * g.n_rows + t.q.row0 + row] = lse;
                win_plain::store4(a.o, paged_out(a, t, row, h) * D + c, a.out_bf16, o[0], o[1], o[2], o[3]);
            }
        }
    }
    if (tid == 0) paged_args().tiles[walk.me] = open;
}

// The pieces of a tile joined, as hexi_attn_merge_lse joins two.  Workgroup (w, y): the tile that range w starts and does not end.  Of few pieces a thread takes four columns of a
// vector and reads them all; of many a workgroup takes a vector at a time, eight or sixteen threads to its columns.
template <int D> __global__ void __launch_bounds__(256) paged_join_kernel(const PagedArgs few, const PagedArgs large, const int n_few)
{
    constexpr int D4 = D / 4, G = 256 / D4, MAX = 512, FEW = 8;
    __shared__ float weight[MAX], reduced[4];
    __shared__ __attribute__((aligned(16))) float sum[G][D];
    const bool second = (int)blockIdx.x >= n_few;
    const PagedArgs& a = second ? large : few;
    const PagedGeom& g = few.g;
    const int w = (int)blockIdx.x - (second ? n_few : 0), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int active = *a.n_active;
    const PagedTile t = a.tiles[w];
    if (w >= active || t.pieces == 0) return;
    const int nv = 1 << a.share.shift, count = g.regular ? g.most : g.first[t.run + 1] - g.first[t.run], left = t.rows * count - t.v0, vectors = left < nv ? left : nv;
    auto piece_of = [&](int i) { return i == 0 ? 2 * w + 1 : 2 * (w + i); };
    auto put = [&](int i, int c, const f32x4& o, float m, float total) {
        const float r = total == 0.f ? 0.f : 1.0f / total;
        const int row = (int)((unsigned)(t.v0 + i) / (unsigned)count), k = t.v0 + i - row * count, h = g.regular ? t.run * count + k : g.head[g.first[t.run] + k];
        if (c == 0 && a.lse) a.lse[(long long)h * g.n_rows + t.row0 + row] = total == 0.f ? -INFINITY : m + logf(total);
        win_plain::store4(a.o, ((long long)(t.row0 + row) * g.nq + h) * D + c, a.out_bf16, o[0] * r, o[1] * r, o[2] * r, o[3] * r);
    };
    if (t.pieces <= FEW) {
        for (int p = (int)blockIdx.y * 256 + tid; p < vectors * D4; p += (int)gridDim.y * 256) {
            const int i = p / D4, c = 4 * (p % D4);
            float l[FEW], m = -INFINITY, total = 0.f;
            f32x4 x[FEW], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < FEW; ++k) {
                const long long at = (long long)piece_of(k < t.pieces ? k : 0) * nv + i;
                l[k] = k < t.pieces ? a.part_lse[at] : -INFINITY;
                x[k] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + c);
            }
#pragma unroll
            for (int k = 0; k < FEW; ++k) m = fmaxf(m, l[k]);
            if (m == -INFINITY) m = 0.f;          // no weight at all, or NaN alone
#pragma unroll
            for (int k = 0; k < FEW; ++k) {
                if (k >= t.pieces) break;
                const float e = expf(l[k] - m);
                total += e;
                o += e * x[k];
            }
            put(i, c, o, m, total);
        }
        return;
    }
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
        if (m == -INFINITY) m = 0.f;
        float total = 0.f;
        for (int p = tid; p < t.pieces; p += 256) {
            const float e = expf(weight[p] - m);
            weight[p] = e;
            total += e;
        }
#pragma unroll
        for (int off = 1; off < 64; off *= 2) total += __shfl_xor(total, off, 64);
        __syncthreads();                          // the maxima have been read
        if (lane == 0) reduced[wave] = total;
        __syncthreads();
        total = (reduced[0] + reduced[1]) + (reduced[2] + reduced[3]);
        const int c = 4 * (tid % D4), p0 = tid / D4;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 16
        for (int p = p0; p < t.pieces; p += G) o += weight[p] * *reinterpret_cast<const f32x4*>(a.part_o + ((long long)piece_of(p) * nv + i) * D + c);
        *reinterpret_cast<f32x4*>(&sum[p0][c]) = o;
        __syncthreads();
        if (tid < D4) {
            o = *reinterpret_cast<const f32x4*>(&sum[0][c]);
#pragma unroll
            for (int x = 1; x < G; ++x) o += *reinterpret_cast<const f32x4*>(&sum[x][c]);
            put(i, c, o, m, total);
        }
        __syncthreads();
    }
}

template <class T, int D, bool FINE> void launch_few(const PagedArgs& a, hipStream_t s)
{
    if (a.share.shift == 4) paged_few_kernel<T, D, 1, FINE><<<a.n_ranges, 64 * NW, 0, s>>>(a);
    else paged_few_kernel<T, D, 2, FINE><<<a.n_ranges, 64 * NW, 0, s>>>(a);
}

}  // namespace

hipError_t hexi_launch_paged_few(const PagedArgs& a, int dtype, int d, hipStream_t s)
{
    if (dtype == HEXI_F32) {
        if (d == 128) launch_few<float, 128, false>(a, s); else launch_few<float, 64, false>(a, s);
    } else if (a.out_bf16) {
        if (d == 128) launch_few<uint16_t, 128, false>(a, s); else launch_few<uint16_t, 64, false>(a, s);
    } else if (d == 128) launch_few<uint16_t, 128, true>(a, s);
    else launch_few<uint16_t, 64, true>(a, s);
    return hipGetLastError();
}

hipError_t hexi_launch_paged_join(const PagedArgs& few, const PagedArgs& large, int d, hipStream_t s)
{
    // few tiles that may have many pieces: a workgroup to a vector; many tiles: they have few pieces
    const long long tiles = few.g.n_runs * (((long long)few.g.n_rows * few.g.most >> 4) + few.g.n_requests);
    const dim3 grid((unsigned)(few.n_ranges + large.n_ranges), tiles <= 32 ? 16u : tiles <= 256 ? 4u : 2u);
    if (d == 128) paged_join_kernel<128><<<grid, 256, 0, s>>>(few, large, few.n_ranges);
    else paged_join_kernel<64><<<grid, 256, 0, s>>>(few, large, few.n_ranges);
    return hipGetLastError();
}
