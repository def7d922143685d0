// Windowed forward for few rows (a token or a handful, every head of them), and the join of split runs of keys.
//
// The query vectors of a kv head are its q heads' rows; a workgroup takes up to 16 of them and a part of the run of keys that some row sees, and its four
// wavefronts split every 64-key block, 16 keys each, without LDS and without a barrier before the end:
//   S^T[key][vector] = K Q^T       lane (g, l): row l of either, 16 bytes of it a load, as the 16-row operands of the matrix instruction take them;
//   a lane then has four keys of ONE vector, so softmax is four values and two exchanges;
//   O^T[column][vector] = V^T P^T  P as it stands; V by rows, 4 g + e of the block, a piece of neighbouring columns a lane: what the four rows hold of a column is an
//   operand (bf16: packed by v_perm_b32), so output row l of product c is column PIECE l + c.  bf16 calls round P to bf16 for it, the only operand the instruction takes beside bf16 V: a
//   weight is off by at most 2^-8 of itself, and the sum that normalises is that of the rounded weights, so o stays an average of V's rows (1.9e-3 of o in all, relative L2, against
//   1.6e-3 with fp32 weights: most of either is o's own rounding).  Statistics, sums and the splits' results are fp32; fp32 calls round nothing.
// What bounds it: latency.  A call of one row is a launch, a read of its arguments (about half a microsecond), two trips to memory one behind the other, of K and V, and
// the join of the splits.  One row of 8/1 heads of 128 columns, 4100 keys (2.1 MB: 0.4 us at a copy's rate): 5.0 us and a join of 3.2; 64-row units in 32 splits 10.8 and the
// join, in one piece 34.5.
#include "hexi_blocks.h"
#include "hexi_f32_common.h"
#include "hexi_window_plain.h"

namespace {

constexpr int NV = 16, KEYS = 64, NW = 4;

// What the kernel reads of its arguments, side by side and through scalar reads: a first read of a line takes about half a microsecond, one behind the other where reads
// depend on each other.  So what the host can work out it does.
struct FewArgs {
    const void *q, *k, *v;
    float *o, *lse;                   // of split 0; the others' o_split and lse_split further
    long long q_tok, q_head, kv_tok, kv_head, o_split, lse_split;
    int lq, nq, last_key, each, rest;      // split s takes blocks [s each + min(s, rest), ..) of the run, `each` or one more
    int merges, rounds, per_row;      // per_row: 2^16 / lq, rounded up
    float scale, c_hi, c_lo;          // scale x log2(e) as two floats
    WinSpan<KEYS> span;
    WinKeys keys[HEXI_WIN_FEW_ROWS];       // of every row
};
// A workgroup's vectors: kv head, heads of the vectors (0xff: none), row of the first one; a head's rows follow each other.
struct FewGroup { int row; unsigned char kvh, pad[3], head[NV]; };
struct FewTable { FewGroup group[HEXI_WIN_FEW_GROUPS]; };

// Operands and products by element type: ROW loads of 16 bytes to a row of q or k per lane; a lane's PIECE of neighbouring columns of a row of v.
template <class T, int D> struct Ops;
template <int D> struct Ops<float, D> {
    static constexpr int ROW = D / 16, PIECE = 4, NC = D / 16;     // (D = 128: the piece is twice 4 columns, 64 apart)
    f32x4 k[ROW], v[4][D / 64];
    // columns 16 i + 4 g .. + 3 of a row
    static __device__ __forceinline__ void row(f32x4 (&x)[ROW], const float* p, int g)
    {
#pragma unroll
        for (int i = 0; i < ROW; ++i) x[i] = *reinterpret_cast<const f32x4*>(p + 16 * i + 4 * g);
    }
    __device__ __forceinline__ void values(int e, const float* p, int l)
    {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) v[e][i] = *reinterpret_cast<const f32x4*>(p + 64 * i + 4 * l);
    }
    __device__ __forceinline__ f32x4 scores(const f32x4 (&q)[ROW]) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROW; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q[i][e], s, 0, 0, 0);
        return s;
    }
    // acc[c] += ...; l: sum of p as it is multiplied
    __device__ __forceinline__ void sums(f32x4 (&acc)[NC], const f32x4& p, float& l) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            l += p[e];
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][c / 4][c % 4], p[e], acc[c], 0, 0, 0);
        }
    }
    // column of row r of product c (r = 4 g + register)
    static __device__ __forceinline__ int column(int c, int r) { return 64 * (c / 4) + 4 * r + c % 4; }
};
template <int D> struct Ops<uint16_t, D> {
    static constexpr int ROW = D / 32, PIECE = D / 16, NC = D / 16;
    bf16x8 k[ROW];
    uint32_t v[4][PIECE / 2];
    static __device__ __forceinline__ void row(bf16x8 (&x)[ROW], const uint16_t* p, int g)
    {
#pragma unroll
        for (int i = 0; i < ROW; ++i) x[i] = *reinterpret_cast<const bf16x8*>(p + 32 * i + 8 * g);
    }
    __device__ __forceinline__ void values(int e, const uint16_t* p, int l)
    {
        if constexpr (PIECE == 8) {
            const uint4 x = *reinterpret_cast<const uint4*>(p + 8 * l);
            v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(p + 4 * l);
            v[e][0] = x.x; v[e][1] = x.y;
        }
    }
    __device__ __forceinline__ f32x4 scores(const bf16x8 (&q)[ROW]) const
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ROW; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q[i], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void sums(f32x4 (&acc)[NC], const f32x4& p, float& l) const
    {
        const bf16x4 b = {(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) l += (float)b[e];
        const s16x4 pb = __builtin_bit_cast(s16x4, b);
#pragma unroll
        for (int i = 0; i < PIECE / 2; ++i) {      // columns 2 i (low halves) and 2 i + 1 (high ones) of the four rows
            const uint2 lo = {__builtin_amdgcn_perm(v[1][i], v[0][i], 0x05040100), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x05040100)};
            const uint2 hi = {__builtin_amdgcn_perm(v[1][i], v[0][i], 0x07060302), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x07060302)};
            acc[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, lo), pb, acc[2 * i], 0, 0, 0);
            acc[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, hi), pb, acc[2 * i + 1], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ int column(int c, int r) { return PIECE * r + c; }
};

__device__ __forceinline__ float over_groups(float x, bool maximum)      // over lanes l, l + 16, l + 32, l + 48
{
    const float y = __shfl_xor(x, 16, 64);
    x = maximum ? fmaxf(x, y) : x + y;
    const float z = __shfl_xor(x, 32, 64);
    return maximum ? fmaxf(x, z) : x + z;
}

template <class T, int D>
__global__ void __launch_bounds__(64 * NW) win_few_kernel(const FewArgs f, const FewTable tb, const WinFwdArgs whole)
{
    using O = Ops<T, D>;
    __shared__ __attribute__((aligned(16))) float acc_of[NW][NV][D + 4];
    __shared__ float stat[3][NW][NV];             // reference, sum of P, sum of P as it was multiplied
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, l16 = lane & 15;
    const int group = (int)blockIdx.x, split = (int)blockIdx.y;
    const uint32_t* entry = reinterpret_cast<const uint32_t*>(&tb.group[group]);
    const int row0 = (int)entry[0], kvh = (int)(entry[1] & 0xff);
    const uint32_t heads0 = entry[2], heads1 = entry[3], heads2 = entry[4], heads3 = entry[5];
    asm volatile("" ::"s"(row0), "s"(f.q), "s"(f.kv_tok), "s"(f.last_key), "s"(f.span.n_sink_blocks), "s"(f.keys[0].lo), "s"(f.keys[HEXI_WIN_FEW_ROWS - 1].hi));      // all lines of the arguments at once
    // vector i of the workgroup: head and row (row0 + i, from row 0 again for the next head)
    auto head_of = [&](int i) {
        // (not an array: the compiler would put it into LDS, and ask the dispatch packet for the workgroup's size to index it: one to five microseconds)
        uint32_t w = heads0;
        if (i >= 4) w = heads1;
        if (i >= 8) w = heads2;
        if (i >= 12) w = heads3;
        return (int)((w >> (8 * (i & 3))) & 0xff);
    };
    auto row_of = [&](int i) {
        const int x = row0 + i;                   // below 8 + 16
        return x - f.lq * (int)(((unsigned)x * (unsigned)f.per_row) >> 16);
    };
    const int b0 = split * f.each + (split < f.rest ? split : f.rest), b1 = b0 + f.each + (split < f.rest ? 1 : 0);
    const int my_head = head_of(l16), my_row = row_of(l16);      // of the lane's vector; of one that is none: row and head are read, and see no key
    WinKeys mine = f.keys[0];
#pragma unroll
    for (int i = 1; i < HEXI_WIN_FEW_ROWS; ++i)
        if (my_row == i) mine = f.keys[i];
    decltype(O::k) q;
    O::row(q, static_cast<const T*>(f.q) + (long long)my_row * f.q_tok + (long long)(my_head == 0xff ? 0 : my_head) * f.q_head, grp);
    const T* k = static_cast<const T*>(f.k) + (long long)kvh * f.kv_head;
    const T* v = static_cast<const T*>(f.v) + (long long)kvh * f.kv_head;
    O ops;
    auto load_block = [&](int b) {                // this wavefront's 16 keys; past the end of the chunk the last key again
        const int j0 = KEYS * f.span.block(b) + 16 * wave, last = f.last_key;
        const int j = j0 + l16 < last ? j0 + l16 : last;
        O::row(ops.k, k + (long long)j * f.kv_tok, grp);
#pragma unroll
        for (int e = 0; e < 4; ++e) ops.values(e, v + (long long)(j0 + 4 * grp + e < last ? j0 + 4 * grp + e : last) * f.kv_tok, l16);
    };
    load_block(b0 < b1 ? b0 : 0);
    if (my_head == 0xff) mine = WinKeys{0, 0, 0};
    const float c_hi = f.c_hi, c_lo = f.c_lo;
    float m = -INFINITY, l = 0.f, l_used = 0.f;
    f32x4 acc[O::NC];
#pragma unroll
    for (int c = 0; c < O::NC; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int b = b0; b < b1; ++b) {
        if (b > b0) load_block(b);
        f32x4 s = ops.scores(q);                  // register e: key 4 grp + e of the wavefront's 16
        const int key = KEYS * f.span.block(b) + 16 * wave + 4 * grp;
        bool seen[4];
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            seen[e] = key + e < mine.sink || (key + e >= mine.lo && key + e < mine.hi);
            if (seen[e]) mx = fmaxf(mx, s[e]);
        }
        mx = fmaxf(m, over_groups(mx, true));
        const float y = m - mx, alpha = mx == -INFINITY ? 1.f : fast_exp2(fmaf(y, c_hi, y == -INFINITY ? 0.f : y * c_lo));
        m = mx;
        l *= alpha;
        l_used *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = s[e] - mx;
            s[e] = !seen[e] || s[e] == -INFINITY ? 0.f : fast_exp2(fmaf(x, c_hi, x == -INFINITY ? 0.f : x * c_lo));
            l += s[e];
        }
#pragma unroll
        for (int c = 0; c < O::NC; ++c) acc[c] *= alpha;
        ops.sums(acc, s, l_used);
    }
    l = over_groups(l, false);
    l_used = over_groups(l_used, false);
    if (grp == 0) { stat[0][wave][l16] = m; stat[1][wave][l16] = l; stat[2][wave][l16] = l_used; }
    float z = 0.f;
#pragma unroll
    for (int c = 0; c < O::NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z = fmaf(acc[c][e], 0.f, z);
            acc_of[wave][l16][O::column(c, 4 * grp + e)] = acc[c][e];
        }
    // (a key that a vector does not see has P = 0, and 0 x inf is NaN: what is not finite is done again element by element)
    if (__syncthreads_or(z != 0.f && my_head != 0xff)) {
        for (int i = 0; i < NV; ++i)
            if (head_of(i) != 0xff) win_plain::fwd_unit<T, D>(whole, head_of(i), row_of(i), 1, win_plain::keys_of_blocks(f.span, b0, b1), split);
        return;
    }
    for (int t = tid; t < NV * D / 4; t += 64 * NW) {       // four columns of a vector: neighbouring lanes of one wavefront
        const int i = t / (D / 4), c = 4 * (t % (D / 4)), h = head_of(i), row = row_of(i);
        if (h == 0xff) continue;
        float mm = -INFINITY, total = 0.f, used = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) mm = fmaxf(mm, stat[0][w][i]);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            // (x is -inf too where the two are finite and far apart: 0, whatever the sign of c_lo)
            const float x = stat[0][w][i] - mm, e = stat[0][w][i] == -INFINITY ? 0.f : fast_exp2(fmaf(x, c_hi, x == -INFINITY ? 0.f : x * c_lo));
            total += e * stat[1][w][i];
            used += e * stat[2][w][i];
            o += e * *reinterpret_cast<const f32x4*>(&acc_of[w][i][c]);
        }
        float lse = total == 0.f ? -INFINITY : fmaf(mm, f.scale, logf(total));
        float wa = 0.f, wb = used == 0.f ? 0.f : 1.0f / used;
        float* lp = f.lse + split * f.lse_split + (long long)h * f.lq + row;
        float* out = f.o + split * f.o_split;
        const long long at = ((long long)row * f.nq + h) * D + c;
        if (f.merges) {
            const float old = *lp, top = fmaxf(old, lse);
            if (top != -INFINITY) {
                const float ea = expf(old - top), eb = expf(lse - top), r = 1.0f / (ea + eb);
                wa = ea * r;
                wb *= eb * r;
                lse = top + logf(ea + eb);
            }
        }
        __builtin_amdgcn_wave_barrier();          // the lanes of a vector have read the old value
        if (c == 0) *lp = lse;
        o *= wb;
        if (f.merges) o += wa * *reinterpret_cast<const f32x4*>(out + at);
        win_plain::store4(out, at, f.rounds, o[0], o[1], o[2], o[3]);
    }
}

// The splits' normalised results joined, as hexi_attn_merge_lse joins two: a workgroup to a (row, head), a thread to four columns of every G-th split.
template <int D> __global__ void __launch_bounds__(256) win_join_kernel(const WinFwdArgs a)
{
    constexpr int D4 = D / 4, G = 256 / D4;
    static_assert(HEXI_WIN_MAX_SPLITS <= 256, "a thread to a split");
    __shared__ float weight[256], part[2][4];
    __shared__ __attribute__((aligned(16))) float sum[G][D];
    const AttnGeom& g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = (int)blockIdx.x / g.nq, h = (int)blockIdx.x - row * g.nq;
    const long long li = (long long)h * g.lq + row, lse_part = (long long)g.nq * g.lq, o_part = lse_part * D, at = (long long)blockIdx.x * D;
    const float old = a.accumulate ? a.lse[li] : -INFINITY;
    const float own = tid < a.n_splits ? a.part_lse[tid * lse_part + li] : -INFINITY;
    float m = own;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) m = fmaxf(m, __shfl_xor(m, off, 64));
    if (lane == 0) part[0][wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3])), old);
    if (m == -INFINITY) m = 0.f;                  // no weight at all, or NaN alone
    const float w = expf(own - m);
    weight[tid] = w;
    float total = w;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) total += __shfl_xor(total, off, 64);
    if (lane == 0) part[1][wave] = total;
    __syncthreads();
    const float w_old = expf(old - m);
    total = ((part[1][0] + part[1][1]) + (part[1][2] + part[1][3])) + w_old;
    const int c = 4 * (tid % D4), s0 = tid / D4;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = s0; s < a.n_splits; s += G) o += weight[s] * *reinterpret_cast<const f32x4*>(a.part_o + s * o_part + at + c);
    *reinterpret_cast<f32x4*>(&sum[s0][c]) = o;
    __syncthreads();
    if (tid >= D4) return;
    o = *reinterpret_cast<const f32x4*>(&sum[0][c]);
#pragma unroll
    for (int i = 1; i < G; ++i) o += *reinterpret_cast<const f32x4*>(&sum[i][c]);
    if (a.accumulate) o += w_old * *reinterpret_cast<const f32x4*>(a.o + at + c);
    o *= total == 0.f ? 0.f : 1.0f / total;
    if (tid == 0) a.lse[li] = total == 0.f ? -INFINITY : m + logf(total);
    win_plain::store4(a.o, at + c, a.out_bf16, o[0], o[1], o[2], o[3]);
}

}  // namespace

hipError_t hexi_launch_win_few(const WinFwdArgs& a, int dtype, hipStream_t s)
{
    const AttnGeom& g = a.g;
    FewTable tb;
    int n = 0;
    for (int kh = 0; kh < g.nkv; ++kh) {
        int used = NV;                            // of the group that is open
        for (int h = 0; h < g.nq; ++h) {
            if (g.kv_of_q[h] != kh) continue;
            for (int row = 0; row < g.lq; ++row) {
                if (used == NV) {
                    if (n == HEXI_WIN_FEW_GROUPS) return hipErrorInvalidValue;
                    FewGroup& open = tb.group[n++];
                    open.row = row;
                    open.kvh = (unsigned char)kh;
                    for (int i = 0; i < NV; ++i) open.head[i] = 0xff;
                    used = 0;
                }
                tb.group[n - 1].head[used++] = (unsigned char)h;
            }
        }
    }
    if (g.lq > HEXI_WIN_FEW_ROWS) return hipErrorInvalidValue;
    WinKeys keys[HEXI_WIN_FEW_ROWS] = {};
    for (int row = 0; row < g.lq; ++row) keys[row] = win_keys_of_row(g.ks, seg_pos_of_row(g.qs, row), a.window, a.n_sink);
    const WinSpan<KEYS> span(keys[0], keys[g.lq - 1], g.lc);
    const float c_hi = g.scale * LOG2E_HI;
    FewArgs f = {a.q, a.k, a.v, a.n_splits > 1 ? a.part_o : a.o, a.n_splits > 1 ? a.part_lse : a.lse, g.q_stride_tok, g.q_stride_head, g.kv_stride_tok, g.kv_stride_head,
                       (long long)g.lq * g.nq * g.d, (long long)g.nq * g.lq, g.lq, g.nq, g.lc - 1, span.n_blocks / a.n_splits, span.n_blocks % a.n_splits,
                       a.n_splits == 1 && a.accumulate, a.n_splits == 1 && a.out_bf16, (65536 + g.lq - 1) / g.lq, g.scale, c_hi, fmaf(g.scale, LOG2E_HI, -c_hi) + g.scale * LOG2E_LO, span, {}};
    for (int row = 0; row < g.lq; ++row) f.keys[row] = keys[row];
    const dim3 grid((unsigned)n, (unsigned)a.n_splits);
    if (dtype == HEXI_F32) {
        if (g.d == 128) win_few_kernel<float, 128><<<grid, 64 * NW, 0, s>>>(f, tb, a);
        else win_few_kernel<float, 64><<<grid, 64 * NW, 0, s>>>(f, tb, a);
    } else if (g.d == 128) win_few_kernel<uint16_t, 128><<<grid, 64 * NW, 0, s>>>(f, tb, a);
    else win_few_kernel<uint16_t, 64><<<grid, 64 * NW, 0, s>>>(f, tb, a);
    return hipGetLastError();
}

hipError_t hexi_launch_win_join(const WinFwdArgs& a, hipStream_t s)
{
    const unsigned grid = (unsigned)a.g.lq * (unsigned)a.g.nq;
    if (a.g.d == 128) win_join_kernel<128><<<grid, 256, 0, s>>>(a);
    else win_join_kernel<64><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}
