// Windowed attention element by element, as its definition says it.
//
// A workgroup of 64 to 1024 threads takes its stationary rows (or keys) eight neighbouring lanes to a row, D / 8 columns each, which walk the row's own runs
// of the other tensor's rows one by one.  No value of a row that the mask excludes is ever read into a sum, so what is not finite there
// stays there.
#pragma once
#include "hexi_window.h"

namespace { namespace win_plain {

constexpr int LANES = 8;      // to a row

template <class T> __device__ __forceinline__ void load4(const T* p, float* x)
{
    if constexpr (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}
template <int N, class T> __device__ __forceinline__ void load_cols(const T* p, float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) load4(p + i, x + i);
}
// columns [at, at + 4) of a dense output, rounded to nearest even where it is bf16
__device__ __forceinline__ void store4(void* out, long long at, bool bf16, float a, float b, float c, float d)
{
    if (bf16) {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        const b4 v = {(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = __builtin_bit_cast(uint2, v);
    } else {
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
    }
}
template <int N> __device__ __forceinline__ float dot(const float (&a)[N], const float (&b)[N])
{
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) s[i & 3] = fmaf(a[i], b[i], s[i & 3]);
    float x = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int off = 1; off < LANES; off *= 2) x += __shfl_xor(x, off, 64);      // the lanes of a row run the same iterations
    return x;
}

// o and lse of rows [row0, row0 + rows) of head h from the keys in [keys.x, keys.y) and [keys.z, keys.w), those of a split of the unit's run of blocks.
template <class T, int D> __device__ __forceinline__ void fwd_unit(const WinFwdArgs& a, const int h, const int row0, const int rows, const int4 keys, const int split)
{
    constexpr int N = D / LANES;
    const AttnGeom& g = a.g;
    const int col = (int)threadIdx.x % LANES * N, end_row = row0 + rows < g.lq ? row0 + rows : g.lq;
    for (int row = row0 + (int)threadIdx.x / LANES; row < end_row; row += (int)blockDim.x / LANES) {
        const WinKeys w = win_keys_of_row(g.ks, seg_pos_of_row(g.qs, row), a.window, a.n_sink);
        const T* k = static_cast<const T*>(a.k) + (long long)g.kv_of_q[h] * g.kv_stride_head + col;
        const T* v = static_cast<const T*>(a.v) + (long long)g.kv_of_q[h] * g.kv_stride_head + col;
        float q[N], acc[N];
        load_cols(static_cast<const T*>(a.q) + (long long)row * g.q_stride_tok + (long long)h * g.q_stride_head + col, q);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
        float m = -INFINITY, l = 0.f;
        for (int part = 0; part < 4; ++part) {
            const int p0 = part & 2 ? keys.z : keys.x, p1 = part & 2 ? keys.w : keys.y, k0 = part & 1 ? w.lo : 0, k1 = part & 1 ? w.hi : w.sink;
            for (int j = k0 > p0 ? k0 : p0, end = k1 < p1 ? k1 : p1; j < end; ++j) {
                float x[N];
                load_cols(k + (long long)j * g.kv_stride_tok, x);
                const float s = dot(q, x) * g.scale;
                load_cols(v + (long long)j * g.kv_stride_tok, x);
                if (s > m) {
                    const float alpha = expf(m - s);   // (m = -inf: 0)
                    m = s;
                    l *= alpha;
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] *= alpha;
                }
                // scores of -inf alone so far weigh nothing; a NaN score, or one of +inf, makes the row NaN
                const float p = s == -INFINITY ? 0.f : expf(s - m);
                l += p;
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = fmaf(p, x[i], acc[i]);
            }
        }
        float lse = l == 0.f ? -INFINITY : m + logf(l);
        float wa = 0.f, wb = l == 0.f ? 0.f : 1.0f / l;
        float* lp = a.out_lse(split) + (long long)h * g.lq + row;
        float* out = a.out_o(split);
        if (a.merges()) {
            const float old = *lp, mm = fmaxf(old, lse);
            if (mm != -INFINITY) {
                const float ea = expf(old - mm), eb = expf(lse - mm), r = 1.0f / (ea + eb);
                wa = ea * r;
                wb *= eb * r;
                lse = mm + logf(ea + eb);
            }
        }
        __builtin_amdgcn_wave_barrier();              // the lanes of a row have read the old value
        if (col == 0) *lp = lse;
        const long long at = ((long long)row * g.nq + h) * D + col;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
            if (a.merges()) old = *reinterpret_cast<const float4*>(out + at + i);
            store4(out, at + i, a.rounds(), wa * old.x + wb * acc[i], wa * old.y + wb * acc[i + 1], wa * old.z + wb * acc[i + 2], wa * old.w + wb * acc[i + 3]);
        }
    }
}

// The keys of blocks [i0, i1) of a unit's run, as fwd_unit takes them.
template <int B> __device__ __forceinline__ int4 keys_of_blocks(const WinSpan<B>& span, int i0, int i1)
{
    const int s = span.n_sink_blocks, first = i0 > s ? i0 : s;
    return make_int4(B * i0, B * (i1 < s ? i1 : s), B * (first + span.skip), i1 > first ? B * (i1 + span.skip) : 0);
}

// dq of rows [row0, row0 + rows) of head h.
template <class T, int D> __device__ __forceinline__ void dq_unit(const WinBwdArgs& a, const int h, const int row0, const int rows)
{
    constexpr int N = D / LANES;
    const AttnGeom& g = a.g;
    const int col = (int)threadIdx.x % LANES * N, end_row = row0 + rows < g.lq ? row0 + rows : g.lq;
    for (int row = row0 + (int)threadIdx.x / LANES; row < end_row; row += (int)blockDim.x / LANES) {
        const WinKeys w = win_keys_of_row(g.ks, seg_pos_of_row(g.qs, row), a.window, a.n_sink);
        const T* k = static_cast<const T*>(a.k) + (long long)g.kv_of_q[h] * g.kv_stride_head + col;
        const T* v = static_cast<const T*>(a.v) + (long long)g.kv_of_q[h] * g.kv_stride_head + col;
        const long long q_at = (long long)row * g.q_stride_tok + (long long)h * g.q_stride_head + col;
        float q[N], d_o[N], acc[N];
        load_cols(static_cast<const T*>(a.q) + q_at, q);
        load_cols(static_cast<const T*>(a.d_o) + q_at, d_o);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
        const float lse = a.lse[(long long)h * g.lq + row], delta = a.delta[(long long)h * g.lq + row];
        const bool live = fabsf(lse) != INFINITY;
        for (int part = 0; part < 2; ++part)
            for (int j = part ? w.lo : 0, end = !live ? 0 : part ? w.hi : w.sink; j < end; ++j) {
                float x[N], y[N];
                load_cols(k + (long long)j * g.kv_stride_tok, x);
                load_cols(v + (long long)j * g.kv_stride_tok, y);
                const float ds = expf(dot(q, x) * g.scale - lse) * (dot(d_o, y) - delta);
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = fmaf(ds, x[i], acc[i]);
            }
        const long long at = ((long long)row * g.nq + h) * D + col;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float4 old = make_float4(0.f, 0.f, 0.f, 0.f);
            if (!a.out_bf16) old = *reinterpret_cast<const float4*>(a.dq + at + i);
            store4(a.dq, at + i, a.out_bf16, fmaf(g.scale, acc[i], old.x), fmaf(g.scale, acc[i + 1], old.y), fmaf(g.scale, acc[i + 2], old.z), fmaf(g.scale, acc[i + 3], old.w));
        }
    }
}

// dk and dv of keys [col0, col0 + keys) of kv head kvh.
template <class T, int D> __device__ __forceinline__ void dkdv_unit(const WinBwdArgs& a, const int kvh, const int col0, const int keys)
{
    constexpr int N = D / LANES;
    const AttnGeom& g = a.g;
    const int col = (int)threadIdx.x % LANES * N, end_key = col0 + keys < g.lc ? col0 + keys : g.lc;
    for (int key = col0 + (int)threadIdx.x / LANES; key < end_key; key += (int)blockDim.x / LANES) {
        const WinRows w = win_rows_of_key(g.qs, seg_pos_of_row(g.ks, key), a.window, a.n_sink);
        const long long kv_at = (long long)key * g.kv_stride_tok + (long long)kvh * g.kv_stride_head + col;
        float k[N], v[N], dk[N], dv[N];
        load_cols(static_cast<const T*>(a.k) + kv_at, k);
        load_cols(static_cast<const T*>(a.v) + kv_at, v);
#pragma unroll
        for (int i = 0; i < N; ++i) { dk[i] = 0.f; dv[i] = 0.f; }
        for (int h = 0; h < g.nq; ++h) {
            if (g.kv_of_q[h] != kvh) continue;
            const T* q = static_cast<const T*>(a.q) + (long long)h * g.q_stride_head + col;
            const T* d_o = static_cast<const T*>(a.d_o) + (long long)h * g.q_stride_head + col;
            for (int i = w.first; i < w.end; ++i) {
                const float lse = a.lse[(long long)h * g.lq + i], delta = a.delta[(long long)h * g.lq + i];
                if (fabsf(lse) == INFINITY) continue;
                float x[N], y[N];
                load_cols(q + (long long)i * g.q_stride_tok, x);
                load_cols(d_o + (long long)i * g.q_stride_tok, y);
                const float p = expf(dot(k, x) * g.scale - lse), ds = p * (dot(v, y) - delta);
#pragma unroll
                for (int c = 0; c < N; ++c) { dv[c] = fmaf(p, y[c], dv[c]); dk[c] = fmaf(ds, x[c], dk[c]); }
            }
        }
        const long long at = ((long long)key * g.nkv + kvh) * D + col;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float4 ok = make_float4(0.f, 0.f, 0.f, 0.f), ov = ok;
            if (a.accumulate) { ok = *reinterpret_cast<const float4*>(a.dk + at + i); ov = *reinterpret_cast<const float4*>(a.dv + at + i); }
            store4(a.dk, at + i, a.out_bf16, fmaf(g.scale, dk[i], ok.x), fmaf(g.scale, dk[i + 1], ok.y), fmaf(g.scale, dk[i + 2], ok.z), fmaf(g.scale, dk[i + 3], ok.w));
            store4(a.dv, at + i, a.out_bf16, dv[i] + ov.x, dv[i + 1] + ov.y, dv[i + 2] + ov.z, dv[i + 3] + ov.w);
        }
    }
}

// dk and dv of keys that no row of the unit's part sees: zeros, to its slot or, unless they would be added, to the outputs.
template <int D> __device__ __forceinline__ void no_dkdv(const WinBwdArgs& a, const WinUnit& unit, const int keys)
{
    for (int i = (int)threadIdx.x; i < keys * (D / 4); i += (int)blockDim.x)
        for (int which = 0; which < 2; ++which) {
            const int key = unit.tile * keys + i / (D / 4);
            if (unit.n_parts > 1) store4(a.part, (unit.slot * 2 + which) * (keys * D) + 4 * i, false, 0.f, 0.f, 0.f, 0.f);
            else if (!a.accumulate && key < a.g.lc) store4(which ? a.dk : a.dv, ((long long)key * a.g.nkv + unit.kvh) * D + 4 * (i % (D / 4)), a.out_bf16, 0.f, 0.f, 0.f, 0.f);
        }
}

} }  // namespace win_plain
