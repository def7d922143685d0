// Rotary positions with several axes on a shard's rows, alone (hexi_rope) and on the way into or out of the ragged all-to-all
// (hexi_rope_a2a_pack / _unpack).  HBM-bound: every element is read once and written once.
//
// A workgroup owns a few tokens: it forms their sines and cosines in LDS, then walks their pieces in the order in which they lie in memory.  A piece is P pairs of
// columns of one head (one 16-byte load of x on either side); head_dim / (2 P) neighbouring threads take a head's row, the next threads the next head.
//
// Angle: position times frequency in quarter turns, t = pos (c_hi + c_lo) with c the frequency times 2 / pi as two doubles.  With q = rint(t)
// the rest r = fma(pos, c_lo, fma(pos, c_hi, -q)) is exact to 2^-53 whatever the position, and |r| <= 1/2 (an eighth of a turn), so fp32 holds it to
// 2^-26: 2.4e-8 rad.  sin and cos of x = r pi / 2 from their power series up to x^9 and x^10 (the next terms are below 2e-9), swapped and negated by q mod 4.
#include "hexi_rope.h"
#include "hexi_mfma.h"

namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef unsigned int u2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void sincos_turns(int pos, double c_hi, double c_lo, float& sn, float& cs)
{
    const double p = (double)pos, q = rint(p * c_hi);
    const float x = (float)fma(p, c_lo, fma(p, c_hi, -q)) * 1.57079632679489662f, x2 = x * x;
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
    const int n = (int)(long long)q & 3;                    // |q| < 2^63: the host refuses frequencies that would exceed it
    const float a = n & 1 ? c : s, b = n & 1 ? s : c;
    sn = n & 2 ? -a : a;
    cs = (n + 1) & 2 ? -b : b;
}

// P columns as floats from / to memory; nontemporal: nothing is read twice.
template <class T, int P> struct Piece;
template <int P> struct Piece<float, P> {
    static __device__ __forceinline__ void load(const float* p, float (&x)[P])
    {
#pragma unroll
        for (int i = 0; i < P; i += 4) {
            const f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + i));
            x[i] = v[0]; x[i + 1] = v[1]; x[i + 2] = v[2]; x[i + 3] = v[3];
        }
    }
    static __device__ __forceinline__ void store(float* p, const float (&x)[P])
    {
#pragma unroll
        for (int i = 0; i < P; i += 4) __builtin_nontemporal_store(f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]}, reinterpret_cast<f32x4*>(p + i));
    }
};
template <int P> struct Piece<uint16_t, P> {
    static __device__ __forceinline__ void load(const uint16_t* p, float (&x)[P])
    {
        static_assert(P == 8, "a 16-byte piece");
        const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4*>(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(v[i] << 16); x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&x)[P])
    {
        unsigned w[P / 2];
#pragma unroll
        for (int i = 0; i < P / 2; ++i) { const bf16x2 t = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]}; w[i] = __builtin_bit_cast(unsigned, t); }
        if constexpr (P == 8) __builtin_nontemporal_store(u4{w[0], w[1], w[2], w[3]}, reinterpret_cast<u4*>(p));
        else __builtin_nontemporal_store(u2{w[0], w[1]}, reinterpret_cast<u2*>(p));
    }
};

// n / d for n < 2^31: (mulhi(n, mul) + n) >> shift, mul = ceil(2^(32 + shift) / d) - 2^32.
struct Divisor {
    unsigned d, mul, shift;
    explicit Divisor(unsigned x) : d(x), shift(0)
    {
        while ((1ull << shift) < x) ++shift;
        mul = (unsigned)(((1ull << 32) * ((1ull << shift) - x)) / x + 1);
    }
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return (__umulhi(n, mul) + n) >> shift; }
};

// Where a slot's row lies on either side, and whether its head is rotated.
template <class X, class Y> struct Where { const X* x; Y* y; bool rotate; };
struct InTensors {
    RopeTensors t;
    template <class X, class Y> __device__ __forceinline__ Where<X, Y> at(int slot, int row, const RopeGeom&) const
    {
        hexi_rope_tensor a = t.t[0];
        int first = 0;
#pragma unroll
        for (int i = 1; i < HEXI_ROPE_MAX_TENSORS; ++i)
            if (i < t.n && slot >= t.first[i]) { a = t.t[i]; first = t.first[i]; }
        const int h = slot - first;
        return {static_cast<const X*>(a.x) + row * a.x_stride_tok + h * a.x_stride_head, static_cast<Y*>(a.y) + row * a.y_stride_tok + h * a.y_stride_head, true};
    }
};
template <bool PACK> struct InParts {
    RopeParts p;
    template <class X, class Y> __device__ __forceinline__ Where<X, Y> at(int slot, int row, const RopeGeom& g) const
    {
        const long long whole = row * p.x_stride_tok + (long long)p.tb.head[slot] * g.head_dim;
        const long long part = ((long long)p.tb.heads_before[slot] * g.rows + (long long)row * p.tb.n_j[slot] + p.tb.local[slot]) * g.head_dim;
        return {static_cast<const X*>(p.src) + (PACK ? whole : part), static_cast<Y*>(p.dst) + (PACK ? part : whole), p.rotate[slot] != 0};
    }
};

// Workgroup: tokens [tokens blockIdx.x, + tokens), all slots; by_token divides by the pieces of a token, by_row by those of a head's row.
template <class X, class Y, class IN, bool ADJACENT>
__global__ void __launch_bounds__(256) rope_kernel(const RopeGeom g, const IN in, const int tokens, const Divisor by_token, const Divisor by_row)
{
    constexpr int P = 16 / sizeof(X), UNROLL = 4;
    extern __shared__ __attribute__((aligned(16))) float cos_of[];      // [tokens][pairs], and the sines behind them
    const int t0 = (int)blockIdx.x * tokens, n_tokens = g.rows - t0 < tokens ? g.rows - t0 : tokens;
    const int pairs = g.rot_dim / 2;
    float* const sin_of = cos_of + tokens * pairs;
    for (int i = threadIdx.x; i < n_tokens * pairs; i += 256) {
        const int tok = i / pairs, p = i - tok * pairs;
        const int pos = g.positions ? g.positions[(long long)g.axis[p] * g.pos_stride + t0 + tok] : seg_pos_of_row(g.range, t0 + tok);
        float sn, cs;
        sincos_turns(pos, g.turn_hi[p], g.turn_lo[p], sn, cs);
        cos_of[i] = cs;
        sin_of[i] = g.inverse ? -sn : sn;
    }
    __syncthreads();
    const unsigned total = (unsigned)n_tokens * by_token.d;
    for (unsigned i0 = threadIdx.x; i0 < total; i0 += 256 * UNROLL) {
        float a[UNROLL][P], b[UNROLL][P];
        Where<X, Y> w[UNROLL];
        int trig[UNROLL], col_a[UNROLL], col_b[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const unsigned i = i0 + 256 * k;
            if (i >= total) break;
            const unsigned tok = by_token(i), piece = i - tok * by_token.d, slot = by_row(piece);
            const int u = (int)(piece - slot * by_row.d);
            const bool rotated = u < pairs / P;             // otherwise 2 P columns that are copied
            col_a[k] = rotated && !ADJACENT ? P * u : 2 * P * u;
            col_b[k] = rotated && !ADJACENT ? pairs + P * u : 2 * P * u + P;
            w[k] = in.template at<X, Y>((int)slot, t0 + (int)tok, g);
            trig[k] = rotated && w[k].rotate ? (int)tok * pairs + P * u : -1;
            Piece<X, P>::load(w[k].x + col_a[k], a[k]);
            Piece<X, P>::load(w[k].x + col_b[k], b[k]);
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            if (i0 + 256 * k >= total) break;
            if (trig[k] >= 0) {
                float cs[P], sn[P];
#pragma unroll
                for (int e = 0; e < P; e += 4) {
                    const f32x4 c4 = *reinterpret_cast<const f32x4*>(&cos_of[trig[k] + e]), s4 = *reinterpret_cast<const f32x4*>(&sin_of[trig[k] + e]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { cs[e + j] = c4[j]; sn[e + j] = s4[j]; }
                }
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    // HALF: pair e is (a[e], b[e]); ADJACENT: the 2 P columns of a and b in a row are its pairs
                    float& x = ADJACENT ? (e < P / 2 ? a[k][(2 * e) % P] : b[k][(2 * e) % P]) : a[k][e];
                    float& y = ADJACENT ? (e < P / 2 ? a[k][(2 * e + 1) % P] : b[k][(2 * e + 1) % P]) : b[k][e];
                    const float x0 = x, y0 = y;
                    x = x0 * cs[e] - y0 * sn[e];
                    y = y0 * cs[e] + x0 * sn[e];
                }
            }
            Piece<Y, P>::store(w[k].y + col_a[k], a[k]);
            Piece<Y, P>::store(w[k].y + col_b[k], b[k]);
        }
    }
}

template <class X, class Y, class IN> hipError_t launch(const RopeGeom& g, const IN& in, int n_slots, hipStream_t s)
{
    if (n_slots == 0) return hipSuccess;
    const unsigned row = (unsigned)g.head_dim / (2 * (16 / sizeof(X)));
    const Divisor by_token(row * (unsigned)n_slots), by_row(row);
    const RopeShape shape = hexi_rope_shape(g.rows, by_token.d);
    const int tokens = shape.tokens;
    const unsigned grid = shape.grid;
    const size_t lds = 2 * sizeof(float) * (size_t)tokens * (size_t)(g.rot_dim / 2);      // 896 pieces of 8 pairs: 56 KB
    if (lds > 65536) return hipErrorInvalidConfiguration;      // (only where the rows are more bytes than there is memory for)
    if (g.adjacent) rope_kernel<X, Y, IN, true><<<grid, 256, lds, s>>>(g, in, tokens, by_token, by_row);
    else rope_kernel<X, Y, IN, false><<<grid, 256, lds, s>>>(g, in, tokens, by_token, by_row);
    return hipGetLastError();
}

}  // namespace

hipError_t hexi_launch_rope(const RopeGeom& g, const RopeTensors& t, int x_dtype, int y_dtype, hipStream_t s)
{
    const InTensors in{t};
    const int n = t.first[t.n];
    if (x_dtype == HEXI_BF16) return y_dtype == HEXI_BF16 ? launch<uint16_t, uint16_t>(g, in, n, s) : launch<uint16_t, float>(g, in, n, s);
    return y_dtype == HEXI_BF16 ? launch<float, uint16_t>(g, in, n, s) : launch<float, float>(g, in, n, s);
}

hipError_t hexi_launch_rope_a2a(bool pack, const RopeGeom& g, const RopeParts& p, int dtype, hipStream_t s)
{
    if (pack) {
        const InParts<true> in{p};
        return dtype == HEXI_BF16 ? launch<uint16_t, uint16_t>(g, in, p.tb.n_slots, s) : launch<float, float>(g, in, p.tb.n_slots, s);
    }
    const InParts<false> in{p};
    return dtype == HEXI_BF16 ? launch<uint16_t, uint16_t>(g, in, p.tb.n_slots, s) : launch<float, float>(g, in, p.tb.n_slots, s);
}
