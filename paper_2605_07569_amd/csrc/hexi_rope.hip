// Rotary positions with several axes on a shard's rows, alone (hexi_rope) and on the way into or out of the ragged all-to-all
// (hexi_rope_a2a_pack / _unpack).  HBM-bound: every element is read once and written once.
//
// A thread owns P pairs of columns of one row (one 16-byte piece of x on either side), forms their sines and cosines once, in registers,
// and walks the heads with them.  A row of a head is head_dim / (2 P) neighbouring threads, so a wavefront reads whole rows of
// 64 / (head_dim / 2 P) tokens.
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

// Where a slot's row lies on either side, and whether its head is rotated.
template <class X, class Y> struct Where { const X* x; Y* y; bool rotate; };
struct InTensors {
    RopeTensors t;
    __device__ __forceinline__ int slots() const { return t.first[t.n]; }
    template <class X, class Y> __device__ __forceinline__ Where<X, Y> at(int slot, int row, const RopeGeom&) const
    {
        int i = 0;
        while (slot >= t.first[i + 1]) ++i;
        const hexi_rope_tensor& a = t.t[i];
        const int h = slot - t.first[i];
        return {static_cast<const X*>(a.x) + row * a.x_stride_tok + h * a.x_stride_head, static_cast<Y*>(a.y) + row * a.y_stride_tok + h * a.y_stride_head, true};
    }
};
template <bool PACK> struct InParts {
    RopeParts p;
    __device__ __forceinline__ int slots() const { return p.tb.n_slots; }
    template <class X, class Y> __device__ __forceinline__ Where<X, Y> at(int slot, int row, const RopeGeom& g) const
    {
        const long long whole = row * p.x_stride_tok + (long long)p.tb.head[slot] * g.head_dim;
        const long long part = ((long long)p.tb.heads_before[slot] * g.rows + (long long)row * p.tb.n_j[slot] + p.tb.local[slot]) * g.head_dim;
        return {static_cast<const X*>(p.src) + (PACK ? whole : part), static_cast<Y*>(p.dst) + (PACK ? part : whole), p.rotate[slot] != 0};
    }
};

// Workgroup (x, y): rows [x rows_per_block, ..), slots [y slots_per_block, ..).
template <class X, class Y, class IN, bool ADJACENT>
__global__ void __launch_bounds__(256) rope_kernel(const RopeGeom g, const IN in, const int rows_per_block, const int slots_per_block)
{
    constexpr int P = 16 / sizeof(X);
    const int units = g.head_dim / (2 * P);                 // threads of a row
    const int local = (int)threadIdx.x / units, u = (int)threadIdx.x - local * units;
    const int row = (int)blockIdx.x * rows_per_block + local;
    if (local >= rows_per_block || row >= g.rows) return;
    const bool rotated = u < g.rot_dim / (2 * P);           // otherwise 2 P columns that are copied
    const int col_a = rotated && !ADJACENT ? P * u : 2 * P * u, col_b = rotated && !ADJACENT ? g.rot_dim / 2 + P * u : 2 * P * u + P;
    float sn[P], cs[P];
    if (rotated) {
        const int own = g.positions ? 0 : seg_pos_of_row(g.range, row);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = P * u + i;
            const int pos = g.positions ? g.positions[(long long)g.axis[p] * g.pos_stride + row] : own;
            sincos_turns(pos, g.turn_hi[p], g.turn_lo[p], sn[i], cs[i]);
            if (g.inverse) sn[i] = -sn[i];
        }
    }
    const int first = (int)blockIdx.y * slots_per_block, end = first + slots_per_block < in.slots() ? first + slots_per_block : in.slots();
    constexpr int UNROLL = 4;
    for (int s = first; s < end; s += UNROLL) {
        float a[UNROLL][P], b[UNROLL][P];
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
            if (s + i < end) {
                const Where<X, Y> w = in.template at<X, Y>(s + i, row, g);
                Piece<X, P>::load(w.x + col_a, a[i]);
                Piece<X, P>::load(w.x + col_b, b[i]);
            }
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
            if (s + i < end) {
                const Where<X, Y> w = in.template at<X, Y>(s + i, row, g);
                if (rotated && w.rotate) {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        // HALF: pair e is (a[e], b[e]); ADJACENT: the 2 P columns of a and b in a row are its pairs
                        float& x = ADJACENT ? (e < P / 2 ? a[i][(2 * e) % P] : b[i][(2 * e) % P]) : a[i][e];
                        float& y = ADJACENT ? (e < P / 2 ? a[i][(2 * e + 1) % P] : b[i][(2 * e + 1) % P]) : b[i][e];
                        const float x0 = x, y0 = y;
                        x = x0 * cs[e] - y0 * sn[e];
                        y = y0 * cs[e] + x0 * sn[e];
                    }
                }
                Piece<Y, P>::store(w.y + col_a, a[i]);
                Piece<Y, P>::store(w.y + col_b, b[i]);
            }
    }
}

template <class X, class Y, class IN> hipError_t launch(const RopeGeom& g, const IN& in, int n_slots, hipStream_t s)
{
    if (n_slots == 0) return hipSuccess;
    const int rows_per_block = 256 / (g.head_dim / (2 * (16 / (int)sizeof(X))));
    const unsigned row_blocks = (unsigned)((g.rows + rows_per_block - 1) / rows_per_block);
    int per = n_slots;
    const dim3 grid(row_blocks, (unsigned)((n_slots + per - 1) / per));
    if (g.adjacent) rope_kernel<X, Y, IN, true><<<grid, 256, 0, s>>>(g, in, rows_per_block, per);
    else rope_kernel<X, Y, IN, false><<<grid, 256, 0, s>>>(g, in, rows_per_block, per);
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
