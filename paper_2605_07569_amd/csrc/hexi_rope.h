// Rotary positions: what the host hands to the kernels of hexi_rope.hip.
#pragma once
#include "hexi_internal.h"
#include "hexi_a2a_table.h"

struct RopeGeom {
    int rows, head_dim, rot_dim;
    int adjacent;                     // pairs (2 p, 2 p + 1) instead of (p, p + rot_dim / 2)
    int inverse;
    SegTable range;
    const int* positions;             // nullptr: global positions
    long long pos_stride;
    // quarter turns per position: inv_freq * 2 / pi as the sum of two doubles
    double turn_hi[HEXI_ROPE_MAX_DIM / 2], turn_lo[HEXI_ROPE_MAX_DIM / 2];
    unsigned char axis[HEXI_ROPE_MAX_DIM / 2];
};

struct RopeTensors {
    int n;
    int first[HEXI_ROPE_MAX_TENSORS + 1];      // slots (heads of all tensors, one after the other) of each tensor
    hexi_rope_tensor t[HEXI_ROPE_MAX_TENSORS];
};

struct RopeParts {
    A2ATable tb;
    unsigned char rotate[HEXI_A2A_MAX_SLOTS];
    const void* src;
    void* dst;
    long long x_stride_tok;           // of the [rows][heads] side, elements
};

// Tokens of a workgroup of 256 threads, and workgroups, for so many pieces (two loads of 16 bytes) a token: 2 or 3 pieces a thread, so that many workgroups are under way at
// different places, unless there are too few rows to go round; and more where the launch would have 2^32 threads.
// us for 1 / 2 / 4 / 16 tokens, 128 columns: 32768 rows of 40 heads (320 pieces a token) 119 / 107 / 112 / 127; 16384 rows of 40 heads packed into 48 slots (384) 79 / 67 / 70 / 78;
// 8191 rows of 32 heads from fp32 to bf16 (512) 38.5 / 40.8 / 43.6 / 43.1.
struct RopeShape { int tokens; unsigned grid; };
inline RopeShape hexi_rope_shape(int rows, unsigned pieces)
{
    const long long n = rows, most = pieces < 896 ? 896 / pieces : 1, share = (n + 1023) / 1024, least = (n + (1 << 24) - 2) / ((1 << 24) - 1);
    long long tokens = most < share ? most : share;
    tokens = tokens > least ? tokens : least;
    return {(int)tokens, (unsigned)((n + tokens - 1) / tokens)};
}

hipError_t hexi_launch_rope(const RopeGeom& g, const RopeTensors& t, int x_dtype, int y_dtype, hipStream_t s);
hipError_t hexi_launch_rope_a2a(bool pack, const RopeGeom& g, const RopeParts& p, int dtype, hipStream_t s);
