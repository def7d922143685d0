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

hipError_t hexi_launch_rope(const RopeGeom& g, const RopeTensors& t, int x_dtype, int y_dtype, hipStream_t s);
hipError_t hexi_launch_rope_a2a(bool pack, const RopeGeom& g, const RopeParts& p, int dtype, hipStream_t s);
