// What the norms around a block share between their call (resnorm.hip) and their kernels (resnorm_kernels.h, built once per element type).
#pragma once

#include "common.h"
#include "values.h"

namespace slicegcn {
namespace resnorm {

constexpr int NONE = SLICEGCN_NORM_NONE, LAYER = SLICEGCN_NORM_LAYER;
constexpr int ELEMS = 8;              // elements of a row per lane, at most: the backward pass holds two rows' operands, parameters and sums
constexpr int WIDE = 1024 * ELEMS;    // wider rows: twice as many
constexpr int FWD_BLOCKS = 4096;      // workgroups of the forward pass, at most: parameters are read once per workgroup
constexpr int PLANES = 4;             // sums over rows: du * hn, du, dH * s * yn, dH * s (without s where the gate is per column)

struct RowPtr {
    char *data;
    int64_t ld;
};

struct Args {
    RowPtr x, y, gate, h, u, dh, du, dx, dy, dgate;
    float *stats;
    const float *post_w, *post_b, *pre_w, *pre_b, *gate_col;
    float *partial;
    int64_t n;
    int32_t width, lanes; // lanes of a row
    int32_t post, pre;
    float residual, eps, inv_width;
    bool sigmoid, past_cache;
    uint32_t planes; // bit p: the sums of plane p are wanted
};

// A row's accesses over lanes: as few lanes as the registers of a row allow (8 at least: a whole line), so that a sum over the row takes few steps.
struct Shape {
    int lanes, accesses; // per row, per lane
    Shape(int32_t width, int v)
    {
        const int all = (width + v - 1) / v, most = v == 1 ? 1 : (width <= WIDE ? ELEMS : 2 * ELEMS) / v;
        lanes = 8;
        while (lanes * most < all) lanes *= 2;
        accesses = (all + lanes - 1) / lanes;
    }
    int threads() const { return lanes > 256 ? lanes : 256; }
    bool full(int32_t width, int v) const { return width == lanes * accesses * v; }
};

inline int access_elems(int32_t width, int32_t type)
{
    const int v = 16 / type_bytes(type);
    return width < v ? 1 : v;
}

// Launches a direction for one element type
template <class T> void launch_fwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream);
template <class T> void launch_bwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream);

} // namespace resnorm
} // namespace slicegcn
