// What the norms around a block share between their call (resnorm.hip) and their kernels (resnorm_kernels.h, built once per element type).
#pragma once

#include "common.h"
#include "values.h"

namespace slicegcn {
namespace resnorm {

constexpr int NONE = SLICEGCN_NORM_NONE, LAYER = SLICEGCN_NORM_LAYER;
constexpr int ELEMS = 8;              // elements of a row per lane, at most: the backward pass holds two rows' operands, parameters and sums
constexpr int WIDE = 1024 * ELEMS;    // wider rows: twice as many
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

// A row's accesses over lanes: as few lanes as the registers of a row allow, so that a sum over the row takes few steps.  A power of two up to 512 (8 at
// least, 4 for rows of four accesses), beyond that whole wavefronts: bf16 rows of 5000 columns on 10 wavefronts, on 16 (RMS norms, forward 3.5 and
// 2.7 TB/s, backward with layer norms 4.1 and 3.5), but of 2500 on 5, on 8 (5.0 and 5.1, 3.3 and 3.5).
// fp32 rows above 8192 columns take all 16: fewer elements a lane count more there (9000 columns, 9 wavefronts, 16: 3.4 and 3.9, 1.7 and 2.3).
struct Shape {
    int lanes, accesses; // per row, per lane
    Shape(int32_t width, int v)
    {
        const int all = (width + v - 1) / v, most = v == 1 ? 1 : (width <= WIDE ? ELEMS : 2 * ELEMS) / v;
        lanes = all <= 4 ? 4 : 8;
        while (lanes < 512 && lanes * most < all) lanes *= 2;
        if (lanes * most < all) lanes = width > WIDE && v == 4 ? 1024 : (all + 64 * most - 1) / (64 * most) * 64;
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

// Whether the workgroups of the forward pass take many rows each, one requested ahead, with parameters and columns found out once: rows of several
// wavefronts, whose wavefronts wait for each other, and 16-bit rows that do not fill their lanes, which are bound by instructions.  Others
// are as fast or faster with a row to each group of lanes.  TB/s of rows read and written, looping / not: bf16 rows of 100 with layer norms
// 4.7 / 3.3, of 256 with RMS norms 5.0 / 5.7, of 4096 (several wavefronts) 5.5 / 5.0, fp32 rows of 256 5.3 / 5.6.
constexpr bool fwd_loops(bool multi, bool full, int bytes) { return multi || (bytes == 2 && !full); }

// Launches a direction for one element type
template <class T> void launch_fwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream);
template <class T> void launch_bwd(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream);

} // namespace resnorm
} // namespace slicegcn
