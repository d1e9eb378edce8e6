// How the products of the projections are cut into tiles and sums, by their sizes.
#pragma once
#include <algorithm>

#include "ops.h"

namespace ndvm {
namespace ops {

constexpr int kStep = 32;       // of the sum, per LDS tile

// How a gated product is cut.  Tiles of 256 x 256, 256 x 128 (n by m) or 128 x 128: by the time of a
// step of the largest tile (1; 8192 x 2048 x 8192), one workgroup a compute unit; the
// others' measured at half and a quarter of the work, the smallest with two workgroups side by
// side.  Their loads take 1.5 and 2 times the bandwidth for the same work, which is what
// holds them back.  Too few tiles for the compute units, and long sums: several workgroups
// share a sum, of 32 steps at least (about 15 us, three times what adding their parts up costs).
struct Gated {
    int64_t ba, bb, splits;
};
inline Gated cut_tiles(int64_t rows, int64_t steps, int64_t columns) {
    const auto tiles = [&](int64_t ba, int64_t bb) { return ceil_div(columns, ba) * ceil_div(rows, bb); };
    const int64_t large = ceil_div(tiles(256, 256), kCus) * 100, middle = ceil_div(tiles(256, 128), kCus) * 56;
    const int64_t few_tiles = tiles(128, 128), small = few_tiles <= kCus ? 40 : ceil_div(few_tiles, 2 * kCus) * 64;
    if (large <= middle && large <= small) return Gated{256, 256, 1};
    if (middle <= small) return Gated{256, 128, 1};
    const int64_t splits = few_tiles ? std::min(2 * kCus / few_tiles, std::min<int64_t>(steps / 32, 16)) : 1;
    return Gated{128, 128, std::max<int64_t>(splits, 1)};
}
inline int64_t steps_of(int dtype, int64_t n_in) { return ceil_div(n_in, kStep) * (dtype == NDVM_F32 ? 6 : 1); }
// (ceil(n_out / 64) = ceil(2 n_out / 128): a gated tile holds both weights' columns)
inline Gated gated_cut(int dtype, int64_t rows, int64_t n_in, int64_t n_out) { return cut_tiles(rows, steps_of(dtype, n_in), 2 * n_out); }
// Of one weight.
inline Gated linear_cut(int dtype, int64_t rows, int64_t n_in, int64_t n_out) { return cut_tiles(rows, steps_of(dtype, n_in), n_out); }

// How the gradient's two plain products are cut: tiles of `tile` squared, each one's sum over so
// many workgroups.  Both have the same number of steps in all.  Unless there are tiles for two
// workgroups a compute unit, sums are cut into pieces of about a compute unit's share, of
// at least 16 steps, but not so many that the pieces' sums cost more traffic than they save.
struct Pieces {
    int64_t tile, dx, dw;
};
inline Pieces cut_gradient(int dtype, int64_t rows, int64_t n_in, int64_t width) {
    const int64_t pairs = dtype == NDVM_F32 ? 6 : 1;
    const int64_t steps_dx = width / kStep * pairs, steps_dw = ceil_div(rows, 64) * 2 * pairs;
    const auto tiles_dx = [&](int64_t t) { return ceil_div(n_in, t) * ceil_div(rows, t); };
    const auto tiles_dw = [&](int64_t t) { return ceil_div(n_in, t) * ceil_div(width, t); };
    const auto work = [&](int64_t t) { return tiles_dx(t) * steps_dx + tiles_dw(t) * steps_dw; };
    Pieces c{work(256) >= 32 * kCus ? 256 : 128, 1, 1};
    if (tiles_dx(c.tile) + tiles_dw(c.tile) >= 4 * kCus) return c;
    const int64_t share = std::max<int64_t>(16, work(c.tile) / kCus);
    const auto cut = [&](int64_t steps) { return std::max<int64_t>(1, std::min<int64_t>(32, (steps + share / 2) / share)); };
    c.dx = cut(steps_dx);
    c.dw = cut(steps_dw);
    return c;
}
inline Pieces pieces(int dtype, int64_t rows, int64_t n_in, int64_t n_out) { return cut_gradient(dtype, rows, n_in, 2 * ceil_div(n_out, 64) * 64); }
// Of one weight.
inline Pieces linear_pieces(int dtype, int64_t rows, int64_t n_in, int64_t n_out) { return cut_gradient(dtype, rows, n_in, ceil_div(n_out, 64) * 64); }

}  // namespace ops
}  // namespace ndvm
