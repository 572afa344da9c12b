// Which kernel takes a product: host code of sizes alone.
#pragma once

#include <algorithm>
#include <cmath>

#include "kernels.h"

namespace craft {

// Which kernel, and the size of its tiles: what is expected to take the least time, from sizes that the host knows.  How rows are
// spread over groups only the GPU knows.  Fitted to times of 70 drawn products of 6 to 3700 rows (1 to 68 groups, every type).  On 70
// others of the same ranges the choice takes 1.01 of the better kernel's time in the geometric mean, units everywhere 1.06 and tiles
// wherever they can be 1.16; on the 23 of them above 10 us 0.99 (at worst 1.08), 1.09 and 1.12.
struct Sizes {
    double rows, groups, columns, slabs;           // groups: those that can have rows
    double matrix;                                 // cycles of a slab's matrix instructions, relative to 16 bits
    double weights;                                // ns that the weights take out of HBM
};
inline Sizes sizes_of(const ProductArgs &a) {
    Sizes z;
    z.rows = (double)a.M;
    z.groups = (double)std::min<int64_t>(a.M, a.G);
    z.columns = a.N;
    z.slabs = (a.row_bytes + 127) / 128;
    z.matrix = a.format == CRAFT_F32 ? 4 : 1;
    z.weights = z.groups * a.N * a.row_bytes * (a.up ? 2 : 1) / 5000;
    return z;
}
// ns of units: their bytes at 60 GB/s a CU, or their matrix instructions; 2 us for a unit that four waves share, 4 to 5.5 for
// four of a wave each, whose results go out at the same time.
inline double stream_time(const ProductArgs &a, const Sizes &z) {
    const double blocks = a.G == 1 ? std::ceil(z.rows / 64) : std::max(z.groups, z.rows / 64 + 0.5 * z.groups);
    const double rows = z.rows / blocks, fx = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const double units = blocks * std::ceil(z.columns / (a.up ? 16 : 32));
    const double bytes = z.slabs * (2 + fx) * 2048, matrix = z.slabs * 4 * fx * 16 / 2 * (z.matrix > 1 ? 8 : 1);
    double time;
    if (units >= 4.0 * a.num_cu) time = std::ceil(units / (4.0 * a.num_cu)) * (std::max(4 * bytes / 60, matrix) + 3500 + 500 * fx);
    else time = std::ceil(units / a.num_cu) * (std::max(bytes / 60, matrix / 4) + 2000);
    return std::max(time, z.weights);
}
// ns of tiles.  A slab of a tile of FW x FX fragments a wave takes 88 FW + 26 FW FX cycles (0.38 us at 4 x 4, 0.77 at 8 x 4, 1.2 at
// 8 x 8), a tile 12000 and 150 for every product of fragments beside its slabs, at 2 GHz.  A third of a tile more for each group is
// assumed, and that behind the first round tiles end at different times; groups of 64 rows in the mean: low tiles.
inline double tile_time(const ProductArgs &a, const Sizes &z, int32_t *width, int32_t *height) {
    double best = 0;
    for (int fw = 8; fw >= 4; fw -= 4)
        for (int fx = fw; fx >= 2; --fx) {
            if (fx == 3) continue;
            const double columns = std::ceil(z.columns / (32 * fw / (a.up ? 2 : 1)));
            const double rows = a.G == 1 ? std::ceil(z.rows / (32 * fx)) : z.rows / (32 * fx) + 0.35 * a.G;
            const double rounds = rows * columns / a.num_cu;
            const double made = rounds <= 1 ? 1 : a.G == 1 ? std::ceil(rounds) : rounds + 0.6;
            const double time = made * (z.slabs * (88 * fw + 26 * fw * fx * z.matrix) + 12000 + 150 * fw * fx) / 2;
            if (best == 0 || time < best) {
                best = time;
                *width = 32 * fw;
                *height = 32 * fx;
            }
        }
    if (z.rows / a.G <= 64) {
        const double rounds = z.groups * std::ceil(z.columns / (a.up ? 64 : 128)) / a.num_cu, fx = z.rows / a.G <= 32 ? 1 : 2;
        best = (rounds < 2 ? std::ceil(rounds) : rounds + 0.5) * (z.slabs * (352 + 104 * fx * z.matrix) + 12500) / 2;
    }
    return std::max(best, z.weights * 5000 / 4500);
}

struct ProductChoice {
    int32_t width, height;                         // of tiles; 0: units
};
inline ProductChoice product_choice(const ProductArgs &a) {
    const bool near = a.src ? a.x_rows * a.x_stride < (int64_t)1 << 32 : a.x_stride < (int64_t)1 << 24;
    ProductChoice c = {};
    if (!near || a.row_bytes < 128 || a.M <= 16) return c;
    const Sizes z = sizes_of(a);
    return tile_time(a, z, &c.width, &c.height) < stream_time(a, z) ? c : ProductChoice{};
}

}  // namespace craft
