// What the products by expert and the 8-bit products share on the host.
#ifndef WPK_GROUPED_H
#define WPK_GROUPED_H

#include "wpk_product.h"
#include "wpk_q8.h"

namespace wpk {

struct Q8Args {
    LinearArgs a;                                     // x and w e4m3; bias, residual and y of the kernel's type
    const float *x_scales, *w_scales;
    int64_t x_scale_stride, w_scale_stride, w_scale_group_stride;
};

// Workgroups for tiles of tile_m rows and tile_n columns of y of products by expert: as many as there could be.
struct GroupedGrid {
    int64_t tiles;
    GroupedGrid(const LinearArgs &a, int tile_m, int tile_n)
    {
        // (each expert has one tile at most that is not full)
        const int64_t tiles_m = ((int64_t)a.m + (int64_t)a.groups * (tile_m - 1)) / tile_m;
        tiles = (tiles_m < a.m ? tiles_m : a.m) * ((a.n + tile_n - 1) / tile_n);
    }
};

int grouped_q8(const Q8Args &q, int y_dtype, bool gated, hipStream_t st);

}  // namespace wpk
#endif
