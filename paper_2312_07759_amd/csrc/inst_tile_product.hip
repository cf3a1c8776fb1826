// Tile products: shapes and types.
#include "layers.h"

namespace idkm {

template <typename T, int BM, int BN, int WM, int WN, int ST>
static TileShape shape() {
    return TileShape{BM, BN, 64 * WM * WN, (size_t)ST * (BM + BN) * TP_STEP, &k_tile_product<T, BM, BN, WM, WN, ST>};
}

template <typename T>
static TileShape shape_of(int which) {
    switch (which) {
        case 0: return shape<T, 256, 256, 2, 4, 2>();
        case 1: return shape<T, 256, 128, 4, 2, 3>();
        case 2: return shape<T, 128, 128, 2, 2, 3>();
        default: return shape<T, 64, 64, 2, 2, 4>();
    }
}

TileShape tile_shape(int dtype, int which) {
    if (dtype == 0) return shape_of<float>(which);
    if (dtype == 1) return shape_of<f16>(which);
    return shape_of<bf16>(which);
}

}  // namespace idkm
