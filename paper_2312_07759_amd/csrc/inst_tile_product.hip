// Tile products: shapes and types.
#include "layers.h"

namespace idkm {

// resident: workgroups that the device holds at once; us: of one step of all of them, measured over products of 512 .. 4096 rows,
// 512 .. 4096 columns and sums of 512 .. 4096.
template <typename T, int BM, int BN, int WM, int WN, int ST>
static TileShape shape(int resident, float us) {
    return TileShape{BM, BN, 64 * WM * WN, (size_t)ST * (BM + BN) * TP_STEP, &k_tile_product<T, BM, BN, WM, WN, ST>, resident, us};
}

template <typename T>
static TileShape shape_of(int which) {
    if constexpr (sizeof(T) == 4) {
        // two wavefronts a SIMD hold 128 x 128 sums; four, and larger tiles, are slower
        switch (which) {
            case 0: return shape<T, 128, 128, 2, 4, 3>(256, 2.03f);
            case 1: return shape<T, 64, 64, 2, 2, 4>(512, 1.1f);
        }
    } else {
        switch (which) {
            case 0: return shape<T, 256, 256, 2, 4, 2>(256, 2.0f);
            case 1: return shape<T, 256, 128, 4, 4, 3>(256, 1.0f);
            case 2: return shape<T, 128, 128, 2, 4, 2>(512, 1.02f);
            case 3: return shape<T, 128, 128, 2, 4, 4>(256, 0.56f);
            case 4: return shape<T, 64, 64, 2, 2, 4>(512, 0.41f);
        }
    }
    return TileShape{};
}

TileShape tile_shape(int dtype, int which) {
    if (dtype == 0) return shape_of<float>(which);
    if (dtype == 1) return shape_of<f16>(which);
    return shape_of<bf16>(which);
}

}  // namespace idkm
