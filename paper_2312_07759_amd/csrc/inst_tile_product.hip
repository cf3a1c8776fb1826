// Tile products: shapes and types.
#include "layers.h"

namespace idkm {

// resident: workgroups that the device holds at once; us: of one step of all of them, measured over products of 512 .. 4096 rows,
// 512 .. 4096 columns and sums of 512 .. 4096.
template <typename T, int BM, int BN, int WM, int WN, int ST, int SC = 0>
static TileShape shape(int resident, float us) {
    return TileShape{BM, BN, 64 * WM * WN, (size_t)ST * ((BM + BN) * TP_STEP + SC * BN * 4), &k_tile_product<T, BM, BN, WM, WN, ST, SC>, resident, us};
}

template <typename T>
static TileShape shape_of(int which, int scaled) {
    if constexpr (sizeof(T) == 4) {
        // two wavefronts a SIMD hold 128 x 128 sums; four, and larger tiles, are slower
        switch (which) {
            case 0: return shape<T, 128, 128, 2, 4, 3>(256, 2.03f);
            case 1: return shape<T, 64, 64, 2, 2, 4>(512, 1.1f);
        }
    } else if (scaled == 0) {
        switch (which) {
            case 0: return shape<T, 256, 256, 2, 4, 2>(256, 2.0f);
            case 1: return shape<T, 256, 128, 4, 4, 3>(256, 1.0f);
            case 2: return shape<T, 128, 128, 2, 4, 2>(512, 1.02f);
            case 3: return shape<T, 128, 128, 2, 4, 4>(256, 0.56f);
            case 4: return shape<T, 64, 64, 2, 2, 4>(512, 0.41f);
        }
    } else if (scaled == 1) {
        // larger tiles are no faster (2048 x 4096 x 4096: 74 us with the first, with 256 x 128 by eight wavefronts 74, by sixteen 75), and 256 x 256
        // leaves no registers for them
        switch (which) {
            case 0: return shape<T, 128, 128, 2, 4, 2, 1>(512, 1.18f);
            case 1: return shape<T, 128, 128, 2, 4, 4, 1>(256, 0.69f);
            case 2: return shape<T, 64, 64, 2, 2, 4, 1>(512, 0.48f);
        }
    } else {
        switch (which) {
            case 0: return shape<T, 128, 128, 2, 4, 2, 2>(512, 1.48f);
            case 1: return shape<T, 128, 128, 2, 4, 4, 2>(256, 0.88f);
            case 2: return shape<T, 64, 64, 2, 2, 4, 2>(512, 0.6f);
        }
    }
    return TileShape{};
}

TileShape tile_shape(int dtype, int which, int scaled) {
    if (dtype == 0) return shape_of<float>(which, scaled);
    if (dtype == 1) return shape_of<f16>(which, scaled);
    return shape_of<bf16>(which, scaled);
}

}  // namespace idkm
