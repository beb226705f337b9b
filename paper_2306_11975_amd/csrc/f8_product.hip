// Tiled products of 8-bit codes with 16-bit results (f8_product.h, gfx950).
#include "f8_product.h"

namespace ozimmu {

hipError_t launch_f8_tiles(const F8Args& a, const F8Choice& c, hipStream_t st) {
    const F8Plan plan{0, 0, c.whole, c.parts, c.part_slabs};
    switch (c.shape) {
        case kF8Tile128: return launch_f8_tile<128, 128, 2, 2, false>(a, plan, st);
        case kF8Tile64x128: return launch_f8_tile<64, 128, 2, 2, false>(a, plan, st);
        case kF8Tile64: return launch_f8_tile<64, 64, 2, 2, false>(a, plan, st);
        default: return launch_f8_tile<32, 64, 2, 2, false>(a, plan, st);
    }
}

}  // namespace ozimmu
