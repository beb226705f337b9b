// Tiled products of 8-bit codes with 32-bit results (f8_product.h, gfx950).
#include "f8_product.h"

namespace ozimmu {

hipError_t launch_f8_tiles_exact(const F8Args& a, hipStream_t st) {
    F8Plan plan{};
    plan.parts = 1;
    plan.part_slabs = a.slabs;
    plan.whole = (int)(((int64_t)(a.rows + 127) / 128) * ((a.n + 127) / 128));
    return launch_f8_tile<128, 128, 2, 2, kF8ReadOnTime, true>(a, plan, st);
}

}  // namespace ozimmu
