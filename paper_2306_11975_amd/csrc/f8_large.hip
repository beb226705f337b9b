// Large tiles of 8-bit codes (f8_large.h, gfx950).
#include "f8_large.h"

namespace ozimmu {
namespace {

template <bool Q_ROWS, int TYPE>
hipError_t launch(const F8Args& a, const F8Plan& plan, int64_t grid, hipStream_t st) {
    constexpr auto kernel = f8_large_kernel<Q_ROWS, TYPE>;
    if (hipError_t e = allow_dynamic_lds<kernel>(kLargeBytes); e != hipSuccess) return e;
    kernel<<<dim3((unsigned)grid), dim3(256), kLargeBytes, st>>>(a, plan);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f8_large(const F8Args& a, hipStream_t st) {
    F8Plan plan{};
    plan.parts = 1;
    plan.part_slabs = a.slabs;
    plan.whole = ((a.rows + kLargeTile - 1) / kLargeTile) * ((a.n + kLargeTile - 1) / kLargeTile);
    const int64_t grid = std::min<int64_t>(kComputeUnits, f8_most_items<kLargeTile, kLargeTile>(a, plan));
    if (grid <= 0 || a.scale_type == OZIMMU_F32 || a.out_type == OZIMMU_F32) return hipErrorInvalidConfiguration;
    if (a.along_rows) return a.out_type == OZIMMU_BF16 ? launch<true, OZIMMU_BF16>(a, plan, grid, st) : launch<true, OZIMMU_F16>(a, plan, grid, st);
    return a.out_type == OZIMMU_BF16 ? launch<false, OZIMMU_BF16>(a, plan, grid, st) : launch<false, OZIMMU_F16>(a, plan, grid, st);
}

}  // namespace ozimmu
