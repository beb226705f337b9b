// Instances of the 16-bit matrix-core product with one slice (weights in four bits, 16-bit types).
#include "nt_product.h"

namespace ozimmu {
hipError_t launch_nt_two_slices(const NtArgs& a, NtResult result, hipStream_t st);   // nt_product_two.hip

hipError_t launch_nt_product(const NtArgs& a, int slices, bool bf16, NtResult result, hipStream_t st) {
    if (slices == 2) return launch_nt_two_slices(a, result, st);
    if (bf16) return result == kOutBf16 ? launch_nt<1, true, kOutBf16>(a, st) : hipErrorInvalidValue;
    return result == kOutF16 ? launch_nt<1, false, kOutF16>(a, st) : hipErrorInvalidValue;
}
}  // namespace ozimmu
