// Instances of the 16-bit matrix-core product with two slices of fp16 (32-bit weights products, orthogonal updates).
#include "nt_product.h"

namespace ozimmu {
hipError_t launch_nt_two_slices(const NtArgs& a, NtResult result, hipStream_t st) {
    switch (result) {
        case kOutF32: return launch_nt<2, false, kOutF32>(a, st);
        case kOutBf16: return launch_nt<2, false, kOutBf16>(a, st);
        case kOutF16: return launch_nt<2, false, kOutF16>(a, st);
        case kOutSlices: return launch_nt<2, false, kOutSlices>(a, st);
    }
    return hipErrorInvalidValue;
}
}  // namespace ozimmu
