// Launchers that launch nothing, for the host-only sanitizer build of the
// operators' C ABI layer (see launch_stubs.cpp).
#include "ops.h"

namespace pa {
hipError_t launch_rope(const RopeParams&, const double*, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_biased(const BiasedParams&, hipStream_t) { return hipErrorNotSupported; }
}  // namespace pa
