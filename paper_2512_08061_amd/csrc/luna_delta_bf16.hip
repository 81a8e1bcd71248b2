// luna_delta_bf16.hip -- the serial passes of the gated delta rule's gradients in bf16 (luna_delta_scan.hpp).
#include "luna_delta_scan.hpp"

namespace luna {

hipError_t launch_delta_both_bf16(const DeltaArgs& a, hipStream_t s) { return launch_scan_all<__bf16, kDeltaBackParts, true>(a, s); }

}  // namespace luna
