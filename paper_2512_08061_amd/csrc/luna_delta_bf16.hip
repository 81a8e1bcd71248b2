// luna_delta_bf16.hip -- the serial passes of the gated delta rule's gradients in bf16 (luna_delta_scan.hpp).
#include "luna_delta_scan.hpp"

namespace luna {

hipError_t launch_delta_both_bf16(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_both_one, __bf16, , kDeltaBackParts); }

}  // namespace luna
