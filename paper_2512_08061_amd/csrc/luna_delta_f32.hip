// luna_delta_f32.hip -- the serial passes of the gated delta rule in fp32 (luna_delta_scan.hpp), and which type's run.
#include "luna_delta_scan.hpp"

namespace luna {

hipError_t launch_delta_fwd_f32(const DeltaArgs& a, hipStream_t s) { return launch_scan_all<float, 1, false>(a, s); }

static hipError_t both(const DeltaArgs& a, hipStream_t s) { return launch_scan_all<float, 1, true>(a, s); }

hipError_t launch_delta_both_bf16(const DeltaArgs& a, hipStream_t s);

hipError_t launch_delta_both(Dt dt, const DeltaArgs& a, hipStream_t s) { return dt == Dt::BF16 ? launch_delta_both_bf16(a, s) : both(a, s); }

}  // namespace luna
