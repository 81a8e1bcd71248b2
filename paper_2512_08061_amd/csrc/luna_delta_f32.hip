// luna_delta_f32.hip -- the serial passes of the gated delta rule in fp32 (luna_delta_scan.hpp), and the choice of the type.
#include "luna_delta_scan.hpp"

namespace luna {

hipError_t launch_delta_fwd_f32(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_scan_one, float, 1, true); }

static hipError_t record(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_scan_one, float, 1, false); }
static hipError_t back(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_back_one, float, 1); }

hipError_t launch_delta_record_bf16(const DeltaArgs& a, hipStream_t s);
hipError_t launch_delta_back_bf16(const DeltaArgs& a, hipStream_t s);

hipError_t launch_delta_record(Dt dt, const DeltaArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_delta_record_bf16(a, s) : record(a, s);
}
hipError_t launch_delta_back(Dt dt, const DeltaArgs& a, hipStream_t s) {
  return dt == Dt::BF16 ? launch_delta_back_bf16(a, s) : back(a, s);
}

}  // namespace luna
