// luna_delta_bf16.hip -- the serial passes of the gated delta rule in bf16 (luna_delta_scan.hpp).
#include "luna_delta_scan.hpp"

namespace luna {

template <typename T, bool EXACT>
static hipError_t out_typed(const DeltaArgs& a, hipStream_t s) {
  LUNA_DELTA_WIDTHS(launch_scan_one, T, EXACT ? kDeltaExactParts : kDeltaParts, true);
}
static hipError_t record(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_scan_one, __bf16, kDeltaBackParts, false); }
static hipError_t back(const DeltaArgs& a, hipStream_t s) { LUNA_DELTA_WIDTHS(launch_back_one, __bf16, kDeltaBackParts); }

hipError_t launch_delta_out_bf16(bool exact, const DeltaArgs& a, hipStream_t s) {
  return exact ? out_typed<__bf16, true>(a, s) : out_typed<__bf16, false>(a, s);
}
hipError_t launch_delta_record_bf16(const DeltaArgs& a, hipStream_t s) { return record(a, s); }
hipError_t launch_delta_back_bf16(const DeltaArgs& a, hipStream_t s) { return back(a, s); }

}  // namespace luna
