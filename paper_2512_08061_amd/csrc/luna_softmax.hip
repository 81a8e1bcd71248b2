// luna_softmax.hip -- causal softmax attention over sequences of different lengths, forward (luna_softmax_fwd.hpp).
#include "luna_softmax_fwd.hpp"

namespace luna {

hipError_t launch_softmax_fwd(Dt dt, const SoftmaxArgs& a, hipStream_t s) { return launch_tiles<false>(dt, a, s); }

}  // namespace luna
