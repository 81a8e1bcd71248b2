// luna_paged_tiles.hip -- causal softmax attention of many rows over pages (luna_softmax_fwd.hpp): keys and values come 16 rows at a
// time, which lie in one page.
#include "luna_softmax_fwd.hpp"

namespace luna {

hipError_t launch_paged_tiles(Dt dt, const SoftmaxArgs& a, hipStream_t s) { return launch_tiles<true>(dt, a, s); }

}  // namespace luna
