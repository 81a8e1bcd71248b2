// luna_decay_f32_norm.hip -- the chunked decay kernel (luna_decay.hpp) in f32, kDecayNorm.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(float, kDecayNorm)
}  // namespace luna
