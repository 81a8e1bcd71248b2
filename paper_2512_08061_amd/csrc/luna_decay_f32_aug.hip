// luna_decay_f32_aug.hip -- the chunked decay kernel (luna_decay.hpp) in f32, kDecayAug.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(float, kDecayAug)
}  // namespace luna
