// luna_decay_bf16_aug.hip -- the chunked decay kernel (luna_decay.hpp) in bf16, kDecayAug.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(__bf16, kDecayAug)
}  // namespace luna
