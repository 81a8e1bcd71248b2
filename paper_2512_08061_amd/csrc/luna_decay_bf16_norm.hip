// luna_decay_bf16_norm.hip -- the chunked decay kernel (luna_decay.hpp) in bf16, kDecayNorm.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(__bf16, kDecayNorm)
}  // namespace luna
