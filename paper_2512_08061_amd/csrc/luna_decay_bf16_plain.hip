// luna_decay_bf16_plain.hip -- the chunked decay kernel (luna_decay.hpp) in bf16, kDecayPlain.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(__bf16, kDecayPlain)
}  // namespace luna
