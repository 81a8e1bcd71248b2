// luna_decay_f32_plain.hip -- the chunked decay kernel (luna_decay.hpp) in f32, kDecayPlain.
#include "luna_decay.hpp"

namespace luna {
LUNA_DECAY_TYPED(float, kDecayPlain)
}  // namespace luna
