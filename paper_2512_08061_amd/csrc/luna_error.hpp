// luna_error.hpp -- the reason behind luna_last_error(), for the host files of the C ABI.
#pragma once

#include "luna.h"

namespace luna {

// Notes why on the calling thread and returns `s`; throws nothing.
luna_status set_error(luna_status s, const char* why) noexcept;
void clear_error() noexcept;

}  // namespace luna
