// What the host sides of the library's translation units share.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace leet {

// The current device, or LEET_ERR_UNSUPPORTED if it is not a gfx950 one.
int current_device(int* dev);

}  // namespace leet
