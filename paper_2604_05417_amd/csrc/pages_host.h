// What the paged 4-bit caches (pages.hip) and the contexts (metasd.hip) know of each other: host side.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/metasd.h"

namespace msd {

// Notes the message of a call without a context and returns its code (metasd.hip).
int fail_global(int code, const char* fmt, ...);

}  // namespace msd
