// Host code that the library's two source files share.
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

#include "../../include/nuq.h"

namespace nuq {

// Address of the sticky error flags on the current device, null on error.
__attribute__((visibility("hidden"))) uint32_t *flags_ptr();

inline int check_launch()
{
    return hipGetLastError() == hipSuccess ? NUQ_OK : NUQ_EHIP;
}

}  // namespace nuq
