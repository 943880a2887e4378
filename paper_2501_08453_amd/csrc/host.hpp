// Host-side helpers shared by the files of the C ABI.
#pragma once

#include <stdint.h>

#include "vc_jointattn.h"

namespace vcja {

// VC_OK if the current device is a gfx950, VC_ERR_DEVICE otherwise.
vc_status check_device();
// Compute units of the current device (after check_device succeeded).
int device_cus();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace vcja
