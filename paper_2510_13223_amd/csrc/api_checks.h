// api_checks.h -- what the entry points of both headers check and report alike (defined in bana_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bana.h"

namespace bana {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Shapes, hints and index ranges of a call's dims.
bana_status check_dims(const bana_dims* d);

// BANA_OK, or BANA_ERR_DEVICE with the HIP error text kept for bana_last_error().
bana_status device_status(hipError_t e);

}  // namespace bana
