// What the entry points of the 4-bit cache (cache_rows, cache_attention, cache_evict) have in common.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "si_internal.h"

namespace si {

// The status of a call whose last HIP call returned e.
inline si_status report(hipError_t e) { return e == hipSuccess ? SI_OK : hip_fail(e); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// One number a batch (lengths, start): read one at a time.
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace si
