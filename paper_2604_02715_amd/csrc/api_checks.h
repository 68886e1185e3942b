// Checks that the entry points of operators on rows have in common.
#pragma once

#include "fluxmoe_internal.h"

namespace fluxmoe {

inline uint32_t elem_bytes(uint32_t type) { return type == FLUXMOE_F32 ? 4 : 2; }
inline bool known(uint32_t type) { return type == FLUXMOE_BF16 || type == FLUXMOE_F32; }
inline bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// Rows of `bytes` per element, `stride` elements apart, each at a 16-byte address; absent tensors do not stand in the way.
inline bool rows_aligned(const void* p, uint64_t stride, uint32_t bytes) { return !p || (aligned(p, 16) && stride * bytes % 16 == 0); }

inline int check_stride(const char* name, uint64_t stride, uint32_t width) {
    if (stride >= width && stride < (1ull << 40)) return FLUXMOE_OK;
    return set_error(FLUXMOE_EINVAL, "%s (%llu) must be at least the row's %u elements", name, (unsigned long long)stride, width);
}

}  // namespace fluxmoe
