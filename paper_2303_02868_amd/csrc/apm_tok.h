// What the calls on tokens share: ids, and checks of arguments.
#pragma once

#include "apm_act.h"

namespace apm {

// An id as the row that it stands for; `rows`, which is below 2^31, where there is no such row.
__device__ __forceinline__ uint32_t row_of(const void* ids, int32_t type, int64_t p, uint32_t rows) {
    const uint64_t id = type == APM_I32 ? (uint64_t)(int64_t)((const int32_t*)ids)[p] : (uint64_t)((const int64_t*)ids)[p];
    return id < rows ? (uint32_t)id : rows;
}

constexpr int64_t kMostCols = (int64_t)1 << 28;  // a row is under 2^31 bytes

inline int check_indices(const char* name, const apm_indices& i) {
    if (!i.data) return fail(APM_EINVAL, "%s is missing", name);
    if (i.type != APM_I32 && i.type != APM_I64) return fail(APM_EINVAL, "%s: bad type %d", name, i.type);
    if ((uintptr_t)i.data % (i.type == APM_I32 ? 4 : 8) != 0) return fail(APM_EINVAL, "%s is not aligned to its elements", name);
    return APM_OK;
}
inline int check_room(const void* workspace, size_t bytes, size_t need) {
    if (bytes < need) return fail(APM_ENOMEM, "the workspace is too small");
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0)) return fail(APM_EINVAL, "the workspace is missing or not aligned to 16 bytes");
    return APM_OK;
}
// Workgroups of one launch, where a call may take several.
int64_t workgroups_of_launch(int threads);
inline bool aligned_to(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

}  // namespace apm
