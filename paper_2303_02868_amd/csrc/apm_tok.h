// What the kernels on tokens share: ids, and matrices taken eight columns at a time.
#pragma once

#include "apm_act.h"

namespace apm {

// An id as the row that it stands for; `rows`, which is below 2^31, where there is no such row.
__device__ __forceinline__ uint32_t row_of(const void* ids, int32_t type, int64_t p, uint32_t rows) {
    const uint64_t id = type == APM_I32 ? (uint64_t)(int64_t)((const int32_t*)ids)[p] : (uint64_t)((const int64_t*)ids)[p];
    return id < rows ? (uint32_t)id : rows;
}

// Vectors of eight columns of a matrix, numbered row by row.  A workgroup divides once, for its first vector, and each lane makes up for what it is
// further on: `at` / vecs is below 2^10 there, so that one correction makes up for the reciprocal's rounding.
struct VecPlace {
    uint32_t row;
    int col, n;  // the first column, and how many of the eight exist
    __device__ __forceinline__ VecPlace(uint32_t row0, uint32_t vec0, uint32_t further, uint32_t vecs, float inv_vecs, int cols) {
        const uint32_t at = vec0 + further;
        uint32_t r = (uint32_t)((float)at * inv_vecs);
        int32_t left = (int32_t)(at - r * vecs);
        if (left < 0) r -= 1, left += (int32_t)vecs;
        else if (left >= (int32_t)vecs) r += 1, left -= (int32_t)vecs;
        row = row0 + r;
        col = left * kVec;
        n = min(kVec, cols - col);
    }
};
constexpr int64_t kMostCols = (int64_t)1 << 30;
constexpr int64_t kMostVecs = (int64_t)1 << 30;  // of a launch

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
inline bool aligned_to(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

}  // namespace apm
