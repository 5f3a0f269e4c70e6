// Host-side checks shared by the entry points.
#ifndef CG_CHECK_H
#define CG_CHECK_H

#include <stddef.h>
#include <stdint.h>

#include "cg.h"

namespace cg {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// do [a, a+na) and [b, b+nb) (bytes) intersect?
inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + nb && pb < pa + na;
}

// element-wise calls: identical pointers are fine (in place), partial overlap is not
inline bool bad_overlap(const void* out, const void* in, uint64_t bytes) {
    return out != in && overlap(out, bytes, in, bytes);
}

inline cg_status check_ptrs(const void* const* ptrs, int count) {
    for (int i = 0; i < count; ++i)
        if (!ptrs[i]) return CG_ERR_NULL;
    for (int i = 0; i < count; ++i)
        if (!aligned(ptrs[i], 8)) return CG_ERR_ALIGN;
    return CG_OK;
}

inline bool all_aligned16(const void* const* ptrs, int count) {
    for (int i = 0; i < count; ++i)
        if (!aligned(ptrs[i], 16)) return false;
    return true;
}

}  // namespace cg
#endif
