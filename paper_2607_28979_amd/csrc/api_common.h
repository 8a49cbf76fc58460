// What the C-ABI entry points share: the calling thread's last error, pointer
// checks.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/mot.h"

namespace mot {

// Sets the calling thread's error text and returns `s`.
mot_status fail(mot_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return na && nb && pa < pb + nb && pb < pa + na;
}

}  // namespace mot
