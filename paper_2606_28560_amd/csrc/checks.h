// Argument checks shared by the C entry points.
#pragma once

#include "../../include/fibattn.h"
#include "common.h"

namespace fibattn {

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// A caller's placement of one tensor: non-negative strides that keep every row 16-byte
// aligned.
inline bool strides_ok(const fibattn_layout_t &l, fibattn_dtype_t dtype) {
    const long long per = dtype == FIBATTN_BF16 ? 8 : 4;  // elements to 16 bytes
    return l.batch >= 0 && l.head >= 0 && l.pos >= 0 && l.batch % per == 0 && l.head % per == 0 && l.pos % per == 0;
}

}  // namespace fibattn
