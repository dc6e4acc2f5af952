// What the host entry points check their arguments with.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "lemo.h"

namespace lemo {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool valid_dtype(int dt) { return dt == LEMO_F32 || dt == LEMO_BF16; }
inline int elems_per_16B(int dt) { return dt == LEMO_BF16 ? 8 : 4; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int hip_rc(int e) { return e == 0 ? LEMO_OK : LEMO_ERR_HIP; }

}  // namespace lemo
