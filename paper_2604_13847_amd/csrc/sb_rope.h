// Checks that every call with rotary positions makes (sb_rope.hip).
#pragma once

#include "sb_cache.h"

namespace sb {

int check_rope(const sb_rope* r, int head_dim);
int check_axes(const sb_rope* r, const sb_rope_axes* a, const int32_t* positions);       // all three are required
int check_pitch(const char* what, int64_t* pitch, int64_t contiguous);                   // 0 becomes contiguous
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace sb
