// What the entry points' host code shares: the calling thread's error detail,
// failure returns, and the argument checks used by more than one source.
#pragma once

#include "common.h"

namespace mla {

void clear_detail();
mla_status fail(mla_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
mla_status hip_fail(hipError_t e, const char* what);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

mla_status check_geom(const mla_geom* g, bool for_oproj);

}  // namespace mla
