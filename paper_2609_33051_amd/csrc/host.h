// Host-side helpers the entry points share: error reporting (the text behind
// sketchssm_last_error) and the checks of shapes, rings and pointers.  Defined
// in abi.hip.
#pragma once

#include <stdint.h>

#include "../../include/sketchssm.h"

namespace skssm {

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int launched(int rc, const char* what);  // the status after a launch (rc -2: no kernel, -3: too large, neither launched)
int check_shape(const skssm_config* c, bool need_rank, bool allow_rank0);
int check_ring(const skssm_config* c, const skssm_ring* r, bool derived_f, bool derived_pi);
inline bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace skssm
