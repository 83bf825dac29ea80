// Status codes shared by the C ABI and the internal C++ code.
#pragma once
#include "../../include/ndvm.h"

namespace ndvm {
// records the calling thread's message for ndvm_last_error (capi.cpp); returns s
ndvm_status set_error(ndvm_status s, const char* message);
}  // namespace ndvm
