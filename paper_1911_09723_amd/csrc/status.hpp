// The calling thread's error message, shared by the files of the C ABI.
#pragma once

#include <hip/hip_runtime_api.h>

#include "spconv.h"

namespace spconv {

void clear_error();
// Both set the message (left as it is where memory runs out) and return a status.
spconv_status set_error(spconv_status st, const char *msg);
spconv_status set_hip_error(const char *what, hipError_t e);

}  // namespace spconv
