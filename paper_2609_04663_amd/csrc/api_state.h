// What the entry points of the C ABI share across source files: the current
// stream, the error message and the workspace (defined in emu_api.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/emu.h"

namespace emu {
hipStream_t api_stream();
void api_clear_error();
int api_fail(int code, const char *msg);                // sets the message, returns code
int api_hip_fail(hipError_t e, const char *what);       // EMU_EHIP with HIP's own text
// Workspace of at least `bytes` (256-byte aligned start) in *p, or an error code.
int api_workspace(size_t bytes, char **p);
}  // namespace emu
