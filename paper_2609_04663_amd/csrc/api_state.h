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
inline int api_done(hipError_t e, const char *what) { return e == hipSuccess ? EMU_OK : api_hip_fail(e, what); }
// Workspace of at least `bytes` (256-byte aligned start) in *p, or an error code.
int api_workspace(size_t bytes, char **p);
// The same for a call that can do without: *p is null where the workspace cannot
// grow (no memory, a limit, a stream under capture), and what is held stays; an
// error code is a HIP error.
int api_try_workspace(size_t bytes, char **p);
}  // namespace emu
