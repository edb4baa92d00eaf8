// The library's cached workspaces, for the entry points whose caller brings
// none (defined in nmspmm_kernels.hip, where their rules are stated).
#ifndef NMSPMM_WORKSPACE_H
#define NMSPMM_WORKSPACE_H

#include <hip/hip_runtime_api.h>

#include <cstddef>

namespace nmspmm {

// A workspace of at least `need` bytes for a call on `stream` (the current
// device), ordered after the buffer's previous use; null when none can be
// had.  ws_done(...) must follow the call's launches.
void *ws_acquire(hipStream_t stream, size_t need, int *slot);

// After the call's launches on `stream`: mark the buffer's last use.
hipError_t ws_done(int slot, hipStream_t stream);

// Whether work on `stream` is being captured into a graph (or that cannot be
// told): such calls take no cached workspace.
bool capturing(hipStream_t stream);

}  // namespace nmspmm

#endif
