// What the entry points of the paged cache share with the rest of the library:
// the record of HIP errors, the device's facts and the workspaces per (device,
// stream, slot) that sparselnr_release() frees.  Defined in library.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <mutex>

namespace slnr {

// Workspace slots of these operators (0 to 2 belong to the sparse products).
// Attention by pages grows with its call, so it has a slot of its own.
enum WorkspaceSlot { kSlotAttend = 3, kSlotPages = 4 };

int hip_error(hipError_t e);  // records e for the calling thread; SPARSELNR_ERR_HIP
int this_device(int *dev);
int device_cu_count(int dev, int *cus);

// A workspace, held until this goes out of scope.  A call is several launches that share it, so
// it holds it from the lookup to the last of them: no call of another host thread comes in between on the
// same stream, and none grows or releases it.  One lock serves all streams, for the few
// microseconds that the launches take.
struct HeldWorkspace {
  std::unique_lock<std::mutex> lock;
  void *ptr = nullptr;
};
int hold_workspace(int dev, hipStream_t stream, size_t bytes, int slot, HeldWorkspace *out);

}  // namespace slnr
