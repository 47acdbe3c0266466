// The translation unit of the sparse products, and what the entry points of the
// paged cache use of it: one record of HIP errors, one set of workspaces, which
// sparselnr_release() frees.  The products' source stays as it is: its counters
// under profiles/ are valid for exactly that text.
#include "../csrc/sparselnr.hip"

#include "runtime.hpp"

namespace slnr {

int hip_error(hipError_t e) { return hip_fail(e); }
int this_device(int *dev) { return current_device(dev); }
int device_cu_count(int dev, int *cus) {
  try {
    return device_cus(dev, cus);
  } catch (...) {  // no memory for a record of it
    return SPARSELNR_ERR_NO_MEMORY;
  }
}

int hold_workspace(int dev, hipStream_t stream, size_t bytes, int slot, HeldWorkspace *out) {
  try {
    for (;;) {
      void *p = nullptr;
      const int rc = get_workspace(dev, stream, bytes, &p, slot);
      if (rc != SPARSELNR_OK) return rc;
      // get_workspace has let go of the lock: another thread may have grown or released it since
      std::unique_lock<std::mutex> lock(g_mu);
      const auto it = g_workspace.find(WsKey{dev, (uintptr_t)stream, slot});
      if (it == g_workspace.end() || it->second.ptr != p || it->second.bytes < bytes) continue;
      out->lock = std::move(lock);
      out->ptr = p;
      return SPARSELNR_OK;
    }
  } catch (...) {  // no memory for a record of it
    return SPARSELNR_ERR_NO_MEMORY;
  }
}

}  // namespace slnr
