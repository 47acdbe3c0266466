// The translation unit of the sparse products, and what the entry points of the
// paged cache use of it: one record of HIP errors, one set of workspaces, which
// sparselnr_release() frees.  The products' source stays as it is: its counters
// under profiles/ are valid for exactly that text.
#include "../csrc/sparselnr.hip"

#include "runtime.hpp"

namespace slnr {

int hip_error(hipError_t e) { return hip_fail(e); }
int this_device(int *dev) { return current_device(dev); }
int device_cu_count(int dev, int *cus) { return device_cus(dev, cus); }
int stream_workspace(int dev, hipStream_t stream, size_t bytes, void **out, int slot) {
  return get_workspace(dev, stream, bytes, out, slot);
}

}  // namespace slnr
