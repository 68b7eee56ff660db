// Products of some ten rows, FP16 weights: routed lists that make few workgroups.
#include "few_rows_instances.hpp"
#include "shared_rows_kernel.hpp"

namespace bolt {
hipError_t launch_shared_rows_f16(const RowsParams& p, int mode, bool gated, hipStream_t stream) {
  if (mode == ROWS_DOWN) return launch_shared_rows<WEIGHTS_F16, ROWS_DOWN, false, 1, 2, 2, 2, 2, 3>(p, stream);
  return gated ? launch_shared_rows<WEIGHTS_F16, ROWS_UP, true, 1, 2, 2, 2, 2, 3>(p, stream)
               : launch_shared_rows<WEIGHTS_F16, ROWS_UP, false, 1, 2, 2, 2, 2, 3>(p, stream);
}
}  // namespace bolt
