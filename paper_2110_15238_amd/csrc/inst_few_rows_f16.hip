// Products of a few rows, FP16 weights: the experts of a routed list.
#include "few_rows_instances.hpp"

namespace bolt {
template <int MODE, bool GATED>
static hipError_t launch(const RowsParams& p, int mb, hipStream_t stream) {
  if (mb == 1) return launch_few_rows<WEIGHTS_F16, MODE, GATED, 1, 1, 2, 8, 3>(p, stream);
  if (mb == 2) return launch_few_rows<WEIGHTS_F16, MODE, GATED, 1, 2, 2, 8, 3>(p, stream);
  return launch_few_rows<WEIGHTS_F16, MODE, GATED, 1, 4, 4, 4, 2>(p, stream);
}
hipError_t launch_few_rows_f16(const RowsParams& p, int mode, bool gated, int mb, hipStream_t stream) {
  if (mode == ROWS_DOWN) return launch<ROWS_DOWN, false>(p, mb, stream);
  return gated ? launch<ROWS_UP, true>(p, mb, stream) : launch<ROWS_UP, false>(p, mb, stream);
}
}  // namespace bolt
