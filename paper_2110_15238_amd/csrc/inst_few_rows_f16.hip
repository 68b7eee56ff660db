// Products of up to 16 rows, FP16 weights: the experts of a routed list.
#include "few_rows_instances.hpp"
#include "few_rows_kernel.hpp"

namespace bolt {
template <int MODE, bool GATED>
static hipError_t launch(const RowsParams& p, hipStream_t stream) {
  const int n = (p.steps + 7) / 8;  // steps of a wave
  if (n == 1) return launch_few_rows_walk<WEIGHTS_F16, MODE, GATED, 1, 2, 8, 1>(p, stream);
  if (n == 2) return launch_few_rows_walk<WEIGHTS_F16, MODE, GATED, 1, 2, 8, 2>(p, stream);
  if (n <= 4) return launch_few_rows_walk<WEIGHTS_F16, MODE, GATED, 1, 2, 8, 4>(p, stream);
  return launch_few_rows<WEIGHTS_F16, MODE, GATED, 1, 2, 8, 3>(p, stream);
}
hipError_t launch_few_rows_f16(const RowsParams& p, int mode, bool gated, hipStream_t stream) {
  if (mode == ROWS_DOWN) return launch<ROWS_DOWN, false>(p, stream);
  return gated ? launch<ROWS_UP, true>(p, stream) : launch<ROWS_UP, false>(p, stream);
}
}  // namespace bolt
