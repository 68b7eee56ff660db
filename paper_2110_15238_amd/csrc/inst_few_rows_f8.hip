// Products of up to 16 rows, E4M3 operands: linear layers.
#include "few_rows_instances.hpp"
#include "few_rows_kernel.hpp"

namespace bolt {
hipError_t launch_few_rows_f8(const RowsParams& p, hipStream_t stream) {
  const int n = (p.steps + 7) / 8;  // steps of a wave
  if (n == 1) return launch_few_rows_walk<WEIGHTS_F8, ROWS_DENSE, false, 1, 2, 8, 1>(p, stream);
  if (n == 2) return launch_few_rows_walk<WEIGHTS_F8, ROWS_DENSE, false, 1, 2, 8, 2>(p, stream);
  if (n <= 4) return launch_few_rows_walk<WEIGHTS_F8, ROWS_DENSE, false, 1, 2, 8, 4>(p, stream);
  if (few_rows_tiles(p.N) == 1) return launch_few_rows<WEIGHTS_F8, ROWS_DENSE, false, 1, 1, 8, 3>(p, stream);
  return launch_few_rows<WEIGHTS_F8, ROWS_DENSE, false, 1, 2, 8, 3>(p, stream);
}
}  // namespace bolt
