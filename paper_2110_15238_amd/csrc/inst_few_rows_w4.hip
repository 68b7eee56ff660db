// Products of a few rows, weights in 4 bits: linear layers, and the experts of a routed list.
#include "few_rows_instances.hpp"

namespace bolt {
template <int MODE, bool GATED, int NG>
static hipError_t launch(const RowsParams& p, int mb, hipStream_t stream) {
  constexpr int NB = NG == 4 ? 2 : 3;  // (registers: four scale quads for each tile and step)
  if (mb == 1) return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 1, 2, 8, NB>(p, stream);
  if (mb == 2) return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 2, 8, 2>(p, stream);
  return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 4, 2, 4, 1>(p, stream);
}
template <int MODE, bool GATED>
static hipError_t launch_group(const RowsParams& p, int group, int mb, hipStream_t stream) {
  if (group == 128) return launch<MODE, GATED, 1>(p, mb, stream);
  if (group == 64) return launch<MODE, GATED, 2>(p, mb, stream);
  return launch<MODE, GATED, 4>(p, mb, stream);
}
hipError_t launch_few_rows_w4(const RowsParams& p, int mode, bool gated, int group, int mb, hipStream_t stream) {
  if (mode == ROWS_DENSE) return launch_group<ROWS_DENSE, false>(p, group, mb, stream);
  if (mode == ROWS_DOWN) return launch_group<ROWS_DOWN, false>(p, group, mb, stream);
  return gated ? launch_group<ROWS_UP, true>(p, group, mb, stream) : launch_group<ROWS_UP, false>(p, group, mb, stream);
}
}  // namespace bolt
