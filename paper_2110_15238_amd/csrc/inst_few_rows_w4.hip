// Products of up to 16 rows, weights in 4 bits: linear layers, and the experts of a routed list.
#include "few_rows_instances.hpp"
#include "few_rows_kernel.hpp"

namespace bolt {
template <int MODE, bool GATED, int NG>
static hipError_t launch(const RowsParams& p, hipStream_t stream) {
  constexpr int NB = NG == 4 ? 2 : 3;  // (registers: four scale quads for each tile and step)
  constexpr int R4 = GATED ? 2 : 1;    // (registers: four steps)
  const int n = (p.steps + 7) / 8;     // steps of a wave
  if (n == 1) return launch_few_rows_walk<WEIGHTS_W4, MODE, GATED, NG, 2, 8, 1>(p, stream);
  if (n == 2) return launch_few_rows_walk<WEIGHTS_W4, MODE, GATED, NG, 2, 8, 2>(p, stream);
  // (four steps of two tiles with groups of 32 do not fit the registers: one token, 8 of 64 experts of 2560 x 1024, gated, 33 us walking
  // with 228 bytes a lane spilled, 21 with the sets of the deep kernel; 2 of 8 experts of 4096 x 4096 40 and 24)
  if constexpr (!(GATED && NG == 4))
    if (n <= 4) return launch_few_rows_walk<WEIGHTS_W4, MODE, GATED, NG, R4, 8, 4>(p, stream);
  if constexpr (MODE == ROWS_DENSE) {
    // us for 1 and 16 rows, tiles of 16 weight rows on 8 waves / of 32 on 16: 2048 x 8192 6.1 and 10.9 / 7.9 and 12.4, 4096 x 6000 6.4 and 8.7 /
    // 7.9 and 9.6, 6152 x 5000 (385 tiles of 16) 7.8 and 10.8 / 6.7 and 8.1, 12288 x 5000 10.9 and 14.9 / 11.8 and 14.4
    if (p.N <= 16 * 256) return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 1, 8, NB>(p, stream);
    return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 16, NB - 1>(p, stream);
  } else {
    return launch_few_rows<WEIGHTS_W4, MODE, GATED, NG, 2, 8, NB>(p, stream);
  }
}
template <int MODE, bool GATED>
static hipError_t launch_group(const RowsParams& p, int group, hipStream_t stream) {
  if (group == 128) return launch<MODE, GATED, 1>(p, stream);
  if (group == 64) return launch<MODE, GATED, 2>(p, stream);
  return launch<MODE, GATED, 4>(p, stream);
}
hipError_t launch_few_rows_w4(const RowsParams& p, int mode, bool gated, int group, hipStream_t stream) {
  if (mode == ROWS_DENSE) return launch_group<ROWS_DENSE, false>(p, group, stream);
  if (mode == ROWS_DOWN) return launch_group<ROWS_DOWN, false>(p, group, stream);
  return gated ? launch_group<ROWS_UP, true>(p, group, stream) : launch_group<ROWS_UP, false>(p, group, stream);
}
// (One tile of columns per workgroup: the walking kernels would wait for the adapters of every tile.)
template <int NG>
static hipError_t launch_lora(const LayerParams& p, hipStream_t stream) {
  constexpr int NB = NG == 4 ? 2 : 3;  // (registers, as above; of two tiles the adapters' operands take the third set's)
  if (few_rows_tiles(p.N) == 1) return launch_few_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 1, 8, NB, true>(p, stream);
  return launch_few_rows<WEIGHTS_W4, ROWS_DENSE, false, NG, 2, 8, 2, true>(p, stream);
}
hipError_t launch_few_rows_w4_lora(const LayerParams& p, int group, hipStream_t stream) {
  if (group == 128) return launch_lora<1>(p, stream);
  if (group == 64) return launch_lora<2>(p, stream);
  return launch_lora<4>(p, stream);
}
}  // namespace bolt
