// Products of more than 16 rows, FP16 weights: linear layers whose rows have adapters.
#include "few_rows_instances.hpp"
#include "moe_pp_kernel.hpp"
#include "rows_tile_kernel.hpp"

namespace bolt {
template <int ADD>
static hipError_t launch(const LayerParams& p, RowsTile tile, hipStream_t stream) {
  switch (tile) {
    // rows, columns, waves along either, stages, sets
    case RowsTile::ROWS64_COLS32: return launch_rows_tiles<WEIGHTS_F16, ADD, 64, 32, 2, 1, 3, 4>(p, stream);
    case RowsTile::ROWS64_COLS64: return launch_rows_tiles<WEIGHTS_F16, ADD, 64, 64, 2, 2, 3, 2>(p, stream);
    case RowsTile::ROWS128_COLS64: return launch_rows_tiles<WEIGHTS_F16, ADD, 128, 64, 4, 1, 3, 2>(p, stream);
    case RowsTile::ROWS128_COLS128: return launch_rows_tiles<WEIGHTS_F16, ADD, 128, 128, 2, 2, 3, 1>(p, stream);
    case RowsTile::ROWS128_COLS256: return launch_rows_tiles<WEIGHTS_F16, ADD, 128, 256, 2, 4, 3, 1>(p, stream);
    default: return launch_moe_pp<ROWS_DENSE, false, WEIGHTS_F16, ADD>(p, stream);
  }
}
hipError_t launch_rows_f16_adapters(const LayerParams& p, RowsTile tile, hipStream_t stream) { return launch<FROM_ADAPTERS>(p, tile, stream); }
hipError_t launch_rows_f16_add(const LayerParams& p, RowsTile tile, hipStream_t stream) { return launch<FROM_ADD>(p, tile, stream); }
}  // namespace bolt
