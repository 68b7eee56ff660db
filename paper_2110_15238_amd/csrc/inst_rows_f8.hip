// Products of any rows, E4M3 operands: linear layers.
#include "few_rows_instances.hpp"
#include "moe_pp_kernel.hpp"
#include "rows_tile_kernel.hpp"
#include "shared_rows_kernel.hpp"

namespace bolt {
hipError_t launch_rows_f8(const LayerParams& p, RowsTile tile, hipStream_t stream) {
  switch (tile) {
    case RowsTile::ROWS16_COLS32: return launch_shared_rows<WEIGHTS_F8, ROWS_DENSE, false, 1, 1, 1, 2, 4, 3>(p, stream);
    case RowsTile::ROWS32_COLS32: return launch_shared_rows<WEIGHTS_F8, ROWS_DENSE, false, 1, 2, 1, 2, 4, 3>(p, stream);
    // rows, columns, waves along either, stages, sets
    case RowsTile::ROWS64_COLS32: return launch_rows_tiles<WEIGHTS_F8, ADD_NOTHING, 64, 32, 2, 1, 3, 4>(p, stream);
    case RowsTile::ROWS64_COLS64: return launch_rows_tiles<WEIGHTS_F8, ADD_NOTHING, 64, 64, 2, 2, 3, 2>(p, stream);
    case RowsTile::ROWS128_COLS64: return launch_rows_tiles<WEIGHTS_F8, ADD_NOTHING, 128, 64, 4, 1, 3, 2>(p, stream);
    case RowsTile::ROWS128_COLS128: return launch_rows_tiles<WEIGHTS_F8, ADD_NOTHING, 128, 128, 2, 2, 3, 1>(p, stream);
    case RowsTile::ROWS128_COLS256: return launch_rows_tiles<WEIGHTS_F8, ADD_NOTHING, 128, 256, 2, 4, 3, 1>(p, stream);
    default: return launch_moe_pp<ROWS_DENSE, false, WEIGHTS_F8>(p, stream);
  }
}
}  // namespace bolt
