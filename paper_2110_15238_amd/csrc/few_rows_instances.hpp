// What launches the products of rows with packed or FP16 weights: one function per family (csrc/inst_few_rows_*.hip,
// csrc/inst_shared_rows_*.hip, csrc/inst_moe_tile.hip).  mode: ROWS_*.
#pragma once
#include "../../include/bolt.h"
#include "routed_rows.hpp"

namespace bolt {
// Activation rows x weight rows of a workgroup's tile (a gated product has half as many output columns).
enum class SharedTile { ROWS16_COLS64, ROWS16_COLS128, ROWS32_COLS32, ROWS32_COLS64, ROWS32_COLS128, ROWS64_COLS128, ROWS128_COLS256 };
struct TileSize {
  int rows, cols;
};
inline TileSize tile_size(SharedTile t) {
  switch (t) {
    case SharedTile::ROWS16_COLS64: return {16, 64};
    case SharedTile::ROWS16_COLS128: return {16, 128};
    case SharedTile::ROWS32_COLS32: return {32, 32};
    case SharedTile::ROWS32_COLS64: return {32, 64};
    case SharedTile::ROWS32_COLS128: return {32, 128};
    case SharedTile::ROWS64_COLS128: return {64, 128};
    default: return {128, 256};
  }
}
enum class ManyTile { ROWS64, ROWS128, ROWS256 };

hipError_t launch_few_rows_f16(const RowsParams& p, int mode, bool gated, hipStream_t stream);
hipError_t launch_few_rows_w4(const RowsParams& p, int mode, bool gated, int group, hipStream_t stream);
hipError_t launch_shared_rows_f16(const RowsParams& p, int mode, bool gated, hipStream_t stream);
hipError_t launch_shared_rows_w4(const RowsParams& p, int mode, bool gated, int group, SharedTile tile, hipStream_t stream);
// A linear layer's outputs whose tiles of 16 weight rows are marked in p.unpacked, and no others.
hipError_t launch_shared_rows_w4_marked(const RowsParams& p, int group, hipStream_t stream);
hipError_t launch_many_rows_f16(const RowsParams& p, int mode, bool gated, ManyTile tile, hipStream_t stream);

// What bolt_gemm_epilogue's own choice of a kernel is estimated to take, in us; false where it has none (csrc/bolt_api.hip).
bool estimate_gemm(const bolt_gemm_desc& d, double* us);
}  // namespace bolt
