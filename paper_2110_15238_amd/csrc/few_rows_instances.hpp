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
hipError_t launch_shared_rows_w4_marked(const LayerParams& p, int group, hipStream_t stream);
hipError_t launch_many_rows_f16(const RowsParams& p, int mode, bool gated, ManyTile tile, hipStream_t stream);

// Linear layers of E4M3 operands: x, ldx, K and steps in pairs (halves); x_scales, w_scales.
enum class RowsTile { ROWS16_COLS32, ROWS32_COLS32, ROWS64_COLS32, ROWS64_COLS64, ROWS128_COLS64, ROWS128_COLS128, ROWS128_COLS256, ROWS256_COLS256 };
hipError_t launch_rows_f8(const LayerParams& p, RowsTile tile, hipStream_t stream);
// Linear layers with FP16 weights, from 64 x 32 to 256 x 256 tiles, that compute the rows' share of their adapters (adapter, low, up, adapters, rank,
// low_parts; on the largest tiles low is one part), or take it from p.add.  The largest start their sums at beta / alpha times the bias.
hipError_t launch_rows_f16_adapters(const LayerParams& p, RowsTile tile, hipStream_t stream);
hipError_t launch_rows_f16_add(const LayerParams& p, RowsTile tile, hipStream_t stream);

// A projection with FP16 weights and a share from p.add on the tile of the smallest estimate; beta / alpha times the bias is finite (csrc/lora_api.hip).
hipError_t launch_projection_f16_add(const LayerParams& p, hipStream_t stream);

// Linear layers of up to 16 rows (some more of narrow ones) whose sums take the rows' adapters (adapter, low, up, adapters, rank).
hipError_t launch_few_rows_f16_lora(const LayerParams& p, hipStream_t stream);
hipError_t launch_few_rows_w4_lora(const LayerParams& p, int group, hipStream_t stream);
// The same on one of the tiles of linear layers: with the share from p.add, or, where that is null and but for 128 x 256, computed there.
hipError_t launch_shared_rows_w4_lora(const LayerParams& p, int group, SharedTile tile, hipStream_t stream);

// bolt_gemm_w4 behind its checks; `add` (M x N floats, or null): added to A . W^T before alpha (csrc/moe_api.hip).
bolt_status check_gemm_w4(const bolt_gemm_w4_desc* d);
bolt_status run_gemm_w4(const bolt_gemm_w4_desc& d, const void* A, const void* packed, const void* bias, const float* add, void* D, void* workspace,
                        void* stream);
SharedTile tile_of_gemm_w4(const bolt_gemm_w4_desc& d);  // where the weights stay packed
LayerParams dense_w4_rows(const bolt_gemm_w4_desc& d, const void* A, const void* packed, const void* bias, void* D, const half_t* none);

// What bolt_gemm_epilogue's own choice of a kernel is estimated to take, in us; false where it has none (csrc/bolt_api.hip).
bool estimate_gemm(const bolt_gemm_desc& d, double* us);
}  // namespace bolt
