// What launches the products of a few rows: one function per kind of weights (csrc/inst_few_rows_*.hip).
#pragma once
#include "few_rows_kernel.hpp"

namespace bolt {
// mode: ROWS_*; mb: 16-row blocks of activations per workgroup, 1, 2 or 4.
hipError_t launch_few_rows_f16(const RowsParams& p, int mode, bool gated, int mb, hipStream_t stream);
hipError_t launch_few_rows_w4(const RowsParams& p, int mode, bool gated, int group, int mb, hipStream_t stream);
}  // namespace bolt
