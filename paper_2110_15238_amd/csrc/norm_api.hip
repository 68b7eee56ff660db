// C ABI of the norm with its residual and of rows in 8 bits.
#include <algorithm>
#include <cmath>

#include "llm_checks.hpp"
#include "norm_kernel.hpp"

namespace bolt {
namespace {

constexpr int kMaxNormWidth = 16 * 64 * 4 * 8;  // 16 waves, four pieces a lane (eight do not fit their 128 registers)

template <int WAVES, int V, bool NORM>
hipError_t launch(const NormParams& p, hipStream_t stream) {
  constexpr int PER = WAVES == 1 ? 4 : 1, NT = WAVES == 1 ? 256 : 64 * WAVES;
  const int64_t blocks = blocks_of(p.rows, PER);
  hipLaunchKernelGGL((norm_kernel<WAVES, V, NORM>), dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(NT), 0, stream, p);
  return hipGetLastError();
}

// Waves and pieces by the width alone: few rows take about 4 us in any form (one round trip), many are fastest where a workgroup's lanes have two to
// four pieces each.  us with the residual, FP16 rows, waves x pieces: 32768 x 1024 1 x 2 47, 2 x 2 48, 4 x 1 56; 32768 x 2048 2 x 2 92, 1 x 4 92, 4 x 1 96, 8 x 1
// 110; 4099 x 5120 4 x 4 34.0, 8 x 2 35.3, 16 x 2 45; 4099 x 8192 4 x 4 48.6, 8 x 2 49.0, 16 x 2 55; 4099 x 12296 16 x 2 74, 8 x 4 90; 1 x 4096 3.9 to 4.2 in six forms.
template <bool NORM>
hipError_t launch_norm(const NormParams& p, hipStream_t stream) {
  const int chunks = p.width / 8;
  if (chunks <= 64) return launch<1, 1, NORM>(p, stream);
  if (chunks <= 128) return launch<1, 2, NORM>(p, stream);
  if (chunks <= 256) return launch<2, 2, NORM>(p, stream);
  if (chunks <= 512) return launch<4, 2, NORM>(p, stream);
  if (chunks <= 1024) return launch<4, 4, NORM>(p, stream);
  if (chunks <= 2048) return launch<16, 2, NORM>(p, stream);
  return launch<16, 4, NORM>(p, stream);
}

bool strides_ok(int width, std::initializer_list<int> strides) {
  return std::all_of(strides.begin(), strides.end(), [&](int s) { return s >= width; });
}

}  // namespace
}  // namespace bolt

using namespace bolt;

extern "C" {

bolt_status bolt_rms_norm(const bolt_rms_norm_desc* desc, const void* x, const void* residual, const void* weight, void* sum, void* y, void* q,
                          void* scales, void* stream) {
  if (!desc || desc->rows < 0 || desc->width <= 0 || !(desc->eps >= 0.f) || !std::isfinite(desc->eps) || !std::isfinite(desc->weight_offset))
    return BOLT_ERR_INVALID_ARG;
  const bolt_rms_norm_desc& d = *desc;
  const int ldr = residual ? d.ldr : d.width, lds = sum ? d.lds : d.width, ldy = y ? d.ldy : d.width, ldq = q ? d.ldq : d.width;
  if (!strides_ok(d.width, {d.ldx, ldr, lds, ldy, ldq})) return BOLT_ERR_INVALID_ARG;
  if ((d.width | d.ldx | ldr | lds | ldy | ldq) & 7) return BOLT_ERR_ALIGNMENT;
  if (d.width > kMaxNormWidth || d.rows > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  if (d.rows == 0) return BOLT_OK;
  if (!x || !weight || (!y && !q) || (q && !scales)) return BOLT_ERR_INVALID_ARG;
  for (const void* at : {x, residual, weight, (const void*)sum, (const void*)y, (const void*)q, (const void*)scales})
    if (!aligned16(at)) return BOLT_ERR_ALIGNMENT;
  // sum and y in the place of an input: row by row, value by value
  const auto in_place = [&](const void* out, int ld) { return d.rows == 1 || ((out != x || ld == d.ldx) && (out != residual || ld == ldr)); };
  if (starts_at(sum, {y, weight, q, scales}) || starts_at(y, {weight, q, scales}) || starts_at(q, {x, residual, weight, scales}) ||
      starts_at(scales, {x, residual, weight}) || (sum && !in_place(sum, lds)) || (y && !in_place(y, ldy)))
    return BOLT_ERR_INVALID_ARG;
  NormParams p{};
  p.x = (const half_t*)x; p.residual = (const half_t*)residual; p.weight = (const half_t*)weight;
  p.sum = (half_t*)sum; p.y = (half_t*)y; p.q = (unsigned char*)q; p.scales = (float*)scales;
  p.ldx = d.ldx; p.ldr = ldr; p.lds = lds; p.ldy = ldy; p.ldq = ldq;
  p.rows = d.rows; p.width = d.width; p.eps = d.eps; p.offset = d.weight_offset;
  return status_of(launch_norm<true>(p, (hipStream_t)stream));
}

bolt_status bolt_quantize_rows(int32_t rows, int32_t width, int32_t ldx, int32_t ldq, const void* x, void* q, void* scales, void* stream) {
  if (rows < 0 || width <= 0 || !strides_ok(width, {ldx, ldq})) return BOLT_ERR_INVALID_ARG;
  if ((width | ldx | ldq) & 7) return BOLT_ERR_ALIGNMENT;
  if (width > kMaxNormWidth || rows > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  if (rows == 0) return BOLT_OK;
  if (!x || !q || !scales) return BOLT_ERR_INVALID_ARG;
  for (const void* at : {x, (const void*)q, (const void*)scales})
    if (!aligned16(at)) return BOLT_ERR_ALIGNMENT;
  if (starts_at(q, {x, scales}) || starts_at(scales, {x})) return BOLT_ERR_INVALID_ARG;
  NormParams p{};
  p.x = (const half_t*)x; p.q = (unsigned char*)q; p.scales = (float*)scales;
  p.ldx = ldx; p.ldq = ldq;
  p.rows = rows; p.width = width;
  return status_of(launch_norm<false>(p, (hipStream_t)stream));
}

}  // extern "C"
