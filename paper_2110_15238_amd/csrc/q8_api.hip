// C ABI of the linear layers whose operands are held in 8 bits.
#include "few_rows_instances.hpp"
#include "llm_checks.hpp"

namespace bolt {
namespace {

bolt_status check_gemm_q8(const bolt_gemm_q8_desc* d) {
  if (!d || d->M < 0 || d->N <= 0 || d->K <= 0 || !known_act(d->act) || d->lda < d->K || d->ldd < d->N) return BOLT_ERR_INVALID_ARG;
  if (((d->N | d->ldd) & 7) || ((d->K | d->lda) & 15)) return BOLT_ERR_ALIGNMENT;
  if (d->lda > kMaxLength || d->ldd > kMaxLength || d->M > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

}  // namespace
}  // namespace bolt

using namespace bolt;

extern "C" {

size_t bolt_gemm_q8_workspace_bytes(const bolt_gemm_q8_desc* desc) {
  if (check_gemm_q8(desc) != BOLT_OK) return 0;
  return 0;
}

bolt_status bolt_gemm_q8(const bolt_gemm_q8_desc* desc, const void* A, const void* a_scales, const void* W, const void* w_scales, const void* bias, void* D,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_gemm_q8(desc); s != BOLT_OK) return s;
  if (desc->M == 0) return BOLT_OK;
  if (!A || !W || !D) return BOLT_ERR_INVALID_ARG;
  for (const void* at : {A, a_scales, W, w_scales, bias, (const void*)D, (const void*)workspace})
    if (!aligned16(at)) return BOLT_ERR_ALIGNMENT;
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  RowsParams p{};
  p.x = (const half_t*)A; p.ldx = desc->lda / 2;
  p.w = (const unsigned char*)W; p.w_stride = (int64_t)desc->N * desc->K;
  p.x_scales = (const float*)a_scales; p.w_scales = (const float*)w_scales;
  p.none = none;
  p.bias = bias ? (const half_t*)bias : none;
  p.bias_on = bias ? 1 : 0;
  p.y = D; p.ldy = desc->ldd;
  p.M = desc->M; p.N = desc->N; p.K = desc->K / 2; p.steps = (int)blocks_of(p.K, 64);
  p.alpha = desc->alpha; p.beta = desc->beta; p.act = desc->act;
  const hipStream_t st = (hipStream_t)stream;
  if (desc->M <= 16) return status_of(launch_few_rows_f8(p, st));
  const bool offsets_fit = p.w_stride <= INT32_MAX;
  TileF8 t = desc->M >= 512 && offsets_fit ? TileF8::ROWS256_COLS256 : desc->M > 128 ? TileF8::ROWS128_COLS256 : desc->M > 64 ? TileF8::ROWS64_COLS128 : TileF8::ROWS32_COLS64;
  return status_of(launch_rows_f8(p, t, st));
}

}  // extern "C"
