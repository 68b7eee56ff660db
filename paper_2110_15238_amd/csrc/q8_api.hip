// C ABI of the linear layers whose operands are held in 8 bits.
#include <algorithm>

#include "layer_tiles.hpp"

namespace bolt {
namespace {

bolt_status check_gemm_q8(const bolt_gemm_q8_desc* d) {
  if (!d || d->M < 0 || d->N <= 0 || d->K <= 0 || !known_act(d->act) || d->lda < d->K || d->ldd < d->N) return BOLT_ERR_INVALID_ARG;
  if (((d->N | d->ldd) & 7) || ((d->K | d->lda) & 15)) return BOLT_ERR_ALIGNMENT;
  if (d->lda > kMaxLength || d->ldd > kMaxLength || d->M > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// Tiles for more than 16 rows.  A fit to 7 shapes (1024 to 12288 outputs, K 2048 to 11008) x 7 row counts from 45 to 2048, weights from memory: the
// choice takes 1.01 times the best tile on average, 1.09 at most; of 77 other sizes 1.003 and 1.08.  us, 32 x 32, 64 x 32, 64 x 64, 128 x 64, 128 x 128, 128 x 256 and 256 x 256: 4096 x 4096, 45
// rows 6.7 / 7.6 / 9.0 / 10.9 / 14.7 / 21 / 37, 333 rows 30 / 20 / 17 / 12.5 / 15.6 / 22 / 38, 2048 rows 184 / 96 / 62 / 49 / 35 / 30 / 41; 12288 x 4096, 1024 rows 302 /
// 179 / 126 / 91 / 68 / 65 / 46.
constexpr LayerTile kLayerTiles[] = {{RowsTile::ROWS32_COLS32, 32, 32, 4, 3.3, 0.39},      {RowsTile::ROWS64_COLS32, 64, 32, 4, 2.9, 0.62},
                                     {RowsTile::ROWS64_COLS64, 64, 64, 2, 3.0, 0.48},      {RowsTile::ROWS128_COLS64, 128, 64, 2, 3.1, 0.70},
                                     {RowsTile::ROWS128_COLS128, 128, 128, 1, 2.85, 0.53}, {RowsTile::ROWS128_COLS256, 128, 256, 1, 3.2, 0.82},
                                     {RowsTile::ROWS256_COLS256, 256, 256, 1, 7.0, 1.24}};
// Up to 16 rows: whole lines to LDS here too.  Weights that go to registers in the order of the operands (few_rows_kernel) take, 1 and 16 rows, here / so
// on the better of one and two tiles of 16: 4096 x 4096 5.2 and 5.4 / 5.4 and 6.2; 6152 x 5008 8.2 and 9.5 / 8.9 and 11.2; 12288 x 4096 12.3 and 12.7 /
// 11.3 and 14.1; 4096 x 11008 13.6 and 14.6 / 12.0 and 13.9; 1024 x 8192 6.8 and 6.9 / 6.9 and 9.3; 12288 x 512 4.4 and 4.3 / 4.2 and 4.4.
constexpr RowsTile kFewRowsTile = RowsTile::ROWS16_COLS32;

}  // namespace
}  // namespace bolt

using namespace bolt;

extern "C" {

size_t bolt_gemm_q8_workspace_bytes(const bolt_gemm_q8_desc* desc) {
  (void)desc;
  return 0;
}

bolt_status bolt_gemm_q8(const bolt_gemm_q8_desc* desc, const void* A, const void* a_scales, const void* W, const void* w_scales, const void* bias, void* D,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_gemm_q8(desc); s != BOLT_OK) return s;
  if (desc->M == 0) return BOLT_OK;
  if (!A || !W || !D) return BOLT_ERR_INVALID_ARG;
  for (const void* at : {A, a_scales, W, w_scales, bias, (const void*)D, (const void*)workspace})
    if (!aligned16(at)) return BOLT_ERR_ALIGNMENT;
  if (starts_at(D, {A, a_scales, W, w_scales, bias})) return BOLT_ERR_INVALID_ARG;
  const LayerTile* const tile = desc->M > 16 ? layer_tile(kLayerTiles, desc->M, desc->N, desc->K, true) : nullptr;
  if (desc->M > 16 && !tile) return BOLT_ERR_UNSUPPORTED;
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  LayerParams p{};
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
  return status_of(launch_rows_f8(p, tile ? tile->tile : kFewRowsTile, st));
}

}  // extern "C"
