// C ABI of projections that are shared by requests with low-rank adapters of their own.
#include <algorithm>
#include <cmath>

#include "layer_tiles.hpp"
#include "lora_kernel.hpp"

namespace bolt {
namespace {

constexpr int kMaxRank = 128;
// Workgroups of 16 rows from which low's reduction is not split any more, and into how many parts at most.
constexpr int kDownGroups = 256, kMostParts = kMostLowParts;

// Whether the projection runs on the kernel for up to 16 rows, which adds the adapters itself: some more rows too, where all of their blocks are on the
// chip at once (2048 x 8192 in 4 bits with 32 adapters, 17 to 32 rows: 19.8 us so, 24 on tiles of 32 rows behind lora_up_kernel; FP16 25 and 25).
// Of wide projections, more than two tiles of 16 columns for each compute unit, the tiles have more than 8 rows (12 where groups of 32 make decoding dearer):
// us, 9 and 16 rows with 32 adapters of rank 24, few rows / tiles: FP16 8200 x 4096 24.8 and 29.1 / 22.0 and 22.5, 12288 x 5000 38.6 and 46.9 / 37.6 and 41.2;
// 4 bits, groups of 128, 21.1 and 24.9 / 18.6 and 19.9, 22.2 and 25.4 / 21.0 and 22.8, of 32 21.9 and 26.4 / 20.4 and 21.8, 22.7 and 26.8 / 23.3 and 25.0;
// FP16 6152 x 5000 with rank 16, 16 rows 20.4 / 22.7.
bool on_few_rows(const bolt_gemm_lora_desc& d) {
  const bool narrow = d.N <= 16 * 512, dear = d.weights == BOLT_WEIGHTS_W4 && d.group == 32;
  return (d.M <= 16 && (narrow || d.M <= (dear ? 12 : 8))) || (d.M <= 64 && blocks_of(d.M, 16) * blocks_of(d.N, 16) <= 256);
}

bolt_gemm_w4_desc base_w4(const bolt_gemm_lora_desc& d) { return {d.M, d.N, d.K, d.lda, d.ldd, d.group, d.alpha, d.beta, d.act}; }

bolt_status check_gemm_lora(const bolt_gemm_lora_desc* d) {
  if (!d || d->M < 0 || d->N <= 0 || d->K <= 0 || d->adapters <= 0 || d->rank <= 0 || d->lda < d->K || d->ldd < d->N) return BOLT_ERR_INVALID_ARG;
  if (!known_act(d->act) || d->act == BOLT_ACT_SILU) return BOLT_ERR_INVALID_ARG;
  if (d->weights != BOLT_WEIGHTS_F16 && d->weights != BOLT_WEIGHTS_W4) return BOLT_ERR_INVALID_ARG;
  if (d->weights == BOLT_WEIGHTS_W4) {
    const bolt_gemm_w4_desc base = base_w4(*d);
    if (bolt_status s = check_gemm_w4(&base); s == BOLT_ERR_INVALID_ARG) return s;
  }
  if ((d->N | d->K | d->lda | d->ldd | d->rank) & 7) return BOLT_ERR_ALIGNMENT;
  if (d->lda > kMaxLength || d->ldd > kMaxLength || d->rank > kMaxRank || d->M > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  // the launches of 64 x 256 outputs and of 16 rows
  if (!launches(blocks_of(d->M, 16)) || !launches(blocks_of(d->M, 64) * blocks_of(d->N, 256))) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// The workspace: low [parts][M][rank], the adapters' share [M][N] in FP32 (whichever kernel runs, so that the size does not fall as M grows) and 4-bit
// weights that may be unpacked.
struct LoraWorkspace {
  int64_t share_at, weights_at, bytes;
};
LoraWorkspace lora_workspace(const bolt_gemm_lora_desc& d) {
  LoraWorkspace w;
  // (a bound of parts * M that does not fall as M grows)
  w.share_at = round_up(std::max<int64_t>(d.M, std::min<int64_t>((int64_t)kMostParts * d.M, 16 * kDownGroups)) * d.rank * 4, 256);
  w.weights_at = w.bytes = w.share_at + round_up((int64_t)d.M * d.N * 4, 256);
  if (d.weights == BOLT_WEIGHTS_W4) {
    const bolt_gemm_w4_desc base = base_w4(d);
    w.bytes += round_up((int64_t)bolt_gemm_w4_workspace_bytes(&base), 256);
  }
  return w;
}

// Over how many workgroups a block's adapters are dealt: as many as the block can have where the launch has few workgroups.
int turns_of(const LoraParams& p, int block_rows, int64_t workgroups) {
  const int64_t most = std::min<int64_t>(std::min(block_rows, p.M), p.adapters);
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, 512 / workgroups));
}

// Tiles of 16 ranks that a workgroup of lora_down_kernel has, 1, 2, 4 or 8: all of them, so that x is read once, unless that leaves compute units without
// work though the reduction is split into kMostParts; rows that are as good as single have one.
int down_tiles(int64_t M, int rank) {
  if (M <= 64) return 1;
  int tiles = rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
  while (tiles > 1 && blocks_of(M, 16) * blocks_of(rank, 16 * tiles) * kMostParts < 160) tiles /= 2;
  return tiles;
}
// Parts of low's reduction, as many as the launch needs to fill the chip.
int down_parts(int64_t M, int rank) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMostParts, kDownGroups / (blocks_of(M, 16) * (M <= 64 ? 1 : blocks_of(rank, 16 * down_tiles(M, rank))))));
}

template <int RT, int NW, int S>
hipError_t launch_down(LoraParams p, hipStream_t stream) {
  auto kern = lora_down_kernel<RT, NW, S>;
  constexpr int LDS_BYTES = NW * S * (2 + 2 * RT) * 1024;
  static_assert(LDS_BYTES <= 160 * 1024 && NW * RT * 1024 <= LDS_BYTES, "stages; the sums take their place");
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, LDS_BYTES); e != hipSuccess) return e;
  const int blocks = p.blocks = (p.M + 15) / 16;
  p.tiles = (p.rank + 16 * RT - 1) / (16 * RT);
  p.turns = turns_of(p, 16, (int64_t)blocks * p.tiles * p.parts);
  hipLaunchKernelGGL(kern, dim3(blocks * p.tiles * p.turns * p.parts), dim3(64 * NW), LDS_BYTES, stream, p);
  return hipGetLastError();
}
hipError_t launch_lora_down(const LoraParams& p, hipStream_t stream) {
  switch (down_tiles(p.M, p.rank)) {
    case 1: return launch_down<1, 4, 4>(p, stream);
    case 2: return launch_down<2, 4, 3>(p, stream);
    case 4: return launch_down<4, 4, 2>(p, stream);
    default: return launch_down<8, 4, 2>(p, stream);
  }
}
template <int MB>
hipError_t launch_up(LoraParams p, hipStream_t stream) {
  const int blocks = p.blocks = (p.M + 16 * MB - 1) / (16 * MB);
  p.tiles = (p.N + 255) / 256;
  p.turns = turns_of(p, 16 * MB, (int64_t)blocks * p.tiles);
  hipLaunchKernelGGL(lora_up_kernel<MB>, dim3(blocks * p.tiles * p.turns), dim3(256), 0, stream, p);
  return hipGetLastError();
}
// (64 rows for a workgroup read up less often, 16 make more workgroups)
hipError_t launch_lora_up(const LoraParams& p, hipStream_t stream) {
  return blocks_of(p.M, 64) * blocks_of(p.N, 256) < 256 ? launch_up<1>(p, stream) : launch_up<4>(p, stream);
}

// ---- which kernels run a projection with FP16 weights on more than 16 rows ----------------------------------------------------
// A fit to 5 shapes (1024 to 8192 outputs, K 2048 to 11008) x 10 row counts from 17 to 3300, with adapters in the tiles and with their share from memory:
// the choice takes the best tile of all 50, and 1.002 times it of 77 other sizes (1.11 at most; 64 x 128 and 256 x 128 tiles beside these would have won 0.6 % there,
// 8 % at most).  us with adapters of rank 32 in runs, 64 x 32, 64 x 64, 128 x 64, 128 x 128, 128 x 256 and 256 x 256: 4096 x 4096, 64
// rows 16.4 / 21.7 / 24.7 / 39 / 55 / -, 700 rows 79 / 57 / 49 / 39 / 51 / 81, 3300 rows 307 / 212 / 174 / 141 / 114 / 97.
constexpr LayerTile kLayerTiles[] = {{RowsTile::ROWS64_COLS32, 64, 32, 4, 2.5, 0.70},      {RowsTile::ROWS64_COLS64, 64, 64, 2, 2.2, 0.49},
                                     {RowsTile::ROWS128_COLS64, 128, 64, 2, 2.0, 0.68},    {RowsTile::ROWS128_COLS128, 128, 128, 1, 1.0, 0.58},
                                     {RowsTile::ROWS128_COLS256, 128, 256, 1, 0.0, 0.90},  {RowsTile::ROWS256_COLS256, 256, 256, 1, 9.4, 1.26}};
template <typename D>
const LayerTile* projection_tile(const D& d) {
  const bool bias_in_sum = d.alpha != 0.f && std::fabs(d.beta) <= 1e30f * std::fabs(d.alpha);
  return layer_tile(kLayerTiles, d.M, d.N, (int64_t)d.K * 2, bias_in_sum);
}
// Whether the tiles compute the adapters' share.  Where the rows of a request lie together a tile has one or two adapters, which cost it 1 to 3 us (256 x 256:
// 7); each further one 0.5 (2.4), and how many there are the host does not know: it asks that the most there can be cost no more than the share's way
// through memory (lora_up_kernel: 7.8 us for 700 x 4104, 45 and more for 4096 x 8192).
bool adapters_in_tiles(const bolt_gemm_lora_desc& d, const LayerTile& t) {
  const double most = std::min(d.adapters, std::min(t.rows, d.M)) * (t.tile == RowsTile::ROWS256_COLS256 ? 2.4 : 0.5);
  return layer_rounds(t, d.M, d.N) * most <= 3.5 + 1.1e-6 * d.M * d.N;
}
// The same for tiles on 4-bit weights, which have fewer waves to hide it behind: while the most adapters a tile can have are few, of low rank.  us, 64 rows
// (32 x 32 and 32 x 64 tiles) and 300 (64 x 128), share through memory / in the tiles: 4096 x 4096, 2 adapters of rank 16 17.0 / 14.0 and 33.6 / 31.0, 8 17.5 /
// 15.6 and 38.6 / 37.9, 32 18.6 / 17.7 and 44.2 / 44.3, 64 18.9 / 18.7 and 45.5 / 46.5; 6152 x 5000, 2 of rank 72 25.0 / 24.1 and 48.5 / 51.4, 8 31.0 / 30.6 and
// 70.5 / 65.4, 32 38.6 / 41.1 and 103 / 102.  128 x 256 tiles lose with two of rank 16 already (12288 x 4096, 300 rows 64 / 75).
bool adapters_in_w4_tiles(const bolt_gemm_lora_desc& d) {
  const bolt_gemm_w4_desc base = base_w4(d);
  const SharedTile tile = tile_of_gemm_w4(base);
  if (bolt_gemm_w4_workspace_bytes(&base) > 0 || tile == SharedTile::ROWS128_COLS256) return false;
  const int rows = tile_size(tile).rows;
  return std::min(d.adapters, std::min(rows, d.M)) * blocks_of(d.rank, 32) <= (rows == 32 ? 16 : 8);
}
// (256 x 256 tiles read low as halves.)
int low_parts(const bolt_gemm_lora_desc& d) {
  if (d.weights == BOLT_WEIGHTS_F16 && !on_few_rows(d))
    if (const LayerTile* t = projection_tile(d); t && t->tile == RowsTile::ROWS256_COLS256) return 1;
  return down_parts(d.M, d.rank);
}

}  // namespace

hipError_t launch_projection_f16_add(const LayerParams& p, hipStream_t stream) {
  const LayerTile* const tile = projection_tile(p);
  return tile ? launch_rows_f16_add(p, tile->tile, stream) : hipErrorInvalidConfiguration;
}

}  // namespace bolt

using namespace bolt;

extern "C" {

size_t bolt_gemm_lora_workspace_bytes(const bolt_gemm_lora_desc* desc) {
  if (check_gemm_lora(desc) != BOLT_OK) return 0;
  return (size_t)lora_workspace(*desc).bytes;
}

bolt_status bolt_gemm_lora(const bolt_gemm_lora_desc* desc, const void* A, const void* W, const void* bias, const void* ids, const void* down,
                           const void* up, const void* scales, void* D, void* workspace, size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_gemm_lora(desc); s != BOLT_OK) return s;
  if (desc->M == 0) return BOLT_OK;
  if (!A || !W || !ids || !down || !up || !D) return BOLT_ERR_INVALID_ARG;
  for (const void* at : {A, W, bias, ids, down, up, scales, (const void*)D, (const void*)workspace})
    if (!aligned16(at)) return BOLT_ERR_ALIGNMENT;
  const bolt_gemm_lora_desc& d = *desc;
  const LoraWorkspace ws = lora_workspace(d);
  if (!workspace || workspace_bytes < (size_t)ws.bytes) return BOLT_ERR_WORKSPACE;
  if (starts_at(D, {A, W, bias, ids, down, up, scales, workspace}) || starts_at(workspace, {A, W, bias, ids, down, up, scales})) return BOLT_ERR_INVALID_ARG;
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  const bool w4 = d.weights == BOLT_WEIGHTS_W4, few = on_few_rows(d);
  const LayerTile* const tile = w4 || few ? nullptr : projection_tile(d);
  if (!w4 && !few && !tile) return BOLT_ERR_UNSUPPORTED;
  const bolt_gemm_w4_desc base = base_w4(d);
  const hipStream_t st = (hipStream_t)stream;
  LoraParams l{};
  l.x = (const half_t*)A; l.ldx = d.lda;
  l.adapter = (const int*)ids;
  l.down = (const half_t*)down; l.up = (const half_t*)up; l.scales = (const float*)scales;
  l.low = workspace;
  l.none = none;
  l.parts = low_parts(d);
  l.M = d.M; l.N = d.N; l.K = d.K; l.adapters = d.adapters; l.rank = d.rank;
  if (launch_lora_down(l, st) != hipSuccess) return BOLT_ERR_LAUNCH;
  LayerParams p{};
  if (w4) {
    p = dense_w4_rows(base, A, W, bias, D, none);
  } else {
    p.x = (const half_t*)A; p.ldx = d.lda;
    p.w = (const unsigned char*)W; p.w_stride = (int64_t)d.N * d.K * 2;
    p.none = none;
    p.bias = bias ? (const half_t*)bias : none;
    p.bias_on = bias ? 1 : 0;
    p.y = D; p.ldy = d.ldd;
    p.M = d.M; p.N = d.N; p.K = d.K; p.steps = (d.K + 63) / 64;
    p.alpha = d.alpha; p.beta = d.beta; p.act = d.act;
  }
  p.adapter = l.adapter; p.low = l.low; p.up = l.up; p.adapters = d.adapters; p.rank = d.rank; p.low_parts = l.parts;
  if (few) return status_of(w4 ? launch_few_rows_w4_lora(p, d.group, st) : launch_few_rows_f16_lora(p, st));
  if (tile && adapters_in_tiles(d, *tile)) return status_of(launch_rows_f16_adapters(p, tile->tile, st));
  if (w4 && adapters_in_w4_tiles(d)) return status_of(launch_shared_rows_w4_lora(p, d.group, tile_of_gemm_w4(base), st));
  l.share = (float*)((char*)workspace + ws.share_at);
  if (launch_lora_up(l, st) != hipSuccess) return BOLT_ERR_LAUNCH;
  if (w4) return run_gemm_w4(base, A, W, bias, l.share, D, (char*)workspace + ws.weights_at, stream);
  p.add = l.share;
  return status_of(launch_rows_f16_add(p, tile->tile, st));
}

}  // extern "C"
