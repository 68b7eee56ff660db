// The experts' products over many rows: a grouped GEMM, each expert's list rows with that expert's weights, on the direct-to-LDS main
// loop of the tiled kernels (dma_main_loop).
//
// Row blocks of BM list rows are counted expert by expert, each expert's last one may be short; the host knows only a bound of their number,
// so a workgroup finds its tile from `offsets` and those past the last tile end at once.  Tiles run row block fastest inside an
// expert, and every XCD takes a contiguous run of them: the row blocks that share a stretch of weights run side by side on one L2.
//   UP: the activation rows are gathered by the loader (one byte offset per row and lane, as for a convolution's pixels); with a gate the
//       weight tile alternates 32 gate rows and the 32 value rows of the same columns, so that a lane holds both factors of an output.
//   DOWN: the rows lie in the list's order; results leave in FP32, to the slot's row.
// What bounds it: a workgroup's own chain of steps, where there is one workgroup for each compute unit.  1000 wide, 2504 hidden, 158 rows for each
// expert, 64 x 128 tiles, the down product's 40 steps: 17.5 us with 24 tiles on the chip, 19 with 96, 22 with 240 (0.37 to 0.46 us a step, of which the
// matrix instructions are 0.11; operands from the caches, 9 TB/s with 240 tiles), so neither bandwidth nor the L2s; 37 with 384 tiles, which are two
// rounds.  Weights that no cache holds add to a step (700 tokens to 2 of 8 experts: 22 and 23 us up and down on the same weights again and again, 25 and
// 31 on changing ones).  Two stages are slower (26 and 40 there), four or six no better, two sets of waves that split the reduction 31 and 30.
#pragma once
#include "routed_rows.hpp"

namespace bolt {

// An operand tile whose rows lie anywhere: one byte offset per row that a lane loads, from a base that all share.
template <int ROWS, int BK, int NW>
struct ListedRowsLoader {
  static constexpr int CH = BK / 8, RPI = 64 / CH, ALL = ROWS / RPI;  // ALL: instructions of a tile
  static constexpr int NI = ALL / NW;                                 // of a wave
  static_assert(BK == 64 && ALL % NW == 0 && NW % 2 == 0, "every wave loads as many pieces, which the main loop's waits count");
  __amdgpu_buffer_rsrc_t rsrc;
  unsigned at[NI];  // kInvalidOffset for rows that do not exist
  int lc, wave, K;
  // offset_of(tile row): byte offset of the row from `base`, or kInvalidOffset
  template <typename F>
  __device__ __forceinline__ void init(const void* base, unsigned bytes, int K_, int wave_, int lane, F&& offset_of) {
    rsrc = make_rsrc(base, bytes);
    K = K_;
    wave = wave_;
    const int lrow = lane / CH;
    lc = (lane % CH) ^ dma_swizzle<BK>(wave * RPI + lrow);
#pragma unroll
    for (int j = 0; j < NI; ++j) at[j] = offset_of((j * NW + wave) * RPI + lrow);
  }
  template <int J0, int J1>
  __device__ __forceinline__ void issue_part(int kt, half_t* dst, const ConvGeom&) {
    const int k = kt * BK + lc * 8;
#pragma unroll
    for (int j = J0; j < J1; ++j) {
      const unsigned off = k < K ? at[j] + (unsigned)k * 2u : kInvalidOffset;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, BOLT_LDS_PTR(dst + (j * NW + wave) * RPI * BK), 16, off, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void issue(int kt, half_t* dst, const ConvGeom& cg) { issue_part<0, NI>(kt, dst, cg); }
  __device__ __forceinline__ void advance(const ConvGeom&) {}
};

template <int BM, int BN, int WAVES_M, int WAVES_N, int NS, int MODE, bool GATED>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void moe_tile_kernel(const RowsParams p) {
  constexpr int BK = 64;
  using T = FpropDmaTraits<BM, BN, BK, WAVES_M, WAVES_N, 0, NS>;
  constexpr int NW = T::NW, WTM = T::WTM, WTN = T::WTN, FM = T::FM, FN = T::FN;
  static_assert(!GATED || FN % 2 == 0, "gated: a wave holds gate and value of its outputs");
  static_assert(MODE != ROWS_DENSE, "routed lists");
  using Loader = ListedRowsLoader<BM, BK, NW>;
  using WLoader = ListedRowsLoader<BN, BK, NW>;
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WAVES_M, wn = wave / WAVES_M, g = lane >> 5, l32 = lane & 31;

  // ---- the tile ---------------------------------------------------------------------------------------------------
  const BlockCounts counts = count_row_blocks<BM>(p.offsets, p.experts, lane);
  const int total = counts.total() * p.col_blocks;
  if ((int)blockIdx.x >= total) return;
  const int tile = xcd_run((int)blockIdx.x, total);
  RowBlock rb;
  if (!find_row_block<BM>(p.offsets, counts, tile / p.col_blocks, &rb)) return;
  const int local = tile - rb.first * p.col_blocks, cb = local / rb.count, block = local - cb * rb.count;
  const int row0 = rb.lo + block * BM, rows = rb.n - block * BM < BM ? rb.n - block * BM : BM;
  constexpr int COLS = GATED ? BN / 2 : BN;
  const int c0 = cb * COLS, outputs = GATED ? p.hidden : p.N;

  // ---- operands ---------------------------------------------------------------------------------------------------
  Loader xl;
  WLoader wl;
  if constexpr (MODE == ROWS_UP) {
    // (the host keeps x under 2 GiB)
    xl.init(p.x, 0x7fffffffu, p.K, wave, lane, [&](int r) {
      return r < rows ? (unsigned)(p.order[row0 + r] / p.top_k) * (unsigned)(p.ldx * 2) : kInvalidOffset;
    });
  } else {
    xl.init(p.x + (int64_t)row0 * p.ldx, (unsigned)(rows * p.ldx * 2), p.K, wave, lane,
            [&](int r) { return r < rows ? (unsigned)(r * p.ldx * 2) : kInvalidOffset; });
  }
  // (and each expert's weights)
  wl.init(p.w + rb.expert * p.w_stride, (unsigned)p.w_stride, p.K, wave, lane, [&](int r) {
    const int c = GATED ? c0 + (r >> 6) * 32 + (r & 31) : c0 + r;
    return c < outputs ? (unsigned)(c + (GATED && (r & 32) ? p.hidden : 0)) * (unsigned)(p.K * 2) : kInvalidOffset;
  });
  floatx16 acc[FN][FM];
#pragma unroll
  for (int a = 0; a < FN; ++a)
#pragma unroll
    for (int b = 0; b < FM; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;

  // this lane's output columns: fragment a, quad q -> column of the tile's outputs
  constexpr int FO = GATED ? FN / 2 : FN;
  auto column = [&](int a, int q) { return wn * (WTN / (GATED ? 2 : 1)) + a * 32 + q * 8 + g * 4; };
  half4 bias[FN][4];
  const ConvGeom none{};
  dma_main_loop<BM, BN, BK, WAVES_M, WAVES_N, NS, 1, T::G, (T::DEEP || NW < 8 ? 2 : 3), false>(
      xl, wl, lds, none, 0, (p.K + BK - 1) / BK, wm, wn, lane, acc, [&] {
#pragma unroll
        for (int a = 0; a < FN; ++a)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = c0 + column(GATED ? a >> 1 : a, q), n = (c < outputs ? c : 0) + (GATED && (a & 1) ? p.hidden : 0);
            bias[a][q] = *(const half4*)(p.bias + (rb.expert * (int64_t)p.N + n) * p.bias_on);
          }
      });

  // ---- out --------------------------------------------------------------------------------------------------------
  auto value = [&](int a, int b, int q) {
    floatx4 v = {acc[a][b][q * 4], acc[a][b][q * 4 + 1], acc[a][b][q * 4 + 2], acc[a][b][q * 4 + 3]};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += (float)bias[a][q][e];
    return v;
  };
  if constexpr (MODE == ROWS_DOWN) {
#pragma unroll
    for (int b = 0; b < FM; ++b) {
      const int r = wm * WTM + b * 32 + l32;
      if (r >= rows) continue;
      const int64_t slot = p.order[row0 + r];
      float* const to = (float*)p.y + slot * p.ldy;
#pragma unroll
      for (int a = 0; a < FO; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0 + column(a, q);
          if (c < outputs) *(floatx4*)(to + c) = value(a, b, q);
        }
    }
  } else {
    // through LDS, so that whole row segments are stored
    constexpr int CPR = COLS / 8, NT = 64 * NW;
    barrier_after_lds_writes();
#pragma unroll
    for (int a = 0; a < FO; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int nl = column(a, q);
#pragma unroll
        for (int b = 0; b < FM; ++b) {
          floatx4 v = value(GATED ? 2 * a : a, b, q);
          v = apply_act4(v, p.act);
          if constexpr (GATED) v *= value(2 * a + 1, b, q);
          half4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
          const int row = wm * WTM + b * 32 + l32;
          *(half4*)(lds + row * COLS + (((nl >> 3) ^ ctile_swizzle<CPR>(row)) << 3) + (nl & 4)) = o;
        }
      }
    barrier_after_lds_writes();
    for (int i = tid; i < BM * CPR; i += NT) {
      const int row = i / CPR, chunk = i % CPR, c = c0 + chunk * 8;
      if (row < rows && c < outputs)
        *(half8*)((half_t*)p.y + (int64_t)(row0 + row) * p.ldy + c) = *(const half8*)(lds + row * COLS + ((chunk ^ ctile_swizzle<CPR>(row)) << 3));
    }
  }
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int NS, int MODE, bool GATED>
hipError_t launch_moe_tiles(RowsParams p, hipStream_t stream) {
  using T = FpropDmaTraits<BM, BN, 64, WAVES_M, WAVES_N, 0, NS>;
  auto kern = moe_tile_kernel<BM, BN, WAVES_M, WAVES_N, NS, MODE, GATED>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, T::LDS_BYTES); e != hipSuccess) return e;
  constexpr int COLS = GATED ? BN / 2 : BN;
  p.col_blocks = ((GATED ? p.hidden : p.N) + COLS - 1) / COLS;
  p.row_blocks = row_blocks<BM>(p, MODE);
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * p.col_blocks), dim3(T::NT), T::LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
