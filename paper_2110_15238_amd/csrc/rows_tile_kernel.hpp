// Linear layers for some ten to some thousand rows on the tiled kernels' direct-to-LDS main loop (dma_main_loop): E4M3 operands, and FP16 ones whose
// rows have adapters.
//   E4M3: the bytes are those of an FP16 layer of half the depth, a matrix instruction has twice the depth and rate; sums are scaled by row and
//   column in front of the epilogue.
//   Adapters: FROM_ADD takes the rows' share from memory, where lora_up_kernel left it; FROM_ADAPTERS computes it, a wave for its own part of the
//   tile, 64 ranks at a time: the rows' low once, then up of one adapter after the other, the next one's on its way.  A sum is taken only where the
//   row's adapter is the one at hand.
// What bounds it: a workgroup's own steps.  A compute unit takes in some 50 to 70 GB/s of operands with 33 workgroups on the chip as with 198, so it is not what
// the L2s give all of them together; whether loads, LDS reads or matrix instructions hold a step up has not been told apart.  So the reduction is split over
// sets of waves (KG) where there are few workgroups.  us, E4M3, best tile here, 4096 x 11008: 128 rows 20, 333 rows 33, 1024 rows 54; 8192 x 2048: 128 rows
// 7.0, 1024 rows 18.4 (128 x 256).  Splitting it over workgroups whose FP32 sums another launch adds up gained in 5 of 54 sizes, 9 % at most, for E4M3; for FP16
// operands with adapters it has not been tried.
#pragma once
#include "routed_rows.hpp"

namespace bolt {

template <int WT, int ADD, int BM, int BN, int WAVES_M, int WAVES_N, int NS, int KG>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N * KG) void rows_tile_kernel(const LayerParams p) {
  constexpr bool F8 = WT == WEIGHTS_F8;
  static_assert(WT != WEIGHTS_W4 && (!F8 || ADD == ADD_NOTHING), "kinds of layers");
  constexpr int BK = 64;  // (E4M3: pairs, 128 values)
  using T = FpropDmaTraits<BM, BN, BK, WAVES_M, WAVES_N, 0, NS, KG>;
  constexpr int WPG = T::WPG, WTM = T::WTM, WTN = T::WTN, FM = T::FM, FN = T::FN;
  using XL = DmaTileLoader<BM, BK, WPG, 0, KG>;
  using WL = DmaTileLoader<BN, BK, WPG, 0, KG>;
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave_all / WPG, wave = wave_all - kg * WPG;
  const int wm = wave % WAVES_M, wn = wave / WAVES_M, g = lane >> 5, l32 = lane & 31;
  int tm, tn;
  tile_of_workgroup(blockIdx.x, p.row_blocks, p.col_blocks, 8, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;

  const ConvGeom none{};
  XL xl;
  WL wl;
  // The sets take the steps by turns, all the same number of turns, beyond the last on zeros.
  const int64_t xrem = ((int64_t)(p.M - m0 - 1) * p.ldx + p.K) * 2, wrem = (int64_t)(p.N - n0) * p.K * 2;
  xl.init(p.x + (int64_t)m0 * p.ldx, (unsigned)(xrem < 0x7fffffff ? xrem : 0x7fffffff), (int)p.ldx, p.M - m0, p.K, none, m0, kg, wave, lane);
  wl.init((const half_t*)p.w + (int64_t)n0 * p.K, (unsigned)(wrem < 0x7fffffff ? wrem : 0x7fffffff), p.K, p.N - n0, p.K, none, n0, kg, wave, lane);

  floatx16 acc[FN][FM];
#pragma unroll
  for (int a = 0; a < FN; ++a)
#pragma unroll
    for (int b = 0; b < FM; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
  // this lane's columns: fragment a, quad q
  auto column = [&](int a, int q) { return wn * WTN + a * 32 + q * 8 + g * 4; };
  half4 bias[FN][4];
  floatx4 col_scale[F8 ? FN : 1][4];
  float row_scale[F8 ? FM : 1];
  floatx4 add[ADD == FROM_ADD ? FN : 1][4][FM];
  dma_main_loop<BM, BN, BK, WAVES_M, WAVES_N, NS, KG, (F8 && T::G < 2 ? 2 : T::G), (T::DEEP || T::NW < 8 ? 2 : 3), false, F8>(
      xl, wl, lds + kg * T::GROUP_HALVES, none, kg, (p.steps + KG - 1) / KG, wm, wn, lane, acc, [&] {
        if (kg > 0) return;
#pragma unroll
        for (int a = 0; a < FN; ++a)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = n0 + column(a, q), n = c < p.N ? c : 0;
            bias[a][q] = *(const half4*)(p.bias + n * p.bias_on);
            if constexpr (F8) col_scale[a][q] = column_scales(p, n);
          }
#pragma unroll
        for (int b = 0; b < FM; ++b) {
          const int m = m0 + wm * WTM + b * 32 + l32, row = m < p.M ? m : p.M - 1;
          if constexpr (F8) row_scale[b] = p.x_scales ? p.x_scales[row] : 1.f;
          if constexpr (ADD == FROM_ADD)
#pragma unroll
            for (int a = 0; a < FN; ++a)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const int c = n0 + column(a, q);
                add[a][q][b] = *(const floatx4*)(p.add + (int64_t)row * p.N + (c < p.N ? c : 0));
              }
        }
      });

  // the sets' sums, added in a fixed order
  if constexpr (KG > 1) {
    float* const red = reinterpret_cast<float*>(lds);  // [KG - 1][WPG][FN * FM * 16][64 lanes]
    barrier_after_lds_writes();
    if (kg > 0) {
      float* const mine = red + ((kg - 1) * WPG + wave) * (FN * FM * 16 * 64) + lane;
#pragma unroll
      for (int a = 0; a < FN; ++a)
#pragma unroll
        for (int b = 0; b < FM; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) mine[((a * FM + b) * 16 + r) * 64] = acc[a][b][r];
    }
    barrier_after_lds_writes();
    if (kg == 0) {
      for (int o = 0; o < KG - 1; ++o) {
        const float* const theirs = red + (o * WPG + wave) * (FN * FM * 16 * 64) + lane;
#pragma unroll
        for (int a = 0; a < FN; ++a)
#pragma unroll
          for (int b = 0; b < FM; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] += theirs[((a * FM + b) * 16 + r) * 64];
      }
    }
  }

  if constexpr (ADD == FROM_ADAPTERS) {
    if (kg == 0) {
      static_assert(WTM <= 64, "a row for each lane");
      const int row0 = m0 + wm * WTM, col0 = n0 + wn * WTN;
      const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < WTM && row0 + lane < p.M);
      const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
      for (int k0 = 0; k0 < p.rank; k0 += 64) {
        // (lane l supplies ranks 8 (l / 32) .. + 7 of every 16; those beyond the last are zero on both sides)
        half8 low[FM][4];
        int of_row[FM];
#pragma unroll
        for (int b = 0; b < FM; ++b) {
          const int m = row0 + b * 32 + l32;
          of_row[b] = __shfl(mine, b * 32 + l32);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k0 + k * 16 >= p.rank) {  // (the same for all lanes)
              low[b][k] = zero;
              continue;
            }
            const int at = k0 + k * 16 + g * 8;
            const half8 v = low_operand(p.low, (int64_t)(m < p.M ? m : p.M - 1) * p.rank + (at < p.rank ? at : 0), p.low_parts, (int64_t)p.M * p.rank);
            low[b][k] = at < p.rank ? v : zero;
          }
        }
        half8 up[2][FN][4];
        auto load = [&](int adapter, half8 (&u)[FN][4]) {
          const half_t* const from = p.up + (int64_t)adapter * p.N * p.rank;
#pragma unroll
          for (int a = 0; a < FN; ++a) {
            const int n = col0 + a * 32 + l32;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (k0 + k * 16 >= p.rank) {
                u[a][k] = zero;
                continue;
              }
              const int at = k0 + k * 16 + g * 8;
              const half8 v = *(const half8*)(from + (int64_t)(n < p.N ? n : p.N - 1) * p.rank + (at < p.rank ? at : 0));
              u[a][k] = at < p.rank ? v : zero;
            }
          }
        };
        unsigned long long left = __ballot(mine >= 0);
        auto take = [&] {  // the next adapter, -1 behind the last
          if (left == 0) return -1;
          const int adapter = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
          left &= ~__ballot(mine == adapter);
          return adapter;
        };
        auto multiply = [&](int adapter, const half8 (&u)[FN][4]) {
#pragma unroll
          for (int a = 0; a < FN; ++a)
#pragma unroll
            for (int b = 0; b < FM; ++b) {
              floatx16 sum;
#pragma unroll
              for (int r = 0; r < 16; ++r) sum[r] = 0.f;
#pragma unroll
              for (int k = 0; k < 4; ++k) sum = mfma_32x32x16(u[a][k], low[b][k], sum);
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[a][b][r] += of_row[b] == adapter ? sum[r] : 0.f;
            }
        };
        int now = take();
        if (now >= 0) load(now, up[0]);
        while (now >= 0) {
          int next = take();
          if (next >= 0) load(next, up[1]);
          multiply(now, up[0]);
          if (next < 0) break;
          now = take();
          if (now >= 0) load(now, up[0]);
          multiply(next, up[1]);
        }
      }
    }
  }

  // out, through LDS, so that whole row segments are stored
  constexpr int CPR = T::CPR;
  barrier_after_lds_writes();
  if (kg == 0) {
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int nl = column(a, q);
#pragma unroll
        for (int b = 0; b < FM; ++b) {
          floatx4 v = {acc[a][b][q * 4], acc[a][b][q * 4 + 1], acc[a][b][q * 4 + 2], acc[a][b][q * 4 + 3]};
          if constexpr (F8) v *= col_scale[a][q] * row_scale[b];
          if constexpr (ADD == FROM_ADD) v += add[a][q][b];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = p.alpha * v[e] + p.beta * (float)bias[a][q][e];
          v = apply_act4(v, p.act);
          half4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
          const int row = wm * WTM + b * 32 + l32;
          *(half4*)(lds + row * BN + (((nl >> 3) ^ ctile_swizzle<CPR>(row)) << 3) + (nl & 4)) = o;
        }
      }
  }
  barrier_after_lds_writes();
  for (int i = tid; i < BM * CPR; i += T::NT) {
    const int row = i / CPR, chunk = i % CPR, n = n0 + chunk * 8;
    if (m0 + row < p.M && n < p.N)
      *(half8*)((half_t*)p.y + (int64_t)(m0 + row) * p.ldy + n) = *(const half8*)(lds + row * BN + ((chunk ^ ctile_swizzle<CPR>(row)) << 3));
  }
}

template <int WT, int ADD, int BM, int BN, int WAVES_M, int WAVES_N, int NS, int KG>
hipError_t launch_rows_tiles(LayerParams p, hipStream_t stream) {
  using T = FpropDmaTraits<BM, BN, 64, WAVES_M, WAVES_N, 0, NS, KG>;
  static_assert(T::LDS_BYTES <= 160 * 1024, "stages");
  auto kern = rows_tile_kernel<WT, ADD, BM, BN, WAVES_M, WAVES_N, NS, KG>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, T::LDS_BYTES); e != hipSuccess) return e;
  p.row_blocks = (p.M + BM - 1) / BM;
  p.col_blocks = (p.N + BN - 1) / BN;
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * p.col_blocks), dim3(T::NT), T::LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
