// Low-rank adapters beside a shared projection, every row with its own: low = scale[a] * x . down[a]^T and, where the projection does not add
// them itself, up[a] . low of every row.
//
// Rows come in blocks, and a block takes its adapters one after the other (usually one or two: the rows of a request lie together), over all
// of its rows: the matrix core's columns are the rows, so what another adapter's rows get is simply not taken.  low is rounded to FP16, as
// every on-chip operand of a second product is here.
#pragma once
#include "routed_rows.hpp"

namespace bolt {

struct LoraParams {
  const half_t* x;
  int64_t ldx;
  const int* adapter;     // [M], none below zero and from `adapters` on
  const half_t* down;     // [adapters][rank][K]
  const half_t* up;       // [adapters][N][rank]
  const float* scales;    // [adapters], or null: 1
  half_t* low;            // [M][rank]
  half_t* y;              // [M][N] (ldy)
  int64_t ldy;
  int M, N, K, adapters, rank;
  int blocks, tiles;      // of rows; of 16 ranks (down) or of columns (up)
};

// f(a, rows of a as this lane's bit) for every adapter that one of the 64 or fewer rows has; lane j holds row j's in `mine`.
template <typename F>
__device__ __forceinline__ void for_adapters(int mine, F&& f) {
  unsigned long long left = __ballot(mine >= 0);
  for (int turn = 0; left != 0; ++turn) {
    const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    left &= ~__ballot(mine == a);
    f(turn, a);
  }
}

// low of 16 rows.  RT tiles of 16 ranks; NW waves take the reduction by turns, U steps of 64 columns at a time, and their sums are added through
// LDS in a fixed order.
//   SPREAD (few rows): a workgroup for each of the block's up to 16 adapters and RT tiles of ranks; those past the last adapter end at once.
//   else: one workgroup for a block, all adapters and ranks.
template <int RT, int NW, int U, bool SPREAD>
__global__ __launch_bounds__(64 * NW) void lora_down_kernel(const LoraParams p) {
  extern __shared__ __attribute__((aligned(16))) float part[];  // [NW][RT][64 lanes][4]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  int block = (int)blockIdx.x, slot = 0, rank0 = 0;
  if constexpr (SPREAD) {
    const int each = 16 * p.tiles;
    block = (int)blockIdx.x / each;
    slot = (int)blockIdx.x - block * each;
    rank0 = slot % p.tiles * (16 * RT);
    slot /= p.tiles;
  }
  const int row0 = block * 16, rows = p.M - row0 < 16 ? p.M - row0 : 16;
  const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < rows);
  const half_t* const x = p.x + (int64_t)(row0 + (l16 < rows ? l16 : rows - 1)) * p.ldx;
  const int steps = (p.K + 63) / 64;
  for_adapters(mine, [&](int turn, int a) {
    if (SPREAD && turn != slot) return;
    const half_t* down[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = rank0 + t * 16 + l16;  // (ranks beyond the last repeat it: their sums are not stored)
      down[t] = p.down + ((int64_t)a * p.rank + (r < p.rank ? r : p.rank - 1)) * p.K;
    }
    floatx4 acc[RT] = {};
    for (int s0 = wave; s0 < steps; s0 += NW * U) {
      half8 xv[U][2], dv[U][2][RT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = (s0 + u * NW) * 64 + h * 32 + g * 8;
          const bool in = k < p.K;
          const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
          const half8 v = *(const half8*)(x + (in ? k : 0));
          xv[u][h] = in ? v : zero;
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const half8 d = *(const half8*)(down[t] + (in ? k : 0));
            dv[u][h][t] = in ? d : zero;
          }
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t] = mfma_16x16x32(dv[u][h][t], xv[u][h], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) *(floatx4*)(part + ((wave * RT + t) * 64 + lane) * 4) = acc[t];
    __syncthreads();
    const float scale = p.scales ? p.scales[a] : 1.f;
    for (int i = tid; i < RT * 64; i += 64 * NW) {
      const int at = i & 63, t = i >> 6, j = at & 15, r = rank0 + t * 16 + (at >> 4) * 4;
      floatx4 v = *(const floatx4*)(part + (t * 64 + at) * 4);
#pragma unroll
      for (int w = 1; w < NW; ++w) v += *(const floatx4*)(part + ((w * RT + t) * 64 + at) * 4);
      if (j >= rows || r >= p.rank || row_adapter(p.adapter, p.adapters, row0 + j, true) != a) continue;
      half4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (half_t)(scale * v[e]);
      *(half4*)(p.low + (int64_t)(row0 + j) * p.rank + r) = o;
    }
    __syncthreads();
  });
}

// y = up[a] . low of every row, zero for rows without an adapter: 64 rows x 256 columns for a workgroup, 64 columns for each of its four
// waves.  Bound by writing y.  The columns of a wave's four tiles are interleaved, so that a lane holds 16 neighbouring ones of a row and
// four lanes a whole line.
__global__ __launch_bounds__(256) void lora_up_kernel(const LoraParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int id = xcd_run((int)blockIdx.x, (int)gridDim.x), block = id / p.tiles;
  const int row0 = block * 64, rows = p.M - row0 < 64 ? p.M - row0 : 64;
  const int col0 = (id - block * p.tiles) * 256 + wave * 64;
  if (col0 >= p.N) return;  // (no barriers here)
  const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < rows);
  int of_row[4];
  const half_t* low[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int j = b * 16 + l16;
    of_row[b] = __shfl(mine, j);
    low[b] = p.low + (int64_t)(row0 + (j < rows ? j : rows - 1)) * p.rank + g * 8;
  }
  const int from = col0 + (l16 >> 2) * 16 + (l16 & 3);  // + 4 t: the column of this lane's weight row in tile t
  floatx4 acc[4][4] = {};
  for_adapters(mine, [&](int, int a) {
    const half_t* const up = p.up + (int64_t)a * p.N * p.rank + g * 8;
    floatx4 sum[4][4] = {};
    for (int k = 0; k < p.rank; k += 32) {
      const bool in = k + g * 8 < p.rank;
      const int at = in ? k : -g * 8;
      const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
      half8 l[4], u[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) l[b] = *(const half8*)(low[b] + at);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int n = from + 4 * t;
        u[t] = *(const half8*)(up + (int64_t)(n < p.N ? n : p.N - 1) * p.rank + at);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) sum[t][b] = mfma_16x16x32(in ? u[t] : zero, in ? l[b] : zero, sum[t][b]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][b][e] = of_row[b] == a ? sum[t][b][e] : acc[t][b][e];
  });
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    if (b * 16 + l16 >= rows) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = col0 + g * 16 + h * 8;
      half8 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (half_t)acc[2 * h][b][e], o[4 + e] = (half_t)acc[2 * h + 1][b][e];
      if (c < p.N) *(half8*)(p.y + (int64_t)(row0 + b * 16 + l16) * p.ldy + c) = o;
    }
  }
}

}  // namespace bolt
