// Low-rank adapters beside a shared projection, every row with its own: low = scale[a] * x . down[a]^T and, where the projection does not add
// them itself, up[a] . low of every row.
//
// Rows come in blocks, and a block takes its adapters one after the other (usually one or two: the rows of a request lie together), over all
// of its rows: the matrix core's columns are the rows, so what another adapter's rows get is simply not taken.  Where there are few blocks, a
// block's adapters are dealt over `turns` workgroups, and the reduction of low over `parts` more: one compute unit alone reads some 30 GB/s, so that
// 128 KB of one adapter take it 4 us.  low is rounded to FP16, as every operand of a second product is here; of several parts whoever reads
// them, which are FP32, adds them up first.
// What bounds it: of few rows the chain of round trips (ids, operands, sums), of many the staging of x: down for one row of 4096 and rank 16 3.6 us on the
// GPU, 29 rows of 5000 with 32 adapters of rank 32 4.6, 700 rows of 4096 with 6 of rank 24 5.0, 4096 rows of 4096 with 4 of rank 64, which it reads once, 18;
// up for 29 rows of 6152 columns 6.0, for 700 x 4104 with 64 of rank 24 7.8, for 4096 x 8192 with 4 of rank 64 45, with 64 of them 73 (134 MB written; with
// halves 6.8, 36 and 59).
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
  const half_t* none;     // eight zeros
  void* low;              // one part: [M][rank] halves, else [parts][M][rank] floats
  float* share;           // [M][N]
  int M, N, K, adapters, rank;
  int parts, turns, tiles, blocks;  // tiles: of 16 RT ranks (down) or of columns (up); blocks: of rows
};

// f(a) for every adapter, by turns of `turns`, that one of up to 64 rows has; lane j holds row j's in `mine`.
template <typename F>
__device__ __forceinline__ void for_adapters(int mine, int turn, int turns, F&& f) {
  unsigned long long left = __ballot(mine >= 0);
  for (int i = 0; left != 0; i = i + 1 == turns ? 0 : i + 1) {
    const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    left &= ~__ballot(mine == a);
    if (i == turn) f(a);
  }
}

// low of 16 rows, RT tiles of 16 ranks.  The NW waves of a block's `parts` workgroups take the reduction by turns, 64 columns a step; every wave
// stages its steps in a ring of its own, S - 1 ahead, in whole lines (in the operand's order, 64 bytes of a row, an L2 gives a third of that),
// without barriers.  A workgroup's sums are added through LDS in a fixed order.
template <int RT, int NW, int S>
__global__ __launch_bounds__(64 * NW) void lora_down_kernel(const LoraParams p) {
  constexpr int PIECES = 2 + 2 * RT, STAGE = PIECES * 512;
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  // (the turns that many blocks do not need come last, so that those they do need are spread over the XCDs)
  int id = (int)blockIdx.x;
  const int part = id % p.parts, rank0 = (id / p.parts) % p.tiles * (16 * RT);
  id /= p.parts * p.tiles;
  const int block = id % p.blocks, turn = id / p.blocks;
  const int row0 = block * 16, rows = p.M - row0 < 16 ? p.M - row0 : 16;
  const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < rows);
  const int first = part * NW + wave, stride = p.parts * NW, steps = (p.K + 63) / 64;
  const int n = steps > first ? (steps - first + stride - 1) / stride : 0;
  half_t* const ring = lds + wave * S * STAGE;

  // Piece h of a tile: rows 8 h .. 8 h + 7, this lane's 16 bytes of row 8 h + lane / 8.  Rows and ranks beyond the last repeat it: their sums are not
  // stored.
  int chunk[2];
  const half_t *x[2], *down[RT][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 8 + (lane >> 3);
    chunk[h] = ((lane & 7) ^ dma_swizzle<64>(r)) * 8;
    x[h] = p.x + (int64_t)(row0 + (r < rows ? r : rows - 1)) * p.ldx;
  }
  for_adapters(mine, turn, p.turns, [&](int a) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = rank0 + t * 16 + h * 8 + (lane >> 3);
        down[t][h] = p.down + ((int64_t)a * p.rank + (r < p.rank ? r : p.rank - 1)) * p.K;
      }
    auto load = [&](int i) {
      half_t* const to = ring + i % S * STAGE;
      const int k0 = (first + i * stride) * 64;
      for_constants<2>([&](auto hc) {
        constexpr int h = decltype(hc)::value;
        const int k = k0 + chunk[h];
        const bool in = k < p.K;  // (beyond K: zeros on both sides)
        lds_load16(in ? x[h] + k : p.none, to + h * 512);
        for_constants<RT>([&](auto tc) {
          constexpr int t = decltype(tc)::value;
          lds_load16(in ? down[t][h] + k : p.none, to + (2 + 2 * t + h) * 512);
        });
      });
    };
    floatx4 acc[RT] = {};
    auto multiply = [&](const half_t* __restrict__ from) {
      for_constants<2>([&](auto sc) {
        const int at = dma_chunk_offset<64>(l16, decltype(sc)::value * 4 + g);
        const half8 b = *(const half8*)(from + at);
        for_constants<RT>([&](auto t) { acc[t] = mfma_16x16x32(*(const half8*)(from + (1 + decltype(t)::value) * 1024 + at), b, acc[t]); });
      });
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
      if (i < n) load(i);
    for (int i = 0; i < n; ++i) {
      // (the step that is loaded next takes the place of the one multiplied last, whose operands have arrived)
      wave_waits_for_reads();
      if (i + S - 1 < n) {
        load(i + S - 1);
        wave_waits_for_loads<(S - 1) * PIECES>();
      } else {
        wave_waits_for_loads<0>();
      }
      multiply(ring + i % S * STAGE);
    }
    __syncthreads();
    float* const sums = (float*)lds;  // [NW][RT][64 lanes][4]
#pragma unroll
    for (int t = 0; t < RT; ++t) *(floatx4*)(sums + ((wave * RT + t) * 64 + lane) * 4) = acc[t];
    __syncthreads();
    const float scale = p.scales ? p.scales[a] : 1.f;
    for (int i = tid; i < RT * 64; i += 64 * NW) {
      const int at = i & 63, t = i >> 6, j = at & 15, r = rank0 + t * 16 + (at >> 4) * 4;
      floatx4 v = *(const floatx4*)(sums + (t * 64 + at) * 4);
#pragma unroll
      for (int w = 1; w < NW; ++w) v += *(const floatx4*)(sums + ((w * RT + t) * 64 + at) * 4);
      if (j >= rows || r >= p.rank || row_adapter(p.adapter, p.adapters, row0 + j, true) != a) continue;
      v *= scale;
      const int64_t to = ((int64_t)part * p.M + row0 + j) * p.rank + r;
      if (p.parts > 1) {
        *(floatx4*)((float*)p.low + to) = v;
      } else {
        half4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
        *(half4*)((half_t*)p.low + to) = o;
      }
    }
    __syncthreads();
  });
}

// share = up[a] . low of every row, zero for rows without an adapter: 16 MB rows x 256 columns for a workgroup, 64 columns for each of its four
// waves, of which four lanes store 64 bytes of a row at a time.
// Each row is stored by the workgroup that has its adapter's turn, those without one by the first.  It stays FP32: what the layer adds it to, and alpha,
// can bring a sum beyond binary16's range back into it, and tiles that compute the share themselves hold it so.
template <int MB>
__global__ __launch_bounds__(256) void lora_up_kernel(const LoraParams p) {
  constexpr int BM = 16 * MB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, l16 = lane & 15;
  const int each = p.blocks * p.tiles, turn = (int)blockIdx.x / each;
  const int id = xcd_run((int)blockIdx.x - turn * each, each), block = id / p.tiles;
  const int row0 = block * BM, rows = p.M - row0 < BM ? p.M - row0 : BM;
  const int col0 = (id - block * p.tiles) * 256 + wave * 64;
  if (col0 >= p.N) return;  // (no barriers here)
  const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < rows);
  int of_row[MB];
  int64_t low[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int j = b * 16 + l16;
    of_row[b] = __shfl(mine, j);
    low[b] = (int64_t)(row0 + (j < rows ? j : rows - 1)) * p.rank + g * 8;
  }
  auto store = [&](int a, const floatx4 (&v)[4][MB]) {
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      if (b * 16 + l16 >= rows || of_row[b] != a) continue;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int c = col0 + t * 16 + g * 4;
        if (c < p.N) *(floatx4*)(p.share + (int64_t)(row0 + b * 16 + l16) * p.N + c) = v[t][b];
      }
    }
  };
  // (low of all ranks once: what the rows have does not depend on the adapter at hand)
  const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  half8 l[4][MB];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      l[k][b] = zero;
      if (k * 32 >= p.rank) continue;
      const bool in = k * 32 + g * 8 < p.rank;
      const half8 v = low_operand(p.low, low[b] + (in ? k * 32 : -g * 8), p.parts, (int64_t)p.M * p.rank);
      l[k][b] = in ? v : zero;
    }
  for_adapters(mine, turn, p.turns, [&](int a) {
    const half_t* const up = p.up + (int64_t)a * p.N * p.rank + g * 8;
    floatx4 sum[4][MB] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k * 32 >= p.rank) break;
      const bool in = k * 32 + g * 8 < p.rank;
      half8 u[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int n = col0 + t * 16 + l16;
        u[t] = *(const half8*)(up + (int64_t)(n < p.N ? n : p.N - 1) * p.rank + (in ? k * 32 : -g * 8));
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int b = 0; b < MB; ++b) sum[t][b] = mfma_16x16x32(in ? u[t] : zero, l[k][b], sum[t][b]);
    }
    store(a, sum);
  });
  if (turn == 0 && __any(lane < rows && mine < 0)) {
    const floatx4 zeros[4][MB] = {};
    store(-1, zeros);
  }
}

}  // namespace bolt
