// Products of some to some hundred rows with weights in 4 bits or FP16: between few_rows_kernel, whose waves each read all of their
// activations, and the kernels for many rows, which stage both operands for all waves.
//
// A workgroup computes 16 MB activation rows x 16 R WN weight rows.  The activation rows are shared by its waves.  The weights are not: a
// wave owns 16 R weight rows, so 4-bit weights are decoded once per workgroup and never stored.  Both go to LDS directly, S - 1 steps
// ahead (a round trip to memory is about 2000 cycles, a step over 32 rows some hundred): the weights into a piece that only their
// wave reads (4-bit ones in the order it reads them, FP16 and E4M3 ones in whole lines), so that no register holds what is on its way and every
// load is one that can be counted.
// KG sets of WN waves split the reduction (step t to set t % KG) where there are few workgroups; their sums are added through LDS in a
// fixed order.  One barrier per step.
// What bounds it: of few rows the instructions of a step (decoding, LDS reads, matrix instructions one behind the other), which several
// workgroups per compute unit cover for each other, so tiles are small; of many rows LDS reads, decoding and matrix instructions are
// about equally long and overlap in part.  Measured in 4 bits: 29 tokens to 8 of 128 experts 2048 x 768, 29 to 32 us for 165 MB of gate and value rows
// (5 TB/s and more) and 19 to 22 us for the 83 MB behind; 3001 tokens to 4 of 32 experts 1536 x 1280, 154 and 93 us (600 and 500 TFLOP/s); 100 x 8192 x 2048
// 9.9 to 10.3 us.  More stages than three cost resident workgroups and are slower (the first 64 us: 75 with four); so are 4 tiles of weight rows
// per wave, which leave one wave per SIMD (64 x 256 tiles, 265 -> 346 us for the second).  FP16 experts, both products, weights staged in the order of the
// operands / in whole lines: 48 tokens to 2 of 4 experts 4096 x 1024 37.2 / 27.9, 200 to 4 of 32 1024 x 768 47.1 / 37.9, gated 100 to 4 of 16 2048 x 512 47.9 / 38.1.
#pragma once
#include "few_rows_kernel.hpp"
#include "moe_tile_kernel.hpp"

namespace bolt {

template <int WT, int MODE, bool GATED, int NG, int MB, int R, int WN, int KG, int S>
struct SharedRowsTraits {
  static constexpr bool W4 = WT == WEIGHTS_W4;
  static constexpr int NW = WN * KG, NT = 64 * NW, BM = 16 * MB;
  static constexpr int COLS = 16 * R * WN / (GATED ? 2 : 1);
  static constexpr int KS = W4 ? 4 : 2;                        // matrix instructions of a step
  static constexpr int HALVES = W4 ? 2 : 1;                    // 64-column activation tiles of a step
  static constexpr int PIECES = R * (W4 ? 1 : KS);             // KB of weights of a wave and step
  static constexpr int METAS = W4 ? (R * NG * 12 + 63) / 64 : 0;  // 256-byte pieces of scales and zero points
  static constexpr int XI = HALVES * (BM / 8) / WN;            // load instructions of a wave and step for the activations
  static constexpr int LOADS = PIECES + METAS + XI;
  static constexpr int X_HALVES = HALVES * BM * 64, W_HALVES = PIECES * 512 + METAS * 128;
  static constexpr int STAGE = X_HALVES + WN * W_HALVES;       // halves of one set of waves
  static constexpr int SUM_BYTES = (KG - 1) * WN * R * MB * 1024;
  static constexpr int PIPE_BYTES = KG * S * STAGE * 2;
  static constexpr int LDS_BYTES = PIPE_BYTES > SUM_BYTES ? PIPE_BYTES : SUM_BYTES;
  static_assert(HALVES * (BM / 8) % WN == 0 && WN % 2 == 0, "every wave loads the same number of activation pieces");
  static_assert(LDS_BYTES <= 160 * 1024 && S >= 3, "stages");
};

// The rows' adapters (linear layers): acc += up[a] . low^T for every adapter a that one of the rows has, adapter i by set i % KG of the waves, 64 ranks at
// a time (of 64 rows 32: registers): the rows' low once, then up of one adapter after the other, the next one's on its way.  A sum is taken only where the
// row's adapter is a.
template <int MB, int R, int KG>
__device__ __forceinline__ void add_adapters_by_sets(const LayerParams& p, int row0, int rows, int col0, int kg, int lane, floatx4 (&acc)[R][MB]) {
  static_assert(MB <= 4, "a row for each lane");
  constexpr int KD = MB < 4 ? 2 : 1;  // matrix instructions, 32 ranks each
  const int g = lane >> 4, l16 = lane & 15;
  const int mine = row_adapter(p.adapter, p.adapters, row0 + lane, lane < rows);
  int of_row[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) of_row[b] = __shfl(mine, b * 16 + l16);
  const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int k0 = 0; k0 < p.rank; k0 += 32 * KD) {
    // (ranks beyond the last are zero on both sides)
    auto at = [&](int k) { return k0 + 32 * k + g * 8; };
    auto any = [&](int k) { return k0 + 32 * k < p.rank; };  // (the same for all lanes)
    auto load = [&](int a, half8 (&u)[R][KD]) {
      const half_t* const up = p.up + (int64_t)a * p.N * p.rank;
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const int n = col0 + t * 16 + l16;
        const half_t* const from = up + (int64_t)(n < p.N ? n : p.N - 1) * p.rank;
#pragma unroll
        for (int k = 0; k < KD; ++k) {
          u[t][k] = zero;
          if (any(k)) u[t][k] = *(const half8*)(from + (at(k) < p.rank ? at(k) : 0));
        }
      }
    };
    unsigned long long left = __ballot(mine >= 0);
    int turn = 0;
    auto take = [&] {  // this set's next adapter, -1 behind its last
      while (left != 0) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        left &= ~__ballot(mine == a);
        const bool ours = turn == kg;
        turn = turn + 1 == KG ? 0 : turn + 1;
        if (ours) return a;
      }
      return -1;
    };
    int now = take();
    if (now < 0) return;
    half8 up[2][R][KD], low[MB][KD];
    load(now, up[0]);
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const int j = b * 16 + l16;
      const int64_t row = (int64_t)(row0 + (j < rows ? j : rows - 1)) * p.rank;
#pragma unroll
      for (int k = 0; k < KD; ++k) {
        low[b][k] = zero;
        if (any(k)) {
          const half8 v = low_operand(p.low, row + (at(k) < p.rank ? at(k) : 0), p.low_parts, (int64_t)p.M * p.rank);
          low[b][k] = at(k) < p.rank ? v : zero;
        }
      }
    }
    auto multiply = [&](int a, const half8 (&u)[R][KD]) {
#pragma unroll
      for (int t = 0; t < R; ++t)
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KD; ++k) sum = mfma_16x16x32(at(k) < p.rank ? u[t][k] : zero, low[b][k], sum);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][b][e] += of_row[b] == a ? sum[e] : 0.f;
        }
    };
    while (now >= 0) {
      const int next = take();
      if (next >= 0) load(next, up[1]);
      multiply(now, up[0]);
      if (next < 0) break;
      now = take();
      if (now >= 0) load(now, up[0]);
      multiply(next, up[1]);
    }
  }
}

// MORE (linear layers of 4-bit weights): the adapters' share, from p.add where that is given, else, up to 64 rows, computed here.
template <int WT, bool MORE>
using SharedParams = std::conditional_t<WT == WEIGHTS_F8 || MORE, LayerParams, RowsParams>;
template <int WT, int MODE, bool GATED, int NG, int MB, int R, int WN, int KG, int S, bool MORE = false>
__device__ __forceinline__ void shared_rows_tile(const SharedParams<WT, MORE>& p, RowsWave<WT, MODE, GATED, NG, MB, R>& w, int wave_all, int cb, half_t* lds) {
  using T = SharedRowsTraits<WT, MODE, GATED, NG, MB, R, WN, KG, S>;
  using Wave = RowsWave<WT, MODE, GATED, NG, MB, R>;
  constexpr int BM = T::BM, KS = T::KS;
  const int lane = w.lane, kg = wave_all / WN, wave = wave_all - kg * WN;
  const int col0 = cb * T::COLS + wave * (16 * R / (GATED ? 2 : 1));  // this wave's first output column
  w.take_columns(col0);
  // Scales and zero points: lane l of piece m loads dword 64 m + l of a wave's step: R * NG * 8 of scales ([tile][quad of rows][group][4
  // rows]), then R * NG * 4 of zero points ([tile][row][group]).
  const unsigned* meta[T::METAS > 0 ? T::METAS : 1];
  int meta_stride[T::METAS > 0 ? T::METAS : 1];
  if constexpr (T::W4) {
    constexpr int SCALES = R * NG * 8, ALL = R * NG * 12;
#pragma unroll
    for (int m = 0; m < T::METAS; ++m) {
      const int d = m * 64 + lane < ALL ? m * 64 + lane : ALL - 1;
      const bool is_scale = d < SCALES;
      const int t = is_scale ? d / (NG * 8) : (d - SCALES) / (NG * 4), in = is_scale ? d % (NG * 8) : (d - SCALES) % (NG * 4);
      const int row = w.first_row(col0, t) + (is_scale ? in / (NG * 2) * 4 : in * 4 / NG);  // the first of the rows it belongs to
      const int at = row < p.N ? row : (p.N - 1) & ~3;
      const int64_t base = w.expert * p.scale_stride + (int64_t)(at >> 4) * p.steps * 16 * NG;
      meta[m] = is_scale ? (const unsigned*)(p.scales + base + ((at & 15) >> 2) * NG * 4) + in % (NG * 2)
                         : (const unsigned*)(p.zeros + base + (at & 15) * NG);
      meta_stride[m] = is_scale ? NG * 8 : NG * 4;
    }
  }

  // ---- activations: tiles of BM rows x 64 columns, 8 rows per load instruction, dealt over the waves of a set -------------------
  constexpr int RG = BM / 8, AT = RG > WN ? RG / WN : 1;
  const int lrow = lane >> 3, lc = (lane & 7) ^ dma_swizzle<64>(wave * 8 + lrow);  // (WN is even)
  __amdgpu_buffer_rsrc_t xrsrc;
  unsigned xat[AT];
  {
    // (UP: the host keeps x below 2 GiB)
    if constexpr (MODE == ROWS_UP) xrsrc = make_rsrc(p.x, 0x7fffffffu);
    else xrsrc = make_rsrc(p.x + (int64_t)w.row0 * p.ldx, (unsigned)(((int64_t)(w.rows - 1) * p.ldx + p.K) * 2));
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      const int r = (j * WN + wave) % RG * 8 + lrow;
      const int from = MODE == ROWS_UP ? p.order[w.row0 + (r < w.rows ? r : w.rows - 1)] / p.top_k : r;
      xat[j] = r < w.rows ? (unsigned)from * (unsigned)(p.ldx * 2) : kInvalidOffset;
    }
  }
  // FP16, E4M3: a tile of 16 weight rows and 64 columns is two pieces of 8 whole lines, swizzled as the activations are.  (Pieces of 16 rows x 64
  // bytes, in the order of the operand, come out of an L2 at a third of the rate.)
  const unsigned char* wline[R][2];
  int wchunk[2];
  if constexpr (!T::W4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = h * 8 + lrow;
      wchunk[h] = (lane & 7) ^ dma_swizzle<64>(r);
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const int row = w.first_row(col0, t) + r;
        wline[t][h] = p.w + w.expert * p.w_stride + (int64_t)(row < p.N ? row : p.N - 1) * p.K * 2;
      }
    }
  }
  half_t* const ring = lds + kg * S * T::STAGE;

  // ---- steps kg, kg + KG, ...: every set of waves runs `turns` of them; one past the end is not multiplied -------------------
  const int last_step = p.steps - 1, turns = (p.steps + KG - 1) / KG;
  auto load = [&](int turn, half_t* stage) {
    const int step = kg + turn * KG, at = step < last_step ? step : last_step;
    half_t* const mine = stage + T::X_HALVES + wave * T::W_HALVES;
    for_constants<R>([&](auto tc) {
      constexpr int t = decltype(tc)::value;
      if constexpr (T::W4) {
        lds_load16(w.wrow[t] + (int64_t)at * W4Format::BLOCK_BYTES, mine + t * 512);
      } else {
        for_constants<2>([&](auto hc) {
          constexpr int h = decltype(hc)::value;
          const int k = at * 64 + wchunk[h] * 8;  // (beyond K: zeros; an infinite weight would make a NaN of the zero it meets)
          lds_load16(k < p.K ? wline[t][h] + (int64_t)k * 2 : (const unsigned char*)p.none, mine + (t * 2 + h) * 512);
        });
      }
    });
    for_constants<T::METAS>([&](auto m) { lds_load4(meta[m] + (int64_t)at * meta_stride[m], mine + T::PIECES * 512 + decltype(m)::value * 128); });
    for_constants<T::XI>([&](auto ic) {
      constexpr int j = decltype(ic)::value;
      const int i = j * WN + wave, h = i / RG;
      const int k = step * 32 * KS + h * 64 + lc * 8;
      const unsigned off = k < p.K ? xat[j % AT] + (unsigned)k * 2u : kInvalidOffset;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xrsrc, BOLT_LDS_PTR(stage + i * 512), 16, off, 0, 0, 0);
    });
  };
  floatx4 acc[R][MB] = {};
  auto multiply = [&](const half_t* __restrict__ xs) {
    const half_t* const mine = xs + T::X_HALVES + wave * T::W_HALVES;
    const half_t* const scales = mine + T::PIECES * 512;
    const unsigned* const zeros = (const unsigned*)(scales + R * NG * 16);
    unsigned zp[R];
    half4 scale[R][NG];
    uintx4 piece[R];
    if constexpr (T::W4) {
      for_constants<R>([&](auto t) {
        piece[t] = *(const uintx4*)(mine + t * 512 + lane * 8);
        zp[t] = zeros[t * NG * 4 + w.l16 * NG / 4] >> (w.l16 * NG % 4 * 8);
        for_constants<NG>([&](auto i) { scale[t][i] = *(const half4*)(scales + t * NG * 16 + (w.g * NG + decltype(i)::value) * 4); });
      });
    }
    if constexpr (WT == WEIGHTS_F8) {
      half8 x[MB][2];
      for_constants<MB>([&](auto b) {
        for_constants<2>([&](auto s) {
          x[b][s] = *(const half8*)(xs + dma_chunk_offset<64>(decltype(b)::value * 16 + w.l16, decltype(s)::value * 4 + w.g));
        });
      });
      for_constants<R>([&](auto t) {
        const half8 a0 = *(const half8*)(mine + t * 1024 + dma_chunk_offset<64>(w.l16, w.g));
        const half8 a1 = *(const half8*)(mine + t * 1024 + dma_chunk_offset<64>(w.l16, 4 + w.g));
        for_constants<MB>([&](auto b) { acc[t][b] = mfma_16x16x128_f8(a0, a1, x[b][0], x[b][1], acc[t][b]); });
      });
      return;
    }
    floatx4 sum[R][MB];
    for_constants<KS>([&](auto sc) {
      constexpr int s = decltype(sc)::value;
      half8 x[MB];
      for_constants<MB>([&](auto b) {
        x[b] = *(const half8*)(xs + (s >> 1) * BM * 64 + dma_chunk_offset<64>(decltype(b)::value * 16 + w.l16, (s & 1) * 4 + w.g));
      });
      for_constants<R>([&](auto tc) {
        constexpr int t = decltype(tc)::value;
        if constexpr (T::W4) {
          constexpr int MPG = Wave::MPG, i = s / MPG;
          const unsigned z = (zp[t] >> (i * 8)) & 0xffu;
          const half8 a = w4_values(piece[t][s], w4_minus1(z), w4_minus16(z));
          for_constants<MB>([&](auto b) { sum[t][b] = mfma_16x16x32(a, x[b], s % MPG == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : sum[t][b]); });
          if constexpr (s % MPG == MPG - 1)
            for_constants<MB>([&](auto b) {
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[t][b][e] += (float)scale[t][i][e] * sum[t][b][e];
            });
        } else {
          const half8 a = *(const half8*)(mine + t * 1024 + dma_chunk_offset<64>(w.l16, s * 4 + w.g));
          for_constants<MB>([&](auto b) { acc[t][b] = mfma_16x16x32(a, x[b], acc[t][b]); });
        }
      });
    });
  };
  // Loads complete in order, so all but the newest (S - 2) * LOADS are there when no more are outstanding.
  constexpr int AHEAD = (S - 2) * T::LOADS < 63 ? (S - 2) * T::LOADS : 63;
#pragma unroll
  for (int t = 0; t < S - 1; ++t) load(t, ring + t * T::STAGE);
  // (while the first steps' loads are on their way)
  if constexpr (MORE && MB <= 4)
    if (!p.add) add_adapters_by_sets<MB, R, KG>(p, w.row0, w.rows, col0, kg, lane, acc);
  int stage = 0, fill = S - 1;
  const int all = KG > 1 ? p.steps / KG : turns;  // turns that every set has
  for (int t = 0; t < all; ++t) {
    // this turn's loads have landed for every wave of the set, and every wave is done with the stage that is filled next
    barrier_after_reads_and_loads<AHEAD>();
    load(t + S - 1, ring + fill * T::STAGE);
    multiply(ring + stage * T::STAGE);
    fill = stage;
    stage = stage + 1 == S ? 0 : stage + 1;
  }
  if (KG > 1 && all < turns) {  // (apart: a branch in the loop costs 4 % at 24 rows of 5800 x 6656)
    barrier_after_reads_and_loads<AHEAD>();
    if (kg + all * KG <= last_step) multiply(ring + stage * T::STAGE);
  }
  barrier_after_reads_and_loads<0>();  // nothing is on its way into LDS any more

  if constexpr (KG > 1) {
    float* const sums = (float*)lds;  // [KG - 1][WN][R * MB][64 lanes][4]
    if (kg > 0) w.put_sums(sums + (kg - 1) * WN * R * MB * 256, wave, acc);
    barrier_after_lds_writes();
    if (kg > 0) return;
#pragma unroll
    for (int k = 0; k < KG - 1; ++k)
#pragma unroll
      for (int a = 0; a < R; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[a][b] += *(const floatx4*)(sums + ((k * WN + wave) * R * MB + a * MB + b) * 256 + lane * 4);
  }

  int g = w.g, l16 = w.l16;
  if constexpr (MORE) {
    // (the lane's number anew: kept through the loop above it would be spilled)
    int elane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    asm volatile("" : "+v"(elane));
    g = elane >> 4;
    l16 = elane & 15;
    // the share from memory, all of a lane's quads asked for together
    if (p.add) {
      const float* const share = p.add + (int64_t)w.row0 * p.N;
#pragma unroll
      for (int a = 0; a < R; ++a) {
        const int col = col0 + a * 16 + g * 4, n = col < p.N ? col : 0;
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          const int j = b * 16 + l16;
          acc[a][b] += *(const floatx4*)(share + ((unsigned)(j < w.rows ? j : w.rows - 1) * (unsigned)p.N + (unsigned)n));  // (128 rows of 2^21 at most)
          asm volatile("" : "+v"(acc[a][b]));  // (added here, not where it is stored)
        }
      }
    }
  }

  // ---- out: four columns of one row per accumulator ------------------------------------------------------------------
  const int outputs = GATED ? p.hidden : p.N;
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int j = b * 16 + l16;
    if (j >= w.rows) continue;
    const int64_t to = MODE == ROWS_DOWN ? p.order[w.row0 + j] : w.row0 + j;
#pragma unroll
    for (int a = 0; a < R; a += GATED ? 2 : 1) {
      const int col = col0 + (GATED ? a / 2 : a) * 16 + g * 4;
      if (col >= outputs) continue;
      auto with_bias = [&](floatx4 v, int n) {
        const half4 hb = *(const half4*)(p.bias + (w.expert * (int64_t)p.N + n) * p.bias_on);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = p.alpha * v[e] + p.beta * (float)hb[e];
        return v;
      };
      if constexpr (WT == WEIGHTS_F8) acc[a][b] *= column_scales(p, col) * (p.x_scales ? p.x_scales[w.row0 + j] : 1.f);
      floatx4 v = with_bias(acc[a][b], col);
      v = apply_act4(v, p.act);
      if constexpr (GATED) v *= with_bias(acc[a + 1][b], p.hidden + col);
      if constexpr (MODE == ROWS_DOWN) {
        *(floatx4*)((float*)p.y + to * p.ldy + col) = v;
      } else {
        half4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
        *(half4*)((half_t*)p.y + to * p.ldy + col) = o;
      }
    }
  }
}

template <int WT, int MODE, bool GATED, int NG, int MB, int R, int WN, int KG, int S, bool MORE = false>
__global__ __launch_bounds__(64 * WN * KG, MORE && MB <= 4 ? 4 : 1) void shared_rows_kernel(const SharedParams<WT, MORE> p) {
  using T = SharedRowsTraits<WT, MODE, GATED, NG, MB, R, WN, KG, S>;
  constexpr int BM = T::BM;
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  RowsWave<WT, MODE, GATED, NG, MB, R> w(p, lane);
  int cb;
  if constexpr (MODE == ROWS_DENSE) {
    const int id = xcd_run((int)blockIdx.x, (int)gridDim.x);
    cb = id / p.row_blocks;
    w.row0 = (id - cb * p.row_blocks) * BM;
    w.rows = p.M - w.row0 < BM ? p.M - w.row0 : BM;
  } else {
    const BlockCounts counts = count_row_blocks<BM>(p.offsets, p.experts, lane);
    const int total = counts.total() * p.col_blocks;
    if ((int)blockIdx.x >= total) return;
    const int tile = xcd_run((int)blockIdx.x, total);
    RowBlock at;
    if (!find_row_block<BM>(p.offsets, counts, tile / p.col_blocks, &at)) return;
    const int local = tile - at.first * p.col_blocks;
    cb = local / at.count;
    const int done = (local - cb * at.count) * BM;
    w.expert = at.expert;
    w.row0 = at.lo + done;
    w.rows = at.n - done < BM ? at.n - done : BM;
  }
  shared_rows_tile<WT, MODE, GATED, NG, MB, R, WN, KG, S, MORE>(p, w, __builtin_amdgcn_readfirstlane(tid >> 6), cb, lds);
}

// The tiles of columns that hold marked weights (w4_unpack_kernel), all rows; a workgroup whose columns hold none reads 16 numbers and ends.
template <int NG, int MB, int R, int WN, int S>
__global__ __launch_bounds__(64 * WN) void shared_rows_marked_kernel(const LayerParams p) {
  using T = SharedRowsTraits<WEIGHTS_W4, ROWS_DENSE, false, NG, MB, R, WN, 1, S>;
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, cb = blockIdx.x;
  const int row = cb * T::COLS + (lane < T::COLS / 16 ? lane : 0) * 16;
  const half_t first = row < p.N ? p.unpacked[(int64_t)row * p.K] : (half_t)0.f;
  if (!__any(first != first)) return;  // (the same for every wave)
  for (int rb = blockIdx.y; rb < p.row_blocks; rb += gridDim.y) {
    RowsWave<WEIGHTS_W4, ROWS_DENSE, false, NG, MB, R> w(p, lane);
    w.row0 = rb * T::BM;
    w.rows = p.M - w.row0 < T::BM ? p.M - w.row0 : T::BM;
    static_assert(MB > 4, "a share is in memory, if there is one");
    shared_rows_tile<WEIGHTS_W4, ROWS_DENSE, false, NG, MB, R, WN, 1, S, true>(p, w, __builtin_amdgcn_readfirstlane(tid >> 6), cb, lds);
  }
}

template <int WT, int MODE, bool GATED, int NG, int MB, int R, int WN, int KG, int S, bool MORE = false>
hipError_t launch_shared_rows(SharedParams<WT, MORE> p, hipStream_t stream) {
  static_assert(!MORE || (WT == WEIGHTS_W4 && MODE == ROWS_DENSE), "adapters: linear layers of 4-bit weights");
  auto kern = shared_rows_kernel<WT, MODE, GATED, NG, MB, R, WN, KG, S, MORE>;
  using T = SharedRowsTraits<WT, MODE, GATED, NG, MB, R, WN, KG, S>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, T::LDS_BYTES); e != hipSuccess) return e;
  p.col_blocks = ((GATED ? p.hidden : p.N) + T::COLS - 1) / T::COLS;
  p.row_blocks = row_blocks<T::BM>(p, MODE);
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * p.col_blocks), dim3(T::NT), T::LDS_BYTES, stream, p);
  return hipGetLastError();
}
template <int NG, int MB, int R, int WN, int S>
hipError_t launch_shared_rows_marked(LayerParams p, hipStream_t stream) {
  auto kern = shared_rows_marked_kernel<NG, MB, R, WN, S>;
  using T = SharedRowsTraits<WEIGHTS_W4, ROWS_DENSE, false, NG, MB, R, WN, 1, S>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, T::LDS_BYTES); e != hipSuccess) return e;
  p.col_blocks = (p.N + T::COLS - 1) / T::COLS;
  p.row_blocks = row_blocks<T::BM>(p, ROWS_DENSE);
  const int per_column = p.col_blocks < 256 ? 256 / p.col_blocks : 1;  // workgroups: one round of the compute units
  hipLaunchKernelGGL(kern, dim3(p.col_blocks, p.row_blocks < per_column ? p.row_blocks : per_column), dim3(T::NT), T::LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
