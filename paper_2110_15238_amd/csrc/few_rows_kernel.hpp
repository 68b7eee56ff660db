// Products of up to 16 rows with a large weight matrix [N][K]: the linear layers of a handful of tokens, with weights in 4 bits
// or in FP16, for one matrix or for the experts that a router chose.
//
// Every weight is used for 16 rows at most, so the product is bound by reading the weights once, and small ones by the launch and one
// round trip to memory.  A workgroup owns 16 R weight rows; its NW waves take the reduction in turns, step by step (a wave's step
// is 128 columns of 4-bit weights or 64 of FP16 ones), so that the workgroup reads its weights as one stream.  Weights and activations go
// straight from memory to registers, several steps ahead, in the operand order of v_mfma_f32_16x16x32_f16, whose 16 columns are the
// activation rows; nothing passes through LDS but the waves' partial sums, which are added in a fixed order.
//   4-bit weights: an operand is q - z, exact in a half; the sum over a group of columns comes out of the matrix core in FP32
//   and is scaled there, so neither scale nor zero point costs accuracy.  (Nine vector instructions make eight operands.)
//   Activation rows beyond the last repeat the last: their columns of the result are not stored.  Columns beyond K are zero on
//   both sides.
// Measured: 4096 x 4096 in 4 bits, one row, 4.2 us (8.7 MB); 6152 x 5000, 13 rows, 7.3 us (17 MB); one token's 8 experts in FP16, 2048 x 1024:
// 16.3 us for 67 MB of gate and value rows (4.1 TB/s; a large copy moves 5.15), 8.5 us for 34 MB behind them.
#pragma once
#include "routed_rows.hpp"
#include "w4_format.hpp"

namespace bolt {

// What both kernels below do alike, for one wave of a workgroup: B = 16 MB activation rows, R tiles of 16 weight rows.
//   WT, NG: kind of weights, groups of a 128-column step (4 bits)
template <int WT, int MODE, bool GATED, int NG, int MB, int R>
struct RowsWave {
  static constexpr int KS = WT == WEIGHTS_W4 ? 4 : 2, STEP = 32 * KS;  // matrix instructions and columns of a step
  static constexpr int MPG = KS / NG;                                  // matrix instructions of a group (4 bits)
  static constexpr int B = 16 * MB, COLS = GATED ? 8 * R : 16 * R;     // rows and outputs of a workgroup's tile
  static constexpr int PIECES = WT == WEIGHTS_W4 ? 1 : KS;             // 16-byte pieces of weights per tile and step
  static_assert(!GATED || R % 2 == 0, "gated: tiles come in pairs");

  struct Weights {  // one step
    uintx4 piece[R][PIECES];
    half4 scale[R][NG];
    unsigned zero[R];
  };
  struct Rows {  // one step
    half8 part[KS][MB];
  };

  const RowsParams& p;
  int lane, g, l16, expert, row0, rows;
  const half_t* xrow[MB];
  const unsigned char* wrow[R];
  __amdgpu_buffer_rsrc_t wtile[R];  // FP16: the rows of a tile, and this lane's place in them
  unsigned wlane[R];
  const half_t* scale_at[R];
  const unsigned char* zero_at[R];

  __device__ __forceinline__ RowsWave(const RowsParams& p_, int lane_) : p(p_), lane(lane_), g(lane_ >> 4), l16(lane_ & 15), expert(0) {}

  // A routed list's block of rows; false beyond the last.
  __device__ __forceinline__ bool take_block(int block) {
    RowBlock at;
    if (!find_row_block<B>(p.offsets, count_row_blocks<B>(p.offsets, p.experts, lane), block, &at)) return false;
    const int done = (block - at.first) * B;
    expert = at.expert;
    row0 = at.lo + done;
    rows = at.n - done < B ? at.n - done : B;
    return true;
  }
  // Rows beyond the last repeat the last: their columns of the result are not stored.
  __device__ __forceinline__ void take_rows() {
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const int j = b * 16 + l16, row = row0 + (j < rows ? j : rows - 1);
      const int64_t from = MODE == ROWS_UP ? p.order[row] / p.top_k : row;
      xrow[b] = p.x + from * p.ldx + g * 8;
    }
  }
  // First weight row of tile t.
  __device__ __forceinline__ int first_row(int col0, int t) const { return GATED ? (t & 1) * p.hidden + col0 + (t >> 1) * 16 : col0 + t * 16; }
  // The tiles of output columns col0 .. col0 + COLS - 1.  Rows beyond the last repeat it.
  __device__ __forceinline__ void take_columns(int col0) {
    const unsigned char* const w = p.w + expert * p.w_stride;
    const int64_t scales = expert * p.scale_stride;
    const int last = p.N - 1;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const int first = first_row(col0, t);
      const int row = first + l16 < last ? first + l16 : last;
      if constexpr (WT == WEIGHTS_W4) {
        wrow[t] = w + (int64_t)(row >> 4) * p.steps * W4Format::BLOCK_BYTES + (g * 16 + (row & 15)) * 16;
        const int quad = first + g * 4 < last ? first + g * 4 : last & ~3;  // (a multiple of 4: the quad lies in one tile)
        scale_at[t] = p.scales + scales + ((int64_t)(quad >> 4) * p.steps * 4 + ((quad & 15) >> 2)) * (NG * 4);
        zero_at[t] = p.zeros + scales + ((int64_t)(row >> 4) * p.steps * 16 + (row & 15)) * NG;
      } else {
        wrow[t] = w + ((int64_t)row * p.K + g * 8) * 2;
        const int base = first < last ? first : last;
        wtile[t] = make_rsrc(w + (int64_t)base * p.K * 2, (unsigned)(16 * p.K * 2));  // (K <= 2^21)
        wlane[t] = (unsigned)(((row - base) * p.K + g * 8) * 2);
      }
    }
  }
  // Step `step` of the weights.  4-bit weights are padded to whole steps.  FP16, RAGGED: columns beyond K are zero (the buffer's range; through
  // one for whole steps too the deep kernel takes 145 registers for 100, and two of 16 experts of 4096 x 2560 99.6 us for 90.7).
  template <bool RAGGED>
  __device__ __forceinline__ void load_weights(int step, Weights& out) const {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      if constexpr (WT == WEIGHTS_W4) {
        out.piece[t][0] = *(const uintx4*)(wrow[t] + (int64_t)step * W4Format::BLOCK_BYTES);
        const half_t* s = scale_at[t] + (int64_t)step * (NG * 16);
#pragma unroll
        for (int i = 0; i < NG; ++i) out.scale[t][i] = *(const half4*)(s + i * 4);
        const unsigned char* z = zero_at[t] + (int64_t)step * (NG * 16);
        if constexpr (NG == 4) out.zero[t] = *(const unsigned*)z;
        else if constexpr (NG == 2) out.zero[t] = *(const unsigned short*)z;
        else out.zero[t] = *z;
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int k = step * STEP + s * 32;
          if constexpr (RAGGED) {
            const unsigned at = k + g * 8 < p.K ? wlane[t] : kInvalidOffset;
            out.piece[t][s] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(wtile[t], at, k * 2, 0));
          } else {
            out.piece[t][s] = *(const uintx4*)(wrow[t] + (int64_t)k * 2);
          }
        }
      }
    }
  }
  template <bool RAGGED>
  __device__ __forceinline__ void load_rows(int step, Rows& out) const {
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const int k = step * STEP + s * 32;
        const bool in = !RAGGED || k + g * 8 < p.K;
        const half8 v = *(const half8*)(xrow[b] + (in ? k : -g * 8));
        out.part[s][b] = in ? v : half8{0, 0, 0, 0, 0, 0, 0, 0};
      }
  }
  // RAGGED: step `step` may not exist; of 4-bit weights another's were read for it then, and it is left out (a scale may be infinite, and would
  // make a NaN of the zero activations).
  template <bool RAGGED>
  __device__ __forceinline__ void multiply(int step, const Weights& w, const Rows& x, floatx4 (&acc)[R][MB]) const {
    if (RAGGED && WT == WEIGHTS_W4 && step >= p.steps) return;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      if constexpr (WT == WEIGHTS_W4) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const unsigned z = NG == 1 ? w.zero[t] : (w.zero[t] >> (i * 8)) & 0xffu;
          const half2v m1 = w4_minus1(z), m16 = w4_minus16(z);
          floatx4 sum[MB];
#pragma unroll
          for (int b = 0; b < MB; ++b) sum[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = i * MPG; s < (i + 1) * MPG; ++s) {
            const half8 a = w4_values(w.piece[t][0][s], m1, m16);
#pragma unroll
            for (int b = 0; b < MB; ++b) sum[b] = mfma_16x16x32(a, x.part[s][b], sum[b]);
          }
          const half4 scale = w.scale[t][i];
#pragma unroll
          for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][b][e] += (float)scale[e] * sum[b][e];
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int b = 0; b < MB; ++b) acc[t][b] = mfma_16x16x32(__builtin_bit_cast(half8, w.piece[t][s]), x.part[s][b], acc[t][b]);
      }
    }
  }
  // part: [waves][R * MB][64 lanes][4] floats
  __device__ __forceinline__ void put_sums(float* part, int wave, const floatx4 (&acc)[R][MB]) const {
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int b = 0; b < MB; ++b) *(floatx4*)(part + ((wave * R * MB + t * MB + b) * 64 + lane) * 4) = acc[t][b];
  }
  // The waves' sums, added in the order of the waves, through the epilogue and out: one thread for a quad of columns of one row.
  template <int NW>
  __device__ __forceinline__ void finish(const float* part, int col0, int tid) const {
    auto sum_of = [&](int t, int b, int at) {
      floatx4 v = *(const floatx4*)(part + ((t * MB + b) * 64 + at) * 4);
#pragma unroll
      for (int k = 1; k < NW; ++k) v += *(const floatx4*)(part + ((k * R * MB + t * MB + b) * 64 + at) * 4);
      return v;
    };
    auto with_bias = [&](floatx4 v, int n) {  // n: weight row of the quad
      const half4 hb = *(const half4*)(p.bias + (expert * (int64_t)p.N + n) * p.bias_on);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = p.alpha * v[e] + p.beta * (float)hb[e];
      return v;
    };
    constexpr int OUT = (GATED ? R / 2 : R) * MB;
    const int outputs = GATED ? p.hidden : p.N;
    for (int i = tid; i < OUT * 64; i += 64 * NW) {
      const int at = i & 63, b = (i >> 6) % MB, t = (i >> 6) / MB;
      const int j = b * 16 + (at & 15), col = col0 + t * 16 + (at >> 4) * 4;
      if (j >= rows || col >= outputs) continue;
      floatx4 v = with_bias(sum_of(GATED ? 2 * t : t, b, at), col);
      v = apply_act4(v, p.act);
      if constexpr (GATED) v *= with_bias(sum_of(2 * t + 1, b, at), p.hidden + col);
      if constexpr (MODE == ROWS_DOWN) {
        *(floatx4*)((float*)p.y + (int64_t)p.order[row0 + j] * p.ldy + col) = v;
      } else {
        half4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
        *(half4*)((half_t*)p.y + (int64_t)(row0 + j) * p.ldy + col) = o;
      }
    }
  }
};

// Deep reductions: a wave's steps pass through NB register sets, one tile of columns per workgroup.
template <int WT, int MODE, bool GATED, int NG, int R, int NW, int NB>
__global__ __launch_bounds__(64 * NW) void few_rows_kernel(const RowsParams p) {
  using Wave = RowsWave<WT, MODE, GATED, NG, 1, R>;
  extern __shared__ __attribute__((aligned(16))) float part[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Wave w(p, tid & 63);
  int cb;
  if constexpr (MODE == ROWS_DENSE) {
    const int id = xcd_run((int)blockIdx.x, (int)gridDim.x);
    cb = id / p.row_blocks;
    w.row0 = (id - cb * p.row_blocks) * Wave::B;
    w.rows = p.M - w.row0 < Wave::B ? p.M - w.row0 : Wave::B;
  } else {
    const int block = (int)blockIdx.x / p.col_blocks;
    cb = (int)blockIdx.x - block * p.col_blocks;
    if (!w.take_block(block)) return;
  }
  const int col0 = cb * Wave::COLS;
  w.take_rows();
  w.take_columns(col0);
  typename Wave::Weights wf[NB];
  typename Wave::Rows xf[NB];
  floatx4 acc[R][1] = {};
  // This wave's steps: wave, wave + NW, ...; a ragged last step is one wave's, behind its whole ones.
  const int whole = p.K / Wave::STEP;
  const int n = whole > wave ? (whole - wave + NW - 1) / NW : 0;
  auto load = [&](int i, auto b) {
    w.template load_weights<false>(wave + i * NW, wf[decltype(b)::value]);
    w.template load_rows<false>(wave + i * NW, xf[decltype(b)::value]);
  };
  auto multiply = [&](auto b) { w.template multiply<false>(0, wf[decltype(b)::value], xf[decltype(b)::value], acc); };
  if (n >= NB) {
    for_constants<NB>([&](auto b) { load(decltype(b)::value, b); });
    int c = 0;
    for (; c + 2 * NB <= n; c += NB)
      for_constants<NB>([&](auto b) {
        multiply(b);
        load(c + NB + decltype(b)::value, b);
      });
    const int left = n - c - NB;  // steps not requested yet, fewer than NB
    for_constants<NB>([&](auto b) {
      multiply(b);
      if (decltype(b)::value < left) load(c + NB + decltype(b)::value, b);
    });
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < left) multiply(b);
    });
  } else {
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < n) load(decltype(b)::value, b);
    });
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < n) multiply(b);
    });
  }
  if (whole < p.steps && whole % NW == wave) {
    w.template load_weights<true>(whole, wf[0]);
    w.template load_rows<true>(whole, xf[0]);
    w.template multiply<true>(whole, wf[0], xf[0], acc);
  }
  w.put_sums(part, wave, acc);
  __syncthreads();
  w.template finish<NW>(part, col0, tid);
}

// Reductions of at most NX steps per wave: the wave's share of the activations stays in registers while the workgroup walks over
// p.walk tiles of columns.  The weights of the next tile are on their way while a tile is multiplied, summed and stored, so the
// cost of finding the rows and of the first round trip to memory is paid once per walk, and the waves' sums have two places, so one
// barrier per tile is enough.  Steps that a wave does not have meet zero activations; their FP16 weights are zero, 4-bit ones are left out.
// (Two workgroups of eight waves share a compute unit with up to 128 registers, which the routed kernels of one group a step and two steps just miss if
// left alone: one token, 8 of 64 experts, 2048 x 2048, no gate, 20.9 us so and 17.7 held to 128; 3 tokens, 3 of 44 experts, 1560 x 664, gated, 14.6
// and 13.7.  Linear layers would spill.)
template <int WT, int MODE, bool GATED, int NG, int R, int NW, int NX>
__global__ __launch_bounds__(64 * NW, WT == WEIGHTS_W4 && MODE != ROWS_DENSE && NG == 1 && NX == 2 ? 4 : 1) void few_rows_walk_kernel(const RowsParams p) {
  using Wave = RowsWave<WT, MODE, GATED, NG, 1, R>;
  constexpr int PART = NW * R * 64 * 4;
  extern __shared__ __attribute__((aligned(16))) float part[];  // [2][PART]
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Wave w(p, tid & 63);
  const int walks = (p.col_blocks + p.walk - 1) / p.walk;
  int cb;
  if constexpr (MODE == ROWS_DENSE) {
    const int id = xcd_run((int)blockIdx.x, (int)gridDim.x), walk = id / p.row_blocks;
    cb = walk * p.walk;
    w.row0 = (id - walk * p.row_blocks) * Wave::B;
    w.rows = p.M - w.row0 < Wave::B ? p.M - w.row0 : Wave::B;
  } else {
    const int block = (int)blockIdx.x / walks;
    cb = ((int)blockIdx.x - block * walks) * p.walk;
    if (!w.take_block(block)) return;
  }
  const int tiles = p.col_blocks - cb < p.walk ? p.col_blocks - cb : p.walk;
  typename Wave::Weights wf[2][NX];
  typename Wave::Rows xf[NX];
  const int last_step = p.steps - 1;
  auto load = [&](int tile, auto set) {
    w.take_columns((cb + tile) * Wave::COLS);
    for_constants<NX>([&](auto i) {
      const int step = wave + decltype(i)::value * NW;
      w.template load_weights<true>(WT == WEIGHTS_F16 || step < last_step ? step : last_step, wf[decltype(set)::value][decltype(i)::value]);
    });
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  load(0, S0{});
  w.take_rows();
  for_constants<NX>([&](auto i) { w.template load_rows<true>(wave + decltype(i)::value * NW, xf[decltype(i)::value]); });
  auto tile = [&](int it, auto set) {
    floatx4 acc[R][1] = {};
    for_constants<NX>([&](auto i) {
      w.template multiply<true>(wave + decltype(i)::value * NW, wf[decltype(set)::value][decltype(i)::value], xf[decltype(i)::value], acc);
    });
    float* const mine = part + decltype(set)::value * PART;
    w.put_sums(mine, wave, acc);
    barrier_after_lds_writes();
    w.template finish<NW>(mine, (cb + it) * Wave::COLS, tid);
  };
  int it = 0;
  for (; it + 2 < tiles; it += 2) {
    load(it + 1, S1{});
    tile(it, S0{});
    load(it + 2, S0{});
    tile(it + 1, S1{});
  }
  if (it + 1 < tiles) {
    load(it + 1, S1{});
    tile(it, S0{});
    tile(it + 1, S1{});
  } else {
    tile(it, S0{});
  }
}

template <int WT, int MODE, bool GATED, int NG, int R, int NW, int NB>
hipError_t launch_few_rows(RowsParams p, hipStream_t stream) {
  auto kern = few_rows_kernel<WT, MODE, GATED, NG, R, NW, NB>;
  using Wave = RowsWave<WT, MODE, GATED, NG, 1, R>;
  constexpr int LDS_BYTES = NW * R * 64 * 16;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, LDS_BYTES); e != hipSuccess) return e;
  p.col_blocks = ((GATED ? p.hidden : p.N) + Wave::COLS - 1) / Wave::COLS;
  p.row_blocks = row_blocks<Wave::B>(p, MODE);
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * p.col_blocks), dim3(64 * NW), LDS_BYTES, stream, p);
  return hipGetLastError();
}
template <int WT, int MODE, bool GATED, int NG, int R, int NW, int NX>
hipError_t launch_few_rows_walk(RowsParams p, hipStream_t stream) {
  auto kern = few_rows_walk_kernel<WT, MODE, GATED, NG, R, NW, NX>;
  using Wave = RowsWave<WT, MODE, GATED, NG, 1, R>;
  constexpr int LDS_BYTES = 2 * NW * R * 64 * 16;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, LDS_BYTES); e != hipSuccess) return e;
  p.col_blocks = ((GATED ? p.hidden : p.N) + Wave::COLS - 1) / Wave::COLS;
  p.row_blocks = row_blocks<Wave::B>(p, MODE);
  // As many walks as the compute units hold at once (two workgroups each).  Routed lists: four times as many, since part of the row
  // blocks that are counted here do not exist (29 tokens to 8 of 128 experts, 2048 x 768 in 4 bits: 112 us so, 96, 92 and 100 with
  // 2, 4 and 8 times).
  const int64_t tiles = (int64_t)p.row_blocks * p.col_blocks, want = 512 * (MODE == ROWS_DENSE ? 1 : 4);
  const int64_t walk = (tiles + want - 1) / want;
  p.walk = (int)(walk < p.col_blocks ? walk : p.col_blocks);
  const int walks = (p.col_blocks + p.walk - 1) / p.walk;
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * walks), dim3(64 * NW), LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
