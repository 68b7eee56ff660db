// Products of a few rows with a large weight matrix [N][K]: the linear layers of a handful of tokens, with weights in 4 bits
// or in FP16, for one matrix or for the experts that a router chose.
//
// With M rows every weight is used M times, so up to about 64 rows the product is bound by reading the weights once.  A
// workgroup owns 16 R weight rows and up to 16 MB activation rows; its NW waves take the reduction in turns, step by step (a
// wave's step is 128 columns of 4-bit weights or 64 of FP16 ones), so that the workgroup reads its weights as one stream.  Weights go
// straight from memory to registers, NB steps ahead, in the operand order of v_mfma_f32_16x16x32_f16, whose 16 columns are the
// activation rows; nothing passes through LDS but the waves' partial sums, which are added in a fixed order.
//   4-bit weights: an operand is q - z, exact in a half; the sum over a group of columns comes out of the matrix core in FP32
//   and is scaled there, so neither scale nor zero point costs accuracy.  (Nine vector instructions make eight operands.)
//   Activation rows beyond the last repeat the last: their columns of the result are not stored.  Columns beyond K are zero on
//   both sides.
#pragma once
#include "fprop_dma_kernel.hpp"
#include "w4_format.hpp"

namespace bolt {

enum { WEIGHTS_F16 = 0, WEIGHTS_W4 = 1 };
// Where a product's rows come from and go to.
//   DENSE: row m of x, to row m of y.
//   UP:    rows of the routed list: token order[i] / top_k of x, to row i of y (the list's order).
//   DOWN:  row i of x, times the slot's weight, to row order[i] of y.
enum { ROWS_DENSE = 0, ROWS_UP = 1, ROWS_DOWN = 2 };

enum { ACT_SILU = 5 };
// v / (1 + exp(-v)) with the hardware exp2 and reciprocal units: relative error about 1e-6 from the argument's rounding, far under a half's.
__device__ __forceinline__ float silu_fast(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504088896340736f));
}
__device__ __forceinline__ float apply_act_or_silu(float v, int act) { return act == ACT_SILU ? silu_fast(v) : apply_act(v, act); }

struct RowsParams {
  const half_t* x;
  int64_t ldx;
  const unsigned char* w;      // FP16: [count][N][K]; 4 bits: the packed weights
  int64_t w_stride;            // bytes from one expert's to the next's
  const half_t* scales;        // 4 bits only
  const unsigned char* zeros;
  int64_t scale_stride;        // scales from one expert's to the next's
  const half_t* bias;          // [count][N]; eight zeros if there is none
  int bias_on;
  half_t* y;
  int64_t ldy;
  int M, N, K, steps;          // N: weight rows; steps of the reduction, the last may be ragged
  int hidden;                  // gated: weight rows [0, hidden) are the gate, [hidden, 2 hidden) the values
  float alpha, beta;
  int act;
  const int* offsets;          // routed lists, see bolt_moe_route
  const int* order;
  const float* slot_weights;
  int experts, top_k;
  int row_blocks, col_blocks;  // grid: row_blocks * col_blocks workgroups
};

// The want-th block of B list rows, blocks counted expert by expert: its expert, first list row and row count.  Every lane of
// a wave calls it; lane l adds up the blocks of `per` neighbouring experts.  False beyond the last block.
template <int B>
__device__ __forceinline__ bool find_row_block(const int* __restrict__ offsets, int experts, int want, int lane, int* expert, int* row0, int* rows) {
  const int per = (experts + 63) >> 6, first = lane * per;
  int mine = 0;
  int at = first <= experts ? offsets[first] : 0;
  for (int i = 0; i < per; ++i) {
    if (first + i < experts) {
      const int next = offsets[first + i + 1];
      mine += (next - at + B - 1) / B;
      at = next;
    }
  }
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  const unsigned long long past = __ballot(upto > want);
  if (past == 0) return false;
  const int owner = __builtin_ctzll(past);
  int left = want - __builtin_amdgcn_readlane(upto - mine, owner);
  int e = owner * per;
  while (true) {  // ends: the owner's experts hold more than `left` blocks
    const int lo = offsets[e], n = offsets[e + 1] - lo, blocks = (n + B - 1) / B;
    if (left < blocks) {
      *expert = e;
      *row0 = lo + left * B;
      *rows = n - left * B < B ? n - left * B : B;
      return true;
    }
    left -= blocks;
    ++e;
  }
}

template <int WT, int MODE, bool GATED, int NG, int MB, int R, int NW, int NB>
__global__ __launch_bounds__(64 * NW) void few_rows_kernel(const RowsParams p) {
  static_assert(!GATED || R % 2 == 0, "gated: tiles come in pairs");
  constexpr int KS = WT == WEIGHTS_W4 ? 4 : 2, STEP = 32 * KS;  // matrix instructions and columns of a step
  constexpr int MPG = KS / NG;                                  // matrix instructions of a group (4 bits)
  constexpr int B = 16 * MB, COLS = GATED ? 8 * R : 16 * R;     // rows and outputs of a workgroup
  extern __shared__ __attribute__((aligned(16))) float part[];  // [NW][R * MB][64 lanes][4]
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // Workgroups: the row blocks of one stretch of weights follow one another on one XCD (ids are dealt round-robin over 8), so the
  // weights come from memory once.  Routed lists: a row block is an expert's, so its stretches follow one another instead.
  int rb, cb, expert = 0, row0, rows;
  if constexpr (MODE == ROWS_DENSE) {
    const int total = (int)gridDim.x, xcd = (int)blockIdx.x & 7, per = total >> 3, rem = total & 7;
    const int id = xcd * per + (xcd < rem ? xcd : rem) + ((int)blockIdx.x >> 3);
    cb = id / p.row_blocks;
    rb = id - cb * p.row_blocks;
    row0 = rb * B;
    rows = p.M - row0 < B ? p.M - row0 : B;
  } else {
    rb = (int)blockIdx.x / p.col_blocks;
    cb = (int)blockIdx.x - rb * p.col_blocks;
    if (!find_row_block<B>(p.offsets, p.experts, rb, lane, &expert, &row0, &rows)) return;
    expert = __builtin_amdgcn_readfirstlane(expert);
    row0 = __builtin_amdgcn_readfirstlane(row0);
    rows = __builtin_amdgcn_readfirstlane(rows);
  }
  const int col0 = cb * COLS;

  // this lane's activation rows and weight rows
  const half_t* xrow[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int j = b * 16 + l16, row = row0 + (j < rows ? j : rows - 1);
    const int64_t from = MODE == ROWS_UP ? p.order[row] / p.top_k : row;
    xrow[b] = p.x + from * p.ldx + g * 8;
  }
  const unsigned char* const w = p.w + expert * p.w_stride;
  auto first_row = [&](int t) { return GATED ? (t & 1) * p.hidden + col0 + (t >> 1) * 16 : col0 + t * 16; };
  const int last_row = p.N - 1;
  const unsigned char* wrow[R];
  int64_t scale_at[R], zero_at[R];
#pragma unroll
  for (int t = 0; t < R; ++t) {
    int row = first_row(t) + l16;
    row = row < last_row ? row : last_row;
    if constexpr (WT == WEIGHTS_W4) {
      wrow[t] = w + (int64_t)(row >> 4) * p.steps * W4Format::BLOCK_BYTES + (g * 16 + (row & 15)) * 16;
      int quad = first_row(t) + g * 4;  // a multiple of 4, so the quad lies in one tile
      quad = quad < last_row ? quad : last_row & ~3;
      const int64_t base = expert * p.scale_stride;
      scale_at[t] = base + ((int64_t)(quad >> 4) * p.steps * 4 + ((quad & 15) >> 2)) * (NG * 4);
      zero_at[t] = base + ((int64_t)(row >> 4) * p.steps * 16 + (row & 15)) * NG;
    } else {
      wrow[t] = w + ((int64_t)row * p.K + g * 8) * 2;
    }
  }

  constexpr int WREGS = WT == WEIGHTS_W4 ? 1 : KS;  // 16-byte pieces of weights per tile and step
  uintx4 wf[NB][R][WREGS];
  half4 sc[NB][R][NG];
  unsigned zp[NB][R];
  half8 xf[NB][KS][MB];
  floatx4 acc[R][MB];
#pragma unroll
  for (int t = 0; t < R; ++t)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[t][b] = floatx4{0.f, 0.f, 0.f, 0.f};

  // Step `step` into register set S; RAGGED: columns at or beyond K are zero (4-bit weights need no such check, zero activations do).
  auto load = [&](int step, auto sc_, auto ragged) {
    constexpr int S = decltype(sc_)::value;
    constexpr bool RAGGED = decltype(ragged)::value;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      if constexpr (WT == WEIGHTS_W4) {
        wf[S][t][0] = *(const uintx4*)(wrow[t] + (int64_t)step * W4Format::BLOCK_BYTES);
        const half_t* s = p.scales + scale_at[t] + (int64_t)step * (NG * 16);
#pragma unroll
        for (int i = 0; i < NG; ++i) sc[S][t][i] = *(const half4*)(s + i * 4);
        const unsigned char* z = p.zeros + zero_at[t] + (int64_t)step * (NG * 16);
        if constexpr (NG == 4) zp[S][t] = *(const unsigned*)z;
        else if constexpr (NG == 2) zp[S][t] = *(const unsigned short*)z;
        else zp[S][t] = *z;
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const bool in = !RAGGED || step * STEP + s * 32 + g * 8 < p.K;
          wf[S][t][s] = in ? *(const uintx4*)(wrow[t] + ((int64_t)step * STEP + s * 32) * 2) : uintx4{0, 0, 0, 0};
        }
      }
    }
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const bool in = !RAGGED || step * STEP + s * 32 + g * 8 < p.K;
        xf[S][s][b] = in ? *(const half8*)(xrow[b] + (int64_t)step * STEP + s * 32) : half8{0, 0, 0, 0, 0, 0, 0, 0};
      }
  };
  auto multiply = [&](auto sc_) {
    constexpr int S = decltype(sc_)::value;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      if constexpr (WT == WEIGHTS_W4) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const unsigned z = NG == 1 ? zp[S][t] : (zp[S][t] >> (i * 8)) & 0xffu;
          const half2v m1 = w4_minus1(z), m16 = w4_minus16(z);
          floatx4 sum[MB];
#pragma unroll
          for (int b = 0; b < MB; ++b) sum[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = i * MPG; s < (i + 1) * MPG; ++s) {
            const half8 a = w4_values(wf[S][t][0][s], m1, m16);
#pragma unroll
            for (int b = 0; b < MB; ++b) sum[b] = mfma_16x16x32(a, xf[S][s][b], sum[b]);
          }
#pragma unroll
          for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][b][e] += (float)sc[S][t][i][e] * sum[b][e];
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int b = 0; b < MB; ++b) acc[t][b] = mfma_16x16x32(__builtin_bit_cast(half8, wf[S][t][s]), xf[S][s][b], acc[t][b]);
      }
    }
  };

  // This wave's steps: wave, wave + NW, ...; a ragged last step is one wave's, behind its whole ones.
  const int whole = p.K / STEP;
  const int n = whole > wave ? (whole - wave + NW - 1) / NW : 0;
  auto step_of = [&](int i) { return wave + i * NW; };
  using False = std::integral_constant<bool, false>;
  using True = std::integral_constant<bool, true>;
  if (n >= NB) {
    for_constants<NB>([&](auto b) { load(step_of(decltype(b)::value), b, False{}); });
    int c = 0;
    for (; c + 2 * NB <= n; c += NB)
      for_constants<NB>([&](auto b) {
        multiply(b);
        load(step_of(c + NB + decltype(b)::value), b, False{});
      });
    const int left = n - c - NB;  // steps not requested yet, fewer than NB
    for_constants<NB>([&](auto b) {
      multiply(b);
      if (decltype(b)::value < left) load(step_of(c + NB + decltype(b)::value), b, False{});
    });
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < left) multiply(b);
    });
  } else {
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < n) load(step_of(decltype(b)::value), b, False{});
    });
    for_constants<NB>([&](auto b) {
      if (decltype(b)::value < n) multiply(b);
    });
  }
  if (whole < p.steps && whole % NW == wave) {
    load(whole, std::integral_constant<int, 0>{}, True{});
    multiply(std::integral_constant<int, 0>{});
  }

  // the waves' sums, in the order of the waves
#pragma unroll
  for (int t = 0; t < R; ++t)
#pragma unroll
    for (int b = 0; b < MB; ++b) *(floatx4*)(part + ((wave * R * MB + t * MB + b) * 64 + lane) * 4) = acc[t][b];
  __syncthreads();
  auto sum_of = [&](int t, int b, int at) {
    floatx4 v = *(const floatx4*)(part + ((t * MB + b) * 64 + at) * 4);
#pragma unroll
    for (int k = 1; k < NW; ++k) v += *(const floatx4*)(part + ((k * R * MB + t * MB + b) * 64 + at) * 4);
    return v;
  };
  auto with_bias = [&](floatx4 v, int n_) {  // n_: weight row of the quad
    const half4 hb = *(const half4*)(p.bias + (expert * (int64_t)p.N + n_) * p.bias_on);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p.alpha * v[e] + p.beta * (float)hb[e];
    return v;
  };
  constexpr int OUT = (GATED ? R / 2 : R) * MB;
  for (int i = tid; i < OUT * 64; i += 64 * NW) {
    const int at = i & 63, b = (i >> 6) % MB, t = (i >> 6) / MB;
    const int j = b * 16 + (at & 15), col = col0 + t * 16 + (at >> 4) * 4;
    const int outputs = GATED ? p.hidden : p.N;
    if (j >= rows || col >= outputs) continue;
    floatx4 v;
    if constexpr (GATED) {
      v = with_bias(sum_of(2 * t, b, at), col);
      const floatx4 u = with_bias(sum_of(2 * t + 1, b, at), p.hidden + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = apply_act_or_silu(v[e], p.act) * u[e];
    } else {
      v = with_bias(sum_of(t, b, at), col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = apply_act_or_silu(v[e], p.act);
    }
    int64_t to = row0 + j;
    if constexpr (MODE == ROWS_DOWN) {
      to = p.order[row0 + j];
      const float s = p.slot_weights[to];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= s;
    }
    half4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
    *(half4*)(p.y + to * p.ldy + col) = o;
  }
}

template <int WT, int MODE, bool GATED, int NG, int MB, int R, int NW, int NB>
hipError_t launch_few_rows(RowsParams p, hipStream_t stream) {
  auto kern = few_rows_kernel<WT, MODE, GATED, NG, MB, R, NW, NB>;
  constexpr int LDS_BYTES = NW * R * MB * 64 * 16, COLS = GATED ? 8 * R : 16 * R;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, LDS_BYTES); e != hipSuccess) return e;
  p.col_blocks = ((GATED ? p.hidden : p.N) + COLS - 1) / COLS;
  // an expert's last block of rows may be short: at most one such block for each expert that has rows
  p.row_blocks = MODE == ROWS_DENSE ? (p.M + 16 * MB - 1) / (16 * MB) : p.M / (16 * MB) + (p.M < p.experts ? p.M : p.experts);
  hipLaunchKernelGGL(kern, dim3(p.row_blocks * p.col_blocks), dim3(64 * NW), LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
