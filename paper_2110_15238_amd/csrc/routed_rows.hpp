// What the products over routed lists share: where rows come from and go to, the experts' blocks of rows, SiLU.
#pragma once
#include <type_traits>

#include "fprop_dma_kernel.hpp"

namespace bolt {

// WEIGHTS_F8: weights and activations in E4M3.  They move as the halves that two of them fill, so lengths of rows and reductions count those
// pairs; two pieces of an FP16 operand make one of v_mfma_f32_16x16x128_f8f6f4.  (A named type: it is part of kernels' names, and one without a name is
// counted differently by the compiler's host and device passes.)
enum WeightKind { WEIGHTS_F16 = 0, WEIGHTS_W4 = 1, WEIGHTS_F8 = 2 };
// Where a product's rows come from and go to.
//   DENSE: row m of x, to row m of y.
//   UP:    rows of the routed list: token order[i] / top_k of x, to row i of y (the list's order).
//   DOWN:  row i of x, to row order[i] of y, in FP32: the rows of a token's slots are still to be weighted and added.
enum { ROWS_DENSE = 0, ROWS_UP = 1, ROWS_DOWN = 2 };

enum { ACT_SILU = 5 };
// v / (1 + exp(-v)) with the hardware exp2 and reciprocal units: relative error about 1e-6 from the argument's rounding, far under a half's.
__device__ __forceinline__ float silu_fast(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504088896340736f));
}
// A quad through the activation: one wave-uniform switch for four values.
__device__ __forceinline__ floatx4 apply_act4(floatx4 v, int act) {
  if (act == ACT_SILU) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = silu_fast(v[e]);
  } else if (act > ACT_RELU) {
    v = apply_act_slow4_inline(v, act);
  } else {
    const float lo = relu_bound(act);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = at_least(v[e], lo);
  }
  return v;
}

struct RowsParams {
  const half_t* x;
  int64_t ldx;
  const unsigned char* w;      // FP16: [count][N][K]; 4 bits: the packed weights
  int64_t w_stride;            // bytes from one expert's to the next's
  const half_t* scales;        // 4 bits only
  const unsigned char* zeros;
  int64_t scale_stride;        // scales from one expert's to the next's
  const half_t* none;          // eight zeros
  const half_t* bias;          // [count][N]; `none` if there is none
  int bias_on;
  void* y;                     // halves; DOWN: floats
  int64_t ldy;
  int M, N, K, steps;          // N: weight rows; steps of the reduction, the last may be ragged
  int hidden;                  // gated: weight rows [0, hidden) are the gate, [hidden, 2 hidden) the values
  float alpha, beta;
  int act;
  const int* offsets;          // routed lists, see bolt_moe_route
  const int* order;
  int experts, top_k;
  int row_blocks, col_blocks;
  const half_t* unpacked;      // [N][K], for the marks of w4_unpack_kernel
  int walk;                    // tiles of columns that a workgroup walks over
};
// What linear layers of E4M3 operands, and those whose rows have adapters, take besides.  (Apart: 90 bytes more of arguments cost the calls of a few us that
// have no use for them 0.1 to 0.2 us.)
struct LayerParams : RowsParams {
  const float* x_scales;       // E4M3: of the rows of x and of w, or null
  const float* w_scales;
  const float* add;            // [M][N], added to the sums before alpha (the adapters' share, where it goes through memory), or null
  // low-rank adapters (linear layers)
  const int* adapter;          // of each row; none below zero and from `adapters` on
  const void* low;             // scale * x . down^T of each row's adapter: [M][rank] halves, or [low_parts][M][rank] floats to be added up
  const half_t* up;            // [adapters][N][rank]
  int adapters, rank, low_parts;
};

// The experts' row blocks: each expert's list rows in blocks of B, counted expert by expert.
struct RowBlock {
  int expert, lo, n;  // the expert's first list row and its rows
  int first, count;   // number of the expert's first block, and of its blocks
};
// Blocks of the experts `per` l .. `per` (l + 1) - 1 (mine) and of those up to and with lane l (upto).
struct BlockCounts {
  int per, mine, upto;
  __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(upto, 63); }
};
template <int B>
__device__ __forceinline__ BlockCounts count_row_blocks(const int* __restrict__ offsets, int experts, int lane) {
  BlockCounts c;
  c.per = (experts + 63) >> 6;
  c.mine = 0;
  const int first = lane * c.per;
  int at = first <= experts ? offsets[first] : 0;
  for (int i = 0; i < c.per; ++i) {
    if (first + i < experts) {
      const int next = offsets[first + i + 1];
      c.mine += (next - at + B - 1) / B;
      at = next;
    }
  }
  c.upto = c.mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(c.upto, d);
    if (lane >= d) c.upto += o;
  }
  return c;
}
// Block `want`; false beyond the last.  Every lane of the wave calls it with the same number.
template <int B>
__device__ __forceinline__ bool find_row_block(const int* __restrict__ offsets, const BlockCounts& c, int want, RowBlock* out) {
  const unsigned long long past = __ballot(c.upto > want);
  if (past == 0) return false;
  const int owner = __builtin_ctzll(past);
  int first = __builtin_amdgcn_readlane(c.upto - c.mine, owner);
  int e = owner * c.per;
  while (true) {  // ends: the owner's experts hold block `want`
    const int lo = offsets[e], n = offsets[e + 1] - lo, blocks = (n + B - 1) / B;
    if (want < first + blocks) {
      out->expert = __builtin_amdgcn_readfirstlane(e);
      out->lo = __builtin_amdgcn_readfirstlane(lo);
      out->n = __builtin_amdgcn_readfirstlane(n);
      out->first = __builtin_amdgcn_readfirstlane(first);
      out->count = __builtin_amdgcn_readfirstlane(blocks);
      return true;
    }
    first += blocks;
    ++e;
  }
}

// The adapter of a row, -1 for none; `exists`: the row does.
__device__ __forceinline__ int row_adapter(const int* ids, int adapters, int row, bool exists) {
  const int id = exists ? ids[row] : -1;
  return id >= 0 && id < adapters ? id : -1;
}

// Eight values from `at` on of low, as the FP16 operand of the product with up: halves where low is one part, else the sums of `parts` floats that
// are `part` apart, all asked for at once.
constexpr int kMostLowParts = 4;
__device__ __forceinline__ half8 low_operand(const void* low, int64_t at, int parts, int64_t part) {
  if (parts == 1) return *(const half8*)((const half_t*)low + at);
  const float* const sums = (const float*)low + at;
  floatx4 v[kMostLowParts][2];
#pragma unroll
  for (int i = 0; i < kMostLowParts; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) v[i][h] = *(const floatx4*)(sums + (i < parts ? i : 0) * part + 4 * h);
  floatx4 a = v[0][0], b = v[0][1];
#pragma unroll
  for (int i = 1; i < kMostLowParts; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = i < parts ? a[e] + v[i][0][e] : a[e];
      b[e] = i < parts ? b[e] + v[i][1][e] : b[e];
    }
  half8 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (half_t)a[e], o[4 + e] = (half_t)b[e];
  return o;
}

// The scales of four columns.
__device__ __forceinline__ floatx4 column_scales(const LayerParams& p, int n) {
  return p.w_scales ? *(const floatx4*)(p.w_scales + n) : floatx4{1.f, 1.f, 1.f, 1.f};
}

// Where a kernel of tiles takes the adapters' share from: nowhere, LayerParams::add, or low and up (computed in the tile).
enum LayerShare { ADD_NOTHING = 0, FROM_ADD = 1, FROM_ADAPTERS = 2 };

// Direct-to-LDS loads from any address: lane l's 16 (4) bytes go to `to` + 16 l (4 l).
__device__ __forceinline__ void lds_load16(const void* from, half_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, BOLT_LDS_PTR(to), 16, 0, 0);
}
__device__ __forceinline__ void lds_load4(const void* from, half_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, BOLT_LDS_PTR(to), 4, 0, 0);
}

// Waits of a wave that stages for itself: its direct-to-LDS loads but for the VM newest have landed; its LDS reads have returned.
template <int VM>
__device__ __forceinline__ void wave_waits_for_loads() {
  static_assert(VM >= 0 && VM < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt((VM & 0xF) | ((VM >> 4) << 14) | 0x0F70);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wave_waits_for_reads() {
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}

// Workgroup ids are dealt round-robin over 8 XCDs: every XCD gets a contiguous run of the `total` tiles.
__device__ __forceinline__ int xcd_run(int id, int total) {
  const int xcd = id & 7, per = total >> 3, rem = total & 7;
  return xcd * per + (xcd < rem ? xcd : rem) + (id >> 3);
}

// How many row blocks there can be.  An expert's last one may be short: at most one such block for each expert that has rows.
template <int B>
inline int row_blocks(const RowsParams& p, int mode) {
  return mode == ROWS_DENSE ? (p.M + B - 1) / B : p.M / B + (p.M < p.experts ? p.M : p.experts);
}

}  // namespace bolt
