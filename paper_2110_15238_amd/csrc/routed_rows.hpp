// What the products over routed lists share: where rows come from and go to, the experts' blocks of rows, SiLU.
#pragma once
#include "fprop_dma_kernel.hpp"

namespace bolt {

enum { WEIGHTS_F16 = 0, WEIGHTS_W4 = 1 };
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

// Direct-to-LDS loads from any address: lane l's 16 (4) bytes go to `to` + 16 l (4 l).
__device__ __forceinline__ void lds_load16(const void* from, half_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, BOLT_LDS_PTR(to), 16, 0, 0);
}
__device__ __forceinline__ void lds_load4(const void* from, half_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, BOLT_LDS_PTR(to), 4, 0, 0);
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
