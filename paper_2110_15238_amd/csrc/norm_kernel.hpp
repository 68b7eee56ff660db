// Root-mean-square norm of rows, with the residual's addition in front and rows in FP16 or in 8 bits behind it:
//   v = x + residual;  n = v / sqrt(mean(v^2) + eps) * (offset + weight);  scale = max |n| / 448;  q = n / scale as E4M3.
//
// One pass: a row is read once into registers, by one wave or one workgroup, and everything leaves from there.  The factor
// 1 / sqrt(...) is one positive number per row, so the largest |n| is that number times the largest |v * (offset + weight)|: the sum of the
// squares and the largest value come out of one reduction, with one barrier.
// Bound by memory where there are many rows, by the launch, one round trip and the reduction where there are few: 32768 x 4096 with the residual, FP16,
// 181 us (5.9 TB/s; a large copy moves 5.0), 4099 x 5120 to 8 bits 30.7 us (4.8 TB/s), one row of 4096 2.9 us on the GPU.
#pragma once
#include "bolt_device.hpp"

namespace bolt {

constexpr float kMostE4m3 = 448.f;  // the largest finite value

struct NormParams {
  const half_t* x;
  const half_t* residual;  // or null
  const half_t* weight;    // or null: quantisation alone
  half_t* sum;             // v in FP16, or null
  half_t* y;               // n in FP16, or null
  unsigned char* q;        // n in E4M3, or null
  float* scales;           // of q
  int64_t ldx, ldr, lds, ldy, ldq;
  int rows, width;
  float eps, offset;
};

// The reduction of a row: the sum of squares, and the largest magnitude as its bits (as integers a NaN is larger than an infinity, which is
// larger than every number, so neither gets lost).
struct RowStats {
  float squares;
  unsigned largest;
};
__device__ __forceinline__ RowStats merge(RowStats a, RowStats b) {
  return {a.squares + b.squares, a.largest > b.largest ? a.largest : b.largest};
}
__device__ __forceinline__ RowStats merge_lanes(RowStats s) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) s = merge(s, {__shfl_xor(s.squares, d), (unsigned)__shfl_xor((int)s.largest, d)});
  return s;
}

// WAVES waves share a row (1: every wave of the workgroup of four has a row of its own), V pieces of eight values a lane.
// NORM: false leaves the rows as they are (quantisation alone).
template <int WAVES, int V, bool NORM>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_kernel(const NormParams p) {
  constexpr int LANES = 64 * WAVES, PER = WAVES == 1 ? 4 : 1;  // lanes of a row, rows at a time
  __shared__ RowStats parts[2][WAVES];
  const int lane = threadIdx.x % LANES, wave = lane >> 6;
  const int chunks = p.width >> 3;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES; row < p.rows; row += (int64_t)gridDim.x * PER, turn ^= 1) {
    // (pieces beyond the row are read as its last one and count as zero)
    half8 in[V], add[V], gain[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = i * LANES + lane, at = (c < chunks ? c : chunks - 1) * 8;
      in[i] = *(const half8*)(p.x + row * p.ldx + at);
      if (NORM) gain[i] = *(const half8*)(p.weight + at);
      if (p.residual) add[i] = *(const half8*)(p.residual + row * p.ldr + at);
    }
    float v[V][8];
    RowStats s = {0.f, 0u};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool on = i * LANES + lane < chunks;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f = (float)in[i][e];
        if (p.residual) f += (float)add[i][e];
        v[i][e] = on ? f : 0.f;
        if (NORM) s.squares += v[i][e] * v[i][e];
      }
      if (p.sum && on) {
        half8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (half_t)v[i][e];
        *(half8*)(p.sum + row * p.lds + (i * LANES + lane) * 8) = o;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (NORM) v[i][e] *= p.offset + (float)gain[i][e];
        const unsigned bits = on ? __builtin_bit_cast(unsigned, v[i][e]) & 0x7fffffffu : 0u;
        s.largest = s.largest > bits ? s.largest : bits;
      }
    }
    s = merge_lanes(s);
    if constexpr (WAVES > 1) {
      // (two places, by turns: a wave that is a row ahead writes where nobody reads any more)
      if ((lane & 63) == 0) parts[turn][wave] = s;
      __syncthreads();
      s = parts[turn][0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s = merge(s, parts[turn][w]);
    }
    const float factor = NORM ? 1.f / sqrtf(s.squares / (float)p.width + p.eps) : 1.f;
    // A row of zeros, or one so small that 448 over it is no number any more, is zero; one that holds an infinity or a NaN has no number for
    // its scale either, so that none of its values is one.
    const float largest = __builtin_bit_cast(float, s.largest) * factor;
    const float to_q = largest < 0x1p-118f ? 0.f : kMostE4m3 / largest;
    if (p.q && lane == 0) p.scales[row] = largest / kMostE4m3;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = i * LANES + lane;
      if (c >= chunks) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= factor;
      if (p.y) {
        half8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (half_t)v[i][e];
        *(half8*)(p.y + row * p.ldy + c * 8) = o;
      }
      if (p.q) {
        // (no value is more than a few units in the last place of FP32 past 448, which rounds to 448)
        int out[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          out[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * h] * to_q, v[i][4 * h + 1] * to_q, out[h], false);
          out[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * h + 2] * to_q, v[i][4 * h + 3] * to_q, out[h], true);
        }
        *(int2*)(p.q + row * p.ldq + c * 8) = int2{out[0], out[1]};
      }
    }
  }
}

}  // namespace bolt
