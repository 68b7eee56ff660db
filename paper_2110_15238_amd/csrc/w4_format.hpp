// Weights held in 4 bits: W[n][k] = s[n][k / G] * (q[n][k] - z[n][k / G]), q and z in 0 .. 15, G = 32, 64 or 128.
//
// The packed form is laid out once, for the matrix core: a block is 16 rows x 128 columns, 1024 bytes, and lane l of a
// wave reads its 16 bytes as one load: row l % 16, and in word s (0 .. 3) the columns 32 s + 8 (l / 16) .. + 7, which is
// the operand of the s-th v_mfma_f32_16x16x32_f16 of the block.  Within a word the eight values lie so that a mask leaves
// two of them where the mantissas of two halves are (nibbles 0 and 4: columns 0 and 1; 1 and 5: 2 and 3; 2 and 6: 4 and 5; 3
// and 7: 6 and 7).  Rows beyond N and columns beyond K hold zeros.
//   weights  [count][tiles][steps][64 lanes][16 bytes]
//   scales   [count][tiles][steps][4 row quads][groups of a step][4 rows] halves: a quad is what a lane's accumulators need
//   zeros    [count][tiles][steps][16 rows][groups of a step] bytes: a lane's row for its operand
// tiles = ceil(N / 16), steps = ceil(K / 128).  Scales of rows and groups that do not exist are zero.
#pragma once
#include "bolt_device.hpp"

namespace bolt {

struct W4Format {
  int N, K, group, tiles, steps, ng;  // ng: groups of a step
  int64_t weight_bytes, scale_count;  // of one matrix; as many zero bytes as scales
  static constexpr int STEP = 128, BLOCK_BYTES = 1024;
  W4Format(int N_, int K_, int group_) : N(N_), K(K_), group(group_) {
    tiles = (N + 15) / 16;
    steps = (K + STEP - 1) / STEP;
    ng = STEP / group;
    weight_bytes = (int64_t)tiles * steps * BLOCK_BYTES;
    scale_count = (int64_t)tiles * steps * ng * 16;
  }
  __host__ __device__ int64_t scales_at(int count) const { return count * weight_bytes; }
  __host__ __device__ int64_t zeros_at(int count) const { return scales_at(count) + count * scale_count * 2; }
  int64_t bytes(int count) const { return zeros_at(count) + count * scale_count; }
};

// Largest scale (in absolute value) of which every multiple up to 15 is finite as a half: 15 * 4364 = 65460, and 15 * 4368 = 65520 rounds to
// infinity.
static constexpr float kW4MostScale = 4364.f;

// Eight values q - z as halves, exact: 0x6400 | q is 1024 + q and 0x6400 | q << 4 is 1024 + 16 q as a half; minus1 holds two
// halves -1024 - z, minus16 two halves -64 - z.  The empty asm keeps the constants in registers: as literals they would make two
// instructions of every (w & mask) | exponent.
__device__ __forceinline__ half8 w4_values(unsigned w, half2v minus1, half2v minus16) {
  const half2v sixteenth = {(half_t)0.0625f, (half_t)0.0625f};
  unsigned lo = 0x000f000fu, hi = 0x00f000f0u, exponent = 0x64006400u;
#if defined(__HIP_DEVICE_COMPILE__)
  asm("" : "+s"(lo));
  asm("" : "+s"(hi));
  asm("" : "+v"(exponent));
#endif
  const unsigned v = w >> 8;
  const half2v a = __builtin_bit_cast(half2v, (w & lo) | exponent) + minus1;
  const half2v b = __builtin_elementwise_fma(__builtin_bit_cast(half2v, (w & hi) | exponent), sixteenth, minus16);
  const half2v c = __builtin_bit_cast(half2v, (v & lo) | exponent) + minus1;
  const half2v d = __builtin_elementwise_fma(__builtin_bit_cast(half2v, (v & hi) | exponent), sixteenth, minus16);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The two constants for a zero point: -1024 - z is 0xe400 + z as a half, -64 - z is 0xd400 + 16 z.
__device__ __forceinline__ half2v w4_minus1(unsigned z) { return __builtin_bit_cast(half2v, 0xe400e400u + z * 0x00010001u); }
__device__ __forceinline__ half2v w4_minus16(unsigned z) { return __builtin_bit_cast(half2v, 0xd400d400u + z * 0x00100010u); }

}  // namespace bolt
