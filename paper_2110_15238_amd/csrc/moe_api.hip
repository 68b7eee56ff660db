// C ABI of the operators of language models: linear layers with weights in 4 bits, routing to experts, the experts' products.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/bolt.h"
#include "few_rows_instances.hpp"
#include "w4_format.hpp"
#include "moe_route_kernel.hpp"

namespace bolt {
namespace {

// Packing, once for a program's weights: one thread a 16-byte piece, then one a scale and its zero point.
__global__ __launch_bounds__(256) void w4_pack_kernel(const unsigned char* q, const half_t* scales, const unsigned char* zeros, unsigned char* packed,
                                                      int count, const W4Format f) {
  const int64_t pieces = (int64_t)count * f.weight_bytes / 16, numbers = (int64_t)count * f.scale_count;
  const int groups = (f.K + f.group - 1) / f.group;
  half_t* const scales_out = (half_t*)(packed + f.scales_at(count));
  unsigned char* const zeros_out = packed + f.zeros_at(count);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces + numbers; i += (int64_t)gridDim.x * 256) {
    if (i < pieces) {
      const int lane = (int)(i & 63);
      const int64_t block = i >> 6;
      const int step = (int)(block % f.steps);
      const int64_t tile = block / f.steps;
      const int row = (int)(tile % f.tiles) * 16 + (lane & 15);
      const int64_t matrix = tile / f.tiles;
      uintx4 out = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = step * W4Format::STEP + s * 32 + (lane >> 4) * 8;
        if (row >= f.N || k >= f.K) continue;
        const unsigned v = *(const unsigned*)(q + ((matrix * f.N + row) * f.K + k) / 2);  // (K % 8 == 0)
        // columns 0 1 2 3 4 5 6 7 -> nibbles 0 4 1 5 2 6 3 7
        out[s] = (v & 0xfu) | (v >> 4 & 0xfu) << 16 | (v >> 8 & 0xfu) << 4 | (v >> 12 & 0xfu) << 20 | (v >> 16 & 0xfu) << 8 |
                 (v >> 20 & 0xfu) << 24 | (v >> 24 & 0xfu) << 12 | (v >> 28) << 28;
      }
      *(uintx4*)(packed + i * 16) = out;
    } else {
      const int64_t n = i - pieces;  // in the order of the zeros: [tile][step][16 rows][ng]
      const int j = (int)(n % f.ng), r = (int)(n / f.ng % 16);
      const int64_t block = n / (f.ng * 16);
      const int step = (int)(block % f.steps);
      const int64_t tile = block / f.steps, matrix = tile / f.tiles;
      const int row = (int)(tile % f.tiles) * 16 + r, group = step * f.ng + j;
      const bool in = row < f.N && group < groups;
      const int64_t from = (matrix * f.N + row) * groups + group;
      scales_out[(block * 4 + (r >> 2)) * f.ng * 4 + j * 4 + (r & 3)] = in ? scales[from] : (half_t)0.f;
      zeros_out[n] = in && zeros ? zeros[from] & 15 : 8;
    }
  }
}


// A packed 4-bit matrix as [N][K] halves, scale * (q - z) rounded once: for problems of so many rows that the matrix cores bound
// them, where decoding once and running on operands in FP16 costs less than decoding in every tile.  The rounding is that of a weight
// held in FP16.  One thread for 16 packed bytes.
// A weight beyond a half's range (a scale above kW4MostScale) has no such form: the first element of a tile of 16 rows with one is left
// a NaN, which no other tile has there, and launch_shared_rows_w4_marked computes those tiles' outputs from the packed weights.
template <int NG>
__global__ __launch_bounds__(256) void w4_unpack_kernel(const unsigned char* packed, half_t* out, const W4Format f) {
  const half_t* const scales = (const half_t*)(packed + f.scales_at(1));
  const unsigned char* const zeros = packed + f.zeros_at(1);
  const int64_t pieces = f.weight_bytes / 16;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
    const int lane = (int)(i & 63), g = lane >> 4, r = lane & 15;
    const int64_t block = i >> 6, tile = block / f.steps;
    const int step = (int)(block - tile * f.steps), row = (int)tile * 16 + r;
    bool marked = false;
    if (step == 0) {  // (the same for all lanes of a wave, which share the tile's scales)
      const half8* const all = (const half8*)(scales + tile * f.steps * (16 * NG));
      for (int j = lane; j < f.steps * (2 * NG); j += 64) {
        const half8 v = all[j];
#pragma unroll
        for (int e = 0; e < 8; ++e) marked |= !(__builtin_fabsf((float)v[e]) <= kW4MostScale);
      }
      marked = __any(marked) && lane == 0;
    }
    if (row >= f.N) continue;
    const uintx4 w = *(const uintx4*)(packed + i * 16);
    half_t* const to = out + (int64_t)row * f.K;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int k = step * W4Format::STEP + s * 32 + g * 8, j = s * NG / 4;
      if (k >= f.K) continue;
      const unsigned z = zeros[(block * 16 + r) * NG + j];
      const half_t scale = scales[((block * 4 + (r >> 2)) * NG + j) * 4 + (r & 3)];
      half8 v = w4_values(w[s], w4_minus1(z), w4_minus16(z)) * scale;
      if (s == 0 && marked) v[0] = __builtin_bit_cast(half_t, (unsigned short)0x7e00);
      *(half8*)(to + k) = v;
    }
  }
}
hipError_t launch_w4_unpack(const void* packed, half_t* out, const W4Format& f, hipStream_t stream) {
  const int64_t pieces = f.weight_bytes / 16;
  const dim3 grid((unsigned)std::min<int64_t>((pieces + 255) / 256, 256 * 32));
  auto kern = f.ng == 1 ? w4_unpack_kernel<1> : f.ng == 2 ? w4_unpack_kernel<2> : w4_unpack_kernel<4>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, (const unsigned char*)packed, out, f);
  return hipGetLastError();
}

// y[t] = sum of weight times row over the token's slots, in FP32, in the order of the slots: one thread for eight columns, the rows of U
// slots requested together: few tokens wait for one round trip after the other (1 token, 8 slots, 2048 wide: 5.9 us with U = 1, 3.8 with 4),
// many are faster one row at a time (8192 tokens, 6 slots: 78 against 86).  Slots without an expert have no row: what lies there is
// read and not used.
template <int U>
__global__ __launch_bounds__(256) void moe_combine_kernel(const float* rows, const int* ids, const float* weights, half_t* y, int tokens, int top_k,
                                                          int width, int64_t ldy) {
  const int chunks = width / 8;
  const int64_t total = (int64_t)tokens * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / chunks;
    const int c = (int)(i - t * chunks) * 8;
    const int64_t first = t * top_k;
    floatx4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    for (int j0 = 0; j0 < top_k; j0 += U) {
      floatx4 a[U], b[U];
      float w[U];
      bool on[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int64_t slot = first + (j0 + j < top_k ? j0 + j : top_k - 1);
        const float* row = rows + slot * width + c;
        a[j] = *(const floatx4*)row;
        b[j] = *(const floatx4*)(row + 4);
        w[j] = weights[slot];
        on[j] = ids[slot] >= 0 && j0 + j < top_k;
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = on[j] ? lo[e] + w[j] * a[j][e] : lo[e];
          hi[e] = on[j] ? hi[e] + w[j] * b[j][e] : hi[e];
        }
    }
    half8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (half_t)lo[e], o[4 + e] = (half_t)hi[e];
    *(half8*)(y + t * ldy + c) = o;
  }
}

__device__ __attribute__((aligned(16))) half_t g_no_bias[8];
const half_t* no_bias() {
  static PerDevice known;
  return (const half_t*)address_on_device(known, g_no_bias);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t blocks_of(int64_t v, int64_t by) { return (v + by - 1) / by; }
bool known_act(int a) { return a >= BOLT_ACT_NONE && a <= BOLT_ACT_SILU; }
bolt_status status_of(hipError_t e) { return e == hipSuccess ? BOLT_OK : BOLT_ERR_LAUNCH; }
constexpr int kMaxLength = 1 << 21;  // of a row, as in the other operators
// Rows and slots: the kernels count them in 32 bits, as far as the end of the last workgroup's share and one stride past it.
constexpr int64_t kMaxRows = (1ll << 31) - (1 << 16);
// Threads of a launch: the runtime counts them in 32 bits.  No workgroup whose number grows with the rows has more than 512.
bool launches(int64_t blocks) { return blocks <= UINT32_MAX / 512; }

bolt_status check_w4_shape(int32_t N, int32_t K, int32_t group) {
  if (N <= 0 || K <= 0 || (group != 32 && group != 64 && group != 128)) return BOLT_ERR_INVALID_ARG;
  if ((N | K) & 7) return BOLT_ERR_ALIGNMENT;
  if (N > kMaxLength || K > kMaxLength) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

bolt_status check_gemm_w4(const bolt_gemm_w4_desc* d) {
  if (!d) return BOLT_ERR_INVALID_ARG;
  if (bolt_status s = check_w4_shape(d->N, d->K, d->group); s == BOLT_ERR_INVALID_ARG) return s;
  if (d->M < 0 || !known_act(d->act) || d->lda < d->K || d->ldd < d->N) return BOLT_ERR_INVALID_ARG;
  if ((d->N | d->K | d->lda | d->ldd) & 7) return BOLT_ERR_ALIGNMENT;
  if (d->lda > kMaxLength || d->ldd > kMaxLength || d->N > kMaxLength || d->M > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

bolt_status check_route(const bolt_moe_route_desc* d) {
  if (!d) return BOLT_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->experts <= 0 || d->top_k <= 0 || d->groups <= 0 || d->top_groups <= 0 || d->top_groups > d->groups)
    return BOLT_ERR_INVALID_ARG;
  if (d->experts % d->groups || d->ld_logits < d->experts) return BOLT_ERR_INVALID_ARG;
  if (d->score != BOLT_SCORE_SOFTMAX && d->score != BOLT_SCORE_SIGMOID) return BOLT_ERR_INVALID_ARG;
  if (d->logits_type != BOLT_TYPE_F16 && d->logits_type != BOLT_TYPE_F32) return BOLT_ERR_INVALID_ARG;
  if ((int64_t)d->top_k > (int64_t)(d->experts / d->groups) * d->top_groups) return BOLT_ERR_INVALID_ARG;
  if (d->experts > kRouteMaxExperts || d->top_k > kRouteMaxTopK || d->groups > kRouteMaxGroups) return BOLT_ERR_UNSUPPORTED;
  if ((int64_t)d->tokens * d->top_k > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// Workgroups of the routing kernel.  Few tokens are one workgroup's, which makes the lists in the same launch; beyond, each workgroup of a second
// launch adds up the counts of all.  One workgroup takes a wave for a token up to 16 tokens and 16 lanes from there, 64 tokens at once.  us, a wave
// each / 16 lanes, FP16 softmax, 28, 128 and 196 (4 groups) experts: 17 tokens 5.6 / 5.1, 6.0 / 5.9 and 8.1 / 9.2, 32 tokens 6.9 / 5.1, 7.5 / 5.9
// and 10.1 / 9.0, 64 tokens 9.7 / 6.0, 10.7 / 7.2 and 15.7 / 11.3.  By 16 lanes 96 tokens take 6.5, 8.0 and 12.7, 256 tokens 10.9, 13.9 and 25.9; two
// launches take 7.9, 8.3 and 12.6 for 257 tokens.  More than 256 experts (32 keys for 16 lanes) keep to waves: 352 and 512 experts in 8 groups, 48 tokens
// 12.5 and 21.3, two launches 13.7 and 20.1 for 49.
struct RoutePlan {
  int blocks, block_tokens, threads, lanes;
};
RoutePlan route_plan(const bolt_moe_route_desc& d) {
  const bool wide = d.experts > 256;
  if (d.tokens <= (wide ? 48 : 64)) return {1, d.tokens, kRouteThreads, wide || d.tokens <= 16 ? 64 : 16};
  const int threads = d.tokens <= 8192 || wide ? 512 : 1024, at_once = threads / 16;
  const int per = (int)blocks_of(d.tokens, at_once * 256) * at_once;
  return {(int)blocks_of(d.tokens, per), per, threads, 16};
}

template <typename T, bool SIGMOID, bool PACKED, bool WIDE, int L, int V, int NT, bool ONE>
hipError_t launch_route(const RouteParams& p, int blocks, hipStream_t stream) {
  auto kern = moe_route_kernel<T, SIGMOID, PACKED, WIDE, L, V, NT, ONE>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, 160 * 1024); e != hipSuccess) return e;
  const int groups = p.top_groups < p.groups ? NT / L * (kRouteMaxGroups + p.experts) : 0;
  const int lists = kRouteWaves * std::max(p.experts, 2 * 64), head = kRouteMaxExperts + 1 + kRouteWaves;
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(NT), (head + (ONE ? std::max(groups, lists) + kRouteKeptIds : groups)) * 4, stream, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || ONE) return e;
  hipLaunchKernelGGL(moe_list_kernel, dim3(blocks), dim3(kRouteThreads), (head + lists) * 4, stream, p);
  return hipGetLastError();
}
template <typename T, bool SIGMOID, bool PACKED>
hipError_t launch_route_keys(const RouteParams& p, const RoutePlan& plan, hipStream_t stream) {
  auto keys = [&](auto v64) {
    constexpr int V = decltype(v64)::value;
    if (plan.lanes == 64) return launch_route<T, SIGMOID, PACKED, false, 64, V, 1024, true>(p, 1, stream);
    if constexpr (V <= 4)
      if (plan.blocks == 1) return launch_route<T, SIGMOID, PACKED, false, 16, 4 * V, 1024, true>(p, 1, stream);
    auto many = [&](auto wide) {
      constexpr bool WIDE = decltype(wide)::value;
      if constexpr (V <= 4)
        if (plan.threads == 1024) return launch_route<T, SIGMOID, PACKED, WIDE, 16, 4 * V, 1024, false>(p, plan.blocks, stream);
      return launch_route<T, SIGMOID, PACKED, WIDE, 16, 4 * V, 512, false>(p, plan.blocks, stream);
    };
    if constexpr (4 * V * sizeof(T) >= 16)
      if (p.experts == 64 * V && p.ld * sizeof(T) % 16 == 0) return many(std::true_type{});  // (logits are 16-byte aligned)
    return many(std::false_type{});
  };
  if (p.experts <= 64) return keys(std::integral_constant<int, 1>{});
  if (p.experts <= 128) return keys(std::integral_constant<int, 2>{});
  if (p.experts <= 256) return keys(std::integral_constant<int, 4>{});
  return keys(std::integral_constant<int, 8>{});
}

bolt_status check_moe(const bolt_moe_desc* d) {
  if (!d) return BOLT_ERR_INVALID_ARG;
  if (d->tokens < 0 || d->experts <= 0 || d->top_k <= 0 || d->top_k > d->experts || d->width <= 0 || d->hidden <= 0) return BOLT_ERR_INVALID_ARG;
  if (!known_act(d->act) || (d->gated != 0 && d->gated != 1) || d->ldx < d->width || d->ldy < d->width) return BOLT_ERR_INVALID_ARG;
  if (d->weights != BOLT_WEIGHTS_F16 && d->weights != BOLT_WEIGHTS_W4) return BOLT_ERR_INVALID_ARG;
  if (d->weights == BOLT_WEIGHTS_W4 && d->group != 32 && d->group != 64 && d->group != 128) return BOLT_ERR_INVALID_ARG;
  if ((d->width | d->hidden | d->ldx | d->ldy) & 7) return BOLT_ERR_ALIGNMENT;
  if (d->experts > kRouteMaxExperts || d->top_k > kRouteMaxTopK) return BOLT_ERR_UNSUPPORTED;
  if (d->ldx > kMaxLength || d->ldy > kMaxLength || d->width > kMaxLength || d->hidden > kMaxLength / 2) return BOLT_ERR_UNSUPPORTED;
  if ((int64_t)d->tokens * d->top_k > kMaxRows) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// ---- which kernel runs a linear layer with 4-bit weights --------------------------------------------------------------------
// Estimated time in us: a fit to 6 shapes x 13 row counts, one workgroup's step in us times its steps and its rounds of 256 workgroups.  Two
// workgroups that share a compute unit (LDS of 78 KB) take 1.55 to 1.6 times as long as one alone.  Measured, rows of A x tile 32 x
// 32, 32 x 64, 64 x 128, 128 x 256 and unpacked: N = K = 4096, 64 rows 9.4 / 12.4 / 28 / 59, 256 rows 32 / 20 / 29 / 62, 1024 rows 150 /
// 77 / 46 / 64 / 78, 2048 rows - / 152 / 92 / 71 / 82; 12288 x 4096, 1024 rows 430 / 225 / 128 / 128 / 108.
struct DenseTile {
  SharedTile tile;
  int rows, cols, sets;  // sets: of waves that split the reduction
  double step_us;
  bool pairs;            // two workgroups fit a compute unit
};
constexpr DenseTile kDenseTiles[] = {{SharedTile::ROWS32_COLS32, 32, 32, 4, 0.72, false},
                                     {SharedTile::ROWS32_COLS64, 32, 64, 2, 0.57, true},
                                     {SharedTile::ROWS64_COLS128, 64, 128, 1, 0.78, true},
                                     {SharedTile::ROWS128_COLS256, 128, 256, 1, 1.73, false}};
// Groups of 32 (64) columns: four (two) times as many sums to scale per step.
double dense_us(const DenseTile& t, int64_t M, int64_t N, int64_t steps, int group) {
  const double rounds = (double)blocks_of(blocks_of(M, t.rows) * blocks_of(N, t.cols), 256);
  const double factor = t.pairs ? (rounds <= 1 ? 1.0 : rounds <= 2 ? 1.55 : 0.8 * rounds) : rounds <= 1 ? 1.0 : 1.2 * rounds;
  return 3.3 + (double)blocks_of(steps, t.sets) * t.step_us * factor * (group == 32 ? 1.4 : group == 64 ? 1.1 : 1.0);
}
const DenseTile& dense_tile(int64_t M, int64_t N, int64_t steps, int group) {
  const DenseTile* best = &kDenseTiles[0];
  for (const DenseTile& t : kDenseTiles)
    if (dense_us(t, M, N, steps, group) < dense_us(*best, M, N, steps, group)) best = &t;
  return *best;
}
// Rows from which unpacking can pay: the caller's buffer for unpacked weights goes by this alone, so that it does not come and go as M grows.
// (Unpacked weights are addressed with 31-bit offsets.)
bool dense_may_unpack(int64_t M, int64_t N, int64_t K) { return M >= 512 && M * N >= 1 << 19 && N * K * 2 <= INT32_MAX; }
// The FP16 layer over unpacked weights.
bolt_gemm_desc unpacked_desc(const bolt_gemm_w4_desc& d) {
  return {d.M, d.N, d.K, d.lda, d.K, d.ldd, d.alpha, d.beta, d.act, BOLT_LAYOUT_NK};
}
// Unpacking, a GEMM on FP16 operands, by the estimate of the GEMM's own kernel, and the launch that looks for marked weights, against the
// best tile on packed ones.  SiLU has one kernel there, 256 x 256 tiles, and an estimate of its own (a fit to the same sizes).  us on packed
// weights / unpacked / unpacked with SiLU, groups of 128: 2048 rows of 256 x 8192 23 / 30 / 133; 512 of 1024 x 12288 32 / 47 / 196; 1536
// of 4096 x 4096 67 / 64 / 84; 4096 of 4096 x 4096 142 / 114 / 119.  Over 221 sizes (256 to 12288 outputs, K 512 to 12288, 512 to 8192
// rows) with groups of 32 and 128 the choice takes 1.012 times the faster side (1.31 at most; packed ones everywhere 1.11 and 1.85), with
// SiLU 1.005 (1.23; 1.03 and 1.31).
bool dense_unpacks(const bolt_gemm_w4_desc& d) {
  if (!dense_may_unpack(d.M, d.N, d.K)) return false;
  const int64_t steps = W4Format(d.N, d.K, d.group).steps;
  // (the packed side's estimate is some 10 % low from a few hundred rows on)
  const double packed = 1.1 * dense_us(dense_tile(d.M, d.N, steps, d.group), d.M, d.N, steps, d.group), weights = (double)d.N * d.K * 1e-6;
  if (d.act == BOLT_ACT_SILU) {
    const double rounds = (double)blocks_of(blocks_of(d.M, 256) * blocks_of(d.N, 256), 256);
    return 13.0 + 0.57 * weights + blocks_of(d.K, 64) * (rounds <= 1 ? 0.95 : 1.29 * rounds) + 0.79e-6 * d.M * d.N < packed;
  }
  double gemm;
  return launches(blocks_of(d.M, 32) * blocks_of(d.N, 32)) && estimate_gemm(unpacked_desc(d), &gemm) && 4.0 + 0.6 * weights + gemm < packed;
}

// ---- which kernels run the experts ------------------------------------------------------------------------------------
// The host does not know the lists: it goes by the experts that the slots reach if all are asked for equally often, and the rows of each.
struct Spread {
  double experts, rows;
  explicit Spread(const bolt_moe_desc& d) {
    const double slots = (double)d.tokens * d.top_k, E = d.experts;
    experts = std::max(1.0, E * (1.0 - std::pow(1.0 - 1.0 / E, slots)));
    rows = slots / experts;
  }
  // workgroups with blocks of `by` rows: every expert's last block is half full on average
  double blocks(int by) const { return experts * std::max(1.0, rows / by + 0.5); }
};
enum class Family { FEW, SHARED, MANY };
struct Choice {
  Family family;
  SharedTile shared;
  ManyTile many;
};
// 4 bits, us for 2048 wide, 1024 hidden, 32 experts, 4 per token, few rows / 16 x 64 / 16 x 128 / 32 x 128 / 64 x 128 / 128 x 256:
// 1 token 15 / 19 / 26; 4 tokens 27 / 23 / 26; 32 tokens 42 / 38 / 34 / 37; 128 tokens 67 / 53 / 45 / 49 / 53 / 68; 512 tokens 157 / 120 / 93 /
// 77 / 90 / 131; 1024 tokens - / - / 162 / 127 / 127 / 143; 2048 tokens - / - / - / - / 246 / 225.  A tile that leaves compute units without a
// workgroup gives way to the next smaller one: groups of 32, no gate, 968 wide, 3592 hidden, 350 tokens, 6 of 6 experts 144 by the rows alone, 114 so;
// groups of 128, gated, 1264 wide, 4072 hidden, 1104 tokens, 3 of 4 experts 186 and 167.  Over 108 sizes (9 shapes, 1 to 8192 tokens) the choice
// takes 1.01 times the best tile for both products, 1.32 at most (4096 tokens, 4 of 16 experts, 512 x 512 without a gate: 103 / 69 / 59 / 65 / 78 by
// 16 x 64 .. 128 x 256, which it takes).
Choice choose_w4(const Spread& s, int weight_rows) {
  if (s.experts * blocks_of(weight_rows, 32) <= 512 && s.rows <= 16) return {Family::FEW, {}, {}};
  const auto fills = [&](int rows, int cols) { return s.blocks(rows) * blocks_of(weight_rows, cols) >= 256; };
  SharedTile t = SharedTile::ROWS16_COLS64;
  if (s.blocks(16) * blocks_of(weight_rows, 64) <= 768) t = SharedTile::ROWS16_COLS64;
  else if (s.rows > 256 && fills(128, 256)) t = SharedTile::ROWS128_COLS256;
  else if (s.rows > 128 && fills(64, 128)) t = SharedTile::ROWS64_COLS128;
  else if (s.rows > 16 && fills(32, 128)) t = SharedTile::ROWS32_COLS128;
  else if (fills(16, 128)) t = SharedTile::ROWS16_COLS128;
  return {Family::SHARED, t, {}};
}
// FP16, us for the first experts above, few rows / shared rows / 64 x 128 / 128 x 128 / 256 x 256: 32 tokens 82 / 90; 128 tokens 116 / 109 / 96 / 98 /
// 109; 512 tokens 183 / 183 / 117 / 140 / 122; 1024 tokens - / - / 142 / 151 / 182; 2048 tokens - / - / 238 / 214 / 189; 4096 tokens - / - / 398 / 348 /
// 285; and 1000 wide, 2504 hidden, no gate, 8 experts, 2 per token: 64 tokens 31 / 31 / 47, 256 tokens - / 51 / 51 / 70 / 100, 1024 tokens - / - /
// 90 / 84 / 114, 4096 tokens - / - / 221 / 200 / 160.
// It does not look at the reduction's length.  Short ones, gated, 4 of 55 experts, 2000 wide, 464 hidden, 64 / 128 / 256 rows: 1024 tokens 130 / 136 /
// 119, 2048 tokens 178 / 169 / 128, 4096 tokens 295 / 256 / 220, 8192 tokens 514 / 427 / 369; 5 of 9 experts, 448 x 424: 2048 tokens 44 / 43 / 48, 8192
// tokens 145 / 123 / 117.  Over 108 sizes (9 shapes, 1 to 8192 tokens) the choice takes 1.03 times the best family for both products, 1.39 at
// most (the 2048 tokens above).
Choice choose_f16(const Spread& s, int weight_rows, bool offsets_fit) {
  if (s.rows <= 10 || !offsets_fit) return {Family::FEW, {}, {}};
  if (s.rows >= 192 && s.blocks(256) * blocks_of(weight_rows, 256) >= 144) return {Family::MANY, {}, ManyTile::ROWS256};
  if (s.rows <= 48 && s.blocks(32) * blocks_of(weight_rows, 64) <= 768) return {Family::SHARED, {}, {}};
  return {Family::MANY, {}, s.rows >= 224 ? ManyTile::ROWS128 : ManyTile::ROWS64};
}

// Whether the launch of a product with N weight rows of K columns can be made; the number of row blocks is the host's bound of it.
bool product_launches(const bolt_moe_desc& d, const Spread& s, int N, int K, bool gate, bool offsets_fit) {
  const bool w4 = d.weights == BOLT_WEIGHTS_W4;
  const Choice c = w4 ? choose_w4(s, N) : choose_f16(s, N, offsets_fit);
  const int64_t slots = (int64_t)d.tokens * d.top_k, short_blocks = std::min<int64_t>(slots, d.experts);
  if (c.family == Family::FEW || !offsets_fit) {
    const int64_t blocks = slots / 16 + short_blocks;
    // walks: each row block once at least, some thousand workgroups otherwise (csrc/inst_few_rows_*.hip)
    const bool walks = blocks_of(K, w4 ? W4Format::STEP : 64) <= (w4 && gate && d.group == 32 ? 16 : 32);
    return launches(walks ? 2 * blocks + 2048 : blocks * blocks_of(N, 32));
  }
  if (c.family == Family::MANY && c.many == ManyTile::ROWS256) return true;  // (one workgroup per compute unit)
  TileSize t = {32, 64};
  if (w4) t = tile_size(c.shared);
  else if (c.family == Family::MANY) t = c.many == ManyTile::ROWS64 ? TileSize{64, 128} : TileSize{128, 128};
  return launches((slots / t.rows + short_blocks) * blocks_of(N, t.cols));
}

struct MoeWorkspace {
  int64_t hidden_at, rows_at, bytes;  // [slots][hidden] halves in the lists' order, [slots][width] floats by slot
};
MoeWorkspace moe_workspace(const bolt_moe_desc& d) {
  const int64_t slots = (int64_t)d.tokens * d.top_k;
  MoeWorkspace w;
  w.hidden_at = 0;
  w.rows_at = round_up(slots * d.hidden * 2, 256);
  w.bytes = w.rows_at + round_up(slots * d.width * 4, 256);
  return w;
}

}  // namespace
}  // namespace bolt

using namespace bolt;

extern "C" {

size_t bolt_w4_packed_bytes(int32_t N, int32_t K, int32_t group, int32_t count) {
  if (check_w4_shape(N, K, group) != BOLT_OK || count <= 0) return 0;
  return (size_t)W4Format(N, K, group).bytes(count);
}

bolt_status bolt_w4_pack(int32_t N, int32_t K, int32_t group, int32_t count, const void* q, const void* scales, const void* zeros, void* packed,
                         size_t packed_bytes, void* stream) {
  if (bolt_status s = check_w4_shape(N, K, group); s != BOLT_OK) return s;
  if (count <= 0 || !q || !scales || !packed) return BOLT_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(scales) || !aligned16(packed)) return BOLT_ERR_ALIGNMENT;
  const W4Format f(N, K, group);
  if (packed_bytes < (size_t)f.bytes(count)) return BOLT_ERR_WORKSPACE;
  const int64_t items = count * (f.weight_bytes / 16 + f.scale_count);
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)std::min<int64_t>((items + 255) / 256, 256 * 16)), dim3(256), 0, (hipStream_t)stream,
                     (const unsigned char*)q, (const half_t*)scales, (const unsigned char*)zeros, (unsigned char*)packed, count, f);
  return status_of(hipGetLastError());
}

size_t bolt_gemm_w4_workspace_bytes(const bolt_gemm_w4_desc* desc) {
  if (check_gemm_w4(desc) != BOLT_OK || !dense_may_unpack(desc->M, desc->N, desc->K)) return 0;
  return (size_t)desc->N * desc->K * 2;
}

bolt_status bolt_gemm_w4(const bolt_gemm_w4_desc* desc, const void* A, const void* packed, const void* bias, void* D, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_gemm_w4(desc); s != BOLT_OK) return s;
  if (desc->M == 0) return BOLT_OK;
  if (!A || !packed || !D) return BOLT_ERR_INVALID_ARG;
  if (!aligned16(A) || !aligned16(packed) || !aligned16(D) || (bias && !aligned16(bias))) return BOLT_ERR_ALIGNMENT;
  const size_t need = bolt_gemm_w4_workspace_bytes(desc);
  if (need > 0 && (!workspace || workspace_bytes < need)) return BOLT_ERR_WORKSPACE;
  if (!aligned16(workspace)) return BOLT_ERR_ALIGNMENT;
  const W4Format f(desc->N, desc->K, desc->group);
  const DenseTile& tile = desc->M > 16 ? dense_tile(desc->M, desc->N, f.steps, desc->group) : kDenseTiles[0];
  // The kernels of many rows start their sums at beta / alpha times the bias, which has to be finite.
  const bool bias_in_sum = desc->alpha != 0.f && std::fabs(desc->beta) <= 1e30f * std::fabs(desc->alpha);
  const bool packed_tiles = desc->M > 16 && (!bias_in_sum || !dense_unpacks(*desc));
  if (packed_tiles && !launches(blocks_of(desc->M, tile.rows) * blocks_of(desc->N, tile.cols))) return BOLT_ERR_UNSUPPORTED;
  const hipStream_t st = (hipStream_t)stream;
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  RowsParams p{};
  p.x = (const half_t*)A;
  p.ldx = desc->lda;
  p.w = (const unsigned char*)packed;
  p.scales = (const half_t*)((const char*)packed + f.scales_at(1));
  p.zeros = (const unsigned char*)packed + f.zeros_at(1);
  p.none = none;
  p.bias = bias ? (const half_t*)bias : none;
  p.bias_on = bias ? 1 : 0;
  p.y = D;
  p.ldy = desc->ldd;
  p.M = desc->M; p.N = desc->N; p.K = desc->K; p.steps = f.steps;
  p.alpha = desc->alpha; p.beta = desc->beta; p.act = desc->act;
  if (desc->M <= 16) return status_of(launch_few_rows_w4(p, ROWS_DENSE, false, desc->group, st));
  if (packed_tiles) return status_of(launch_shared_rows_w4(p, ROWS_DENSE, false, desc->group, tile.tile, st));
  if (launch_w4_unpack(packed, (half_t*)workspace, f, st) != hipSuccess) return BOLT_ERR_LAUNCH;
  if (desc->act != BOLT_ACT_SILU) {
    const bolt_gemm_desc g = unpacked_desc(*desc);
    if (bolt_status s = bolt_gemm_epilogue(&g, A, workspace, bias, D, nullptr, nullptr, 0, stream); s != BOLT_OK) return s;
  } else {
    RowsParams u = p;
    u.w = (const unsigned char*)workspace;
    u.w_stride = (int64_t)p.N * p.K * 2;
    if (launch_many_rows_f16(u, ROWS_DENSE, false, ManyTile::ROWS256, st) != hipSuccess) return BOLT_ERR_LAUNCH;
  }
  p.unpacked = (const half_t*)workspace;
  return status_of(launch_shared_rows_w4_marked(p, desc->group, st));
}

size_t bolt_moe_route_workspace_bytes(const bolt_moe_route_desc* desc) {
  if (check_route(desc) != BOLT_OK) return 0;
  if (route_plan(*desc).blocks == 1) return 0;
  // a bound of the plan's workgroups that does not fall as tokens grow: a buffer for the largest batch is enough for all
  return (size_t)std::min<int64_t>(256, blocks_of(desc->tokens, 32)) * desc->experts * sizeof(int);
}

bolt_status bolt_moe_route(const bolt_moe_route_desc* desc, const void* logits, const void* bias, const void* mask, void* ids, void* weights,
                           void* offsets, void* order, void* workspace, size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_route(desc); s != BOLT_OK) return s;
  if (!offsets || (desc->tokens > 0 && (!logits || !ids || !weights || !order))) return BOLT_ERR_INVALID_ARG;
  for (const void* q : {logits, bias, (const void*)ids, (const void*)weights, (const void*)offsets, (const void*)order, (const void*)workspace})
    if (!aligned16(q)) return BOLT_ERR_ALIGNMENT;
  const size_t need = bolt_moe_route_workspace_bytes(desc);
  if (need > 0 && (!workspace || workspace_bytes < need)) return BOLT_ERR_WORKSPACE;
  const RoutePlan plan = route_plan(*desc);
  RouteParams p{};
  p.logits = logits; p.bias = (const float*)bias; p.mask = (const unsigned char*)mask;
  p.ids = (int*)ids; p.weights = (float*)weights; p.offsets = (int*)offsets; p.order = (int*)order; p.counts = (int*)workspace;
  p.ld = desc->ld_logits;
  p.tokens = desc->tokens; p.experts = desc->experts; p.top_k = desc->top_k; p.groups = desc->groups; p.top_groups = desc->top_groups;
  p.renormalize = desc->renormalize; p.scale = desc->scale; p.block_tokens = plan.block_tokens;
  const bool sigmoid = desc->score == BOLT_SCORE_SIGMOID;
  const hipStream_t st = (hipStream_t)stream;
  if (desc->logits_type == BOLT_TYPE_F32)
    return status_of(sigmoid ? launch_route_keys<float, true, false>(p, plan, st) : launch_route_keys<float, false, false>(p, plan, st));
  if (bias)
    return status_of(sigmoid ? launch_route_keys<half_t, true, false>(p, plan, st) : launch_route_keys<half_t, false, false>(p, plan, st));
  return status_of(sigmoid ? launch_route_keys<half_t, true, true>(p, plan, st) : launch_route_keys<half_t, false, true>(p, plan, st));
}

size_t bolt_moe_workspace_bytes(const bolt_moe_desc* desc) {
  if (check_moe(desc) != BOLT_OK) return 0;
  return (size_t)moe_workspace(*desc).bytes;
}

bolt_status bolt_moe_experts(const bolt_moe_desc* desc, const void* x, const void* w_up, const void* b_up, const void* w_down, const void* b_down,
                             const void* ids, const void* weights, const void* offsets, const void* order, void* y, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_moe(desc); s != BOLT_OK) return s;
  if (desc->tokens == 0) return BOLT_OK;
  if (!x || !w_up || !w_down || !ids || !weights || !offsets || !order || !y) return BOLT_ERR_INVALID_ARG;
  for (const void* q : {x, w_up, b_up, w_down, b_down, ids, weights, offsets, order, (const void*)y, (const void*)workspace})
    if (!aligned16(q)) return BOLT_ERR_ALIGNMENT;
  const MoeWorkspace ws = moe_workspace(*desc);
  if (!workspace || workspace_bytes < (size_t)ws.bytes) return BOLT_ERR_WORKSPACE;
  const bool w4 = desc->weights == BOLT_WEIGHTS_W4, gated = desc->gated != 0;
  const int slots = desc->tokens * desc->top_k, E = desc->experts;
  const int up_rows = gated ? 2 * desc->hidden : desc->hidden;
  // the kernels that stage rows address x, an expert's weights and a tile's rows with 31-bit byte offsets
  const int64_t most = (1ll << 31) - 1;
  const bool offsets_fit = (int64_t)desc->tokens * desc->ldx * 2 <= most && (int64_t)up_rows * desc->width * 2 <= most &&
                           (int64_t)desc->width * desc->hidden * 2 <= most && (int64_t)256 * desc->hidden * 2 <= most;
  // (beyond them the kernel of few rows runs)
  const Spread spread(*desc);
  if (!product_launches(*desc, spread, up_rows, desc->width, gated, offsets_fit) ||
      !product_launches(*desc, spread, desc->width, desc->hidden, false, offsets_fit))
    return BOLT_ERR_UNSUPPORTED;
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  const hipStream_t st = (hipStream_t)stream;

  RowsParams p{};
  p.M = slots;
  p.offsets = (const int*)offsets; p.order = (const int*)order;
  p.experts = E; p.top_k = desc->top_k;
  p.none = none;
  p.alpha = p.beta = 1.f;
  auto product = [&](int N, int K, const void* w, const void* b, int mode) {
    const bool gate = mode == ROWS_UP && gated;
    p.N = N; p.K = K;
    p.w = (const unsigned char*)w;
    p.bias = b ? (const half_t*)b : none;
    p.bias_on = b ? 1 : 0;
    if (w4) {
      const W4Format f(N, K, desc->group);
      p.w_stride = f.weight_bytes; p.scale_stride = f.scale_count; p.steps = f.steps;
      p.scales = (const half_t*)((const char*)w + f.scales_at(E));
      p.zeros = (const unsigned char*)w + f.zeros_at(E);
      const Choice c = choose_w4(spread, N);
      if (c.family == Family::FEW || !offsets_fit) return launch_few_rows_w4(p, mode, gate, desc->group, st);
      return launch_shared_rows_w4(p, mode, gate, desc->group, c.shared, st);
    }
    p.w_stride = (int64_t)N * K * 2; p.steps = (K + 63) / 64;
    const Choice c = choose_f16(spread, N, offsets_fit);
    if (c.family == Family::FEW) return launch_few_rows_f16(p, mode, gate, st);
    if (c.family == Family::SHARED) return launch_shared_rows_f16(p, mode, gate, st);
    return launch_many_rows_f16(p, mode, gate, c.many, st);
  };
  half_t* const hidden = (half_t*)((char*)workspace + ws.hidden_at);
  float* const rows = (float*)((char*)workspace + ws.rows_at);
  p.x = (const half_t*)x; p.ldx = desc->ldx; p.y = hidden; p.ldy = desc->hidden; p.hidden = desc->hidden; p.act = desc->act;
  if (hipError_t e = product(up_rows, desc->width, w_up, b_up, ROWS_UP); e != hipSuccess) return BOLT_ERR_LAUNCH;
  p.x = hidden; p.ldx = desc->hidden; p.y = rows; p.ldy = desc->width; p.act = BOLT_ACT_NONE;
  if (hipError_t e = product(desc->width, desc->hidden, w_down, b_down, ROWS_DOWN); e != hipSuccess) return BOLT_ERR_LAUNCH;
  const int64_t chunks = (int64_t)desc->tokens * (desc->width / 8);
  hipLaunchKernelGGL(chunks <= 256 * 1024 ? moe_combine_kernel<4> : moe_combine_kernel<1>, dim3((unsigned)std::min<int64_t>((chunks + 255) / 256, 256 * 32)), dim3(256), 0, st, rows,
                     (const int*)ids, (const float*)weights, (half_t*)y, desc->tokens, desc->top_k, desc->width, desc->ldy);
  return status_of(hipGetLastError());
}

}  // extern "C"
