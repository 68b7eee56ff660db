// C ABI of the operators of language models: linear layers with weights in 4 bits, routing to experts, the experts' products.
#include <algorithm>
#include <cstdint>

#include "../../include/bolt.h"
#include "few_rows_instances.hpp"
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


// y[t] = sum of the slots' rows (which carry their weights already), in FP32, in the order of the slots: one thread for eight columns.
// Slots without an expert have no row.
__global__ __launch_bounds__(256) void moe_combine_kernel(const half_t* rows, const int* ids, half_t* y, int tokens, int top_k, int width, int64_t ldy) {
  const int chunks = width / 8;
  const int64_t total = (int64_t)tokens * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / chunks;
    const int c = (int)(i - t * chunks) * 8;
    float sum[8] = {};
    for (int j = 0; j < top_k; ++j) {
      const int64_t slot = t * top_k + j;
      if (ids[slot] < 0) continue;
      const half8 v = *(const half8*)(rows + slot * width + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += (float)v[e];
    }
    half8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (half_t)sum[e];
    *(half8*)(y + t * ldy + c) = o;
  }
}

__device__ __attribute__((aligned(16))) half_t g_no_bias[8];
const half_t* no_bias() {
  static const half_t* ptr = [] {
    void* q = nullptr;
    return hipGetSymbolAddress(&q, HIP_SYMBOL(g_no_bias)) == hipSuccess ? (const half_t*)q : nullptr;
  }();
  return ptr;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
bool known_act(int a) { return a >= BOLT_ACT_NONE && a <= BOLT_ACT_SILU; }
bolt_status status_of(hipError_t e) { return e == hipSuccess ? BOLT_OK : BOLT_ERR_LAUNCH; }
constexpr int kMaxLength = 1 << 21;  // of a row, as in the other operators
constexpr int64_t kMaxGrid = (1ll << 31) - 1;

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
  if (d->lda > kMaxLength || d->ldd > kMaxLength || d->N > kMaxLength) return BOLT_ERR_UNSUPPORTED;
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
  if ((int64_t)d->tokens * d->top_k > INT32_MAX) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// Tokens per workgroup of the routing kernel.  One workgroup makes the lists in the same launch.
struct RoutePlan {
  int blocks, block_tokens;
};
RoutePlan route_plan(const bolt_moe_route_desc& d) {
  if (d.tokens <= 256) return {1, d.tokens};
  const int blocks = std::min(256, (d.tokens + 63) / 64), per = (d.tokens + blocks - 1) / blocks;
  return {(d.tokens + per - 1) / per, per};
}

template <typename T, bool SIGMOID, int L, int V>
hipError_t launch_route(const RouteParams& p, int blocks, hipStream_t stream) {
  constexpr int TEAMS = kRouteThreads / L;
  const int groups = p.top_groups < p.groups ? TEAMS * (kRouteMaxGroups + p.experts) : 0;
  const int lists = kRouteWaves * p.experts, head = kRouteMaxExperts + 1 + kRouteWaves;
  constexpr int MOST = 160 * 1024;
  auto one = moe_route_kernel<T, SIGMOID, L, V, true>;
  auto many = moe_route_kernel<T, SIGMOID, L, V, false>;
  static LdsOptIn opt_in[2];
  if (hipError_t e = opt_in[0].ensure((const void*)one, MOST); e != hipSuccess) return e;
  if (hipError_t e = opt_in[1].ensure((const void*)many, MOST); e != hipSuccess) return e;
  if (blocks == 1) {
    hipLaunchKernelGGL(one, dim3(1), dim3(kRouteThreads), (head + std::max(groups, lists)) * 4, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(many, dim3(blocks), dim3(kRouteThreads), (head + groups) * 4, stream, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(moe_list_kernel, dim3(blocks), dim3(kRouteThreads), (head + lists) * 4, stream, p);
  return hipGetLastError();
}
template <typename T, bool SIGMOID>
hipError_t launch_route_keys(const RouteParams& p, int blocks, hipStream_t stream) {
  if (p.experts <= 64) return launch_route<T, SIGMOID, 64, 1>(p, blocks, stream);
  if (p.experts <= 128) return launch_route<T, SIGMOID, 64, 2>(p, blocks, stream);
  if (p.experts <= 256) return launch_route<T, SIGMOID, 64, 4>(p, blocks, stream);
  return launch_route<T, SIGMOID, 64, 8>(p, blocks, stream);
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
  if ((int64_t)d->tokens * d->top_k > INT32_MAX) return BOLT_ERR_UNSUPPORTED;
  return BOLT_OK;
}

// Rows of a workgroup in 16s, from the rows that share a weight matrix.
int row_blocks_of(double rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

struct MoeWorkspace {
  int64_t hidden_at, rows_at, bytes;  // [slots][hidden] in the lists' order, [slots][width] by slot, halves
};
MoeWorkspace moe_workspace(const bolt_moe_desc& d) {
  const int64_t slots = (int64_t)d.tokens * d.top_k;
  MoeWorkspace w;
  w.hidden_at = 0;
  w.rows_at = round_up(slots * d.hidden * 2, 256);
  w.bytes = w.rows_at + round_up(slots * d.width * 2, 256);
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
  (void)desc;
  return 0;
}

bolt_status bolt_gemm_w4(const bolt_gemm_w4_desc* desc, const void* A, const void* packed, const void* bias, void* D, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (bolt_status s = check_gemm_w4(desc); s != BOLT_OK) return s;
  if (!A || !packed || !D) return BOLT_ERR_INVALID_ARG;
  if (!aligned16(A) || !aligned16(packed) || !aligned16(D) || (bias && !aligned16(bias))) return BOLT_ERR_ALIGNMENT;
  (void)workspace;
  (void)workspace_bytes;
  if (desc->M == 0) return BOLT_OK;
  const W4Format f(desc->N, desc->K, desc->group);
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  RowsParams p{};
  p.x = (const half_t*)A;
  p.ldx = desc->lda;
  p.w = (const unsigned char*)packed;
  p.scales = (const half_t*)((const char*)packed + f.scales_at(1));
  p.zeros = (const unsigned char*)packed + f.zeros_at(1);
  p.bias = bias ? (const half_t*)bias : none;
  p.bias_on = bias ? 1 : 0;
  p.y = (half_t*)D;
  p.ldy = desc->ldd;
  p.M = desc->M; p.N = desc->N; p.K = desc->K; p.steps = f.steps;
  p.alpha = desc->alpha; p.beta = desc->beta; p.act = desc->act;
  const int mb = row_blocks_of(desc->M);
  if ((int64_t)((desc->M + 15) / 16) * ((desc->N + 15) / 16) > kMaxGrid) return BOLT_ERR_UNSUPPORTED;
  return status_of(launch_few_rows_w4(p, ROWS_DENSE, false, desc->group, mb, (hipStream_t)stream));
}

size_t bolt_moe_route_workspace_bytes(const bolt_moe_route_desc* desc) {
  if (check_route(desc) != BOLT_OK) return 0;
  const RoutePlan plan = route_plan(*desc);
  return plan.blocks == 1 ? 0 : (size_t)plan.blocks * desc->experts * sizeof(int);
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
  if (desc->logits_type == BOLT_TYPE_F16)
    return status_of(sigmoid ? launch_route_keys<half_t, true>(p, plan.blocks, st) : launch_route_keys<half_t, false>(p, plan.blocks, st));
  return status_of(sigmoid ? launch_route_keys<float, true>(p, plan.blocks, st) : launch_route_keys<float, false>(p, plan.blocks, st));
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
  const half_t* none = no_bias();
  if (!none) return BOLT_ERR_LAUNCH;
  const bool w4 = desc->weights == BOLT_WEIGHTS_W4, gated = desc->gated != 0;
  const int slots = desc->tokens * desc->top_k, E = desc->experts;
  const int mb = row_blocks_of((double)slots / E);
  const int up_rows = gated ? 2 * desc->hidden : desc->hidden;
  if (((int64_t)slots / 16 + E) * ((std::max(desc->hidden, desc->width) + 15) / 16) > kMaxGrid) return BOLT_ERR_UNSUPPORTED;

  RowsParams p{};
  p.M = slots;
  p.offsets = (const int*)offsets; p.order = (const int*)order; p.slot_weights = (const float*)weights;
  p.experts = E; p.top_k = desc->top_k;
  p.alpha = p.beta = 1.f;
  auto product = [&](int N, int K, const void* w, const void* b, int mode) {
    p.N = N; p.K = K;
    p.w = (const unsigned char*)w;
    p.bias = b ? (const half_t*)b : none;
    p.bias_on = b ? 1 : 0;
    if (w4) {
      const W4Format f(N, K, desc->group);
      p.w_stride = f.weight_bytes; p.scale_stride = f.scale_count; p.steps = f.steps;
      p.scales = (const half_t*)((const char*)w + f.scales_at(E));
      p.zeros = (const unsigned char*)w + f.zeros_at(E);
      return launch_few_rows_w4(p, mode, mode == ROWS_UP && gated, desc->group, mb, (hipStream_t)stream);
    }
    p.w_stride = (int64_t)N * K * 2; p.steps = (K + 63) / 64;
    return launch_few_rows_f16(p, mode, mode == ROWS_UP && gated, mb, (hipStream_t)stream);
  };
  half_t* const hidden = (half_t*)((char*)workspace + ws.hidden_at);
  half_t* const rows = (half_t*)((char*)workspace + ws.rows_at);
  p.x = (const half_t*)x; p.ldx = desc->ldx; p.y = hidden; p.ldy = desc->hidden; p.hidden = desc->hidden; p.act = desc->act;
  if (hipError_t e = product(up_rows, desc->width, w_up, b_up, ROWS_UP); e != hipSuccess) return BOLT_ERR_LAUNCH;
  p.x = hidden; p.ldx = desc->hidden; p.y = rows; p.ldy = desc->width; p.act = BOLT_ACT_NONE;
  if (hipError_t e = product(desc->width, desc->hidden, w_down, b_down, ROWS_DOWN); e != hipSuccess) return BOLT_ERR_LAUNCH;
  const int64_t chunks = (int64_t)desc->tokens * (desc->width / 8);
  hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)std::min<int64_t>((chunks + 255) / 256, 256 * 32)), dim3(256), 0, (hipStream_t)stream, rows,
                     (const int*)ids, (half_t*)y, desc->tokens, desc->top_k, desc->width, desc->ldy);
  return status_of(hipGetLastError());
}

}  // extern "C"
