// Routing of tokens to experts, and the lists that the experts' products walk.
//
// Per token: scores over E experts (softmax or sigmoid of the logits, FP32), a key for the choice (the logit itself, whose order is the
// scores', or score + bias), optionally the best groups of experts first, then the top_k largest keys, ties to the lowest index.
// L lanes share a token and hold its keys in registers; a place is one maximum over the keys and one minimum over the indices that
// have it.  FP16 logits that are keys themselves are packed with their index into 32 bits that order as (key, lower index first), so that a
// place is one maximum of unsigned numbers, and the next one the maximum of their distances below the last.  Only the chosen
// scores are computed where no sum or key needs the others.  What bounds it: the instructions of the choice (65536 tokens over 128
// experts, 4 places: 14.3 us; the logits alone are 3.3 us of memory traffic) and one round trip to memory after the other.
//
// Lists: slot t * top_k + j belongs to expert ids[t][j]; order holds the slots by expert, within an expert ascending, offsets where each
// expert's begin.  Positions come from counts, never from the order in which workgroups or atomics happen to run: a workgroup
// counts its slots per wave, adds up the counts of the waves and workgroups before it, and ranks 64 slots at a time by comparing ids.
#pragma once
#include <float.h>

#include "bolt_device.hpp"

namespace bolt {

struct RouteParams {
  const void* logits;
  const float* bias;
  const unsigned char* mask;
  int* ids;
  float* weights;
  int* offsets;
  int* order;
  int* counts;  // [blocks][experts], several workgroups only
  int64_t ld;
  int tokens, experts, top_k, groups, top_groups, renormalize;
  float scale;
  int block_tokens;  // tokens of a workgroup
};

static constexpr int kRouteMaxExperts = 512, kRouteMaxTopK = 16, kRouteMaxGroups = 16;
static constexpr int kRouteKeptIds = 1024;  // a single workgroup keeps its ids in LDS: 64 tokens of 16 slots
static constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;  // of a workgroup that makes lists

// exp(x) for x <= 0 (softmax) or of either sign (sigmoid) to about 2 units in the last place: the product with log2 e in two parts.
__device__ __forceinline__ float route_exp(float x) {
  x = fmaxf(x, -200.f);  // exp is zero from -104 on; minus infinity would make a NaN of the second part
  const float hi = x * 1.44269504088896340736f;
  const float lo = __builtin_fmaf(x, 1.44269504088896340736f, -hi) + x * 1.9259629911266175e-8f;
  const float p = __builtin_amdgcn_exp2f(hi);
  return p + p * (lo * 0.69314718055994530942f);
}
__device__ __forceinline__ float route_sigmoid(float x) {
  // exp(-x) overflows below -88.7228: the score is zero there; the quotient is the hardware's correctly rounded division
  return x < -88.72f ? 0.f : 1.f / (1.f + route_exp(-x));
}

struct MaxU { __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return a > b ? a : b; } };
struct MaxF { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct SumF { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct MinI { __device__ __forceinline__ int operator()(int a, int b) const { return a < b ? a : b; } };
// f over the L lanes of a token, to each of them: lanes exchanged inside rows of 16 (1, 2, 7 and 15 apart by mirroring), then between
// the four rows.  (Shuffles through LDS take ten times as long as these exchanges, and a token's choice is a chain of them.)
template <int L, typename T, typename F>
__device__ __forceinline__ T route_reduce(T v, F f) {
  static_assert(L == 16 || L == 64, "lanes of a token");
  auto with = [&](auto ctrl) {
    const int o = __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true);
    v = f(v, __builtin_bit_cast(T, o));
  };
  with(std::integral_constant<int, 0xb1>{});   // quad_perm 1 0 3 2
  with(std::integral_constant<int, 0x4e>{});   // quad_perm 2 3 0 1
  with(std::integral_constant<int, 0x141>{});  // row_half_mirror
  with(std::integral_constant<int, 0x140>{});  // row_mirror
  if constexpr (L == 64) {
    auto row = [&](int r) { return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), r * 16)); };
    v = f(f(row(0), row(1)), f(row(2), row(3)));
  }
  return v;
}

// LDS written by some lanes of a wave is read by others of the same wave.
__device__ __forceinline__ void route_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A half as 16 bits that order as the numbers do: NaN as minus infinity, minus zero as zero.
__device__ __forceinline__ unsigned route_ordered(half_t h) {
  const unsigned b = __builtin_bit_cast(unsigned short, h == h ? h + (half_t)0.f : (half_t)-INFINITY);
  return b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
}
__device__ __forceinline__ float route_unordered(unsigned o) {
  const unsigned short b = (unsigned short)(o & 0x8000u ? o & 0x7fffu : ~o);
  return (float)__builtin_bit_cast(half_t, b);
}

// One token on L lanes (l: this lane's number among them), V = ceil(experts / L) keys each, `raw`: key v is that of expert v * L + l, or
// l * V + v (WIDE: experts = L * V and aligned rows, so that a lane's logits are one piece of memory).  `shared` holds
// kRouteMaxGroups + experts floats of LDS for this token (groups only).  PACKED: FP16 logits and no bias.  Returns lane j's id and
// weight, j < top_k.
template <typename T, bool SIGMOID, bool PACKED, bool WIDE, int L, int V>
__device__ __forceinline__ void route_token(const RouteParams& p, const T* row, const T (&raw)[V], int l, float* shared, int* id_out, float* weight_out) {
  const int E = p.experts;
  auto expert_of = [&](int v) { return WIDE ? l * V + v : v * L + l; };
  // NaN counts as the lowest value, infinities as the largest finite ones, so a row of nothing but masked experts still has a choice
  auto clamped = [](float x) { return fminf(fmaxf(x, -FLT_MAX), FLT_MAX); };
  auto logit = [&](int e) { return clamped((float)row[e]); };
  float key[V];
  unsigned packed[PACKED ? V : 1];
  float top = -FLT_MAX;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = expert_of(v);
    key[v] = e < E ? clamped((float)raw[v]) : -INFINITY;
    if constexpr (PACKED) packed[v] = e < E ? route_ordered(raw[v]) << 16 | (0xffffu - e) : 0u;
    if constexpr (!SIGMOID) top = fmaxf(top, key[v]);
  }
  float total = 1.f;
  if constexpr (!SIGMOID) {
    top = route_reduce<L>(top, MaxF{});
    if (!p.renormalize || p.bias) {
      total = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) total += route_exp(key[v] - top);  // (0 for experts that do not exist)
      total = route_reduce<L>(total, SumF{});
    }
  }
  auto score = [&](float x) { return SIGMOID ? route_sigmoid(x) : route_exp(x - top) / total; };
  if (p.bias) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = expert_of(v);
      if (e < E) key[v] = fmaxf(score(key[v]) + p.bias[e], -FLT_MAX);
    }
  }
  if (p.top_groups < p.groups) {
    // a group's value: its best key (softmax), or the sum of its two best scores with bias (sigmoid); one lane per group
    const int size = E / p.groups;
    float* const keys = shared + kRouteMaxGroups;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = expert_of(v);
      if (e < E) keys[e] = SIGMOID && !p.bias ? score(key[v]) : key[v];
    }
    route_wave_sync();
    float value = -INFINITY;
    if (l < p.groups) {
      float first = -INFINITY, second = -INFINITY;
      for (int i = 0; i < size; ++i) {
        const float k = keys[l * size + i];
        second = fmaxf(second, fminf(first, k));
        first = fmaxf(first, k);
      }
      value = SIGMOID && size > 1 ? first + second : first;
      shared[l] = value;
    }
    route_wave_sync();
    // a group stays if fewer than top_groups go before it
    int ahead = 0;
    for (int i = 0; i < p.groups; ++i) {
      const float o = shared[i];
      ahead += o > value || (o == value && i < l);
    }
    route_wave_sync();
    if (l < p.groups) shared[l] = ahead < p.top_groups ? 1.f : 0.f;
    route_wave_sync();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = expert_of(v);
      if (e < E && shared[e / size] == 0.f) {
        key[v] = -INFINITY;
        if constexpr (PACKED) packed[v] = 0u;
      }
    }
    route_wave_sync();
  }
  int id = 0;
  float chosen = 0.f;  // lane j: the key of place j, which is the logit if there is no bias
  if constexpr (PACKED) {
    unsigned last = 0u;
    for (int j = 0; j < p.top_k; ++j) {
      // the largest below `last`: the largest key - last modulo 2^32 (for the first place the largest of all)
      unsigned best = packed[0] - last;
#pragma unroll
      for (int v = 1; v < V; ++v) best = MaxU{}(best, packed[v] - last);
      last += route_reduce<L>(best, MaxU{});
      id = l == j ? (int)(0xffffu - (last & 0xffffu)) : id;
      chosen = l == j ? clamped(route_unordered(last >> 16)) : chosen;
    }
  } else {
    for (int j = 0; j < p.top_k; ++j) {
      float best = -INFINITY;
#pragma unroll
      for (int v = 0; v < V; ++v) best = fmaxf(best, key[v]);
      best = route_reduce<L>(best, MaxF{});
      int at = 0x7fffffff;
#pragma unroll
      for (int v = V - 1; v >= 0; --v) at = key[v] == best ? expert_of(v) : at;
      at = route_reduce<L>(at, MinI{});
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = expert_of(v) == at ? -INFINITY : key[v];
      id = l == j ? at : id;
      chosen = l == j ? best : chosen;
    }
  }
  float w = 0.f;
  if (l < p.top_k) {
    const float x = p.bias ? logit(id) : chosen;
    w = SIGMOID ? route_sigmoid(x) : route_exp(x - top);
  }
  if (p.renormalize) {
    const float sum = route_reduce<L>(w, SumF{});
    w = sum > 0.f ? w / sum : 0.f;
  } else if (!SIGMOID) {
    w /= total;
  }
  *id_out = id;
  *weight_out = w * p.scale;
}

template <typename T, bool WIDE, int L, int V>
__device__ __forceinline__ void route_load(const T* row, int E, int l, T (&raw)[V]) {
  if constexpr (WIDE) {
    constexpr int N = 16 / sizeof(T);
    typedef T piece __attribute__((ext_vector_type(N)));
    static_assert(V % N == 0, "whole pieces");
#pragma unroll
    for (int v = 0; v < V; v += N) {
      const piece q = *(const piece*)(row + l * V + v);
#pragma unroll
      for (int i = 0; i < N; ++i) raw[v + i] = q[i];
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = v * L + l < E ? row[v * L + l] : (T)0.f;
  }
}

// Exclusive sums over the experts of n[e] (LDS, in place), all threads of the workgroup; the total goes to n[experts].
__device__ __forceinline__ void route_scan(int* n, int* wave_sums, int experts, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  __syncthreads();
  const int mine = tid < experts ? n[tid] : 0;
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += wave_sums[w];
  if (tid < experts) n[tid] = before + upto - mine;
  if (tid == kRouteThreads - 1) n[experts] = before + upto;
  __syncthreads();
}

// Slots [s0, s1) into their places: base[e] (LDS) is the place of the workgroup's first slot of expert e.  per_wave: LDS, kRouteWaves *
// experts.  Each wave takes a run of the slots.  id_of(slot) gives -1 for slots that are in no list.
__device__ __forceinline__ int route_run(int s0, int s1) { return ((s1 - s0 + 63) / 64 + kRouteWaves - 1) / kRouteWaves * 64; }  // slots of a wave
template <typename F>
__device__ __forceinline__ void route_place(F id_of, int s0, int s1, const int* base, int* per_wave, int experts, int* order, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  const int run = route_run(s0, s1);
  const int a = s0 + wave * run, z = a + run < s1 ? a + run : s1;
  int* const mine = per_wave + wave * experts;
  for (int i = tid; i < kRouteWaves * experts; i += kRouteThreads) per_wave[i] = 0;
  __syncthreads();
  for (int s = a + lane; s < z; s += 64) {
    const int e = id_of(s);
    if (e >= 0) atomicAdd(&mine[e], 1);
  }
  __syncthreads();
  if (tid < experts) {
    int at = base[tid];
    for (int w = 0; w < kRouteWaves; ++w) {
      const int n = per_wave[w * experts + tid];
      per_wave[w * experts + tid] = at;
      at += n;
    }
  }
  __syncthreads();
  for (int s = a; s < z; s += 64) {  // (the same trip count for all lanes of a wave)
    const int slot = s + lane, e = slot < z ? id_of(slot) : -1;
    unsigned long long same = __ballot(e >= 0);
    for (int bit = 1; bit < experts; bit <<= 1) {
      const unsigned long long has = __ballot((e & bit) != 0);
      same &= e & bit ? has : ~has;
    }
    if (e >= 0) {
      const int leader = __builtin_ctzll(same);
      int at = 0;
      if (lane == leader) at = atomicAdd(&mine[e], (int)__popcll(same));
      at = __shfl(at, leader);
      order[at + (int)__popcll(same & ((1ull << lane) - 1))] = slot;
    }
  }
}

// `block_tokens` tokens per workgroup, NT / L at a time.  ONE: a single workgroup, which makes the lists as well; otherwise the
// workgroup's counts per expert go to `counts` for moe_list_kernel.
template <typename T, bool SIGMOID, bool PACKED, bool WIDE, int L, int V, int NT, bool ONE>
__global__ __launch_bounds__(NT) void moe_route_kernel(const RouteParams p) {
  static_assert(!ONE || NT == kRouteThreads, "lists");
  extern __shared__ __attribute__((aligned(16))) int route_lds[];
  int* const n = route_lds;                        // [experts + 1]
  int* const wave_sums = n + kRouteMaxExperts + 1;  // [kRouteWaves]
  int* const kept = wave_sums + kRouteWaves;       // [kRouteKeptIds], ONE only
  int* const rest = kept + (ONE ? kRouteKeptIds : 0);
  const int tid = threadIdx.x, l = tid % L, team = tid / L;
  constexpr int TEAMS = NT / L;
  float* const shared = (float*)rest + team * (kRouteMaxGroups + p.experts);
  for (int e = tid; e <= p.experts; e += NT) n[e] = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * p.block_tokens;
  const int64_t t1 = t0 + p.block_tokens < p.tokens ? t0 + p.block_tokens : p.tokens;
  // the next token's logits are on their way while one is routed (65536 tokens over 128 experts, four rounds, with the packed keys and
  // whole pieces of logits: 18.2 -> 14.3 us)
  auto row_of = [&](int64_t t) { return (const T*)p.logits + t * p.ld; };
  T next[V];
  if (t0 + team < t1) route_load<T, WIDE, L, V>(row_of(t0 + team), p.experts, l, next);
  for (int64_t t = t0 + team; t < t1; t += TEAMS) {
    T raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = next[v];
    if (!ONE) route_load<T, WIDE, L, V>(row_of(t + TEAMS < t1 ? t + TEAMS : t), p.experts, l, next);
    else if (t + TEAMS < t1) route_load<T, WIDE, L, V>(row_of(t + TEAMS), p.experts, l, next);
    int id;
    float w;
    route_token<T, SIGMOID, PACKED, WIDE, L, V>(p, row_of(t), raw, l, shared, &id, &w);
    if (l < p.top_k) {
      const bool on = !p.mask || p.mask[t];
      p.ids[t * p.top_k + l] = on ? id : -1;
      if (ONE) kept[t * p.top_k + l] = on ? id : -1;
      p.weights[t * p.top_k + l] = on ? w : 0.f;
      if (on) atomicAdd(&n[id], 1);
    }
  }
  if constexpr (ONE) {
    route_scan(n, wave_sums, p.experts, tid);  // (its first barrier: the ids are kept)
    for (int e = tid; e <= p.experts; e += kRouteThreads) p.offsets[e] = n[e];
    const int slots = p.tokens * p.top_k;
    for (int s = n[p.experts] + tid; s < slots; s += kRouteThreads) p.order[s] = -1;
    route_place([&](int s) { return kept[s]; }, 0, slots, n, rest, p.experts, p.order, tid);
  } else {
    __syncthreads();
    for (int e = tid; e < p.experts; e += NT) p.counts[(int64_t)blockIdx.x * p.experts + e] = n[e];
  }
}

// The lists of several workgroups' tokens: each adds up the counts of all workgroups, for where the experts' lists begin, and of those before
// it, for where its own slots go.
__global__ __launch_bounds__(kRouteThreads) void moe_list_kernel(const RouteParams p) {
  extern __shared__ __attribute__((aligned(16))) int route_lds[];
  int* const n = route_lds;
  int* const wave_sums = n + kRouteMaxExperts + 1;
  int* const rest = wave_sums + kRouteWaves;
  const int tid = threadIdx.x, E = p.experts;
  const int64_t first = (int64_t)blockIdx.x * p.block_tokens * p.top_k, end = first + (int64_t)p.block_tokens * p.top_k;
  const int slots = p.tokens * p.top_k, s0 = (int)first, s1 = end < slots ? (int)end : slots;
  // this lane's first slot in route_place, requested together with the counts
  const int mine = s0 + (tid >> 6) * route_run(s0, s1) + (tid & 63), kept = mine < s1 ? p.ids[mine] : -1;
  // a thread adds up every SLICES-th workgroup's counts of one expert
  int pad = 64;
  while (pad < E) pad *= 2;
  const int slices = kRouteThreads / pad, e = tid & (pad - 1), slice = tid / pad;
  int all = 0, before = 0;
  if (e < E) {
#pragma unroll 16
    for (int b = slice; b < (int)gridDim.x; b += slices) {
      const int c = p.counts[(int64_t)b * E + e];
      all += c;
      before += b < (int)blockIdx.x ? c : 0;
    }
  }
  rest[tid] = all;
  rest[kRouteThreads + tid] = before;
  __syncthreads();
  all = before = 0;
  if (tid < E)
    for (int i = 0; i < slices; ++i) {
      all += rest[i * pad + tid];
      before += rest[kRouteThreads + i * pad + tid];
    }
  if (tid < E) n[tid] = all;
  route_scan(n, wave_sums, E, tid);
  if (blockIdx.x == 0)
    for (int i = tid; i <= E; i += kRouteThreads) p.offsets[i] = n[i];
  const int listed = n[E];
  __syncthreads();
  if (tid < E) n[tid] += before;
  for (int s = (s0 > listed ? s0 : listed) + tid; s < s1; s += kRouteThreads) p.order[s] = -1;
  route_place([&](int s) { return s == mine ? kept : p.ids[s]; }, s0, s1, n, rest, E, p.order, tid);
}

}  // namespace bolt
