// The experts' products over many rows, on the two-wave-group ("ping-pong"), persistent scheme of fprop_pp_kernel: a 256 x 256 tile
// on 8 waves, group 0 (waves 0-3) and group 1 (waves 4-7) sharing the SIMDs pairwise; a wave alternates between a phase that reads
// fragments and issues direct-to-LDS loads and a phase of nothing but MFMAs, a workgroup barrier after every phase, group 1 one phase
// behind.  Stages, waits and the epilogue's LDS are as described there: W(t + 1) is loaded by group 0 in phase M(t), X(t + 2) by group 1;
// the first k-tiles of the next output tile go out before a tile's epilogue, which uses the stages they leave free.
//
// What differs: a workgroup finds its tiles from `offsets` (the host knows a bound of their number only); the activation rows may be
// gathered; with a gate the weight tile alternates 16 gate rows and the 16 value rows of the same columns, so that neighbouring
// fragments of a wave are the two factors of an output; results leave as halves in the list's order or as FP32 rows by slot.
// Tiles run in bands of 8 row blocks of an expert, and an XCD's 32 workgroups walk neighbouring tiles: a band's rows stay in its L2 while
// the expert's weights stream through.
// Measured: 8192 tokens to 6 of 64 experts, 2048 x 1024, gated: up 400 to 470 us (880 to 1030 TFLOP/s of what was asked for, 1.18 times that with the
// blocks' padding), down 280 to 310 us (670 to 740: 400 MB of FP32 rows leave it).  The matrix cores work 69 and 50 % of the cycles at 1.7 to 1.8 GHz,
// the L2s miss 31 and 37 % of the requests.  No effect: tiles from a counter instead of dealt out (7.1 rounds take 8), wave groups
// without rows that leave their MFMAs out, XCDs that start apart, rows stored from registers or through LDS.
#pragma once
#include <type_traits>
#include <utility>

#include "fprop_pp_kernel.hpp"
#include "routed_rows.hpp"

namespace bolt {

template <int MODE, bool GATED>
__global__ __launch_bounds__(512) void moe_pp_kernel(const RowsParams p) {
  using T = FpropPpTraits;
  constexpr int BM = 256, BN = T::BN, BK = T::BK, WTM = BM / 2, WTN = T::WTN;
  constexpr int FM = WTM / 16, FN = WTN / 16, KS = BK / 32;
  constexpr int L = 8;  // load instructions per k-tile of a wave: 4 waves x 8 rows of 256 each
  constexpr int COLS = GATED ? BN / 2 : BN;
  constexpr bool FLOATS = MODE == ROWS_DOWN;

  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  half_t* const wring = lds;
  half_t* const xring = lds + T::W_STAGES * T::W_HALVES;
  half_t* const free0 = wring + T::W_HALVES;
  half_t* const free1 = xring + 2 * T::X_HALVES;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2, wq = wave & 3;
  const int g = lane >> 4, lr = lane & 15;
  const int n_tiles = (p.K + BK - 1) / BK;
  const int outputs = GATED ? p.hidden : p.N;

  BlockCounts counts;
  if constexpr (MODE != ROWS_DENSE) counts = count_row_blocks<BM>(p.offsets, p.experts, lane);
  const int total = (MODE == ROWS_DENSE ? p.row_blocks : counts.total()) * p.col_blocks;

  // ---- this wave's loader: rows (j * 4 + wq) * 8 + lane / 8 of ONE operand tile, one byte offset per row ---------------------
  const int lrow = lane >> 3;
  const int lc16 = ((lane & 7) ^ dma_swizzle<BK>(wq * 8 + lrow)) << 4;
  unsigned st[L];
  __amdgpu_buffer_rsrc_t rsrc;
  const int k_limit_bytes = p.K * 2;
  // An output tile.  The next one is looked up while the first loads of a tile are on their way, not between two tiles.
  struct Tile {
    int expert, row0, rows, c0;
  };
  auto find_tile = [&](int id) {
    const int tile = xcd_run(id, total);
    RowBlock at = {0, 0, p.M, 0, p.row_blocks};
    if constexpr (MODE != ROWS_DENSE) find_row_block<BM>(p.offsets, counts, tile / p.col_blocks, &at);  // (tile < total)
    // bands of 8 row blocks, in a band the row block fastest
    const int local = tile - at.first * p.col_blocks, band = local / (8 * p.col_blocks), in_band = local - band * 8 * p.col_blocks;
    const int height = at.count - band * 8 < 8 ? at.count - band * 8 : 8;
    const int cb = in_band / height, block = band * 8 + in_band - cb * height;
    return Tile{at.expert, at.lo + block * BM, at.n - block * BM < BM ? at.n - block * BM : BM, cb * COLS};
  };
  // UP: the byte offset of one row of the tile's tokens per lane, of those this wave loads: row (lane / 8 * 4 + wq) * 8 + lane % 8.
  auto find_row = [&](const Tile& t) {
    const int r = (lane >> 3) * 32 + wq * 8 + (lane & 7);
    const unsigned token = (unsigned)(p.order[t.row0 + (r < t.rows ? r : t.rows - 1)] / p.top_k);
    return r < t.rows ? token * (unsigned)(p.ldx * 2) : kInvalidOffset;
  };
  Tile cur, next;
  unsigned next_row = 0;
  auto setup_tile = [&](const Tile& t, unsigned row) {
    if (grp == 0) {
      rsrc = make_rsrc(p.w + t.expert * p.w_stride, (unsigned)p.w_stride);
#pragma unroll
      for (int j = 0; j < L; ++j) {
        const int r = (j * 4 + wq) * 8 + lrow;
        const int c = GATED ? t.c0 + (r >> 5) * 16 + (r & 15) : t.c0 + r;
        st[j] = c < outputs ? (unsigned)(c + (GATED && (r & 16) ? p.hidden : 0)) * (unsigned)(p.K * 2) : kInvalidOffset;
      }
    } else if (MODE == ROWS_UP) {
      rsrc = make_rsrc(p.x, 0x7fffffffu);  // (the host keeps x below 2 GiB)
#pragma unroll
      for (int j = 0; j < L; ++j) st[j] = (unsigned)__shfl((int)row, j * 8 + lrow);
    } else {
      rsrc = make_rsrc(p.x + (int64_t)t.row0 * p.ldx, (unsigned)(((int64_t)(t.rows - 1) * p.ldx + p.K) * 2));
#pragma unroll
      for (int j = 0; j < L; ++j) {
        const int r = (j * 4 + wq) * 8 + lrow;
        st[j] = r < t.rows ? (unsigned)(r * p.ldx * 2) : kInvalidOffset;
      }
    }
  };
  auto issue_one = [&](auto jc, int kt, half_t* dst) {
    constexpr int j = decltype(jc)::value;
    half_t* slot = dst + (j * 4) * 8 * BK + wq * 8 * BK;
    unsigned sj = st[j];  // (the empty asm: see fprop_pp_kernel, nothing derived from it is to live through the k loop)
    asm volatile("" : "+v"(sj));
    const int kb = kt * (BK * 2) + lc16;
    const unsigned off = (sj + (unsigned)kb) | (kb < k_limit_bytes ? 0u : kInvalidOffset);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, BOLT_LDS_PTR(slot), 16, off, 0, 0, 0);
  };
  auto issue_first_tiles = [&]() {
    if (grp == 0) {
      for_constants<L>([&](auto jc) { issue_one(jc, 0, wring); });
    } else {
      for_constants<L>([&](auto jc) { issue_one(jc, 0, xring); });
      for_constants<L>([&](auto jc) { issue_one(jc, 1, xring + T::X_HALVES); });
    }
  };

  floatx4 acc[FN][FM];
  half8 xf[KS][FM], wf[KS][FN];
  constexpr int NREAD = KS * (FM + FN);
  auto read_one = [&](const half_t* xs, const half_t* ws, auto rc) {
    constexpr int r = decltype(rc)::value, k = r / (FM + FN), i = r % (FM + FN);
    const int chunk = k * 4 + g;
    if constexpr (i < FM) xf[k][i] = *(const half8*)(xs + dma_chunk_offset<BK>(grp * WTM + i * 16 + lr, chunk));
    else wf[k][i - FM] = *(const half8*)(ws + dma_chunk_offset<BK>(wq * WTN + (i - FM) * 16 + lr, chunk));
  };
  auto m_phase = [&](half_t* dst, int kt, const half_t* xs, const half_t* ws) {
    for_constants<L>([&](auto jc) {
      constexpr int j = decltype(jc)::value, r0 = j * NREAD / L, r1 = (j + 1) * NREAD / L;
      issue_one(jc, kt, dst);
      for_constants<r1 - r0>([&](auto ic) { read_one(xs, ws, std::integral_constant<int, r0 + decltype(ic)::value>{}); });
    });
    for_constants<L>([&](auto jc) {
      constexpr int j = decltype(jc)::value;
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                            // one load
      __builtin_amdgcn_sched_group_barrier(0x100, (j + 1) * NREAD / L - j * NREAD / L, 0);  // its share of reads
    });
  };
  auto c_phase = [&]() {
    for_constants<KS * FM * FN>([&](auto ic) {
      constexpr int i = decltype(ic)::value, k = i / (FM * FN), a = (i / FM) % FN, b = i % FM;
      acc[a][b] = mfma_16x16x32(wf[k][a], xf[k][b], acc[a][b]);
    });
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto wait_reads = [] { __builtin_amdgcn_s_waitcnt(0xC07F); };          // lgkmcnt(0)
  auto wait_loads_0 = [] { __builtin_amdgcn_s_waitcnt(0x0F70); };        // vmcnt(0)
  auto wait_loads_x = [] { __builtin_amdgcn_s_waitcnt(0x0F70 | L); };    // vmcnt(L): all but the newest activation tile

  // The accumulators of a tile start at the bias.
  half4 bias_q[FN];
  auto column = [&](int a, int gl) { return GATED ? wq * (WTN / 2) + (a >> 1) * 16 + gl * 4 : wq * WTN + a * 16 + gl * 4; };
  auto load_bias = [&](const Tile& t) {
#pragma unroll
    for (int a = 0; a < FN; ++a) {
      const int c = t.c0 + column(a, g), n = (c < outputs ? c : 0) + (GATED && (a & 1) ? p.hidden : 0);
      bias_q[a] = *(const half4*)(p.bias + (t.expert * (int64_t)p.N + n) * p.bias_on);
    }
  };

  // Halves: a wave group moves its rows through its own free stage (32 KB), R at a time, so that whole row segments are stored.
  // Floats (DOWN): a quad per lane straight to the slot's row, 64 bytes of a row by four lanes; slot[b] is that of row 16 b + lane % 16.
  auto epilogue = [&](const Tile& t, const int (&slot)[FM]) {
    int elane = lane;
    asm volatile("" : "+v"(elane));  // (as in fprop_pp_kernel: the addresses below are not to live through the k loop)
    const int eg = elane >> 4, elr = elane & 15, gtid = wq * 64 + elane, r_half = grp * WTM;
    if constexpr (FLOATS) {
#pragma unroll
      for (int b = 0; b < FM; ++b) {
        if (r_half + b * 16 + elr >= t.rows) continue;
        float* const to = (float*)p.y + (int64_t)slot[b] * p.ldy;
#pragma unroll
        for (int a = 0; a < FN; ++a) {
          const int c = t.c0 + column(a, eg);
          if (c < outputs) *(floatx4*)(to + c) = acc[a][b];
        }
      }
      return;
    }
    half_t* const stage = grp == 0 ? free0 : free1;
    constexpr int R = (GATED ? 128 : 64) < WTM ? (GATED ? 128 : 64) : WTM;
    constexpr int CPR = COLS / 8;  // 16-byte chunks of a row
    for_constants<WTM / R>([&](auto sc) {
      constexpr int sp = decltype(sc)::value;
      barrier_after_lds_writes();
#pragma unroll
      for (int a = 0; a < FN; a += GATED ? 2 : 1)
#pragma unroll
        for (int bb = 0; bb < R / 16; ++bb) {
          const int b = sp * (R / 16) + bb, srow = bb * 16 + elr, nl = column(a, eg);
          floatx4 v = acc[a][b];
          if constexpr (MODE == ROWS_DENSE) v *= p.alpha;
          v = apply_act4(v, p.act);
          if constexpr (GATED) v *= acc[a + 1][b];
          half4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (half_t)v[e];
          *(half4*)(stage + srow * COLS + (((nl >> 3) ^ ctile_swizzle<CPR>(srow)) << 3) + (nl & 4)) = o;
        }
      barrier_after_lds_writes();
      const int chunk = gtid % CPR, first = gtid / CPR, c = t.c0 + chunk * 8;
      if (c < outputs) {
#pragma unroll
        for (int i = 0; i < R * CPR / 256; ++i) {
          const int srow = first + i * (256 / CPR), r = r_half + sp * R + srow;
          if (r < t.rows)
            *(half8*)((half_t*)p.y + (int64_t)(t.row0 + r) * p.ldy + c) = *(const half8*)(stage + srow * COLS + ((chunk ^ ctile_swizzle<CPR>(srow)) << 3));
        }
      }
    });
  };

  int tile = blockIdx.x;
  if (tile >= total) return;
  cur = find_tile(tile);
  setup_tile(cur, MODE == ROWS_UP ? find_row(cur) : 0);
  load_bias(cur);
  issue_first_tiles();
  while (true) {
    const bool more = tile + (int)gridDim.x < total;
    if (more) {
      next = find_tile(tile + gridDim.x);
      if (MODE == ROWS_UP && grp == 1) next_row = find_row(next);
    }
    if (grp == 0) wait_loads_0();
    else wait_loads_x();
    wait_reads();
    const float bias_scale = MODE == ROWS_DENSE ? p.beta / p.alpha : 1.f;  // (the host keeps it finite)
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
      for (int b = 0; b < FM; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][b][e] = (float)bias_q[a][e] * bias_scale;
    raw_barrier();
    if (grp == 1) raw_barrier();
    int ws_cur = 0, xs_cur = 0;
    for (int t = 0; t < n_tiles; ++t) {
      const int ws_next = ws_cur ^ 1;
      const int xs_fill = xs_cur == 0 ? 2 : xs_cur - 1;
      const half_t* xs = xring + xs_cur * T::X_HALVES;
      const half_t* ws = wring + ws_cur * T::W_HALVES;
      fence();
      // both groups run the same code on their own rows, offsets and stage
      m_phase(grp == 0 ? wring + ws_next * T::W_HALVES : xring + xs_fill * T::X_HALVES, t + 1 + grp, xs, ws);
      wait_reads();
      if (grp == 1) wait_loads_x();  // X(t + 1) has landed
      fence();
      raw_barrier();
      fence();
      __builtin_amdgcn_s_setprio(1);
      c_phase();
      __builtin_amdgcn_s_setprio(0);
      if (grp == 0) wait_loads_0();  // W(t + 1) has landed
      fence();
      raw_barrier();
      ws_cur = ws_next;
      xs_cur = xs_cur == 2 ? 0 : xs_cur + 1;
    }
    if (grp == 0) raw_barrier();
    // nothing of this workgroup is on its way into LDS any more, and nobody reads a stage
    wait_loads_0();
    raw_barrier();
    int slot[FM];  // (requested ahead of the next tile's operands, which they would have to wait for)
    if constexpr (FLOATS) {
      int elane = lane;
      asm volatile("" : "+v"(elane));
#pragma unroll
      for (int b = 0; b < FM; ++b) {
        const int r = grp * WTM + b * 16 + (elane & 15);
        slot[b] = p.order[cur.row0 + (r < cur.rows ? r : cur.rows - 1)];
      }
    }
    if (more) {
      setup_tile(next, next_row);
      load_bias(next);
      issue_first_tiles();
    }
    epilogue(cur, slot);
    tile += gridDim.x;
    cur = next;
    if (!more) break;
  }
}

template <int MODE, bool GATED>
hipError_t launch_moe_pp(RowsParams p, hipStream_t stream) {
  auto kern = moe_pp_kernel<MODE, GATED>;
  static LdsOptIn opt_in;
  if (hipError_t e = opt_in.ensure((const void*)kern, FpropPpTraits::LDS_BYTES); e != hipSuccess) return e;
  constexpr int COLS = GATED ? FpropPpTraits::BN / 2 : FpropPpTraits::BN, kComputeUnits = 256;
  p.col_blocks = ((GATED ? p.hidden : p.N) + COLS - 1) / COLS;
  p.row_blocks = row_blocks<256>(p, MODE);
  const int64_t most = (int64_t)p.row_blocks * p.col_blocks;
  hipLaunchKernelGGL(kern, dim3((unsigned)(most < kComputeUnits ? most : kComputeUnits)), dim3(512), FpropPpTraits::LDS_BYTES, stream, p);
  return hipGetLastError();
}

}  // namespace bolt
