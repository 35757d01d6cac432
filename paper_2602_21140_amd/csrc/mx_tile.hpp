// Grouped product of microscaled 4-bit activations and weights for many rows per expert: both operands through LDS.
//
// Same contract and the same results (bit for bit) as mx_stream_kernel (mx_stream.hpp).  A workgroup of 8 wavefronts (2 x 4)
// computes 256 x 256 outputs (EPI_H: 128 gate and the 128 up columns that go with them), a wavefront 128 x 64, in steps of 128
// K-elements.  A step's codes (32 KiB) come by asynchronous copies through a ring of four stages, three steps ahead; the
// scales of four steps (8 KiB) through two buffers of their own, once in four steps, a copy per wavefront.  Sums stay in
// registers and the results leave from there: the weights' row order (mx_row) gives a lane eight columns side by side.
//
// LDS: weights lie in operand order, as in memory.  Activation row r is at r * 64 bytes, its 16-byte chunk c at chunk
// c ^ ((r >> 2) & 3): a copy then fetches a row's 64 bytes with four neighbouring lanes, and the 16 rows of a fragment read
// cover all banks once.
#pragma once

#include "gemm_bf16.hpp"
#include "mx_stream.hpp"

namespace revive {

constexpr int kMxTile = 256;                       // rows, and weight rows, of a workgroup
constexpr int kMxStage = 2 * kMxTile * 64;         // bytes of a step: A, then B
constexpr int kMxScales = 2 * kMxTile * 16;        // bytes of a group's scales: A's, then B's
constexpr size_t kMxTileLds = 4 * kMxStage + 2 * kMxScales;

template <int EPI>
__global__ __launch_bounds__(512) void mx_tile_kernel(MxArgs a) {
  constexpr int TM = 8, TN = 4, WAVES_M = 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  typedef __attribute__((address_space(3))) void* lptr;
  const bool dense = blockIdx.x < static_cast<unsigned>(a.dense.blocks);
  const MxProblem g = dense ? a.dense : a.grouped;
  const int b = dense ? blockIdx.x : blockIdx.x - a.dense.blocks;
  int n_idx, row_begin, row_end;
  const uint8_t* B;
  if (dense) {
    // each XCD (workgroup i runs on XCD i % 8) takes a contiguous eighth of the tiles
    const int at = (b & 7) * (g.blocks >> 3) + (b >> 3);
    const int m_idx = at / g.n_col_tiles;
    n_idx = at - m_idx * g.n_col_tiles;
    row_begin = m_idx * kMxTile;
    row_end = min(g.M, row_begin + kMxTile);
    if (row_begin >= row_end) return;
    B = static_cast<const uint8_t*>(g.B_one);
  } else {
    const GridTile t = grid_tile(a.slot_offsets, a.P, kMxTile, g.n_col_tiles, b, g.B_tab);
    if (t.group < 0) return;
    n_idx = t.n_idx;
    row_begin = t.row_begin;
    row_end = t.row_end;
    B = static_cast<const uint8_t*>(t.w);
  }
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, kb = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int KR = mx_steps(g.K), NG = mx_groups(g.K);
  // Whole groups: steps past K repeat the last one with scales of 2^-127 on both sides, and products of 2^-249 at most add
  // nothing to a sum in fp32.
  const int KT = NG * 4;
  const int rows = row_end - row_begin;

  // ---- copies.  Of a step: two blocks of 16 weight rows and two of 16 rows of A per wavefront; of a group's scales: 64 rows
  // of A's (wavefronts 0 to 3) or half a panel of B's (4 to 7).
  auto source = [&](int r) -> uint32_t {  // row of A; rows past the tile read its last row again
    const int row = min(r, rows - 1);
    return g.src_of ? g.src_of[row_begin + row] / g.k : row;
  };
  auto uniform64 = [](uint64_t v) {
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32)));
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
    return (static_cast<uint64_t>(hi) << 32) | lo;
  };
  const int n_panels = (g.n_out + kMxPanel - 1) / kMxPanel;
  auto matrix = [&](int half) {  // where panel `half` of this workgroup begins: its first weights, and its first scales
    const int panel = EPI == EPI_H ? n_idx : min(n_idx * 2 + half, n_panels - 1);
    const uint8_t* m = B + (EPI == EPI_H && half ? g.b_half : 0);
    struct { const uint8_t *codes, *scales; } p = {m + static_cast<int64_t>(panel) * KR * kMxPanelStep, m + g.b_codes + static_cast<int64_t>(panel) * NG * kMxPanelScales};
    return p;
  };
  uint32_t a_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (wave * 2 + i) * 16 + (lane >> 2);
    a_off[i] = source(row) * static_cast<uint32_t>(g.a_row) + (((lane & 3) ^ swz32(row)) << 4);
  }
  const int64_t first = g.src_of ? 0 : row_begin;  // the row that `source` counts from
  uint64_t base_a = uniform64(reinterpret_cast<uint64_t>(g.A) + first * g.a_row);
  uint64_t base_b = uniform64(reinterpret_cast<uint64_t>(matrix(wave >> 2).codes) + (wave & 3) * 2048);
  const int scale_row = mx_scale_row(g.K);
  const uint32_t s_off = wave < 4 ? source(wave * 64 + lane) * static_cast<uint32_t>(scale_row) : lane * 16;
  uint64_t base_s = wave < 4 ? uniform64(reinterpret_cast<uint64_t>(g.A_scales) + first * scale_row)
                             : uniform64(reinterpret_cast<uint64_t>(matrix((wave >> 1) & 1).scales) + (wave & 1) * 1024);
  const uint32_t s_step = wave < 4 ? 16 : kMxPanelScales;
  const uint32_t lane16 = lane * 16;
  // Five wait states before a copy may read a scalar register that a vector instruction wrote.
  asm volatile("s_nop 4" : "+s"(base_a), "+s"(base_b), "+s"(base_s));
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lptr)smem));
  const uint32_t dst_a = __builtin_amdgcn_readfirstlane(lds0 + wave * 2048), dst_s = __builtin_amdgcn_readfirstlane(lds0 + 4 * kMxStage + wave * 1024);
  // Step kt into stage PH = kt % 4; with the first step of a group, its scales.
  auto copy = [&](int kt, auto ph_tag) {
    constexpr int PH = decltype(ph_tag)::value;
    const uint64_t k = min(kt, KR - 1);
    const uint64_t src_a = base_a + k * g.a_step, src_b = base_b + k * kMxPanelStep;
    if (PH == 0) copy_to_lds_16B(__builtin_amdgcn_readfirstlane(dst_s + ((kt >> 2) & 1) * kMxScales), base_s + static_cast<uint64_t>(kt >> 2) * s_step, s_off);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      copy_to_lds_16B(__builtin_amdgcn_readfirstlane(dst_a + PH * kMxStage + kMxTile * 64 + i * 1024), src_b + i * 1024, lane16);
      copy_to_lds_16B(__builtin_amdgcn_readfirstlane(dst_a + PH * kMxStage + i * 1024), src_a, a_off[i]);
    }
  };

  // ---- fragments: immediate offsets below 64 KiB from the lane's place in stage 0 or in stage 2
  const unsigned char* fa = smem + (wm * 16 + r16) * 64 + ((kb ^ swz32(r16)) << 4);
  const unsigned char* fb = smem + kMxTile * 64 + wn * (EPI == EPI_H ? 2048 : 4096) + lane * 16;
  const unsigned char* fs = smem + 4 * kMxStage;
  constexpr int A_STEP = WAVES_M * 16 * 64;
  auto b_sub = [](int tn) { return EPI == EPI_H ? (tn >> 1) * 8 + (tn & 1) : tn; };
  auto frag = [](const unsigned char* p) { return *reinterpret_cast<const mx_u32x4*>(p); };
  mx_f32x4 acc[TM][TN];
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
  // 16-row sub-tiles are dealt round-robin to the two wavefront rows; those without a valid row are not multiplied
  const int n_sub = (rows + 15) >> 4;
  const int tm_valid = max(0, (n_sub - wm + WAVES_M - 1) / WAVES_M);

  auto run = [&](auto tmv_tag, auto early_tag) {
    constexpr int TMV = decltype(tmv_tag)::value;
    constexpr bool EARLY = decltype(early_tag)::value;
    constexpr int H0 = (TMV + 1) / 2, H1 = TMV / 2;
    mx_u32x4 af0[TM], af1[TM], bf[TN];
    uint32_t xs[TM], ws[TN];
    const uint32_t tail_mask = (KR & 3) ? (1u << (8 * (KR & 3))) - 1u : ~0u;  // A's scales past K are not written
    auto load_scales = [&](int q, uint32_t* x, uint32_t* w) {
      const unsigned char* p = fs + (q & 1) * kMxScales;
      const uint32_t mask = q == NG - 1 ? tail_mask : ~0u;
#pragma unroll
      for (int tm = 0; tm < TMV; ++tm) x[tm] = *reinterpret_cast<const uint32_t*>(p + ((tm * WAVES_M + wm) * 16 + r16) * 16 + kb * 4) & mask;
#pragma unroll
      for (int tn = 0; tn < TN; ++tn)
        w[tn] = *reinterpret_cast<const uint32_t*>(p + kMxTile * 16 + (wn * (EPI == EPI_H ? 2 : 4) + b_sub(tn)) * 256 + lane * 4);
    };
    auto wait_barrier = [&](auto vm_tag) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(decltype(vm_tag)::value));
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    // Step kt = 4 q + PH.  Two phases: the first half of the row sub-tiles times all column tiles, then the rest.  What a phase
    // does not have yet is read while the one before multiplies: phase 0 reads the second half's activations, phase 1, after
    // the barrier that publishes the next step, that step's first half and weights.  The wavefronts that share a SIMD (w and
    // w + 4) issue their copies at different ends of the step, so that one's run under the other's MFMAs.
    // left_tag: steps from this one to the last, as far as they matter here (8: enough).
    auto step = [&](int kt, auto ph_tag, auto left_tag) {
      constexpr int PH = decltype(ph_tag)::value, LEFT = decltype(left_tag)::value;
      // copies that may still be on their way at the barrier: those of steps kt + 2 and kt + 3, and scales that go with one
      constexpr int VM = LEFT > 3 ? (PH == 1 || PH == 2 ? 9 : 8) : LEFT > 2 ? (PH == 2 ? 5 : 4) : 0;
      constexpr int NX = (PH + 1) & 3;
      const unsigned char* pa = fa + (PH >= 2 ? 2 * kMxStage : 0) + (PH & 1) * kMxStage;
      const unsigned char *na = fa + (NX >= 2 ? 2 * kMxStage : 0) + (NX & 1) * kMxStage, *nb = fb + (NX >= 2 ? 2 * kMxStage : 0) + (NX & 1) * kMxStage;
      if (EARLY && LEFT > 3) copy(kt + 3, std::integral_constant<int, (PH + 3) & 3>{});
      __builtin_amdgcn_sched_barrier(0);
      if (TMV > 0) {
#pragma unroll
        for (int i = 0; i < H0 * TN; ++i) {
          const int tn = i / H0, tm = (tn & 1) ? H0 - 1 - i % H0 : i % H0;
          acc[tm][tn] = mx_mfma<PH, PH>(bf[tn], af0[tm], acc[tm][tn], ws[tn], xs[tm]);
          if (i < H1) af1[i] = frag(pa + (H0 + i) * A_STEP);
        }
#pragma unroll
        for (int i = 0; i < H1; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, H0 * TN - H1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (LEFT > 1) {
        wait_barrier(std::integral_constant<int, VM>{});
        if (!EARLY && LEFT > 4) copy(kt + 4, ph_tag);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (TMV > 0) {
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) {
#pragma unroll
          for (int i = 0; i < H1; ++i) {
            const int tm = (tn & 1) ? H1 - 1 - i : i;
            acc[H0 + tm][tn] = mx_mfma<PH, PH>(bf[tn], af1[tm], acc[H0 + tm][tn], ws[tn], xs[H0 + tm]);
            if (LEFT > 1 && tn == 0) af0[i] = frag(na + i * A_STEP);
          }
          if (LEFT > 1 && tn == 0 && H0 > H1) af0[H0 - 1] = frag(na + (H0 - 1) * A_STEP);
          if (LEFT > 1) bf[tn] = frag(nb + b_sub(tn) * 1024);
        }
        if (LEFT > 1) {
#pragma unroll
          for (int i = 0; i < H1; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
          if (H0 > H1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
          for (int i = 1; i < TN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (H1 > 0) __builtin_amdgcn_sched_group_barrier(0x008, H1, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          if (PH == 3) {
            __builtin_amdgcn_sched_barrier(0);
            load_scales((kt + 1) >> 2, xs, ws);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    using P3 = std::integral_constant<int, 3>;
    if (!EARLY) copy(3, P3{});
    if (TMV > 0) {
      load_scales(0, xs, ws);
#pragma unroll
      for (int tm = 0; tm < H0; ++tm) af0[tm] = frag(fa + tm * A_STEP);
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) bf[tn] = frag(fb + b_sub(tn) * 1024);
    }
    using Enough = std::integral_constant<int, 8>;
    int kt = 0;
    for (; kt + 8 <= KT; kt += 4) mx_for(std::make_integer_sequence<int, 4>{}, [&](auto i) { step(kt + i.value, i, Enough{}); });
    mx_for(std::make_integer_sequence<int, 4>{}, [&](auto i) { step(kt + i.value, i, std::integral_constant<int, 4 - decltype(i)::value>{}); });
    // The sums are made here: without this the last products move down to the stores, under their conditions, and what they
    // are made of spills.
#pragma unroll
    for (int tm = 0; tm < TMV; ++tm)
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) asm volatile("" : "+v"(acc[tm][tn]));

    // a lane holds eight consecutive output columns of activation row l % 16
#pragma unroll
    for (int tm = 0; tm < TMV; ++tm) {
      const int row = row_begin + (tm * WAVES_M + wm) * 16 + r16;
      if (EPI == EPI_H) {
        uint32_t byte;
        const uint32_t codes = mx_swiglu_codes(acc[tm][0], acc[tm][1], acc[tm][2], acc[tm][3], byte);
        if (row >= row_end) continue;
        *reinterpret_cast<uint32_t*>(g.H + (static_cast<int64_t>(n_idx) * g.h_rows + row) * 64 + wn * 16 + kb * 4) = codes;
        if (kb == 0) g.H_scales[static_cast<int64_t>(row) * mx_scale_row(g.n_out) + mx_scale_at(n_idx * 4 + wn)] = static_cast<uint8_t>(byte);
      } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int col = n_idx * 256 + wn * 64 + p * 32 + kb * 8;
          if (row >= row_end || col >= g.n_out) continue;
          const mx_f32x4 &v0 = acc[tm][2 * p], &v1 = acc[tm][2 * p + 1];
          const mx_u32x4 o = {pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
          *reinterpret_cast<mx_u32x4*>(g.Y + static_cast<int64_t>(row) * g.n_out + col) = o;
        }
      }
    }
  };

  using Q0 = std::integral_constant<int, 0>;
  using Q1 = std::integral_constant<int, 1>;
  using Q2 = std::integral_constant<int, 2>;
  copy(0, Q0{});
  copy(1, Q1{});
  copy(2, Q2{});
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(8));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  auto pick = [&](auto early) {
    switch (tm_valid) {
      case 0: run(std::integral_constant<int, 0>{}, early); break;
      case 1: run(std::integral_constant<int, 1>{}, early); break;
      case 2: run(std::integral_constant<int, 2>{}, early); break;
      case 3: run(std::integral_constant<int, 3>{}, early); break;
      case 4: run(std::integral_constant<int, 4>{}, early); break;
      case 5: run(std::integral_constant<int, 5>{}, early); break;
      case 6: run(std::integral_constant<int, 6>{}, early); break;
      case 7: run(std::integral_constant<int, 7>{}, early); break;
      default: run(std::integral_constant<int, TM>{}, early); break;
    }
  };
  if (wave < 4) pick(std::true_type{});
  else pick(std::false_type{});
}

template <int EPI>
int launch_mx_tile(revive_ctx* ctx, const MxArgs& args, hipStream_t stream) {
  const int grid = args.dense.blocks + args.grouped.blocks;
  if (grid <= 0) return REVIVE_OK;
  auto kern = mx_tile_kernel<EPI>;
  REVIVE_HIP(ctx, allow_dynamic_lds(reinterpret_cast<const void*>(kern), kMxTileLds));
  hipLaunchKernelGGL(kern, dim3(grid), dim3(512), kMxTileLds, stream, args);
  return check_hip(ctx, hipGetLastError(), "mx_tile launch");
}

}  // namespace revive
