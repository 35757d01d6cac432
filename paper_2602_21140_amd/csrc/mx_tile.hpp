// Grouped product of microscaled 4-bit activations and weights for many rows per expert: both operands through LDS.
//
// Same contract and the same results (bit for bit) as mx_stream_kernel (mx_stream.hpp).  A workgroup of 8 wavefronts (2 x 4)
// computes 256 x 256 outputs (EPI_H: 128 gate and the 128 up columns that go with them), a wavefront 128 x 64, in steps of 128
// K-elements.  Asynchronous copies bring a step's weights (16 KiB) three steps ahead through a ring of four stages, the
// activations of two steps (32 KiB) two to three steps ahead through two, and the scales of four steps (8 KiB) through two.
//
// What bounds it is the memory system: a CU's loads return in order, so that activations, which the L2 has, wait behind weights,
// which HBM has, and every request counts.  Two steps of activations at a time are 128 bytes of a row, a whole line: 16 KiB of
// weights from HBM and 16 KiB of activations from the L2 take 0.69 us (256 CUs together), with 64 bytes of a row at a time
// 0.85.  Results leave through LDS for the same reason, 64 or 128 bytes of a row by neighbouring lanes.
//
// us of the two products of 8192 tokens, 288 slots, H = 7168, I = 2048 (2.16e12 and 1.08e12 multiply-adds: 3.5 and 2.8 PFLOP/s;
// 4.5 and 2.2 GB of weights): 1240 and 780; the copies alone 1070 and 680, everything but the copies 860 and 600, and what a
// tile costs before its first and after its last step 210 and 320.  Weights that all slots share (so that no HBM is read) 1020
// and 600.
//
// LDS: weights lie in operand order, as in memory.  Activation row r is at r * 128 bytes, its 16-byte chunk c at chunk
// c ^ ((r >> 1) & 7): a fragment read (16 rows, four chunks) meets no bank twice in any of its four passes, whose lanes are 0-3,
// 12-15, 20-27 and so on.
#pragma once

#include "mx_stream.hpp"

namespace revive {

constexpr int kMxTile = 256;                  // rows, and weight rows, of a workgroup
constexpr int kMxStageA = kMxTile * 128;      // two steps
constexpr int kMxStageB = kMxTile * 64;       // a step
constexpr int kMxScales = 2 * kMxTile * 16;   // a group's scales: A's, then B's
constexpr int kMxLdsB = 2 * kMxStageA, kMxLdsScales = kMxLdsB + 4 * kMxStageB, kMxLdsOut = kMxLdsScales + 2 * kMxScales;
constexpr size_t kMxTileLds = kMxLdsOut + 8 * 2048;

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
  // nothing to a sum in fp32.  They cost what others do: K = 1408 takes 12 steps for 11, 576 8 for 5, 64 4 for 1.
  const int KT = NG * 4;
  const int rows = row_end - row_begin;

  // ---- copies.  Of two steps: four blocks of 8 rows of A per wavefront; of a step: two blocks of 16 weight rows; of a group's
  // scales: 64 rows of A's (wavefronts 0 to 3) or half a panel of B's (4 to 7).
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
  auto matrix = [&](int half, bool scales) {  // the workgroup's panel `half`: its first weights, or its first scales
    const int panel = EPI == EPI_H ? n_idx : min(n_idx * 2 + half, n_panels - 1);
    const uint8_t* m = B + (EPI == EPI_H && half ? g.b_half : 0);
    return reinterpret_cast<uint64_t>(scales ? m + g.b_codes + static_cast<int64_t>(panel) * NG * kMxPanelScales
                                             : m + static_cast<int64_t>(panel) * KR * kMxPanelStep);
  };
  uint32_t a_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = wave * 32 + i * 8 + (lane >> 3);
    a_off[i] = source(row) * static_cast<uint32_t>(g.a_row) + (((lane & 7) ^ swz(row)) << 4);
  }
  const int64_t first = g.src_of ? 0 : row_begin;  // the row that `source` counts from
  const int scale_row = mx_scale_row(g.K);
  const uint32_t s_off = wave < 4 ? source(wave * 64 + lane) * static_cast<uint32_t>(scale_row) : lane * 16;
  uint64_t base_a = uniform64(reinterpret_cast<uint64_t>(g.A) + first * g.a_row);
  uint64_t base_b = uniform64(matrix(wave >> 2, false) + (wave & 3) * 2048);
  uint64_t base_s = uniform64(wave < 4 ? reinterpret_cast<uint64_t>(g.A_scales) + first * scale_row : matrix((wave >> 1) & 1, true) + (wave & 1) * 1024);
  // Five wait states before a copy may read a scalar register that a vector instruction wrote.
  asm volatile("s_nop 4" : "+s"(base_a), "+s"(base_b), "+s"(base_s));
  const uint32_t s_step = wave < 4 ? 16 : kMxPanelScales;
  const uint32_t lane16 = lane * 16;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lptr)smem));
  auto to = [&](uint32_t at) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(lds0 + at))); };
  // Steps kt and kt + 1 (kt even, kt % 4 = PH) of A.
  auto copy_a = [&](int kt, auto ph_tag) {
    constexpr int PH = decltype(ph_tag)::value;
    const uint64_t src = base_a + static_cast<uint64_t>(min(kt, KR - 1) >> 1) * g.a_pair;
#pragma unroll
    for (int i = 0; i < 4; ++i) copy_to_lds_16B(to((PH >> 1) * kMxStageA + wave * 4096 + i * 1024), src, a_off[i]);
  };
  // Step kt (kt % 4 = PH) of B; with the first step of a group, its scales.
  auto copy_b = [&](int kt, auto ph_tag) {
    constexpr int PH = decltype(ph_tag)::value;
    const uint64_t src = base_b + static_cast<uint64_t>(min(kt, KR - 1)) * kMxPanelStep;
    if (PH == 0) copy_to_lds_16B(to(kMxLdsScales + ((kt >> 2) & 1) * kMxScales + wave * 1024), base_s + static_cast<uint64_t>(kt >> 2) * s_step, s_off);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_to_lds_16B(to(kMxLdsB + PH * kMxStageB + wave * 2048 + i * 1024), src + i * 1024, lane16);
  };

  // ---- fragments: immediate offsets below 64 KiB from the lane's places
  const unsigned char* fa0 = smem + (wm * 16 + r16) * 128 + ((kb ^ swz(r16)) << 4);        // even steps
  const unsigned char* fa1 = smem + (wm * 16 + r16) * 128 + (((kb + 4) ^ swz(r16)) << 4);  // odd steps
  const unsigned char* fb = smem + kMxLdsB + wn * (EPI == EPI_H ? 2048 : 4096) + lane * 16;
  const unsigned char* fs = smem + kMxLdsScales;
  constexpr int A_STEP = WAVES_M * 16 * 128;
  auto b_sub = [](int tn) { return EPI == EPI_H ? (tn >> 1) * 8 + (tn & 1) : tn; };
  auto frag = [](const unsigned char* p) { return *reinterpret_cast<const mx_u32x4*>(p); };
  // 16-row sub-tiles are dealt round-robin to the two wavefront rows; those without a valid row are not multiplied
  const int tm_valid = max(0, (((rows + 15) >> 4) - wm + WAVES_M - 1) / WAVES_M);

  auto run = [&](auto tmv_tag) {
    constexpr int TMV = decltype(tmv_tag)::value;
    constexpr int H0 = (TMV + 1) / 2, H1 = TMV / 2;
    mx_f32x4 acc[TM][TN];
#pragma unroll
    for (int tm = 0; tm < TMV; ++tm)
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
    mx_u32x4 af0[TM], af1[TM], bf[TN];
    uint32_t xs[TM], ws[TN];
    const uint32_t tail_mask = (KR & 3) ? (1u << (8 * (KR & 3))) - 1u : ~0u;  // A's scales past K are not written
    auto load_scales = [&](int q) {
      const unsigned char* p = fs + (q & 1) * kMxScales;
      const uint32_t mask = q == NG - 1 ? tail_mask : ~0u;
#pragma unroll
      for (int tm = 0; tm < TMV; ++tm) xs[tm] = *reinterpret_cast<const uint32_t*>(p + ((tm * WAVES_M + wm) * 16 + r16) * 16 + kb * 4) & mask;
#pragma unroll
      for (int tn = 0; tn < TN; ++tn)
        ws[tn] = *reinterpret_cast<const uint32_t*>(p + kMxTile * 16 + (wn * (EPI == EPI_H ? 2 : 4) + b_sub(tn)) * 256 + lane * 4);
    };
    // Step kt = 4 q + PH; left_tag: steps from this one to the last, as far as they matter here (8: enough).  Two phases: the first
    // half of the row sub-tiles times all column tiles, then the rest.  What a phase does not have yet is read while the one
    // before multiplies: phase 0 reads the second half's activations, phase 1, after the barrier that publishes the next step,
    // that step's first half and weights.
    auto step = [&](int kt, auto ph_tag, auto left_tag) {
      constexpr int PH = decltype(ph_tag)::value, LEFT = decltype(left_tag)::value, NX = (PH + 1) & 3;
      // Copies that may still be on their way at the barrier.  An even step needs the next step's weights: younger are four of A
      // and the weights of two steps; an odd one the next two steps' A too: the weights of two steps.  And scales among them.
      constexpr int VM = LEFT > 3 ? ((PH & 1) ? 4 : 8) + (PH == 1 || PH == 2) : LEFT > 2 ? 2 : 0;
      const unsigned char* pa = ((PH & 1) ? fa1 : fa0) + (PH >> 1) * kMxStageA;
      const unsigned char *na = ((NX & 1) ? fa1 : fa0) + (NX >> 1) * kMxStageA, *nb = fb + NX * kMxStageB;
      if (LEFT > 3) copy_b(kt + 3, std::integral_constant<int, (PH + 3) & 3>{});
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
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(VM));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // everybody is done with the step before this one, and with this one: an odd step's pair of stages is free
        if ((PH & 1) && LEFT > 3) copy_a(kt + 3, std::integral_constant<int, (PH + 3) & 3>{});
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
            load_scales((kt + 1) >> 2);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    if (TMV > 0) {
      load_scales(0);
#pragma unroll
      for (int tm = 0; tm < H0; ++tm) af0[tm] = frag(fa0 + tm * A_STEP);
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

    // A lane holds eight consecutive output columns 8 (l / 16) of activation row l % 16, in each set of 32 columns.
    if (EPI == EPI_H) {
      // the workgroup's 256 rows of 64 bytes; row r's 16-byte word w (wavefront column w) at word w ^ ((r >> 2) & 3)
      unsigned char* out = smem + kMxLdsOut;
#pragma unroll
      for (int tm = 0; tm < TMV; ++tm) {
        const int row = (tm * WAVES_M + wm) * 16 + r16;
        uint32_t byte;
        const uint32_t codes = mx_swiglu_codes(acc[tm][0], acc[tm][1], acc[tm][2], acc[tm][3], byte);
        *reinterpret_cast<uint32_t*>(out + row * 64 + ((wn ^ swz32(row)) << 4) + kb * 4) = codes;
        if (kb == 0 && row < rows) g.H_scales[static_cast<int64_t>(row_begin + row) * mx_scale_row(g.n_out) + mx_scale_at(n_idx * 4 + wn)] = static_cast<uint8_t>(byte);
      }
    } else {
      // 16 rows of 128 bytes at a time, in the wavefront's own part
      unsigned char* out = smem + kMxLdsOut + wave * 2048;
#pragma unroll
      for (int tm = 0; tm < TMV; ++tm) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const mx_f32x4 &v0 = acc[tm][2 * p], &v1 = acc[tm][2 * p + 1];
          const mx_u32x4 o = {pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
          *reinterpret_cast<mx_u32x4*>(out + r16 * 128 + (((p * 4 + kb) ^ swz(r16)) << 4)) = o;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = i * 8 + (lane >> 3), row = row_begin + (tm * WAVES_M + wm) * 16 + r, col = n_idx * 256 + wn * 64 + (lane & 7) * 8;
          const mx_u32x4 o = *reinterpret_cast<const mx_u32x4*>(out + r * 128 + (((lane & 7) ^ swz(r)) << 4));
          if (row < row_end && col < g.n_out) *reinterpret_cast<mx_u32x4*>(g.Y + static_cast<int64_t>(row) * g.n_out + col) = o;
        }
      }
    }
  };

  copy_a(0, std::integral_constant<int, 0>{});
  copy_b(0, std::integral_constant<int, 0>{});
  copy_b(1, std::integral_constant<int, 1>{});
  copy_a(2, std::integral_constant<int, 2>{});
  copy_b(2, std::integral_constant<int, 2>{});
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(8));  // the first step has landed
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  switch (tm_valid) {
    case 0: run(std::integral_constant<int, 0>{}); break;
    case 1: run(std::integral_constant<int, 1>{}); break;
    case 2: run(std::integral_constant<int, 2>{}); break;
    case 3: run(std::integral_constant<int, 3>{}); break;
    case 4: run(std::integral_constant<int, 4>{}); break;
    case 5: run(std::integral_constant<int, 5>{}); break;
    case 6: run(std::integral_constant<int, 6>{}); break;
    case 7: run(std::integral_constant<int, 7>{}); break;
    default: run(std::integral_constant<int, TM>{}); break;
  }
  if (EPI == EPI_H) {
    __syncthreads();
    const unsigned char* out = smem + kMxLdsOut;
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // four neighbouring lanes: the 64 bytes of a row
      const int row = i * 128 + (tid >> 2);
      const mx_u32x4 o = *reinterpret_cast<const mx_u32x4*>(out + row * 64 + (((tid & 3) ^ swz32(row)) << 4));
      if (row < rows) *reinterpret_cast<mx_u32x4*>(g.H + mx_h_at(n_idx, g.h_rows, row_begin + row) + (tid & 3) * 16) = o;
    }
  }
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
