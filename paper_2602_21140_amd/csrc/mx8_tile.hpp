// Product of microscaled 8-bit activations and weights for many rows: both operands through LDS.
//
// A workgroup of 8 wavefronts (2 x 4) computes 256 x 64 TN outputs (EPI8_H: half as many columns, gate and up of each), a
// wavefront 128 x 16 TN, in steps of 128 K-elements.  Asynchronous copies bring the steps' operands into two stages.
//
// A step goes through its row sub-tiles in four pairs: while one is multiplied the next one's activations are read from LDS, and
// during the last pair the next step's weights, all of them, and first activations.  So a stage is done with piece by piece, and
// each piece is filled again at once, a step and a half before it is needed: at barrier X, after the first pair, the weights and
// the activations of the first two pairs (everybody has read them), at barrier Y, after the third, those of the other two.  Each
// barrier also publishes what was ordered a step and a half before; what was ordered since stays on its way.  With one barrier a
// step, everything ordered at once, the copies and the products took turns (8192 x 7168 x 7168 488 us, with the second barrier 424, with
// the copies ordered one by one between the products 398, with bias and residual asked for early 380).
//
// What bounds it: 8192 x 7168 x 7168 takes 376 us, 2.24 PFLOP/s; 896 tiles are 3.5 rounds of the 256 CUs, and a step of a whole round takes 1.6 us, of
// which the matrix instructions alone, on a chip that they fill, take 1.4 (power: on a quarter of the CUs they take 1.1).
// With fewer workgroups than CUs a step still takes 1.0 us (TN = 2: 0.7 to 0.9), as long as LDS is read: 192 KiB of operands (160) and
// 64 KiB of copies (48) at 128 bytes a cycle.  A third stage, tiles of 128 x 128 with four stages and one barrier: the same within 10 %, but for
// 190 to 256 such tiles (512 x 7168 x 7168: 45 instead of 54 us).
//
// LDS: weights lie in operand order, as in memory.  Activation row r is at r * 128 bytes, its 16-byte chunk c at chunk
// c ^ ((r >> 1) & 7): a fragment read (16 rows, four chunks) meets no bank twice in any of its four passes.  A step's scales of
// the weights come with them, those of the activations for four steps at a time.
#pragma once

#include "mx8_product.hpp"

namespace revive {

// As copy_to_lds_16B, past the caches' retention: for weights that one workgroup, or a few at the same time, read.
__device__ __forceinline__ void mx8_copy_once(uint32_t dst, uint64_t src, uint32_t off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(off), "s"(src), "s"(dst) : "memory", "m0");
}

constexpr int kMx8Tile = 256;  // rows of a workgroup
template <int TN>
struct Mx8TileShape {
  static constexpr int TM = 8, BM = kMx8Tile, BN = 64 * TN, PANELS = BN / kMx8Panel;
  static constexpr int STAGE_A = BM * kMx8Step, STAGE_B = BN * kMx8Step, STAGE_WS = PANELS * kMx8PanelScales, STAGE_XS = BM * 16;
  static constexpr int B = 2 * STAGE_A, WS = B + 2 * STAGE_B, XS = WS + 2 * STAGE_WS;
  static constexpr size_t LDS = XS + 2 * STAGE_XS;
};

// Whether a product's rows of scales can be copied by words, four steps at a time.
inline bool mx8_word_scales(const Mx8Problem& p) {
  return p.K % kMx8Step == 0 && p.K >= 4 * kMx8Step && reinterpret_cast<uintptr_t>(p.A_scales) % 4 == 0;
}

// WORD_SCALES: both problems' are (mx8_word_scales).  Otherwise they go through registers, a step's at a time: loads that the
// compiler waits for, and every copy with them, so that what was ordered since the last step does not stay on its way.
template <int TN, int EPI, bool WORD_SCALES>
__global__ __launch_bounds__(512, 2) void mx8_tile_kernel(Mx8Args a) {
  using S = Mx8TileShape<TN>;
  constexpr int TM = S::TM;
  static_assert((TN == 2 || TN == 4) && (EPI != EPI8_H || TN == 4), "whole panels");
  // K is two blocks at least, a row of A can be reached by 32 bits: the host sees to it.
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  typedef __attribute__((address_space(3))) void* lptr;
  const bool dense = blockIdx.x < static_cast<unsigned>(a.dense.blocks);
  const Mx8Problem g = dense ? a.dense : a.grouped;
  const Mx8Tile t = mx8_tile_of(a, g, dense, S::BM);
  if (t.row_begin >= t.row_end) return;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, kb = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int KT = mx8_steps(g.K), k_blocks = g.K / kMx8Block;
  const int rows = t.row_end - t.row_begin;

  // ---- copies of a step, by each wavefront: of either half of A's rows, 16, 8 at a time; of B, an eighth of the panels and of
  // their scales
  constexpr int CP_B = S::STAGE_B / 8192;
  auto source = [&](int r) -> int64_t {  // row of A; rows past the tile read its last row again
    const int row = min(r, rows - 1);
    return g.src_of ? g.src_of[t.row_begin + row] / g.k : row;
  };
  const int64_t first = g.src_of ? 0 : t.row_begin;  // the row that `source` counts from
  const int left = g.K & (kMx8Step - 1);             // K-elements of a last step that is not whole
  // copy i of A: rows 128 (i / 2) + 16 wave + 8 (i % 2) + l / 8
  auto a_row = [&](int i) { return (i >> 1) * 128 + wave * 16 + (i & 1) * 8; };
  auto a_chunk = [&](int i) { return (lane & 7) ^ swz((i & 1) * 8 + (lane >> 3)); };  // that the copy puts where the lane's 16 bytes go
  uint32_t a_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) a_off[i] = static_cast<uint32_t>(source(a_row(i) + (lane >> 3)) * g.a_row) + (a_chunk(i) << 4);
  const int n_panels = (g.n_out + kMx8Panel - 1) / kMx8Panel;
  auto matrix = [&](int p) {  // the workgroup's panel p
    return EPI == EPI8_H ? t.n_idx : min(t.n_idx * S::PANELS + p, n_panels - 1);
  };
  constexpr int WAVES_A_PANEL = 8 / S::PANELS;
  const int own_panel = wave / WAVES_A_PANEL;
  uint64_t base_a = mx8_uniform(reinterpret_cast<uint64_t>(g.A) + first * g.a_row);
  uint64_t base_b = mx8_uniform(reinterpret_cast<uint64_t>(t.B) + (EPI == EPI8_H && own_panel ? g.b_half : 0) +
                              static_cast<int64_t>(matrix(own_panel)) * KT * kMx8PanelStep + (wave % WAVES_A_PANEL) * (CP_B * 1024));
  // of the scales, lanes 0 to 31 take the first panel's, the others the second's; a wavefront 8 / PANELS of each
  constexpr int WS_LANES = 4 * S::PANELS;
  const int ws_lane = wave * WS_LANES + (lane & (WS_LANES - 1));
  const uint32_t ws_off = static_cast<uint32_t>(ws_lane >= 32 ? (EPI == EPI8_H ? g.b_half : static_cast<int64_t>(matrix(1) - matrix(0)) * KT * kMx8PanelScales) : 0) + (ws_lane & 31) * 16;
  uint64_t base_ws = mx8_uniform(reinterpret_cast<uint64_t>(t.B) + g.b_codes + static_cast<int64_t>(matrix(0)) * KT * kMx8PanelScales);
  const uint32_t xs_off = static_cast<uint32_t>(source(wave * 32 + (lane & 31)) * k_blocks);
  uint64_t base_xs = mx8_uniform(reinterpret_cast<uint64_t>(g.A_scales) + first * k_blocks);
  // Five wait states before a copy may read a scalar register that a vector instruction wrote.
  asm volatile("s_nop 4" : "+s"(base_a), "+s"(base_b), "+s"(base_ws), "+s"(base_xs));
  const uint32_t lane16 = lane * 16;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lptr)smem));
  auto to = [&](uint32_t at) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(lds0 + at))); };
  // Copy i of A (0, 1: of the first half of the rows), copy i of B, a step's scales of B.
  auto copy_a = [&](int kt, int stage, int i) {
    // chunks past the row: the step's first one instead, cleared below
    const int end = left && kt == KT - 1 ? left : kMx8Step;
    const uint32_t off = a_chunk(i) * 16 >= end ? a_off[i] - (a_chunk(i) << 4) : a_off[i];
    copy_to_lds_16B(to(stage * S::STAGE_A + a_row(i) * 128), base_a + static_cast<uint64_t>(kt) * kMx8Step, off);
  };
  auto copy_b = [&](int kt, int stage, int i) {
    const uint32_t dst = to(S::B + stage * S::STAGE_B + (wave * CP_B + i) * 1024);
    const uint64_t src = base_b + static_cast<uint64_t>(kt) * kMx8PanelStep + i * 1024;
    if (EPI == EPI8_LINEAR) copy_to_lds_16B(dst, src, lane16);
    else mx8_copy_once(dst, src, lane16);  // 279 slots of 228 rows 3690 -> 3610 us, 108 slots of 450 2560 -> 2510, 12 of 1400 the same
  };
  auto copy_ws = [&](int kt, int stage) {
    if (lane < WS_LANES) copy_to_lds_16B(to(S::WS + stage * S::STAGE_WS + wave * (WS_LANES * 16)), base_ws + static_cast<uint64_t>(kt) * kMx8PanelScales, ws_off);
  };
  constexpr int CP_X = 2 + CP_B + 1, CP_Y = 2;  // copies that a wavefront orders after either barrier
  auto copy_x = [&](int kt, int stage, int n) {  // number n of X's
    if (n < 2) copy_a(kt, stage, n);
    else if (n < 2 + CP_B) copy_b(kt, stage, n - 2);
    else if (n < CP_X) copy_ws(kt, stage);
  };
  auto copy_y = [&](int kt, int stage, int n) { copy_a(kt, stage, 2 + n); };
  // ---- scales of the activations.  WORD_SCALES: group q (steps 4 q to 4 q + 3), 16 bytes a row, in one of two places; the last
  // group is the row's last 16 bytes.
  auto xs_from = [&](int q) { return min(q * 16, k_blocks - 16); };
  auto copy_xs = [&](int q) {
    if (lane < 32) copy_to_lds_16B(to(S::XS + (q & 1) * S::STAGE_XS + wave * 512), base_xs + xs_from(q), xs_off);
  };
  // Otherwise: a thread half of a row's four bytes of a step, zeros past the row's end, in one of four places.
  const uint8_t* xs_row = g.A_scales + (first + source(tid >> 1)) * k_blocks;
  auto load_xs = [&](int kt) -> uint32_t {
    typedef uint16_t any __attribute__((aligned(1)));
    const int at = min(kt * 4 + (tid & 1) * 2, k_blocks + 1), from = min(at, k_blocks - 2);
    return static_cast<uint32_t>(*reinterpret_cast<const __attribute__((address_space(1))) any*>(reinterpret_cast<uintptr_t>(xs_row + from))) >> (8 * (at - from));
  };
  auto store_xs = [&](int kt, uint32_t w) { *reinterpret_cast<uint16_t*>(smem + S::XS + (kt & 3) * (S::STAGE_XS / 4) + tid * 2) = static_cast<uint16_t>(w); };
  // Where step kt's four scales are, from row 0's first.
  constexpr int XS_ROW = WORD_SCALES ? 16 : 4;
  auto xs_at = [&](int kt) { return WORD_SCALES ? ((kt >> 2) & 1) * S::STAGE_XS + kt * 4 - xs_from(kt >> 2) : (kt & 3) * (S::STAGE_XS / 4); };
  // The last step's chunks past the row, of this wavefront's own copies, once these have landed.
  auto clear_rest = [&](int stage, int half) {
#pragma unroll
    for (int i = 2 * half; i < 2 * half + 2; ++i)
      if (a_chunk(i) * 16 >= left) *reinterpret_cast<mx8_u32x4*>(smem + stage * S::STAGE_A + a_row(i) * 128 + lane16) = mx8_u32x4{0u, 0u, 0u, 0u};
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
  };

  // ---- fragments: immediate offsets below 64 KiB from the lane's places
  const unsigned char* fa0 = smem + (wm * 16 + r16) * 128 + ((kb ^ swz(r16)) << 4);        // first halves
  const unsigned char* fa1 = smem + (wm * 16 + r16) * 128 + (((kb + 4) ^ swz(r16)) << 4);  // second halves
  const unsigned char* fb = smem + S::B + (EPI == EPI8_H ? wn * 2 : wn * TN) * 2048 + lane16;
  const unsigned char* fx = smem + S::XS + (wm * 16 + r16) * XS_ROW + kb;
  auto b_block = [](int tn) { return EPI == EPI8_H ? (tn >> 1) * 8 + (tn & 1) : tn; };
  auto frag16 = [](const unsigned char* p) { return *reinterpret_cast<const mx8_u32x4*>(p); };
  auto load_ws = [&](int stage) -> uint32_t {  // bytes: the scales of the wavefront's 16-row blocks
    const unsigned char* p = smem + S::WS + stage * S::STAGE_WS + lane * 8;
    if (EPI == EPI8_H) return *reinterpret_cast<const uint16_t*>(p + wn * 2) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p + kMx8PanelScales + wn * 2)) << 16;
    if (TN == 2) return *reinterpret_cast<const uint16_t*>(p + wn * 2);
    return *reinterpret_cast<const uint32_t*>(p + (wn >> 1) * kMx8PanelScales + (wn & 1) * 4);
  };
  // 16-row sub-tiles are dealt round-robin to the two wavefront rows; of the four pairs none, two or all are multiplied
  const int pairs = max(0, ((((rows + 15) >> 4) - wm + 1) / 2 + 1) / 2);

  mx8_f32x4 acc[TM][TN];
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = mx8_f32x4{0.f, 0.f, 0.f, 0.f};
  // The pair's sums are made here: without this their products move down past the barriers, with all that they need.
  auto pin = [&](auto q) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) {
        mx8_f32x4& sum = acc[2 * q.value + i][tn];
        asm volatile("" : "+v"(sum));
      }
  };

  // Rows that all are of the first half: the other one is not copied.
  const bool half = rows <= S::BM / 2;
  auto run = [&](auto q_tag, auto half_tag) {
    constexpr int Q = decltype(q_tag)::value, Y = decltype(half_tag)::value ? 0 : CP_Y;  // even: a step ends with the second buffer of activations, and the next one begins with the first
    Mx8Frag af[2][2], bf[TN];
    uint32_t xs[2][2], ws = 0, xw = 0;
    auto read_a = [&](int q, int stage, int x_at, Mx8Frag* f, uint32_t* x) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[i] = mx8_frag(frag16(fa0 + stage * S::STAGE_A + (2 * q + i) * 4096), frag16(fa1 + stage * S::STAGE_A + (2 * q + i) * 4096));
        x[i] = fx[x_at + (2 * q + i) * (32 * XS_ROW)];
      }
    };
    auto read_b = [&](int tn, int stage) {
      const unsigned char* p = fb + stage * S::STAGE_B + b_block(tn) * 2048;
      bf[tn] = mx8_frag(frag16(p), frag16(p + 1024));
    };
    // Step kt, in stage kt % 2; MORE: there are two steps behind it.  Copies go out one at a time between the products: ordered
    // all at once behind the barrier they held the wavefronts up.
    auto step = [&](int kt, auto more_tag) {
      const int now = kt & 1, next = now ^ 1;
      constexpr bool MORE = decltype(more_tag)::value;
      const int x_at = xs_at(kt);
      auto pair = [&](auto q_at, auto between) {  // multiply pair q, read the next one
        constexpr int q = decltype(q_at)::value;
        read_a(q + 1, now, x_at, af[(q + 1) & 1], xs[(q + 1) & 1]);
        mx8_for_blocks<TN>([&](auto tn) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int f = (tn.value & 1) ? 1 - i : i;
            acc[2 * q + f][tn.value] = mx8_mfma<tn.value, 0>(bf[tn.value], af[q & 1][f], acc[2 * q + f][tn.value], ws, xs[q & 1][f]);
          }
          between(tn.value);
        });
        pin(q_at);
        __builtin_amdgcn_sched_barrier(0);
      };
      // All of this wavefront's copies but those since the barrier before the last have landed, and its reads are done; then
      // everybody's.
      auto meet = [&](int clear_half) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(MORE ? CP_X + Y : 0));
        if (!MORE && left && kt == KT - 1 - (clear_half ^ 1) && (Y || !clear_half)) clear_rest(clear_half ? now : next, clear_half);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      };
      auto nothing = [](int) {};
      // n copies of `copy` from number `from` on
      auto copies = [&](auto copy, int from, int n) {
        if (!MORE) return;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < n; ++i) copy(kt + 2, now, from + i);
        __builtin_amdgcn_sched_barrier(0);
      };
      if constexpr (Q > 0) pair(std::integral_constant<int, 0>{}, nothing);
      meet(1);  // X: the second half of this step's rows is there
      if (WORD_SCALES) {
        if ((kt & 3) == 0 && kt + 4 < KT) copy_xs((kt >> 2) + 1);
      } else {
        store_xs(kt + 2, xw);  // read after the next barriers
        xw = load_xs(kt + 3);
      }
      if constexpr (Q == 4) {
        constexpr int EACH = (CP_X + 2 * TN - 1) / (2 * TN);
        pair(std::integral_constant<int, 1>{}, [&](int tn) { copies(copy_x, tn * EACH, EACH); });
        pair(std::integral_constant<int, 2>{}, [&](int tn) { copies(copy_x, (TN + tn) * EACH, EACH); });
      } else {
        copies(copy_x, 0, CP_X);
      }
      meet(0);  // Y: the next step's weights and first half of rows are there
      if constexpr (Q > 0) {
        read_a(0, next, xs_at(kt + 1), af[0], xs[0]);
        const uint32_t ws_next = load_ws(next);
        mx8_for_blocks<TN>([&](auto tn) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int f = (tn.value & 1) ? 1 - i : i;
            acc[2 * (Q - 1) + f][tn.value] = mx8_mfma<tn.value, 0>(bf[tn.value], af[1][f], acc[2 * (Q - 1) + f][tn.value], ws, xs[1][f]);
          }
          __builtin_amdgcn_sched_barrier(0);  // the registers of these weights take the next step's
          read_b(tn.value, next);
          if (tn.value < Y) copies(copy_y, tn.value, 1);
        });
        pin(std::integral_constant<int, Q - 1>{});
        ws = ws_next;
      } else {
        copies(copy_y, 0, Y);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    if (!WORD_SCALES) xw = load_xs(2);
    if constexpr (Q > 0) {
      read_a(0, 0, xs_at(0), af[0], xs[0]);
      ws = load_ws(0);
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) read_b(tn, 0);
    }
    int kt = 0;
    for (; kt + 2 < KT; ++kt) step(kt, std::true_type{});
    for (; kt < KT; ++kt) step(kt, std::false_type{});
  };

  if (WORD_SCALES) {
    copy_xs(0);
  } else {
    store_xs(0, load_xs(0));
    store_xs(1, load_xs(1));
  }
  for (int kt = 0; kt < min(KT, 2); ++kt) {
#pragma unroll
    for (int n = 0; n < CP_X; ++n) copy_x(kt, kt, n);
    if (half) continue;
#pragma unroll
    for (int n = 0; n < CP_Y; ++n) copy_y(kt, kt, n);
  }
  asm volatile("" ::: "memory");
  if (KT > 1 && half) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(CP_X));
  else if (KT > 1) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(CP_X + 2 * CP_Y));  // the first step's weights and first half have landed
  else __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
  if (left && KT == 1) clear_rest(0, 0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (pairs > 2) run(std::integral_constant<int, 4>{}, std::false_type{});
  else if (!half) run(std::integral_constant<int, 2>{}, std::false_type{});
  else if (pairs > 0) run(std::integral_constant<int, 2>{}, std::true_type{});
  else run(std::integral_constant<int, 0>{}, std::true_type{});

  // A lane holds eight consecutive output columns 8 (l / 16) of activation row l % 16, in each set of 32 columns.  Results leave
  // through LDS, by whole lines.
  __syncthreads();  // the stages are free
  if (EPI == EPI8_H) {
    // the workgroup's rows of 128 bytes; 8-byte word w of row r at word w ^ (r & 15)
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
      if (tm >= 2 * pairs) break;
      const int row = (tm * 2 + wm) * 16 + r16, col = t.n_idx * kMx8Panel + wn * 32;
      uint32_t byte;
      const uint2 codes = mx8_swiglu_codes(acc[tm][0], acc[tm][1], acc[tm][TN > 2 ? 2 : 0], acc[tm][TN > 2 ? 3 : 0], byte);
      *reinterpret_cast<uint2*>(smem + row * 128 + (((wn * 4 + kb) ^ r16) << 3)) = codes;
      if (kb == 0 && row < rows && col < g.n_out) g.H_scales[static_cast<int64_t>(t.row_begin + row) * (g.n_out >> 5) + (col >> 5)] = static_cast<uint8_t>(byte);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::BM / 64; ++i) {  // eight neighbouring lanes: the 128 bytes of a row
      const int row = i * 64 + (tid >> 3), w = (tid & 7) * 2, col = t.n_idx * kMx8Panel + w * 8;
      const uint2 lo = *reinterpret_cast<const uint2*>(smem + row * 128 + ((w ^ (row & 15)) << 3));
      const uint2 hi = *reinterpret_cast<const uint2*>(smem + row * 128 + (((w + 1) ^ (row & 15)) << 3));
      if (row < rows && col < g.n_out) *reinterpret_cast<mx8_u32x4*>(g.H + static_cast<int64_t>(t.row_begin + row) * g.n_out + col) = mx8_u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  } else {
    // 16 rows of 16 TN fp32 numbers at a time, in the wavefront's own part; 16-byte word w of row r at word w ^ r
    unsigned char* out = smem + wave * (TN * 1024);
    constexpr int LANES = 2 * TN, WORDS = 4 * TN, COLS = 16 * TN;  // lanes to a row, with eight columns each; words, columns of a row
    constexpr int TURNS = 16 * LANES / 64;
    const int r0 = lane / LANES, c = lane % LANES, col0 = t.n_idx * S::BN + wn * COLS, col = col0 + c * 8;
    auto word = [&](int r, int w) { return reinterpret_cast<mx8_f32x4*>(out + r * (TN * 64) + ((w ^ (r & (WORDS - 1))) << 4)); };
    const bool whole = col + 8 <= g.n_out;
    if (EPI == EPI8_LINEAR) {
      // all of the residual at once, so that its latency shows once
      mx8_u32x4 res[TM][TURNS];
      if (g.residual) {
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
          for (int i = 0; i < TURNS; ++i) {
            const int row = min((tm * 2 + wm) * 16 + i * (64 / LANES) + r0, rows - 1);
            res[tm][i] = mx8_residual8(g, t.row_begin + row, col);
          }
      }
      uint32_t bias[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
      const bool plain = g.activation == REVIVE_ACT_NONE;
      if (g.bias && plain) mx8_load8<float, false>(g.bias, col, g.n_out, bias);
      const int own_col = col0 + lane % COLS;
      const float own_bias = g.bias && own_col < g.n_out ? g.bias[own_col] : 0.f;
#pragma unroll
      for (int tm = 0; tm < TM; ++tm) {
        if (tm >= 2 * pairs) break;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) *word(r16, (tn >> 1) * 8 + kb * 2 + (tn & 1)) = acc[tm][tn];
        __builtin_amdgcn_wave_barrier();
        if (!plain) {  // a lane its column, number by number
#pragma unroll 1
          for (int r = lane / COLS; r < 16; r += 64 / COLS) {
            float* v = reinterpret_cast<float*>(word(r, (lane % COLS) >> 2)) + (lane & 3);
            *v = mx8_activated(*v + own_bias, g.activation);
          }
          __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
          const int r = i * (64 / LANES) + r0, row = (tm * 2 + wm) * 16 + r;
          const mx8_f32x4 v0 = *word(r, 2 * c), v1 = *word(r, 2 * c + 1);
          float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          if (row >= rows) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += __uint_as_float(bias[j]);
          if (col < g.n_out) mx8_finish8(g, t.row_begin + row, col, v, res[tm][i]);
        }
      }
    } else {
#pragma unroll
      for (int tm = 0; tm < TM; ++tm) {
        if (tm >= 2 * pairs) break;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) *word(r16, (tn >> 1) * 8 + kb * 2 + (tn & 1)) = acc[tm][tn];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
          const int r = i * (64 / LANES) + r0, row = (tm * 2 + wm) * 16 + r;
          const mx8_f32x4 v0 = *word(r, 2 * c), v1 = *word(r, 2 * c + 1);
          const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          if (row < rows && whole) mx8_store8<uint16_t, false>(g.Y + static_cast<int64_t>(t.row_begin + row) * g.n_out, col, g.n_out, v);
        }
      }
    }
  }
}

template <int TN, int EPI, bool WORD_SCALES>
int launch_mx8_tile_as(const revive_ctx* ctx, const Mx8Args& args, hipStream_t stream) {
  constexpr size_t lds = Mx8TileShape<TN>::LDS;
  auto kern = mx8_tile_kernel<TN, EPI, WORD_SCALES>;
  REVIVE_HIP(ctx, allow_dynamic_lds(reinterpret_cast<const void*>(kern), lds));
  hipLaunchKernelGGL(kern, dim3(args.dense.blocks + args.grouped.blocks), dim3(512), lds, stream, args);
  return check_hip(ctx, hipGetLastError(), "mx8_tile launch");
}
template <int TN, int EPI>
int launch_mx8_tile(const revive_ctx* ctx, const Mx8Args& args, hipStream_t stream) {
  if (args.dense.blocks + args.grouped.blocks <= 0) return REVIVE_OK;
  const bool words = (args.dense.blocks == 0 || mx8_word_scales(args.dense)) && (args.grouped.blocks == 0 || mx8_word_scales(args.grouped));
  return words ? launch_mx8_tile_as<TN, EPI, true>(ctx, args, stream) : launch_mx8_tile_as<TN, EPI, false>(ctx, args, stream);
}

}  // namespace revive
