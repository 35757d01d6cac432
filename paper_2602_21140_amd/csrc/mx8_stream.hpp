// Product of microscaled 8-bit activations and weights for few rows: the weights are streamed once, straight into registers.
//
// A workgroup covers up to 16 TMX rows and W 16-row blocks of weight rows (EPI8_H: half of them gate, half up).  Its NW
// wavefronts share K, each with a contiguous part of the steps of 128, and add up their sums through LDS at the end, in the
// wavefronts' order.  So the K loop has no barrier, and a product of few columns still has many wavefronts: what bounds it is how
// fast HBM is read, and in the smallest calls latency.  Weights and activations of the next D steps are on their way in registers.
//
// How fast a CU's loads come goes by the lines that each touches.  Weights lie in the order in which the matrix cores want them;
// of the activations a load takes whole lines, 8 rows of 128 bytes, and the wavefront turns them to operand order in LDS of its
// own (as operands straight from memory, 16 rows of 64 bytes, a product of 64 rows takes twice as long).  Their scales come for
// 16 steps at once.
//
// EPI8_H multiplies in bf16, which holds both operands' numbers, scales included (from 2^-126 on, below 2^128), and whose products are added up
// in fp32.  An h that is off by the 3e-5 of the 8-bit instruction is rounded to another code, 2^-4 away, some 17 times in 10 000: with few rows
// a single one of them shows (y of 8 rows, I = 896: relative error 0.0030, of which bf16's rounding is 0.0017).  While weights come
// from HBM there is time for it: 64 tokens on 279 slots of 7168 x 2048 take the same 1.52 ms; a token on 72 slots of 2048 x 1408 24 instead of 22 us,
// 256 tokens 141 instead of 133.
//
// Measured: that FFN of 64 tokens streams its 10.8 GB at 7.1 TB/s at the cases' 1.52 ms; 64 x 7168 x 7168 takes 13 us, 4 TB/s: too short a
// stream, of which 3 us are a launch's start and end.
#pragma once

#include "mx8_product.hpp"

namespace revive {

constexpr int kMx8ScaleSteps = 16, kMx8ScaleRow = kMx8ScaleSteps + 1;  // words of a row's scales in LDS, and from row to row
template <int TM>
constexpr int mx8_stream_wave_lds() { return 16 * TM * (kMx8Step + 4 * kMx8ScaleRow); }  // a wavefront's activations and their scales
template <int TMX, int W, int NW>
constexpr size_t mx8_stream_lds() {
  const int loop = NW * mx8_stream_wave_lds<TMX>(), sums = NW * W * TMX * 1024;
  return loop > sums ? loop : sums;
}

// WIDE: rows of A that are reached by 64 bits (otherwise all of A, or of a dense problem's tile, is within 4 GiB).
template <int TMX, int W, int NW, int D, int EPI, bool WIDE>
__global__ __launch_bounds__(64 * NW, 2) void mx8_stream_kernel(Mx8Args a) {
  static_assert(W % 2 == 0 && W <= 4 && (EPI != EPI8_H || W == 4) && NW > 1, "output columns in sets of 32, sums by way of LDS");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const bool dense = blockIdx.x < static_cast<unsigned>(a.dense.blocks);
  const Mx8Problem g = dense ? a.dense : a.grouped;
  const Mx8Tile t = mx8_tile_of(a, g, dense, 16 * TMX);
  if (t.row_begin >= t.row_end) return;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, kb = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = t.row_end - t.row_begin;
  const int KT = mx8_steps(g.K), blocks = g.K / kMx8Block;

  // 16-row blocks of weights: where a lane's codes and scales of step 0 are
  constexpr int PER = W < 4 ? W : W / (EPI == EPI8_H ? 2 : 1);  // blocks side by side in a panel
  const int block0 = t.n_idx * PER, panel = block0 >> 3, sub0 = block0 & 7;
  constexpr int HALVES = EPI == EPI8_H ? 2 : 1;
  uint64_t codes[HALVES], scales[HALVES];
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    const uint64_t matrix = reinterpret_cast<uint64_t>(t.B) + (h ? g.b_half : 0);
    codes[h] = mx8_uniform(matrix + static_cast<int64_t>(panel) * KT * kMx8PanelStep + sub0 * 2048);
    scales[h] = mx8_uniform(matrix + g.b_codes + static_cast<int64_t>(panel) * KT * kMx8PanelScales + sub0);
  }
  const uint32_t lane16 = lane * 16, lane8 = lane * 8;
  auto source = [&](int r) -> int64_t {  // row of A; rows past the tile read its last row again
    const int row = t.row_begin + min(r, rows - 1);
    return g.src_of ? g.src_of[row] / g.k : row;
  };

  auto run = [&](auto tm_tag, auto once_tag) {
    constexpr int TM = decltype(tm_tag)::value;
    constexpr bool ONCE = decltype(once_tag)::value;  // streamed past the caches' retention (non-temporal)
    // load j of row-tile i: rows 16 i + 8 j + l / 8, chunk l % 8
    typedef typename std::conditional<WIDE, int64_t, uint32_t>::type Off;
    const int64_t origin = g.src_of ? 0 : t.row_begin;
    const uint64_t A = mx8_uniform(reinterpret_cast<uint64_t>(g.A) + origin * g.a_row), A_scales = mx8_uniform(reinterpret_cast<uint64_t>(g.A_scales) + origin * blocks);
    Off x[TM][2], xs[TM];  // scales: rows 16 i + l / 4
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) x[i][j] = static_cast<Off>((source(i * 16 + j * 8 + (lane >> 3)) - origin) * g.a_row + (lane & 7) * 16);
      xs[i] = static_cast<Off>((source(i * 16 + (lane >> 2)) - origin) * blocks);
    }
    unsigned char* own = smem + wave * mx8_stream_wave_lds<TM>();
    uint32_t* own_scales = reinterpret_cast<uint32_t*>(own + 16 * TM * kMx8Step);
    // row r at r * 128 bytes, its chunk c at chunk c ^ ((r >> 1) & 7)
    auto place = [&](int row, int chunk) { return reinterpret_cast<mx8_u32x4*>(own + row * 128 + ((chunk ^ swz(row)) << 4)); };
    // What the wavefront finishes: TM row-tiles of PAIRS sets of 32 columns are dealt round-robin.  A lane holds eight consecutive
    // output columns 8 (l / 16) of activation row l % 16.  Bias and residual are asked for now.
    constexpr int PAIRS = EPI == EPI8_H ? 1 : W / 2, ITEMS = (TM * PAIRS + NW - 1) / NW;
    static_assert(NW % PAIRS == 0, "a wavefront's columns are the same in all of its row-tiles");
    auto row_of = [&](int n) { return t.row_begin + (wave + n * NW) / PAIRS * 16 + r16; };
    auto col_of = [&]() { return (block0 + 2 * (wave % PAIRS)) * 16 + kb * 8; };
    uint32_t bias[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    mx8_u32x4 residual[ITEMS];
    if (EPI == EPI8_LINEAR && wave < TM * PAIRS) {
      if (g.bias) mx8_load8<float, false>(g.bias, col_of(), g.n_out, bias);
#pragma unroll
      for (int n = 0; n < ITEMS; ++n) residual[n] = mx8_residual8(g, min(row_of(n), t.row_end - 1), col_of());
    }
    mx8_f32x4 acc[W][TM];
#pragma unroll
    for (int s = 0; s < W; ++s)
#pragma unroll
      for (int i = 0; i < TM; ++i) acc[s][i] = mx8_f32x4{0.f, 0.f, 0.f, 0.f};

    struct Step { Mx8Frag w[W]; uint32_t ws[HALVES]; mx8_u32x4 x[TM][2]; };  // EPI8_H: ws of the two halves of K
    typedef uint32_t any32 __attribute__((aligned(1)));
#define REVIVE_GLOBAL(type, base, offset) reinterpret_cast<const __attribute__((address_space(1))) type*>((base) + (offset))
    auto load_w = [&](Step& b, int step) {
#pragma unroll
      for (int s = 0; s < W; ++s) {
        const auto p = REVIVE_GLOBAL(mx8_u32x4, codes[HALVES * s / W] + static_cast<uint64_t>(step) * kMx8PanelStep + s % PER * 2048, lane16);
        b.w[s] = ONCE ? mx8_frag(__builtin_nontemporal_load(p), __builtin_nontemporal_load(p + 64)) : mx8_frag(p[0], p[64]);
      }
      const uint64_t at = static_cast<uint64_t>(step) * kMx8PanelScales;
      if (EPI == EPI8_H) {  // of the lane's own K-elements, 16 (l / 16) on: blocks l / 32 and 2 + l / 32
        const uint32_t of_block = ((kb >> 1) * 16 + r16) * 8;
#pragma unroll
        for (int k = 0; k < HALVES; ++k)
          b.ws[k] = *REVIVE_GLOBAL(uint16_t, scales[0] + at + k * 256, of_block) | static_cast<uint32_t>(*REVIVE_GLOBAL(uint16_t, scales[HALVES - 1] + at + k * 256, of_block)) << 16;
      }
      else if (W == 2) b.ws[0] = *REVIVE_GLOBAL(uint16_t, scales[0] + at, lane8);
      else b.ws[0] = *REVIVE_GLOBAL(any32, scales[0] + at, lane8);
    };
    auto load = [&](Step& b, int step) {  // a whole step
      load_w(b, step);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) b.x[i][j] = *REVIVE_GLOBAL(mx8_u32x4, A + static_cast<uint64_t>(step) * kMx8Step, x[i][j]);
    };
    auto multiply = [&](const Step& b, int at) {  // `at`: the step's place among the scales
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *place(i * 16 + j * 8 + (lane >> 3), lane & 7) = b.x[i][j];
      auto scale = [&](int i, int block) -> uint32_t { return reinterpret_cast<const uint8_t*>(own_scales + (i * 16 + r16) * kMx8ScaleRow + at)[block]; };
      if constexpr (EPI == EPI8_H) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          Mx8Wide f[TM];
#pragma unroll
          for (int i = 0; i < TM; ++i) f[i] = mx8_widened(*place(i * 16 + r16, kb + 4 * k), scale(i, 2 * k + (kb >> 1)));
#pragma unroll
          for (int s = 0; s < W; ++s) {
            const mx8_u32x4 codes = {static_cast<uint32_t>(b.w[s][4 * k]), static_cast<uint32_t>(b.w[s][4 * k + 1]), static_cast<uint32_t>(b.w[s][4 * k + 2]), static_cast<uint32_t>(b.w[s][4 * k + 3])};
            const Mx8Wide w = mx8_widened(codes, (b.ws[k] >> (8 * s)) & 255u);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
              for (int n = 0; n < 2; ++n) acc[s][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[n], f[i].part[n], acc[s][i], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);  // or all blocks are widened first, and kept
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const Mx8Frag f = mx8_frag(*place(i * 16 + r16, kb), *place(i * 16 + r16, kb + 4));
          const uint32_t own = scale(i, kb);
          mx8_for_blocks<W>([&](auto s) { acc[s.value][i] = mx8_mfma<s.value, 0>(b.w[s.value], f, acc[s.value][i], b.ws[0], own); });
        }
      }
    };

    const int whole = g.K / kMx8Step;
    const int begin = static_cast<int>(static_cast<int64_t>(wave) * whole / NW), end = static_cast<int>(static_cast<int64_t>(wave + 1) * whole / NW);
    for (int first = begin; first < end; first += kMx8ScaleSteps) {
      const int last = min(first + kMx8ScaleSteps, end);
      uint32_t scale[TM][kMx8ScaleSteps / 4];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int p = 0; p < kMx8ScaleSteps / 4; ++p) scale[i][p] = *REVIVE_GLOBAL(any32, A_scales, xs[i] + static_cast<Off>(min(first + 4 * p + (lane & 3), last - 1) * 4));
      Step b[D];
#pragma unroll
      for (int u = 0; u < D; ++u)
        if (first + u < last) load(b[u], first + u);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int p = 0; p < kMx8ScaleSteps / 4; ++p) own_scales[(i * 16 + (lane >> 2)) * kMx8ScaleRow + 4 * p + (lane & 3)] = scale[i][p];
      int s = first;
      for (; s + 2 * D <= last; s += D) {  // every load unconditional, so that the compiler's count of loads in flight stays exact
#pragma unroll
        for (int u = 0; u < D; ++u) {
          multiply(b[u], s + u - first);
          load(b[u], s + u + D);
        }
      }
#pragma unroll
      for (int u = 0; u < 2 * D; ++u) {  // fewer than twice as many are left
        if (s + u < last) multiply(b[u % D], s + u - first);
        if (u < D && s + u + D < last) load(b[u % D], s + u + D);
      }
    }
    if (wave == NW - 1 && whole < KT) {  // what is left of K, a multiple of 32: zeros behind it, and scales of 2^-127
      Step b;
      load_w(b, whole);
      const int left = g.K - whole * kMx8Step;
      const bool in = (lane & 7) * 16 < left;  // chunks past the row: its first one, not used
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const mx8_u32x4 v = *REVIVE_GLOBAL(mx8_u32x4, A, in ? x[i][j] + static_cast<Off>(whole) * kMx8Step : x[i][j] - (lane & 7) * 16);
          b.x[i][j] = in ? v : mx8_u32x4{0u, 0u, 0u, 0u};
        }
        const int block = lane & 3;
        reinterpret_cast<uint8_t*>(own_scales + (i * 16 + (lane >> 2)) * kMx8ScaleRow)[block] =
            block * 32 < left ? *REVIVE_GLOBAL(uint8_t, A_scales, xs[i] + static_cast<Off>(whole * 4 + block)) : 0;
      }
      multiply(b, 0);
    }
#undef REVIVE_GLOBAL

    // the wavefronts' sums, tile by tile; NW tiles at a time are added up, a wavefront each its own
    mx8_f32x4* part = reinterpret_cast<mx8_f32x4*>(smem);
    __syncthreads();  // the activations are done with
#pragma unroll
    for (int s = 0; s < W; ++s)
#pragma unroll
      for (int i = 0; i < TM; ++i) part[((wave * W + s) * TM + i) * 64 + lane] = acc[s][i];
    __syncthreads();
    auto total = [&](int s, int i) {
      mx8_f32x4 v = part[(s * TM + i) * 64 + lane];
      for (int w = 1; w < NW; ++w) v += part[((w * W + s) * TM + i) * 64 + lane];
      return v;
    };
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      const int item = wave + n * NW, i = item / PAIRS, p = item % PAIRS;
      if (item >= TM * PAIRS) break;
      const int row = row_of(n), col = col_of();
      const mx8_f32x4 v0 = total(2 * p, i), v1 = total(2 * p + 1, i);
      if (EPI == EPI8_H) {
        uint32_t byte;
        const uint2 out = mx8_swiglu_codes(v0, v1, total(2, i), total(3, i), byte);
        if (row >= t.row_end || col >= g.n_out) continue;
        *reinterpret_cast<uint2*>(g.H + static_cast<int64_t>(row) * g.n_out + col) = out;
        if (kb == 0) g.H_scales[static_cast<int64_t>(row) * (g.n_out >> 5) + (col >> 5)] = static_cast<uint8_t>(byte);
      } else if (row < t.row_end && col < g.n_out) {
        float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
        if (EPI == EPI8_LINEAR) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += __uint_as_float(bias[j]);
          if (g.activation != REVIVE_ACT_NONE)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = mx8_activated(v[j], g.activation);
          mx8_finish8(g, row, col, v, residual[n]);
        } else {
          mx8_store8<uint16_t, false>(g.Y + static_cast<int64_t>(row) * g.n_out, col, g.n_out, v);
        }
      }
    }
  };
  using Y = std::true_type;
  if (!t.once) run(std::integral_constant<int, TMX>{}, std::false_type{});
  else if (TMX == 1 || rows <= 16) run(std::integral_constant<int, 1>{}, Y{});
  else if (TMX == 2 || rows <= 32) run(std::integral_constant<int, (TMX < 2 ? TMX : 2)>{}, Y{});
  else run(std::integral_constant<int, TMX>{}, Y{});
}

template <int TMX, int W, int NW, int D, int EPI, bool WIDE = false>
int launch_mx8_stream(const revive_ctx* ctx, const Mx8Args& args, hipStream_t stream) {
  const int grid = args.dense.blocks + args.grouped.blocks;
  if (grid <= 0) return REVIVE_OK;
  constexpr size_t lds = mx8_stream_lds<TMX, W, NW>();
  static_assert(lds <= 64 * 1024, "what a kernel has without asking for more");
  auto kern = mx8_stream_kernel<TMX, W, NW, D, EPI, WIDE>;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * NW), lds, stream, args);
  return check_hip(ctx, hipGetLastError(), "mx8_stream launch");
}

}  // namespace revive
