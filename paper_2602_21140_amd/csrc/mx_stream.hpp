// Grouped product of microscaled 4-bit activations and weights for few rows per expert: the weights are streamed once,
// straight into registers.
//
//   C[rows of tile, n] = sum_k A[row, k] * B_group[n, k], fp32 sums
//
// Two epilogues: EPI_H: B holds gate and up; store silu(gate) * up as microscaled 4-bit numbers (the next product's
// activations).  EPI_Y: store bf16.
//
// A workgroup of NW wavefronts covers up to 16 TMX rows; each wavefront has W 16-row blocks of weight rows of its own (EPI_H:
// half of them gate, half up).  A block of weights (16 rows, 128 K-elements) is one KiB that the wavefront loads in address
// order and feeds to the matrix cores as it is.  Activations come through LDS, 512 K-elements at a time, in two buffers.
// What bounds it is how fast HBM is read: the next 512 K-elements of weights are on their way in registers.  64 tokens on 237
// matrices of H = 7168, I = 2048: gate and up in 525 us (7.0 TB/s), down in 285 (6.5); one token on 9 of them 25 and 12
// (5.7 in both: workgroups start and end together).
//
// BF16: A is the bf16 rows themselves, and a thread rounds blocks of 32 numbers to 4 bits on their way to LDS.  Every workgroup
// does that for its rows, which with few tokens is less than a launch of its own (kMxFewTokens).
#pragma once

#include <type_traits>

#include "ctx.hpp"
#include "gemm_bf16.hpp"
#include "mx.hpp"
#include "row_tiles.hpp"

namespace revive {

enum { EPI_H = 0, EPI_Y = 1 };

// Of a row-tile with up to so many rows no more are copied and rounded; the other lanes multiply what the LDS holds, for results
// that are not stored.
constexpr int kMxFewRows = 4;

// h, the activations of the second product: [pairs of steps][rows][128 bytes]; where the 64 bytes of step s of a row begin.
__host__ __device__ inline int64_t mx_h_at(int s, int64_t rows, int64_t row) { return (static_cast<int64_t>(s >> 1) * rows + row) * 128 + (s & 1) * 64; }

struct MxProblem {
  const uint8_t* A;          // codes of row r, step s: A + r * a_row + s / 2 * a_pair + s % 2 * 64, 64 bytes; BF16: row r at A + r * a_row
  int64_t a_row, a_pair;
  const uint8_t* A_scales;   // rows of mx_scale_row(K) bytes
  const int32_t* src_of;     // not null: row r of the product is row src_of[r] / k of A
  int k;
  const void* const* B_tab;  // device table slot -> packed weights (grouped), or
  const void* B_one;         // the one packed matrix (dense)
  int64_t b_half;            // EPI_H: bytes from the gate matrix to the up matrix
  int64_t b_codes;           // bytes from a matrix' codes to its scales
  uint8_t* H; uint8_t* H_scales;  // EPI_H: codes at mx_h_at, scales [h_rows][mx_scale_row(n_out)]
  int64_t h_rows;
  uint16_t* Y;               // EPI_Y: bf16 [rows, n_out]
  int n_out, K;
  int n_col_tiles;
  int blocks;                // workgroups of the grid that belong to this problem
  int M;                     // rows (dense)
};

struct MxArgs {
  MxProblem dense;              // served by the first dense.blocks workgroups
  MxProblem grouped;            // served by the others
  const int32_t* slot_offsets;  // [P + 1]: rows of every slot (grouped)
  int P;
};

typedef const __attribute__((address_space(1))) mx_u32x4* mx_gptr;
typedef const __attribute__((address_space(1))) uint32_t* mx_gptr1;
__device__ __forceinline__ mx_u32x4 mx_load16(const uint8_t* p) { return *reinterpret_cast<mx_gptr>(reinterpret_cast<uintptr_t>(p)); }
__device__ __forceinline__ uint32_t mx_load4(const uint8_t* p) { return *reinterpret_cast<mx_gptr1>(reinterpret_cast<uintptr_t>(p)); }

// The lane's eight columns of gate and up of one row, of a block of 32 columns that the lanes l, l ^ 16, l ^ 32, l ^ 48 share
// -> a word of codes, and the block's scale byte.
__device__ __forceinline__ uint32_t mx_swiglu_codes(const mx_f32x4& g0, const mx_f32x4& g1, const mx_f32x4& u0, const mx_f32x4& u1, uint32_t& byte) {
  float v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = i < 4 ? silu_f32(g0[i & 3]) * u0[i & 3] : silu_f32(g1[i & 3]) * u1[i & 3];
    m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  }
  m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
  m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
  byte = mx_scale_byte(m);
  return mx_codes(v, mx_scale_f32(byte));
}

// A block of 32 bf16 numbers -> four words of codes, and its scale byte.
typedef uint32_t mx_u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ mx_u32x4 mx_block_codes(const mx_u32x4* x, uint32_t& byte) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i >> 2][i & 3] & 0x7FFF7FFFu));
  byte = mx_scale_byte(static_cast<uint32_t>(m[0] > m[1] ? m[0] : m[1]) << 16);
  const float scale = mx_scale_f32(byte);
  mx_u32x4 o;
  auto two = [](uint32_t v) { return __builtin_bit_cast(bf16x2, v); };
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, two(x[w][0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x[w][1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x[w][2]), scale, 2);
    o[w] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(x[w][3]), scale, 3);
  }
  return o;
}

template <typename F, int... S>
__device__ __forceinline__ void mx_for(std::integer_sequence<int, S...>, F f) { (f(std::integral_constant<int, S>{}), ...); }

template <int TMX, int W, int NW, int EPI, bool BF16>
__global__ __launch_bounds__(64 * NW, 2) void mx_stream_kernel(MxArgs a) {
  constexpr int NT = 64 * NW, PAIRS = EPI == EPI_H ? W / 4 : W / 2;  // sets of 32 output columns per wavefront
  static_assert(PAIRS >= 1, "output columns in sets of 32");
  constexpr int ROWS = TMX * 16 * 256;  // bytes of a buffer's codes; BF16: its scales, 16 bytes a row, follow
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][ROWS + (BF16 ? TMX * 256 : 0)];
  const bool dense = blockIdx.x < static_cast<unsigned>(a.dense.blocks);
  const MxProblem g = dense ? a.dense : a.grouped;
  const int b = dense ? blockIdx.x : blockIdx.x - a.dense.blocks;
  int n_idx, row_begin, row_end;
  const uint8_t* B;
  bool once = true;  // nobody else reads these weights
  if (dense) {
    const int m_idx = b / g.n_col_tiles;
    n_idx = b - m_idx * g.n_col_tiles;
    row_begin = m_idx * (16 * TMX);
    row_end = min(g.M, row_begin + 16 * TMX);
    if (row_begin >= row_end) return;  // the grid is filled up to a multiple of 8
    B = static_cast<const uint8_t*>(g.B_one);
    once = g.M <= 16 * TMX;
  } else {
    const GridTile t = grid_tile(a.slot_offsets, a.P, 16 * TMX, g.n_col_tiles, b, g.B_tab);
    if (t.group < 0) return;
    n_idx = t.n_idx;
    row_begin = t.row_begin;
    row_end = t.row_end;
    B = static_cast<const uint8_t*>(t.w);
    once = t.in_group == 1;
  }
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, kb = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = row_end - row_begin;
  const int KT = mx_steps(g.K), NG = mx_groups(g.K);
  // sets of 32 output columns; EPI_H: all of the last panel, whose rows past the matrix are zeros
  const int n_sets = EPI == EPI_H ? (g.n_out + kMxPanel - 1) / kMxPanel * 4 : (g.n_out + 31) >> 5;
  const int own_set = (n_idx * NW + wave) * PAIRS;

  // 16-row blocks of weights: byte offsets of a lane's codes and scales, for step and group 0
  uint32_t w_off[W], s_off[W];
#pragma unroll
  for (int s = 0; s < W; ++s) {
    const int pair = EPI == EPI_H ? (s % (W / 2)) >> 1 : s >> 1;
    const int set = min(own_set + pair, n_sets - 1);  // past the last column: the last ones again, not stored
    const int sub = (set & 3) * 2 + (s & 1), panel = set >> 2;
    const uint32_t half = EPI == EPI_H && s >= W / 2 ? static_cast<uint32_t>(g.b_half) : 0u;
    w_off[s] = half + static_cast<uint32_t>(panel) * KT * kMxPanelStep + sub * 1024 + lane * 16;
    s_off[s] = half + static_cast<uint32_t>(g.b_codes) + static_cast<uint32_t>(panel) * NG * kMxPanelScales + sub * 256 + lane * 4;
  }

  auto source = [&](int r) -> int64_t {  // row of A; rows past the tile read its last row again
    const int row = row_begin + min(r, rows - 1);
    return g.src_of ? g.src_of[row] / g.k : row;
  };

  auto run = [&](auto tm_tag, auto once_tag, auto rows_tag) {
    constexpr int TM = decltype(tm_tag)::value;
    constexpr bool ONCE = decltype(once_tag)::value;  // streamed past the caches' retention (non-temporal)
    constexpr int WORDS = decltype(rows_tag)::value * 16;  // 16-byte words of one group of activations
    constexpr int NA = (WORDS + NT - 1) / NT;         // per thread
    const uint8_t* a_src[NA];
    uint32_t a_dst[NA], s_dst[NA];
    int a_part[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int w = (i * NT + tid) % WORDS;
      const int row = w >> 4, c = w & 15;
      a_part[i] = BF16 ? c : c >> 2;
      a_src[i] = g.A + source(row) * g.a_row + (BF16 ? 0 : (c & 3) * 16);
      a_dst[i] = row * 256 + ((c ^ (row & 15)) << 4);
      s_dst[i] = ROWS + row * 16 + mx_scale_at(c);
    }
    const uint8_t* x_src[TM];
    if (!BF16)
#pragma unroll
      for (int i = 0; i < TM; ++i) x_src[i] = g.A_scales + source(i * 16 + r16) * mx_scale_row(g.K) + kb * 4;
    mx_f32x4 acc[W][TM];
#pragma unroll
    for (int s = 0; s < W; ++s)
#pragma unroll
      for (int i = 0; i < TM; ++i) acc[s][i] = mx_f32x4{0.f, 0.f, 0.f, 0.f};

    mx_u32x4 wf[4][W], af[NA][BF16 ? 4 : 1];
    uint32_t ws[W], xs[TM], ws_next[W], xs_next[TM];
    auto load_a = [&](int q) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        if (BF16) {  // blocks past the row: the last one again, for weights of zero
          const uint8_t* block = a_src[i] + min(q * 16 + a_part[i], g.K / kMxBlock - 1) * 64;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            af[i][w] = *reinterpret_cast<const __attribute__((address_space(1))) mx_u32x4_any*>(reinterpret_cast<uintptr_t>(block + w * 16));
        } else {
          const int s = min(q * 4 + a_part[i], KT - 1);
          af[i][0] = mx_load16(a_src[i] + (s >> 1) * g.a_pair + (s & 1) * 64);
        }
      }
    };
    auto load_scales = [&](int q, uint32_t* w, uint32_t* x) {
#pragma unroll
      for (int s = 0; s < W; ++s) w[s] = mx_load4(B + s_off[s] + static_cast<int64_t>(q) * kMxPanelScales);
      if (!BF16)
#pragma unroll
        for (int i = 0; i < TM; ++i) x[i] = mx_load4(x_src[i] + q * 16);
    };
    auto load_w = [&](int step, int h) {
      const uint8_t* wp = B + static_cast<int64_t>(min(step, KT - 1)) * kMxPanelStep;
#pragma unroll
      for (int s = 0; s < W; ++s) {
        const mx_gptr p = reinterpret_cast<mx_gptr>(reinterpret_cast<uintptr_t>(wp + w_off[s]));
        wf[h][s] = ONCE ? __builtin_nontemporal_load(p) : *p;
      }
    };
    auto stage = [&](int buf) {
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        if (BF16) {
          uint32_t byte;
          *reinterpret_cast<mx_u32x4*>(lds[buf] + a_dst[i]) = mx_block_codes(af[i], byte);
          lds[buf][s_dst[i]] = static_cast<uint8_t>(byte);
        } else {
          *reinterpret_cast<mx_u32x4*>(lds[buf] + a_dst[i]) = af[i][0];
        }
      }
    };
    auto publish = [&]() {  // this wavefront's LDS accesses are done; then everybody's are
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    // Every load is unconditional, so that the compiler's count of loads in flight stays exact: past the last group or
    // step the last one is fetched again and not multiplied.
    load_a(0);
    load_scales(0, ws, xs);
    mx_for(std::make_integer_sequence<int, 4>{}, [&](auto step) { load_w(step.value, step.value); });
    stage(0);
    load_a(min(1, NG - 1));
    publish();
    for (int q = 0; q < NG; ++q) {
      load_scales(min(q + 1, NG - 1), ws_next, xs_next);
      if (BF16)
#pragma unroll
        for (int i = 0; i < TM; ++i) xs[i] = *reinterpret_cast<const uint32_t*>(lds[q & 1] + ROWS + (i * 16 + r16) * 16 + kb * 4);
      mx_for(std::make_integer_sequence<int, 4>{}, [&](auto step) {
        constexpr int h = decltype(step)::value;
        if (q * 4 + h < KT) {
          const unsigned char* base = lds[q & 1] + r16 * 256 + (((h * 4 + kb) ^ r16) << 4);
#pragma unroll
          for (int i = 0; i < TM; ++i) {
            const mx_u32x4 x = *reinterpret_cast<const mx_u32x4*>(base + i * (16 * 256));
#pragma unroll
            for (int s = 0; s < W; ++s) acc[s][i] = mx_mfma<h, h>(wf[h][s], x, acc[s][i], ws[s], xs[i]);
          }
        }
        load_w(q * 4 + 4 + h, h);
        __builtin_amdgcn_sched_barrier(0);
      });
      stage((q + 1) & 1);
      load_a(min(q + 2, NG - 1));
#pragma unroll
      for (int s = 0; s < W; ++s) ws[s] = ws_next[s];
      if (!BF16)
#pragma unroll
        for (int i = 0; i < TM; ++i) xs[i] = xs_next[i];
      publish();
    }

    // a lane holds eight consecutive output columns 8 (l / 16) of activation row l % 16
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = row_begin + i * 16 + r16;
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        const int set = own_set + p;
        if (EPI == EPI_H) {
          uint32_t byte;
          const uint32_t codes = mx_swiglu_codes(acc[2 * p][i], acc[2 * p + 1][i], acc[W / 2 + 2 * p][i], acc[W / 2 + 2 * p + 1][i], byte);
          if (row >= row_end || set >= n_sets) continue;
          *reinterpret_cast<uint32_t*>(g.H + mx_h_at(set >> 2, g.h_rows, row) + (set & 3) * 16 + kb * 4) = codes;
          if (kb == 0) g.H_scales[static_cast<int64_t>(row) * mx_scale_row(g.n_out) + mx_scale_at(set)] = static_cast<uint8_t>(byte);
        } else {
          const int col = set * 32 + kb * 8;
          if (row >= row_end || col >= g.n_out) continue;
          const mx_f32x4 &v0 = acc[2 * p][i], &v1 = acc[2 * p + 1][i];
          const mx_u32x4 o = {pack_bf16(v0[0], v0[1]), pack_bf16(v0[2], v0[3]), pack_bf16(v1[0], v1[1]), pack_bf16(v1[2], v1[3])};
          *reinterpret_cast<mx_u32x4*>(g.Y + static_cast<int64_t>(row) * g.n_out + col) = o;
        }
      }
    }
  };
  using Y = std::true_type;
  auto tiles = [&](auto tm, auto once_tag) { run(tm, once_tag, std::integral_constant<int, 16 * decltype(tm)::value>{}); };
  if (!once) tiles(std::integral_constant<int, TMX>{}, std::false_type{});
  else if (TMX == 1 && rows <= kMxFewRows) run(std::integral_constant<int, 1>{}, Y{}, std::integral_constant<int, kMxFewRows>{});
  else if (TMX == 1 || rows <= 16) tiles(std::integral_constant<int, 1>{}, Y{});
  else if (TMX == 2 || rows <= 32) tiles(std::integral_constant<int, (TMX < 2 ? TMX : 2)>{}, Y{});
  else tiles(std::integral_constant<int, TMX>{}, Y{});
}

template <int TMX, int W, int NW, int EPI, bool BF16>
int launch_mx_stream(revive_ctx* ctx, const MxArgs& args, hipStream_t stream) {
  const int grid = args.dense.blocks + args.grouped.blocks;
  if (grid <= 0) return REVIVE_OK;
  hipLaunchKernelGGL((mx_stream_kernel<TMX, W, NW, EPI, BF16>), dim3(grid), dim3(64 * NW), 0, stream, args);
  return check_hip(ctx, hipGetLastError(), "mx_stream launch");
}

}  // namespace revive
