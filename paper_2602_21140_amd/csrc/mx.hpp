// Microscaled 4-bit floats (MXFP4): blocks of 32 numbers along K, each number as an E2M1 code, each block with a power of
// two as its scale (E8M0).
//
//   amax = largest magnitude of the block;  e = clamp(floor(log2 amax) - 2, -127, 127);  scale byte = e + 127
//   code = the E2M1 number nearest to x / 2^e, ties to the even code, at most 6  (codes 0..7: 0 0.5 1 1.5 2 3 4 6; 8: sign)
//
// The exponent puts amax into [4, 8), so what saturates is off by a quarter at most.  A block with an infinity or a NaN has
// scale byte 255 and stands for 32 NaNs; the matrix cores read it as that, too.  A block of zeros has scale byte 0.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace revive {

constexpr int kMxBlock = 32;
constexpr int kMxStep = 128;   // K-elements of one MFMA: 64 bytes of codes per row
constexpr int kMxGroup = 512;  // K-elements whose scales a lane takes in one word: four steps
constexpr int kMxPanel = 128;  // weight rows that are stored together
constexpr int kMxPanelStep = kMxPanel * kMxStep / 2;            // bytes of a panel's codes for one step
constexpr int kMxPanelScales = kMxPanel * kMxGroup / kMxBlock;  // bytes of a panel's scales for one group

__host__ __device__ inline int64_t mx_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
__host__ __device__ inline int mx_steps(int K) { return (K + kMxStep - 1) / kMxStep; }
__host__ __device__ inline int mx_groups(int K) { return (K + kMxGroup - 1) / kMxGroup; }

// Packed weights: [panels][steps][8][64][16] bytes of codes, then [panels][groups][8][64][4] bytes of scales.  A block of 16
// rows and 128 K-elements is one contiguous KiB in the order in which the matrix cores want it: lane l holds row l % 16,
// K-elements 32 (l / 16) to 32 (l / 16) + 31, and in its word of scales byte s is that of step s of the group.
inline int64_t mx_packed_codes(int rows, int K) { return mx_up(rows, kMxPanel) * mx_steps(K) * (kMxStep / 2); }
inline int64_t mx_packed_bytes(int rows, int K) { return mx_packed_codes(rows, K) + mx_up(rows, kMxPanel) * mx_groups(K) * (kMxGroup / kMxBlock); }

// Of 32 rows, MFMA row m of the 16-row block s.  An MFMA gives a lane results of four consecutive rows m; dealt this way the
// lane's results of both blocks are eight consecutive rows of the matrix, i.e. output columns: a word of codes, 16 bytes of bf16.
__host__ __device__ inline int mx_row(int s, int m) { return 8 * (m >> 2) + 4 * s + (m & 3); }

// Bytes of a row's codes where the kernels keep activations: whole pairs of steps, whole lines.
__host__ __device__ inline int64_t mx_code_row(int K) { return static_cast<int64_t>((mx_steps(K) + 1) / 2) * kMxStep; }

// Bytes of a row's scales where the kernels keep activations: [groups][4 blocks of a step][4 steps].
__host__ __device__ inline int mx_scale_row(int K) { return mx_groups(K) * (kMxGroup / kMxBlock); }
__host__ __device__ inline int mx_scale_at(int block) { return (block & ~15) + ((block & 3) << 2) + ((block >> 2) & 3); }

// Scale byte of a block from its largest magnitude's bits (a NaN's are above infinity's).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t magnitude) {
  const uint32_t e = magnitude >> 23;
  return e == 255u ? 255u : (e > 2u ? e : 2u) - 2u;
}
// The scale as the conversion instructions take it: they read its exponent, 0 as 2^-127.
__device__ __forceinline__ float mx_scale_f32(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight numbers -> a word of codes, the first one lowest.  The instruction rounds to the nearest, ties to even, and saturates.
__device__ __forceinline__ uint32_t mx_codes(const float* v, float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

typedef int32_t mx_i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));

// acc[4 (l / 16) + i of the first operand's rows][l % 16 of the second's] += 128 products; byte S of each scale word.
template <int SW, int SX>
__device__ __forceinline__ mx_f32x4 mx_mfma(mx_u32x4 w, mx_u32x4 x, mx_f32x4 acc, uint32_t w_scale, uint32_t x_scale) {
  const mx_i32x8 a = {static_cast<int>(w[0]), static_cast<int>(w[1]), static_cast<int>(w[2]), static_cast<int>(w[3]), 0, 0, 0, 0};
  const mx_i32x8 b = {static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, SW, static_cast<int>(w_scale), SX, static_cast<int>(x_scale));
}

}  // namespace revive
