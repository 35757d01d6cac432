// Microscaled 8-bit floats (MXFP8): blocks of 32 numbers along K, each number as an E4M3 code, each block with a power of two
// as its scale (E8M0).
//
//   amax = largest magnitude of the block;  e = the smallest with amax <= 448 * 2^e, at least -127;  scale byte = e + 127
//   code = the E4M3 number nearest to x / 2^e, ties to the even code
//
// 448 is E4M3's largest number: nothing saturates, every number is off by half a step (2^-4 of it, or 2^-10 * 2^e) at most.  With
// floor(log2 amax) - 8 for e, as the 4-bit form has it, a block's largest numbers would be cut off by up to an eighth.  A block
// with an infinity or a NaN has scale byte 255 and stands for 32 NaNs; the matrix cores read it as that, too.  A block of zeros
// has scale byte 0.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace revive {

constexpr int kMx8Block = 32;
constexpr int kMx8Step = 128;                           // K-elements of one MFMA, and bytes of a row's codes
constexpr int kMx8Panel = 128;                          // weight rows that are stored together
constexpr int kMx8PanelStep = kMx8Panel * kMx8Step;     // bytes of a panel's codes for one step
constexpr int kMx8PanelScales = kMx8Panel * kMx8Step / kMx8Block;

constexpr int kMx8MaxK = 1 << 24;                       // of a product: the kernels reach 256 rows of codes by 32 bits

__host__ __device__ inline int mx8_steps(int K) { return (K + kMx8Step - 1) / kMx8Step; }

// Packed weights: [panels][steps][8][2][64][16] bytes of codes, then [panels][steps][64][8] bytes of scales.  A block of 16 rows
// and 128 K-elements is two contiguous KiB in the order in which the matrix cores want it: of its half h, lane l holds row l % 16,
// K-elements 64 h + 16 (l / 16) to + 15; byte b of its scales is that of the panel's block b, row l % 16, K-elements 32 (l / 16)
// to + 31 (the instruction takes a lane's scale for these, not for the lane's own codes).
inline int64_t mx8_packed_codes(int rows, int K) { return (static_cast<int64_t>(rows) + kMx8Panel - 1) / kMx8Panel * mx8_steps(K) * kMx8PanelStep; }
inline int64_t mx8_packed_bytes(int rows, int K) { return mx8_packed_codes(rows, K) / kMx8Block * (kMx8Block + 1); }

// Of 32 rows, MFMA row m of the 16-row block s.  An MFMA gives a lane results of four consecutive rows m; dealt this way the
// lane's results of both blocks are eight consecutive rows of the matrix, i.e. output columns.
__host__ __device__ inline int mx8_row(int s, int m) { return 8 * (m >> 2) + 4 * s + (m & 3); }

// Scale byte of a block from its largest magnitude's bits (a NaN's are above infinity's).  The mantissas above 1.75 carry over.
__device__ __forceinline__ uint32_t mx8_scale_byte(uint32_t magnitude) {
  const uint32_t e = (magnitude + 0x1FFFFFu) >> 23;
  return magnitude >= 0x7F800000u ? 255u : (e > 8u ? e : 8u) - 8u;
}
// The scale as the conversion instructions take it: they read its exponent, 0 as 2^-127.
__device__ __forceinline__ float mx8_scale_f32(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four numbers -> a word of codes, the first one lowest.  The instruction rounds to the nearest, ties to even.
__device__ __forceinline__ uint32_t mx8_codes(float a, float b, float c, float d, float scale) {
  typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
  i16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
// Eight numbers -> two words of codes; of a block that is not finite, codes of NaN.
__device__ __forceinline__ uint2 mx8_codes8(const float* v, uint32_t byte) {
  const float scale = mx8_scale_f32(byte);
  const uint32_t lo = mx8_codes(v[0], v[1], v[2], v[3], scale), hi = mx8_codes(v[4], v[5], v[6], v[7], scale);
  return byte == 255u ? make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu) : make_uint2(lo, hi);
}

// Lanes of four: largest value among them.
__device__ __forceinline__ uint32_t mx8_quad_max(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, false)));
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, false)));
}

// 16 bytes at any address that fits the element: the hardware takes unaligned ones, at the cost of the lines they straddle.
typedef uint32_t mx8_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t mx8_u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <bool ONCE>  // ONCE: past the caches' retention
__device__ __forceinline__ mx8_u32x4 mx8_load_any(const void* p) {
  const auto q = reinterpret_cast<const __attribute__((address_space(1))) mx8_u32x4_any*>(reinterpret_cast<uintptr_t>(p));
  return ONCE ? __builtin_nontemporal_load(q) : *q;
}
template <bool ONCE>
__device__ __forceinline__ void mx8_store_any(void* p, mx8_u32x4 v) {
  const auto q = reinterpret_cast<__attribute__((address_space(1))) mx8_u32x4_any*>(reinterpret_cast<uintptr_t>(p));
  if (ONCE) __builtin_nontemporal_store(v, q);
  else *q = v;
}

// Eight numbers of a row of n from column k0 on as fp32 bits, those past the row as zeros.  El: float, or uint16_t for bf16.
template <typename El, bool ONCE>
__device__ __forceinline__ void mx8_load8(const El* row, int64_t k0, int64_t n, uint32_t* bits) {
  if (k0 + 8 <= n) {
    if (sizeof(El) == 4) {
      const mx8_u32x4 a = mx8_load_any<ONCE>(row + k0), b = mx8_load_any<ONCE>(row + k0 + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) { bits[j] = a[j]; bits[4 + j] = b[j]; }
    } else {
      const mx8_u32x4 a = mx8_load_any<ONCE>(row + k0);
#pragma unroll
      for (int j = 0; j < 8; ++j) bits[j] = (j & 1) ? a[j / 2] & 0xFFFF0000u : a[j / 2] << 16;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      bits[j] = 0;
      if (k0 + j < n) bits[j] = sizeof(El) == 4 ? reinterpret_cast<const uint32_t*>(row)[k0 + j] : static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[k0 + j]) << 16;
    }
  }
}

// Two fp32 -> one word of two bf16, round-to-nearest-even.
__device__ __forceinline__ uint32_t mx8_pack_bf16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// The way back: eight numbers, rounded to El once, those past the row left out.
template <typename El, bool ONCE>
__device__ __forceinline__ void mx8_store8(El* row, int64_t k0, int64_t n, const float* v) {
  uint32_t w[8];
  if (sizeof(El) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = mx8_pack_bf16(v[2 * j], v[2 * j + 1]);
  }
  if (k0 + 8 <= n) {
    mx8_store_any<ONCE>(row + k0, mx8_u32x4{w[0], w[1], w[2], w[3]});
    if (sizeof(El) == 4) mx8_store_any<ONCE>(row + k0 + 4, mx8_u32x4{w[4], w[5], w[6], w[7]});
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (k0 + j >= n) continue;
      if (sizeof(El) == 4) reinterpret_cast<uint32_t*>(row)[k0 + j] = w[j];
      else reinterpret_cast<uint16_t*>(row)[k0 + j] = static_cast<uint16_t>(w[j / 2] >> (16 * (j & 1)));
    }
  }
}

}  // namespace revive
