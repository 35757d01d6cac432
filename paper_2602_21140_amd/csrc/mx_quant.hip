// Microscaled 4-bit floats: quantisation of rows, the way back, and the packed layout of weights (mx.hpp has the format).
#include <algorithm>

#include "ctx.hpp"
#include "mx.hpp"
#include "mx_quant.hpp"

namespace revive {

namespace {

// 16 bytes at any address that fits the element: the hardware takes unaligned ones, at the cost of the lines they straddle.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <bool ONCE>  // ONCE: past the caches' retention
__device__ __forceinline__ u32x4 load_16B(const void* p) {
  const auto q = reinterpret_cast<const __attribute__((address_space(1))) u32x4_any*>(reinterpret_cast<uintptr_t>(p));
  return ONCE ? __builtin_nontemporal_load(q) : *q;
}
template <bool ONCE>
__device__ __forceinline__ void store_16B(void* p, u32x4 v) {
  const auto q = reinterpret_cast<__attribute__((address_space(1))) u32x4_any*>(reinterpret_cast<uintptr_t>(p));
  if (ONCE) __builtin_nontemporal_store(v, q);
  else *q = v;
}

// Lanes of four: largest value among them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, false)));
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, false)));
}

struct QuantArgs {
  const void* x;
  int64_t rows, ld;       // elements between rows
  int K, units;           // units of eight numbers a row is stored in, the last ones zeros
  int row_threads_log2;   // threads side by side on a row
  uint8_t* codes;
  int64_t code_row;       // bytes between rows of codes
  uint8_t* scales;
  int64_t scale_row;
};

// A thread takes units of eight numbers, four threads a block: 16 (32) bytes in, four bytes of codes out, so that a wavefront
// reads and writes in address order.  kUnits of them are in flight.  TILED: the scales' order is that of the kernels'
// activations.
//
// Bound by HBM: 32 768 x 7168 bf16 to codes in 91 us (6.5 TB/s) and back in 84 (7.0).  ONCE (rows larger than the last-level cache):
// non-temporal loads, here and for the way back non-temporal stores, leave the caches to the codes.
constexpr int kUnits = 4;
constexpr int64_t kOnceBytes = 256ll << 20;
template <typename El, bool ONCE, bool TILED>
__global__ __launch_bounds__(256) void mx_quantize_kernel(QuantArgs a) {
  const int tr = 1 << a.row_threads_log2, col = threadIdx.x & (tr - 1);
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) >> a.row_threads_log2;
  if (row >= a.rows) return;
  const El* x = static_cast<const El*>(a.x) + row * a.ld;
  const int u0 = blockIdx.y * (tr * kUnits) + col;
  uint32_t raw[kUnits][sizeof(El) * 2];  // eight numbers
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i * tr, k0 = u * 8;
#pragma unroll
    for (int w = 0; w < static_cast<int>(sizeof(El)) * 2; ++w) raw[i][w] = 0;
    if (k0 + 8 <= a.K) {
#pragma unroll
      for (int w = 0; w < static_cast<int>(sizeof(El)) / 2; ++w) {
        const u32x4 v = load_16B<ONCE>(x + k0 + w * (16 / sizeof(El)));
        raw[i][w * 4] = v[0]; raw[i][w * 4 + 1] = v[1]; raw[i][w * 4 + 2] = v[2]; raw[i][w * 4 + 3] = v[3];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (k0 + j >= a.K) continue;
        if (sizeof(El) == 4) raw[i][j] = reinterpret_cast<const uint32_t*>(x)[k0 + j];
        else raw[i][j / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(x)[k0 + j]) << (16 * (j & 1));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i * tr;
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = sizeof(El) == 4 ? raw[i][j] : (j & 1) ? raw[i][j / 2] & 0xFFFF0000u : raw[i][j / 2] << 16;
      m = max(m, b & 0x7FFFFFFFu);
      v[j] = __uint_as_float(b);
    }
    const uint32_t byte = mx_scale_byte(quad_max(m));
    if (u >= a.units) continue;
    *reinterpret_cast<uint32_t*>(a.codes + row * a.code_row + u * 4) = mx_codes(v, mx_scale_f32(byte));
    if ((u & 3) == 0) a.scales[row * a.scale_row + (TILED ? mx_scale_at(u >> 2) : u >> 2)] = static_cast<uint8_t>(byte);
  }
}

// A grid has fewer than 2^32 threads in x (a launch of more runs what is left of them modulo 2^32, without an error): rows that
// one launch can take.
constexpr int64_t kMaxThreads = (1ll << 32) - 256;
int64_t rows_of_launch(int row_threads_log2) { return kMaxThreads >> row_threads_log2; }
dim3 grid_of(int64_t rows, int units, int row_threads_log2) {
  return dim3(static_cast<uint32_t>(((rows << row_threads_log2) + 255) / 256), ceil_div(units, kUnits << row_threads_log2));
}
int row_threads_log2_of(int units) {
  int n = 2;
  while (n < 8 && (kUnits << n) < units) ++n;
  return n;
}

template <typename El, bool TILED>
int launch_quantize(const QuantArgs& base, hipStream_t stream, const revive_ctx* ctx) {
  QuantArgs a = base;
  if (a.units == 0) return REVIVE_OK;
  a.row_threads_log2 = row_threads_log2_of(a.units);
  const bool once = base.rows * a.K * static_cast<int64_t>(sizeof(El)) > kOnceBytes;
  for (int64_t row = 0; row < base.rows; row += a.rows) {
    a.rows = std::min(base.rows - row, rows_of_launch(a.row_threads_log2));
    a.x = static_cast<const El*>(base.x) + row * a.ld;
    a.codes = base.codes + row * a.code_row;
    a.scales = base.scales + row * a.scale_row;
    const dim3 grid = grid_of(a.rows, a.units, a.row_threads_log2);
    if (once) hipLaunchKernelGGL((mx_quantize_kernel<El, true, TILED>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((mx_quantize_kernel<El, false, TILED>), grid, dim3(256), 0, stream, a);
    const int rc = check_hip(ctx, hipGetLastError(), "mx_quantize launch");
    if (rc != REVIVE_OK) return rc;
  }
  return REVIVE_OK;
}

struct DequantArgs {
  const uint8_t* codes; const uint8_t* scales;
  void* out;
  int64_t rows, ld;
  int K, blocks, units, row_threads_log2;
};

template <typename El, bool ONCE>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(DequantArgs a) {
  const int tr = 1 << a.row_threads_log2, col = threadIdx.x & (tr - 1);
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) >> a.row_threads_log2;
  if (row >= a.rows) return;
  El* out = static_cast<El*>(a.out) + row * a.ld;
  const int u0 = blockIdx.y * (tr * kUnits) + col;
  uint32_t word[kUnits], byte[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = min(u0 + i * tr, a.units - 1);
    word[i] = *reinterpret_cast<const uint32_t*>(a.codes + row * a.blocks * 16 + u * 4);
    byte[i] = a.scales[row * a.blocks + (u >> 2)];
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i * tr, k0 = u * 8;
    if (u >= a.units) continue;
    const float s = mx_scale_f32(byte[i]);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], s, 3)};
    uint32_t b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = byte[i] == 255u ? 0x7FC00000u : __float_as_uint(p[j / 2][j & 1]);
    if (k0 + 8 <= a.K) {
      if (sizeof(El) == 4) {
        store_16B<ONCE>(out + k0, u32x4{b[0], b[1], b[2], b[3]});
        store_16B<ONCE>(out + k0 + 4, u32x4{b[4], b[5], b[6], b[7]});
      } else {  // two significant bits: bf16 holds every value, subnormal ones too
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (b[2 * j] >> 16) | (b[2 * j + 1] & 0xFFFF0000u);
        store_16B<ONCE>(out + k0, u32x4{w[0], w[1], w[2], w[3]});
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (k0 + j >= a.K) continue;
        if (sizeof(El) == 4) reinterpret_cast<uint32_t*>(out)[k0 + j] = b[j];
        else reinterpret_cast<uint16_t*>(out)[k0 + j] = static_cast<uint16_t>(b[j] >> 16);
      }
    }
  }
}

template <typename El>
int launch_dequantize(const DequantArgs& base, hipStream_t stream) {
  DequantArgs a = base;
  a.row_threads_log2 = row_threads_log2_of(a.units);
  const bool once = base.rows * a.K * static_cast<int64_t>(sizeof(El)) > kOnceBytes;
  for (int64_t row = 0; row < base.rows; row += a.rows) {
    a.rows = std::min(base.rows - row, rows_of_launch(a.row_threads_log2));
    a.codes = base.codes + row * a.blocks * 16;
    a.scales = base.scales + row * a.blocks;
    a.out = static_cast<El*>(base.out) + row * a.ld;
    const dim3 grid = grid_of(a.rows, a.units, a.row_threads_log2);
    if (once) hipLaunchKernelGGL((mx_dequantize_kernel<El, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((mx_dequantize_kernel<El, false>), grid, dim3(256), 0, stream, a);
    const int rc = check_hip(nullptr, hipGetLastError(), "mx_dequantize launch");
    if (rc != REVIVE_OK) return rc;
  }
  return REVIVE_OK;
}

// Rows of codes and scales into the packed layout: a thread moves the 16 bytes of a lane, or a lane's word of scales.  Done
// once per matrix, so nothing here is tuned.
__global__ __launch_bounds__(256) void mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K,
                                                      uint8_t* __restrict__ packed, int64_t n_codes, int64_t n_scales) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int blocks = K / kMxBlock;
  auto row_of = [](int64_t panel, int sub, int lane) { return panel * kMxPanel + (sub >> 1) * 32 + mx_row(sub & 1, lane & 15); };
  if (i < n_codes) {
    const int lane = i & 63, sub = (i >> 6) & 7;
    const int64_t rest = i >> 9;
    const int steps = mx_steps(K), step = static_cast<int>(rest % steps);
    const int64_t row = row_of(rest / steps, sub, lane);
    const int block = step * 4 + (lane >> 4);
    u32x4 v = {0u, 0u, 0u, 0u};
    if (row < rows && block < blocks) v = load_16B<false>(codes + (row * blocks + block) * 16);
    reinterpret_cast<u32x4*>(packed)[i] = v;
  } else if (i < n_codes + n_scales) {
    const int64_t o = i - n_codes;
    const int lane = o & 63, sub = (o >> 6) & 7;
    const int64_t rest = o >> 9;
    const int groups = mx_groups(K), group = static_cast<int>(rest % groups);
    const int64_t row = row_of(rest / groups, sub, lane);
    uint32_t w = 0;
    for (int s = 0; s < 4; ++s) {
      const int block = (group * 4 + s) * 4 + (lane >> 4);
      if (row < rows && block < blocks) w |= static_cast<uint32_t>(scales[row * blocks + block]) << (8 * s);
    }
    reinterpret_cast<uint32_t*>(packed + n_codes * 16)[o] = w;
  }
}

}  // namespace

int launch_mx_quantize_tiled(revive_ctx* ctx, const void* x, int64_t rows, int K, uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  QuantArgs a{};
  a.x = x; a.rows = rows; a.ld = K; a.K = K;
  a.units = mx_steps(K) * (kMxStep / 8);
  a.codes = codes; a.code_row = mx_code_row(K);
  a.scales = scales; a.scale_row = mx_scale_row(K);
  KernelTimer timer(ctx, REVIVE_K_MX_QUANTIZE, stream);
  return launch_quantize<uint16_t, true>(a, stream, ctx);
}

}  // namespace revive

using namespace revive;

extern "C" {

int revive_mx_quantize(const void* x, int32_t dtype, int64_t rows, int32_t K, int64_t ld, uint8_t* codes, uint8_t* scales, revive_stream stream) {
  if (dtype != REVIVE_DTYPE_F32 && dtype != REVIVE_DTYPE_BF16) return fail(nullptr, REVIVE_EINVAL, "revive_mx_quantize: dtype must be 0 (fp32) or 1 (bf16)");
  if (rows < 0 || K <= 0 || K > (1 << 24) || ld < K) return fail(nullptr, REVIVE_EINVAL, "revive_mx_quantize: rows >= 0, 0 < K <= 2^24 and ld >= K required");
  if (rows == 0) return REVIVE_OK;
  if (!x || !codes || !scales) return fail(nullptr, REVIVE_EINVAL, "revive_mx_quantize: null argument");
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0) return fail(nullptr, REVIVE_EINVAL, "revive_mx_quantize: codes must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(x) % (dtype == REVIVE_DTYPE_F32 ? 4 : 2) != 0) return fail(nullptr, REVIVE_EINVAL, "revive_mx_quantize: x is not aligned to its elements");
  const int blocks = ceil_div(K, kMxBlock);
  QuantArgs a{};
  a.x = x; a.rows = rows; a.ld = ld; a.K = K; a.units = blocks * 4;
  a.codes = codes; a.code_row = static_cast<int64_t>(blocks) * 16;
  a.scales = scales; a.scale_row = blocks;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == REVIVE_DTYPE_F32 ? launch_quantize<float, false>(a, s, nullptr) : launch_quantize<uint16_t, false>(a, s, nullptr);
}

int revive_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t K, int32_t dtype, void* out, int64_t ld, revive_stream stream) {
  if (dtype != REVIVE_DTYPE_F32 && dtype != REVIVE_DTYPE_BF16) return fail(nullptr, REVIVE_EINVAL, "revive_mx_dequantize: dtype must be 0 (fp32) or 1 (bf16)");
  if (rows < 0 || K <= 0 || K > (1 << 24) || ld < K) return fail(nullptr, REVIVE_EINVAL, "revive_mx_dequantize: rows >= 0, 0 < K <= 2^24 and ld >= K required");
  if (rows == 0) return REVIVE_OK;
  if (!out || !codes || !scales) return fail(nullptr, REVIVE_EINVAL, "revive_mx_dequantize: null argument");
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0) return fail(nullptr, REVIVE_EINVAL, "revive_mx_dequantize: codes must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(out) % (dtype == REVIVE_DTYPE_F32 ? 4 : 2) != 0) return fail(nullptr, REVIVE_EINVAL, "revive_mx_dequantize: out is not aligned to its elements");
  DequantArgs a{};
  a.codes = codes; a.scales = scales; a.out = out; a.rows = rows; a.ld = ld; a.K = K;
  a.blocks = ceil_div(K, kMxBlock);
  a.units = a.blocks * 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == REVIVE_DTYPE_F32 ? launch_dequantize<float>(a, s) : launch_dequantize<uint16_t>(a, s);
}

int revive_mx_packed_bytes(int32_t rows, int32_t K, size_t* bytes) {
  if (!bytes) return fail(nullptr, REVIVE_EINVAL, "revive_mx_packed_bytes: null argument");
  if (rows <= 0 || K <= 0 || K % kMxBlock != 0 || static_cast<int64_t>(rows) * K >= (1ll << 32))
    return fail(nullptr, REVIVE_EINVAL, "revive_mx_packed_bytes: rows > 0, K a multiple of 32 and rows * K < 2^32 required");
  *bytes = static_cast<size_t>(mx_packed_bytes(rows, K));
  return REVIVE_OK;
}

int revive_mx_pack(const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t K, void* packed, revive_stream stream) {
  size_t bytes = 0;
  const int rc = revive_mx_packed_bytes(rows, K, &bytes);
  if (rc != REVIVE_OK) return rc;
  if (!codes || !scales || !packed) return fail(nullptr, REVIVE_EINVAL, "revive_mx_pack: null argument");
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0 || reinterpret_cast<uintptr_t>(packed) % 16 != 0)
    return fail(nullptr, REVIVE_EINVAL, "revive_mx_pack: codes and packed must be 16-byte aligned");
  const int64_t n_codes = mx_packed_codes(rows, K) / 16, n_scales = (static_cast<int64_t>(bytes) - n_codes * 16) / 4;
  hipLaunchKernelGGL(mx_pack_kernel, dim3(static_cast<uint32_t>((n_codes + n_scales + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream),
                     codes, scales, rows, K, static_cast<uint8_t*>(packed), n_codes, n_scales);
  return check_hip(nullptr, hipGetLastError(), "mx_pack launch");
}

}  // extern "C"
