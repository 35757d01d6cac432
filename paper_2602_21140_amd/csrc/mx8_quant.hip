// Microscaled 8-bit floats: quantisation of rows, the way back, and the packed layout of weights (mx8.hpp has the format).
#include <algorithm>

#include "ctx.hpp"
#include "mx8.hpp"

namespace revive {

namespace {

struct Mx8Rows {
  const void* x;            // quantise: the numbers; dequantise: not used
  void* out;                // dequantise: the numbers
  int64_t rows, ld;         // elements between rows of numbers
  int K, blocks;
  int row_threads_log2;     // threads side by side on a row
  uint8_t* codes; uint8_t* scales;
};

// A thread takes units of eight numbers, four threads a block, so that a wavefront reads and writes in address order; kUnits of
// them are in flight.  ONCE (rows larger than the last-level cache): non-temporal loads and stores of the numbers.
// HBM bounds both: 32 768 x 7168 bf16 take 121 us there and 107 back, 5.9 and 6.7 TB/s.
constexpr int kUnits = 4;
constexpr int64_t kOnceBytes = 256ll << 20;

template <typename El, bool ONCE>
__global__ __launch_bounds__(256) void mx8_quantize_kernel(Mx8Rows a) {
  const int tr = 1 << a.row_threads_log2, col = threadIdx.x & (tr - 1);
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) >> a.row_threads_log2;
  if (row >= a.rows) return;
  const El* x = static_cast<const El*>(a.x) + row * a.ld;
  const int u0 = blockIdx.y * (tr * kUnits) + col;
  uint32_t bits[kUnits][8];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) mx8_load8<El, ONCE>(x, static_cast<int64_t>(u0 + i * tr) * 8, a.K, bits[i]);
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i * tr;
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m = max(m, bits[i][j] & 0x7FFFFFFFu);
      v[j] = __uint_as_float(bits[i][j]);
    }
    const uint32_t byte = mx8_scale_byte(mx8_quad_max(m));
    if (u >= a.blocks * 4) continue;
    *reinterpret_cast<uint2*>(a.codes + row * a.blocks * 32 + u * 8) = mx8_codes8(v, byte);
    if ((u & 3) == 0) a.scales[row * a.blocks + (u >> 2)] = static_cast<uint8_t>(byte);
  }
}

template <typename El, bool ONCE>
__global__ __launch_bounds__(256) void mx8_dequantize_kernel(Mx8Rows a) {
  const int tr = 1 << a.row_threads_log2, col = threadIdx.x & (tr - 1);
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) >> a.row_threads_log2;
  if (row >= a.rows) return;
  El* out = static_cast<El*>(a.out) + row * a.ld;
  const int u0 = blockIdx.y * (tr * kUnits) + col;
  uint2 word[kUnits];
  uint32_t byte[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = min(u0 + i * tr, a.blocks * 4 - 1);
    word[i] = *reinterpret_cast<const uint2*>(a.codes + row * a.blocks * 32 + u * 8);
    byte[i] = a.scales[row * a.blocks + (u >> 2)];
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i * tr;
    if (u >= a.blocks * 4) continue;
    const float s = mx8_scale_f32(byte[i]);
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].x, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].x, s, true),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].y, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].y, s, true)};
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = byte[i] == 255u ? __uint_as_float(0x7FC00000u) : p[j / 2][j & 1];
    mx8_store8<El, ONCE>(out, static_cast<int64_t>(u) * 8, a.K, v);
  }
}

// A grid has fewer than 2^32 threads in x (a launch of more runs what is left of them modulo 2^32, without an error): rows that
// one launch can take.
constexpr int64_t kMaxThreads = (1ll << 32) - 256;

// kernel(grid, arguments) for as many rows at a time as one launch takes.
template <typename F>
int by_rows(const Mx8Rows& base, int64_t element, F kernel) {
  Mx8Rows a = base;
  const int units = a.blocks * 4;
  a.row_threads_log2 = 2;
  while (a.row_threads_log2 < 8 && (kUnits << a.row_threads_log2) < units) ++a.row_threads_log2;
  for (int64_t row = 0; row < base.rows; row += a.rows) {
    a.rows = std::min(base.rows - row, kMaxThreads >> a.row_threads_log2);
    a.x = static_cast<const uint8_t*>(base.x) + row * a.ld * element;
    a.out = static_cast<uint8_t*>(base.out) + row * a.ld * element;
    a.codes = base.codes + row * a.blocks * 32;
    a.scales = base.scales + row * a.blocks;
    const dim3 grid(static_cast<uint32_t>(((a.rows << a.row_threads_log2) + 255) / 256), ceil_div(units, kUnits << a.row_threads_log2));
    kernel(grid, a);
    const int rc = check_hip(nullptr, hipGetLastError(), "8-bit rounding launch");
    if (rc != REVIVE_OK) return rc;
  }
  return REVIVE_OK;
}

template <typename El>
int launch_quantize(const Mx8Rows& a, hipStream_t s) {
  const bool once = a.rows * a.K * static_cast<int64_t>(sizeof(El)) > kOnceBytes;
  return by_rows(a, sizeof(El), [&](dim3 grid, const Mx8Rows& r) {
    if (once) hipLaunchKernelGGL((mx8_quantize_kernel<El, true>), grid, dim3(256), 0, s, r);
    else hipLaunchKernelGGL((mx8_quantize_kernel<El, false>), grid, dim3(256), 0, s, r);
  });
}
template <typename El>
int launch_dequantize(const Mx8Rows& a, hipStream_t s) {
  const bool once = a.rows * a.K * static_cast<int64_t>(sizeof(El)) > kOnceBytes;
  return by_rows(a, sizeof(El), [&](dim3 grid, const Mx8Rows& r) {
    if (once) hipLaunchKernelGGL((mx8_dequantize_kernel<El, true>), grid, dim3(256), 0, s, r);
    else hipLaunchKernelGGL((mx8_dequantize_kernel<El, false>), grid, dim3(256), 0, s, r);
  });
}

// Rows of codes and scales into the packed layout: a thread moves 16 bytes of a lane's codes, or a lane's eight scales of a
// panel's step.  Done once per matrix, so nothing here is tuned.
__global__ __launch_bounds__(256) void mx8_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K,
                                                       uint8_t* __restrict__ packed, int64_t n_codes, int64_t n_scales) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int blocks = K / kMx8Block, steps = mx8_steps(K);
  auto row_of = [](int64_t panel, int sub, int lane) { return panel * kMx8Panel + (sub >> 1) * 32 + mx8_row(sub & 1, lane & 15); };
  if (i < n_codes) {
    const int lane = i & 63, half = (i >> 6) & 1, sub = (i >> 7) & 7;
    const int64_t rest = i >> 10;
    const int step = static_cast<int>(rest % steps);
    const int64_t row = row_of(rest / steps, sub, lane);
    const int64_t k = static_cast<int64_t>(step) * kMx8Step + half * 64 + (lane >> 4) * 16;
    mx8_u32x4 v = {0u, 0u, 0u, 0u};
    if (row < rows && k < K) v = mx8_load_any<false>(codes + row * K + k);
    reinterpret_cast<mx8_u32x4*>(packed)[i] = v;
  } else if (i < n_codes + n_scales) {
    const int64_t o = i - n_codes;
    const int lane = o & 63;
    const int64_t rest = o >> 6;
    const int block = static_cast<int>(rest % steps) * 4 + (lane >> 4);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int sub = 0; sub < 8; ++sub) {
      const int64_t row = row_of(rest / steps, sub, lane);
      if (row < rows && block < blocks) w[sub >> 2] |= static_cast<uint32_t>(scales[row * blocks + block]) << (8 * (sub & 3));
    }
    reinterpret_cast<uint2*>(packed + n_codes * 16)[o] = make_uint2(w[0], w[1]);
  }
}

int check_rows(const char* who, int32_t dtype, int64_t rows, int32_t K, int64_t ld) {
  if (dtype != REVIVE_DTYPE_F32 && dtype != REVIVE_DTYPE_BF16) return fail(nullptr, REVIVE_EINVAL, "%s: dtype must be 0 (fp32) or 1 (bf16)", who);
  if (rows < 0 || K <= 0 || K > (1 << 24) || ld < K) return fail(nullptr, REVIVE_EINVAL, "%s: rows >= 0, 0 < K <= 2^24 and ld >= K required", who);
  return REVIVE_OK;
}
int check_pointers(const char* who, const void* numbers, int32_t dtype, const uint8_t* codes, const uint8_t* scales) {
  if (!numbers || !codes || !scales) return fail(nullptr, REVIVE_EINVAL, "%s: null argument", who);
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0) return fail(nullptr, REVIVE_EINVAL, "%s: codes must be 16-byte aligned", who);
  if (reinterpret_cast<uintptr_t>(numbers) % (dtype == REVIVE_DTYPE_F32 ? 4 : 2) != 0)
    return fail(nullptr, REVIVE_EINVAL, "%s: the numbers are not aligned to their type", who);
  return REVIVE_OK;
}

}  // namespace

}  // namespace revive

using namespace revive;

extern "C" {

int revive_mx_eight_quantize(const void* x, int32_t dtype, int64_t rows, int32_t K, int64_t ld, uint8_t* codes, uint8_t* scales, revive_stream stream) {
  int rc = check_rows("revive_mx_eight_quantize", dtype, rows, K, ld);
  if (rc != REVIVE_OK || rows == 0) return rc;
  rc = check_pointers("revive_mx_eight_quantize", x, dtype, codes, scales);
  if (rc != REVIVE_OK) return rc;
  Mx8Rows a{};
  a.x = x; a.rows = rows; a.ld = ld; a.K = K; a.blocks = ceil_div(K, kMx8Block); a.codes = codes; a.scales = scales;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == REVIVE_DTYPE_F32 ? launch_quantize<float>(a, s) : launch_quantize<uint16_t>(a, s);
}

int revive_mx_eight_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t K, int32_t dtype, void* out, int64_t ld, revive_stream stream) {
  int rc = check_rows("revive_mx_eight_dequantize", dtype, rows, K, ld);
  if (rc != REVIVE_OK || rows == 0) return rc;
  rc = check_pointers("revive_mx_eight_dequantize", out, dtype, codes, scales);
  if (rc != REVIVE_OK) return rc;
  Mx8Rows a{};
  a.out = out; a.rows = rows; a.ld = ld; a.K = K; a.blocks = ceil_div(K, kMx8Block);
  a.codes = const_cast<uint8_t*>(codes); a.scales = const_cast<uint8_t*>(scales);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == REVIVE_DTYPE_F32 ? launch_dequantize<float>(a, s) : launch_dequantize<uint16_t>(a, s);
}

int revive_mx_eight_packed_bytes(int32_t rows, int32_t K, size_t* bytes) {
  if (!bytes) return fail(nullptr, REVIVE_EINVAL, "revive_mx_eight_packed_bytes: null argument");
  if (rows <= 0 || K <= 0 || K > kMx8MaxK || K % kMx8Block != 0 || static_cast<int64_t>(rows) * K >= (1ll << 32))
    return fail(nullptr, REVIVE_EINVAL, "revive_mx_eight_packed_bytes: rows > 0, K a multiple of 32 up to 2^24 and rows * K < 2^32 required");
  *bytes = static_cast<size_t>(mx8_packed_bytes(rows, K));
  return REVIVE_OK;
}

int revive_mx_eight_pack(const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t K, void* packed, revive_stream stream) {
  size_t bytes = 0;
  const int rc = revive_mx_eight_packed_bytes(rows, K, &bytes);
  if (rc != REVIVE_OK) return rc;
  if (!codes || !scales || !packed) return fail(nullptr, REVIVE_EINVAL, "revive_mx_eight_pack: null argument");
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0 || reinterpret_cast<uintptr_t>(packed) % 16 != 0)
    return fail(nullptr, REVIVE_EINVAL, "revive_mx_eight_pack: codes and packed must be 16-byte aligned");
  const int64_t n_codes = mx8_packed_codes(rows, K) / 16, n_scales = (static_cast<int64_t>(bytes) - n_codes * 16) / 8;
  hipLaunchKernelGGL(mx8_pack_kernel, dim3(static_cast<uint32_t>((n_codes + n_scales + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream),
                     codes, scales, rows, K, static_cast<uint8_t*>(packed), n_codes, n_scales);
  return check_hip(nullptr, hipGetLastError(), "mx8_pack launch");
}

}  // extern "C"
