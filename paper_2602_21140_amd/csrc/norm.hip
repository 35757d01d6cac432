// Root-mean-square norm in front of the layer, with the residual's addition and an 8-bit output.
//
//   s = x + residual, rounded to dtype (the residual stream as it goes on)
//   y = s / sqrt(mean(s^2) + eps) * weight, rounded to dtype (what the router reads)
//   codes, scales = the microscaled 8-bit form of y (what the 8-bit experts and products read)
#include <algorithm>

#include "ctx.hpp"
#include "mx8.hpp"

namespace revive {

namespace {

struct NormArgs {
  const void* x; const void* residual; const void* weight;
  int64_t rows, ld_x, ld_residual;  // elements between rows
  int H;
  double eps;
  void* sum; void* y;               // [rows, H]
  uint8_t* codes; uint8_t* scales;  // [rows, 32 blocks], [rows, blocks]
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) v += __shfl_xor(v, i);
  return v;
}

// TPR threads share a row, each with U units of eight numbers at a time, TPR units apart.  HELD: that is the whole row, which
// stays in registers; otherwise the row is read twice.
//
// The squares are summed in fp64: no row is too large or too small for it, and the result does not hang on the order of the
// sum, so that y's last bit, and with it the 8-bit form of a number next to a border, is the same for every shape of the kernel.
template <typename El, int TPR, int U, bool HELD>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rms_norm_kernel(NormArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1, WAVES = TPR / 64;
  __shared__ double part[WAVES];
  const int t = threadIdx.x & (TPR - 1);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
  if (row >= a.rows) return;  // with WAVES > 1, the whole workgroup
  const El* x = static_cast<const El*>(a.x) + row * a.ld_x;
  const El* residual = a.residual ? static_cast<const El*>(a.residual) + row * a.ld_residual : nullptr;
  const El* weight = static_cast<const El*>(a.weight);
  El* sum = a.sum ? static_cast<El*>(a.sum) + row * a.H : nullptr;
  El* y = a.y ? static_cast<El*>(a.y) + row * a.H : nullptr;
  const int blocks = (a.H + 31) >> 5;

  float v[U][8];
  auto rounded = [](float f) { return sizeof(El) == 4 ? f : __uint_as_float(mx8_pack_bf16(f, f) << 16); };
  auto load = [&](int c, bool first) {  // s of the units from c on
    uint32_t bx[U][8], br[U][8];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int64_t k = static_cast<int64_t>(c + i * TPR + t) * 8;
      mx8_load8<El, false>(x, k, a.H, bx[i]);
      if (residual) mx8_load8<El, false>(residual, k, a.H, br[i]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = __uint_as_float(bx[i][j]);
        if (residual) v[i][j] = rounded(v[i][j] + __uint_as_float(br[i][j]));
      }
      if (first && sum) mx8_store8<El, false>(sum, static_cast<int64_t>(c + i * TPR + t) * 8, a.H, v[i]);
    }
  };
  const int units = blocks * 4;
  double square = 0;
  for (int c = 0; c < units; c += U * TPR) {
    load(c, true);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) square = fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), square);
  }
  square = wave_sum(square);
  if (WAVES > 1) {
    if ((t & 63) == 0) part[t >> 6] = square;
    __syncthreads();
    square = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) square += part[w];
  }
  const double inverse = 1.0 / sqrt(square / a.H + a.eps);
  const float inv = static_cast<float>(inverse);
  const bool plain = inv > 0x1p-100f && inv < 0x1p+100f;  // else the product with s may be in fp32's range where inv is not
  for (int c = 0; c < units; c += U * TPR) {
    if (!HELD) {
      if (sum) { x = sum; residual = nullptr; }  // where x or the residual was, if sum replaces it
      load(c, false);
    }
    uint32_t bw[U][8];
#pragma unroll
    for (int i = 0; i < U; ++i) mx8_load8<El, false>(weight, static_cast<int64_t>(c + i * TPR + t) * 8, a.H, bw[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = c + i * TPR + t;
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = plain ? v[i][j] * inv : static_cast<float>(static_cast<double>(v[i][j]) * inverse);
        v[i][j] = static_cast<int64_t>(u) * 8 + j < a.H ? rounded(n * __uint_as_float(bw[i][j])) : 0.f;
        m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
      }
      const uint32_t byte = mx8_scale_byte(mx8_quad_max(m));
      if (u >= units) continue;
      if (y) mx8_store8<El, false>(y, static_cast<int64_t>(u) * 8, a.H, v[i]);
      if (a.codes) {
        *reinterpret_cast<uint2*>(a.codes + (row * blocks * 4 + u) * 8) = mx8_codes8(v[i], byte);
        if ((u & 3) == 0) a.scales[row * blocks + (u >> 2)] = static_cast<uint8_t>(byte);
      }
    }
  }
}

// A grid has fewer than 2^32 threads in x (a launch of more runs what is left of them modulo 2^32, without an error).
constexpr int64_t kMaxThreads = (1ll << 32) - 1024;

template <typename El, int TPR, int U, bool HELD>
int launch(const NormArgs& base, hipStream_t stream) {
  constexpr int NT = TPR < 256 ? 256 : TPR;
  NormArgs a = base;
  const int blocks = ceil_div(a.H, 32);
  for (int64_t row = 0; row < base.rows; row += a.rows) {
    a.rows = std::min<int64_t>(base.rows - row, kMaxThreads / TPR);
    a.x = static_cast<const El*>(base.x) + row * a.ld_x;
    if (a.residual) a.residual = static_cast<const El*>(base.residual) + row * a.ld_residual;
    if (a.sum) a.sum = static_cast<El*>(base.sum) + row * a.H;
    if (a.y) a.y = static_cast<El*>(base.y) + row * a.H;
    if (a.codes) { a.codes = base.codes + row * blocks * 32; a.scales = base.scales + row * blocks; }
    const uint32_t grid = static_cast<uint32_t>((a.rows * TPR + NT - 1) / NT);
    hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, HELD>), dim3(grid), dim3(NT), 0, stream, a);
    const int rc = check_hip(nullptr, hipGetLastError(), "add_rms_norm launch");
    if (rc != REVIVE_OK) return rc;
  }
  return REVIVE_OK;
}

template <typename El>
int launch_norm(const NormArgs& a, hipStream_t s) {
  const int units = ceil_div(a.H, 32) * 4;
  if (units <= 64) return launch<El, 64, 1, true>(a, s);
  if (units <= 256) return launch<El, 256, 1, true>(a, s);
  if (units <= 512) return launch<El, 256, 2, true>(a, s);
  if (units <= 1024) return launch<El, 256, 4, true>(a, s);
  if (units <= 2048) return launch<El, 1024, 2, true>(a, s);
  return launch<El, 1024, 2, false>(a, s);
}

}  // namespace

}  // namespace revive

using namespace revive;

extern "C" {

int revive_add_rms_norm(const void* x, const void* residual, const void* weight, int32_t dtype, int64_t rows, int32_t H, int64_t ld_x,
                        int64_t ld_residual, float eps, void* sum, void* y, uint8_t* codes, uint8_t* scales, revive_stream stream) {
  const char* who = "revive_add_rms_norm";
  if (dtype != REVIVE_DTYPE_F32 && dtype != REVIVE_DTYPE_BF16) return fail(nullptr, REVIVE_EINVAL, "%s: dtype must be 0 (fp32) or 1 (bf16)", who);
  if (rows < 0 || H <= 0 || H > (1 << 24) || ld_x < H || (residual && ld_residual < H))
    return fail(nullptr, REVIVE_EINVAL, "%s: rows >= 0, 0 < H <= 2^24 and rows at least H elements apart required", who);
  if (!(eps >= 0.f && eps <= 3.4e38f)) return fail(nullptr, REVIVE_EINVAL, "%s: eps must be finite and not negative", who);
  if (rows == 0) return REVIVE_OK;
  if (!x || !weight || (!y && !codes)) return fail(nullptr, REVIVE_EINVAL, "%s: null argument", who);
  if (!codes != !scales) return fail(nullptr, REVIVE_EINVAL, "%s: codes and scales come together", who);
  if (sum && !residual) return fail(nullptr, REVIVE_EINVAL, "%s: a sum without a residual", who);
  if ((x == sum || x == y) && ld_x != H) return fail(nullptr, REVIVE_EINVAL, "%s: in place, rows are H elements apart", who);
  if (residual && (residual == sum || residual == y) && ld_residual != H)
    return fail(nullptr, REVIVE_EINVAL, "%s: in place, rows are H elements apart", who);
  if (sum && sum == y) return fail(nullptr, REVIVE_EINVAL, "%s: sum and y are one buffer", who);
  const uintptr_t element = dtype == REVIVE_DTYPE_F32 ? 4 : 2;
  for (const void* p : {x, residual, weight, static_cast<const void*>(sum), static_cast<const void*>(y)})
    if (reinterpret_cast<uintptr_t>(p) % element != 0) return fail(nullptr, REVIVE_EINVAL, "%s: a pointer is not aligned to its elements", who);
  if (reinterpret_cast<uintptr_t>(codes) % 16 != 0) return fail(nullptr, REVIVE_EINVAL, "%s: codes must be 16-byte aligned", who);
  const NormArgs a{x, residual, weight, rows, ld_x, ld_residual, H, static_cast<double>(eps), sum, y, codes, scales};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == REVIVE_DTYPE_F32 ? launch_norm<float>(a, s) : launch_norm<uint16_t>(a, s);
}

}  // extern "C"
