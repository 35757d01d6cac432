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

// Sum over the wavefront, the same in every lane: four exchanges inside the rows of 16 lanes by cross-lane operands (through LDS,
// as a shuffle goes, each takes ten times as long), then the rows' sums by scalar registers.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_mov_dpp(static_cast<int>(b), CTRL, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_mov_dpp(static_cast<int>(b >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp<0xB1>(v);   // lane ^ 1
  v += dpp<0x4E>(v);   // lane ^ 2
  v += dpp<0x141>(v);  // the half row mirrored
  v += dpp<0x140>(v);  // the row mirrored
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// Sum over the TPR threads of a row; `part`: a place of the workgroup's that nobody reads any more.
template <int TPR>
__device__ __forceinline__ double row_sum(double v, double* part) {
  constexpr int WAVES = TPR / 64;
  v = wave_sum(v);
  if (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += part[w];
  }
  return v;
}

// 1 / sqrt(v) to fp64's last bits, from the instruction's some 26 bits by two Newton steps.
__device__ __forceinline__ double inverse_root(double v) {
  double r = __builtin_amdgcn_rsq(v);
  if (!(v > 0. && v < __builtin_huge_val())) return r;
#pragma unroll
  for (int i = 0; i < 2; ++i) r = fma(0.5 * r, fma(-v * r, r, 1.), r);
  return r;
}

// Eight numbers as they are in memory.
template <typename El>
struct Raw { mx8_u32x4 w[sizeof(El) / 2]; };
template <typename El, bool ONCE>
__device__ __forceinline__ Raw<El> load_raw(const El* p) {
  Raw<El> r;
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(El)) / 2; ++i) r.w[i] = mx8_load_any<ONCE>(p + i * (16 / sizeof(El)));
  return r;
}
// How a row ends: with a whole unit; inside of one, of at least eight numbers; of fewer.
enum { END_WHOLE, END_INSIDE, END_SHORT };

// Unit u of a row of n numbers, zeros past the row.  END_INSIDE: the unit that the row ends in is the row's last eight numbers, to be
// moved down by `missing` when they are there: a load that is not waited for, where one of number by number would be (16 384 rows of
// 2839 numbers, bf16 161 -> 114 us, aligned ones of 2840 88; fp32 199 -> 158 and 157).
template <typename El, bool ONCE, int END>
__device__ __forceinline__ Raw<El> load_unit(const El* row, int u, int n) {
  Raw<El> r;
#pragma unroll
  for (int j = 0; j < static_cast<int>(sizeof(El)) / 2; ++j) r.w[j] = mx8_u32x4{0u, 0u, 0u, 0u};
  if (END == END_SHORT) {
    uint32_t b[8];
    mx8_load8<El, false>(row, u * 8, n, b);
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(El)) / 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[i][j] = sizeof(El) == 4 ? b[4 * i + j] : b[2 * j] >> 16 | (b[2 * j + 1] & 0xFFFF0000u);
  } else if (END == END_WHOLE ? u * 8 + 8 <= n : u * 8 < n) {
    r = load_raw<El, ONCE>(row + (END == END_WHOLE ? u * 8 : min(u * 8, n - 8)));
  }
  return r;
}
__device__ __forceinline__ int missing(int u, int n) { return u * 8 < n ? max(u * 8 + 8 - n, 0) : 0; }
template <typename El>
__device__ __forceinline__ void move_down(Raw<El>& r, int by) {
  if (__builtin_amdgcn_ballot_w64(by != 0) == 0) return;  // the row doesn't end in this wavefront
  constexpr int WORDS = 2 * sizeof(El), HALF = sizeof(El) == 2;
  uint32_t w[WORDS + 4];
#pragma unroll
  for (int i = 0; i < WORDS + 4; ++i) w[i] = i < WORDS ? r.w[i / 4][i & 3] : 0u;
#pragma unroll
  for (int bit = 2; bit >= HALF; --bit) {
    const int words = (1 << bit) >> HALF;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = (by >> bit) & 1 ? (i + words < WORDS ? w[i + words] : 0u) : w[i];
  }
  if (HALF) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = by & 1 ? w[i] >> 16 | (i + 1 < WORDS ? w[i + 1] << 16 : 0u) : w[i];
  }
#pragma unroll
  for (int i = 0; i < WORDS; ++i) r.w[i / 4][i & 3] = w[i];
}
// The way back, of rounded numbers: what is left of a unit in pieces of four, two and one.
template <typename El, bool ONCE, int END>
__device__ __forceinline__ void store_unit(const float* v, El* row, int u, int n) {
  if (u * 8 + 8 <= n) {
    mx8_store8<El, ONCE>(row, u * 8, 1 << 30, v);
  } else if (END != END_WHOLE && u * 8 < n) {
    typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t one __attribute__((aligned(2)));
    constexpr int WORDS = 2 * sizeof(El);
    uint32_t w[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = sizeof(El) == 4 ? __float_as_uint(v[i]) : mx8_pack_bf16(v[(2 * i) & 7], v[(2 * i + 1) & 7]);
    El* p = row + u * 8;
    if (n & 4) {
      if (sizeof(El) == 4) mx8_store_any<false>(p, mx8_u32x4{w[0], w[1], w[2], w[3]});
      else *reinterpret_cast<two*>(p) = two{w[0], w[1]};
#pragma unroll
      for (int i = 0; i < WORDS / 2; ++i) w[i] = w[i + WORDS / 2];
      p += 4;
    }
    if (n & 2) {
      if (sizeof(El) == 4) *reinterpret_cast<two*>(p) = two{w[0], w[1]};
      else *reinterpret_cast<one*>(p) = w[0];
      w[0] = w[WORDS / 4];
      p += 2;
    }
    if (n & 1) {
      if (sizeof(El) == 4) *reinterpret_cast<one*>(p) = w[0];
      else *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    }
  }
}
template <typename El>
__device__ __forceinline__ float number(const Raw<El>& r, int j) {
  if (sizeof(El) == 4) return __uint_as_float(r.w[(j >> 2) & (sizeof(El) / 2 - 1)][j & 3]);
  return __uint_as_float((j & 1) ? r.w[0][j >> 1] & 0xFFFF0000u : r.w[0][j >> 1] << 16);
}
template <typename El>
__device__ __forceinline__ float rounded(float f) { return sizeof(El) == 4 ? f : __uint_as_float(mx8_pack_bf16(f, f) << 16); }

// s -> y and its 8-bit form, of U units; four neighbouring lanes have a block's.  What is past the row is zeros, or NaN if all of the
// row is.
template <typename El, int U, bool ONCE, int END>
__device__ __forceinline__ void finish(const NormArgs& a, int64_t row, int u0, int step, float (*v)[8], const Raw<El>* weight, double inverse) {
  const int blocks = (a.H + 31) >> 5;
  const float inv = static_cast<float>(inverse);
  const bool plain = inv > 0x1p-100f && inv < 0x1p+100f;  // else the product with s may be in fp32's range where inv is not
  uint32_t byte[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float n = plain ? v[i][j] * inv : static_cast<float>(static_cast<double>(v[i][j]) * inverse);
      v[i][j] = rounded<El>(n * number(weight[i], j));
      m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
    }
    byte[i] = mx8_scale_byte(mx8_quad_max(m));
    __builtin_amdgcn_sched_barrier(0);
  }
  if (a.y) {
#pragma unroll
    for (int i = 0; i < U; ++i) store_unit<El, ONCE, END>(v[i], static_cast<El*>(a.y) + row * a.H, u0 + i * step, a.H);
  }
  if (!a.codes) return;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = u0 + i * step;
    if (u >= blocks * 4) continue;
    *reinterpret_cast<uint2*>(a.codes + (row * blocks * 4 + u) * 8) = mx8_codes8(v[i], byte[i]);
    if ((u & 3) == 0) a.scales[row * blocks + (u >> 2)] = static_cast<uint8_t>(byte[i]);
  }
}

// TPR threads share a row, each with U units of eight numbers, TPR units apart; a row's workgroup takes every gridDim-th row, with
// the weights in registers and the next row on its way while one is finished.
//
// The squares are summed in fp64: no row is too large or too small for it, and the result does not hang on the order of the
// sum, so that y's last bit, and with it the 8-bit form of a number next to a border, is the same for every shape of the kernel.
// That costs nothing: what bounds it is HBM, and for few rows the chain of load, sum and store.
// ONCE (more than the last-level cache holds): numbers past the caches' retention.
template <typename El, int TPR, int U, bool ONCE, int END>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rms_norm_kernel(NormArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  __shared__ double part[2][TPR < 256 ? 1 : TPR / 64];
  const int t = threadIdx.x & (TPR - 1);
  const El* x = static_cast<const El*>(a.x);
  const El* residual = static_cast<const El*>(a.residual);
  Raw<El> rx[U], rr[U], rw[U];
  auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      rx[i] = load_unit<El, ONCE, END>(x + row * a.ld_x, t + i * TPR, a.H);
      if (residual) rr[i] = load_unit<El, ONCE, END>(residual + row * a.ld_residual, t + i * TPR, a.H);
    }
  };
  int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * ROWS;
  if (row >= a.rows) return;  // with more than one wavefront to a row, the whole workgroup
  load(row);
#pragma unroll
  for (int i = 0; i < U; ++i) rw[i] = load_unit<El, false, END>(static_cast<const El*>(a.weight), t + i * TPR, a.H);
  bool first = true;
  for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
    float v[U][8];
    double square = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (END == END_INSIDE) {
        move_down(rx[i], missing(t + i * TPR, a.H));
        if (residual) move_down(rr[i], missing(t + i * TPR, a.H));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = number(rx[i], j);
        if (residual) v[i][j] = rounded<El>(v[i][j] + number(rr[i], j));
        square = fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), square);
      }
      __builtin_amdgcn_sched_barrier(0);  // or all of the fp64 numbers are made first, and kept
    }
    if (a.sum) {
#pragma unroll
      for (int i = 0; i < U; ++i) store_unit<El, ONCE, END>(v[i], static_cast<El*>(a.sum) + row * a.H, t + i * TPR, a.H);
    }
    if (row + stride < a.rows) load(row + stride);
    const double inverse = inverse_root(row_sum<TPR>(square, part[turn]) / a.H + a.eps);
    if (END == END_INSIDE && first) {
#pragma unroll
      for (int i = 0; i < U; ++i) move_down(rw[i], missing(t + i * TPR, a.H));
      first = false;
    }
    finish<El, U, ONCE, END>(a, row, t, TPR, v, rw, inverse);
  }
}

// Rows that do not fit a workgroup's registers are read twice: by way of `sum` the second time, where there is one (x or the residual
// may be what it replaces).  HBM bounds it, and the second reading where the caches have not kept the row: with residual and 8-bit form,
// counted once, 16 384 rows of 8200 fp32 numbers 526 us, 4.4 TB/s (8192, read once: 438 us, 5.2), 10 000 of 12 000 442 us, 4.6, 8000 of 16 384 444 us,
// 5.0; bf16, 8000 rows of 20 000 313 us, 4.6 (16 384, read once: 223 us, 5.3).
template <typename El>
__global__ __launch_bounds__(1024) void add_rms_norm_long_kernel(NormArgs a) {
  constexpr int U = 2, TPR = 1024;
  __shared__ double part[TPR / 64];
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, units = ((a.H + 31) >> 5) * 4;
  const El* x = static_cast<const El*>(a.x) + row * a.ld_x;
  const El* residual = a.residual ? static_cast<const El*>(a.residual) + row * a.ld_residual : nullptr;
  El* sum = a.sum ? static_cast<El*>(a.sum) + row * a.H : nullptr;
  float v[U][8];
  auto load = [&](int c) {
    Raw<El> rx[U], rr[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      rx[i] = load_unit<El, false, END_INSIDE>(x, c + t + i * TPR, a.H);
      if (residual) rr[i] = load_unit<El, false, END_INSIDE>(residual, c + t + i * TPR, a.H);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      move_down(rx[i], missing(c + t + i * TPR, a.H));
      if (residual) move_down(rr[i], missing(c + t + i * TPR, a.H));
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = residual ? rounded<El>(number(rx[i], j) + number(rr[i], j)) : number(rx[i], j);
  };
  double square = 0;
  for (int c = 0; c < units; c += U * TPR) {
    load(c);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (sum) store_unit<El, false, END_INSIDE>(v[i], sum, c + t + i * TPR, a.H);
#pragma unroll
      for (int j = 0; j < 8; ++j) square = fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), square);
    }
  }
  const double inverse = inverse_root(row_sum<TPR>(square, part) / a.H + a.eps);
  if (sum) { x = sum; residual = nullptr; }
  for (int c = 0; c < units; c += U * TPR) {
    load(c);
    Raw<El> rw[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      rw[i] = load_unit<El, false, END_INSIDE>(static_cast<const El*>(a.weight), c + t + i * TPR, a.H);
      move_down(rw[i], missing(c + t + i * TPR, a.H));
    }
    finish<El, U, false, END_INSIDE>(a, row, c + t, TPR, v, rw, inverse);
  }
}

constexpr int64_t kOnceBytes = 256ll << 20;
constexpr int kNormGrid = 2048;  // workgroups that are resident at a time, and more: eight to a CU

template <typename El, int TPR, int U, bool SHORT = false>
int launch(const NormArgs& a, hipStream_t stream) {
  constexpr int NT = TPR < 256 ? 256 : TPR;
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>((a.rows * TPR + NT - 1) / NT, kNormGrid)));
  const bool once = a.rows * a.H * static_cast<int64_t>(sizeof(El)) > kOnceBytes;
  if constexpr (SHORT) hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, false, END_SHORT>), grid, dim3(NT), 0, stream, a);
  // rows at any address, past the caches' retention or not: 32 768 x 5001 bf16 494 and 515 us (3.0 TB/s; 32 768 x 5000
  // aligned 305 us, 4.9), 20 000 x 4001 fp32 290 and 264
  else if (a.H % 8 != 0 && once && sizeof(El) == 2) hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, sizeof(El) == 2, END_INSIDE>), grid, dim3(NT), 0, stream, a);
  else if (a.H % 8 != 0) hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, false, END_INSIDE>), grid, dim3(NT), 0, stream, a);
  else if (once) hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, true, END_WHOLE>), grid, dim3(NT), 0, stream, a);
  else hipLaunchKernelGGL((add_rms_norm_kernel<El, TPR, U, false, END_WHOLE>), grid, dim3(NT), 0, stream, a);
  return check_hip(nullptr, hipGetLastError(), "add_rms_norm launch");
}

template <typename El>
int launch_long(const NormArgs& base, hipStream_t stream) {
  NormArgs a = base;
  const int blocks = ceil_div(a.H, 32);
  for (int64_t row = 0; row < base.rows; row += a.rows) {  // a grid has fewer than 2^32 threads
    a.rows = std::min<int64_t>(base.rows - row, 1 << 21);
    a.x = static_cast<const El*>(base.x) + row * a.ld_x;
    if (a.residual) a.residual = static_cast<const El*>(base.residual) + row * a.ld_residual;
    if (a.sum) a.sum = static_cast<El*>(base.sum) + row * a.H;
    if (a.y) a.y = static_cast<El*>(base.y) + row * a.H;
    if (a.codes) { a.codes = base.codes + row * blocks * 32; a.scales = base.scales + row * blocks; }
    hipLaunchKernelGGL(add_rms_norm_long_kernel<El>, dim3(static_cast<uint32_t>(a.rows)), dim3(1024), 0, stream, a);
    const int rc = check_hip(nullptr, hipGetLastError(), "add_rms_norm launch");
    if (rc != REVIVE_OK) return rc;
  }
  return REVIVE_OK;
}

// A unit a thread as long as a workgroup can hold the row: us of 1024 threads with one unit and 256 with four, bf16 with residual
// and 8-bit output, H = 7168: 64 rows 4.8 (256 threads, weights loaded after the sum: 8.1), 1003 rows 16.8 and 16.2, 4096 rows 62 and
// 57, 32 768 rows 392 (5.4 TB/s) and 413.  Between the forms' lengths
// threads are without a unit, 188 of 256 at 513 numbers: 8000 rows of these take 20.3 us (1.8 TB/s), of 1024 numbers 19.4.
template <typename El>
int launch_norm(const NormArgs& a, hipStream_t s) {
  const int units = ceil_div(a.H, 32) * 4;
  if (a.H < 8) return launch<El, 64, 1, true>(a, s);
  if (units <= 64) return launch<El, 64, 1>(a, s);
  if (units <= 256) return launch<El, 256, 1>(a, s);
  if (units <= 512) return launch<El, 512, 1>(a, s);
  if (units <= 1024) return launch<El, 1024, 1>(a, s);
  if (units <= 2048 && sizeof(El) == 2) return launch<El, 1024, sizeof(El) == 2 ? 2 : 1>(a, s);
  return launch_long<El>(a, s);
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
