// Matrix product of microscaled 8-bit activations and weights with bias, activation and residual in its epilogue:
//   out = act(x W^T + bias) + residual
#include "ctx.hpp"
#include "mx8_stream.hpp"
#include "mx8_tile.hpp"

namespace revive {

namespace {

// Workgroups of a form with tiles of `tile_m` rows and `width` columns.
int64_t workgroups(const Mx8Problem& p, int tile_m, int width) { return static_cast<int64_t>(ceil_div(p.M, tile_m)) * ceil_div(p.n_out, width); }

int too_large() { return fail(nullptr, REVIVE_EINVAL, "revive_mx_eight_linear: rows times N is more than one launch takes"); }

template <int TMX, int W, int NW, int D>
int linear_stream(const Mx8Problem& base, hipStream_t stream) {
  Mx8Args a{};
  a.dense = base;
  if (!mx8_cut(a.dense, ceil_div(base.M, 16 * TMX), 16 * W, 64 * NW)) return too_large();
  return launch_mx8_stream<TMX, W, NW, D, EPI8_LINEAR>(nullptr, a, stream);
}

template <int TN>
int linear_tile(const Mx8Problem& base, hipStream_t stream) {
  Mx8Args a{};
  a.dense = base;
  if (!mx8_cut(a.dense, ceil_div(base.M, kMx8Tile), 64 * TN, 512)) return too_large();
  return launch_mx8_tile<TN, EPI8_LINEAR>(nullptr, a, stream);
}

// The larger a workgroup's tile, the less is read per product, but a CU without a workgroup does nothing.  us of 256 x 256 and 256 x 128
// through LDS, 64 x 64, 32 x 64, 16 x 64, 16 x 32, K = N = 7168: 16 rows - - 19 18 18 13.9, 32 rows - - 21 20 12.4 13.0, 64 rows - - 24 13.9
// 20 19, 128 rows 64 41 18 20 34 30, 256 rows 79 50 27 35 59 55, 512 rows 82 55 54 61, 768 rows 82 61 76 88, 1024 rows 87 68 92 118, 1536
// rows 95 113 137, 2048 rows 102 127 173 221; K = N = 2048: 2048 rows 30 21.2 21.2 26, 4096 rows 33 26 38 47; 8192 rows, K = N = 1024 23 18 27 33;
// 1003 rows, K = 2048, N = 1411 37 25 13 14; 64 rows, K = 16384, N = 576 - - 42 21 17 12.5.
// So the tiles through LDS, which multiply fastest, where they give half of the CUs one, those of 128 columns as long as none gets
// two; else the largest form that gives nearly every CU one.
// Between 112 and 223 workgroups the larger of two forms is the faster one as well, and this rule passes over it.  K = 7168, 32 x 64 (144, 160,
// 192, 220, 224 workgroups), 16 x 64 (twice as many), 64 rows: N = 4608 12.4 17.8, 5120 12.5 17.9, 6144 12.9 18.2, 7040 13.5 18.6, 7168 13.5 18.3; 16 x 64 (as
// many), 16 x 32 (twice as many), 32 rows: 10.5 13.1, 10.7 13.3, 11.0 13.6, 11.7 14.0, 11.5 13.8; 64 x 64 (144 to 224), 32 x 64, 128 rows: 16.8 18.7, 17.0 19.0, 17.4
// 19.2, 17.3 19.8, 17.3 19.3.  A second workgroup on some of the CUs is what costs: up to 256 of them the smaller form wins (48 rows, 16 x 64 and 32 x 64:
// N = 4608, 216 workgroups, 10.6 12.1, N = 6144, 288, 18.0 12.5).
constexpr int kMx8Cus = 256, kMx8HalfGrid = 128, kMx8FullGrid = 224;

int linear(const Mx8Problem& p, hipStream_t s) {
  const int64_t tiles = p.K >= 2 * kMx8Block ? workgroups(p, kMx8Tile, 128) : 0;  // they take K from two blocks on
  if (tiles > kMx8Cus) return linear_tile<4>(p, s);
  if (tiles >= kMx8HalfGrid) return linear_tile<2>(p, s);
  if (workgroups(p, 64, 64) >= kMx8FullGrid) return linear_stream<4, 4, 4, 1>(p, s);
  if (workgroups(p, 32, 64) >= kMx8FullGrid) return linear_stream<2, 4, 4, 2>(p, s);
  if (workgroups(p, 16, 64) >= kMx8FullGrid) return linear_stream<1, 4, 8, 2>(p, s);
  return linear_stream<1, 2, 8, 2>(p, s);
}

}  // namespace

}  // namespace revive

using namespace revive;

extern "C" int revive_mx_eight_linear(const uint8_t* x, const uint8_t* x_scales, int32_t rows, int32_t K, const void* w, int32_t N, const float* bias,
                                 int32_t activation, const void* residual, int64_t ld_residual, void* out, int64_t ld_out,
                                 revive_stream stream) {
  const char* who = "revive_mx_eight_linear";
  if (activation < REVIVE_ACT_NONE || activation > REVIVE_ACT_GELU) return fail(nullptr, REVIVE_EINVAL, "%s: unknown activation %d", who, activation);
  if (rows < 0 || rows > (1 << 30) || K <= 0 || K > kMx8MaxK || K % kMx8Block != 0 || N <= 0 || static_cast<int64_t>(N) * K >= (1ll << 32))
    return fail(nullptr, REVIVE_EINVAL, "%s: 0 <= rows <= 2^30, N > 0, K a positive multiple of 32 up to 2^24 and N * K < 2^32 required", who);
  if (ld_out < N || (residual && ld_residual < N)) return fail(nullptr, REVIVE_EINVAL, "%s: rows at least N elements apart required", who);
  if (residual && residual == out && ld_residual != ld_out) return fail(nullptr, REVIVE_EINVAL, "%s: in place, out and residual have the same distance of rows", who);
  if (rows == 0) return REVIVE_OK;
  if (!x || !x_scales || !w || !out) return fail(nullptr, REVIVE_EINVAL, "%s: null argument", who);
  if (reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w) % 16 != 0)
    return fail(nullptr, REVIVE_EINVAL, "%s: codes and weights must be 16-byte aligned", who);
  if (reinterpret_cast<uintptr_t>(out) % 2 != 0 || reinterpret_cast<uintptr_t>(residual) % 2 != 0 || reinterpret_cast<uintptr_t>(bias) % 4 != 0)
    return fail(nullptr, REVIVE_EINVAL, "%s: a pointer is not aligned to its elements", who);
  Mx8Problem p{};
  p.A = x; p.a_row = K; p.A_scales = x_scales;
  p.B_one = w;
  p.b_codes = mx8_packed_codes(N, K);
  p.Y = static_cast<uint16_t*>(out); p.ldy = ld_out;
  p.bias = bias; p.residual = static_cast<const uint16_t*>(residual); p.ld_residual = ld_residual;
  p.activation = activation;
  p.n_out = N; p.K = K; p.M = rows;
  return linear(p, static_cast<hipStream_t>(stream));
}
