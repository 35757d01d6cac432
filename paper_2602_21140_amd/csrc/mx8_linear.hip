// Matrix product of microscaled 8-bit activations and weights with bias, activation and residual in its epilogue:
//   out = act(x W^T + bias) + residual
#include "ctx.hpp"
#include "mx8_stream.hpp"
#include "mx8_tile.hpp"

namespace revive {

namespace {

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

}  // namespace

}  // namespace revive

using namespace revive;

extern "C" int revive_mx_eight_linear(const uint8_t* x, const uint8_t* x_scales, int32_t rows, int32_t K, const void* w, int32_t N, const float* bias,
                                 int32_t activation, const void* residual, int64_t ld_residual, void* out, int64_t ld_out,
                                 revive_stream stream) {
  const char* who = "revive_mx_eight_linear";
  if (activation < REVIVE_ACT_NONE || activation > REVIVE_ACT_GELU) return fail(nullptr, REVIVE_EINVAL, "%s: unknown activation %d", who, activation);
  if (rows < 0 || K <= 0 || K % kMx8Block != 0 || N <= 0 || static_cast<int64_t>(N) * K >= (1ll << 32))
    return fail(nullptr, REVIVE_EINVAL, "%s: rows >= 0, N > 0, K a positive multiple of 32 and N * K < 2^32 required", who);
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (rows <= 16) return linear_stream<1, 2, 8, 2>(p, s);
  if (rows <= 128 || K < 64) return linear_stream<2, 4, 4, 2>(p, s);  // the tiles take K from two blocks on
  if (static_cast<int64_t>(rows) * N < 256 * 256 * 128) return linear_stream<2, 4, 4, 2>(p, s);
  return linear_tile<4>(p, s);
}
