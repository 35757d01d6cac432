// Grouped SwiGLU expert FFN on microscaled 8-bit weights and activations.
//
// Paper: Sec. 2.1 (each expert acts as an FFN).  With Q the rounding of mx8.hpp, every slot p with rows
// [slot_offsets[p], slot_offsets[p+1]) computes h = Q(silu(x G_p) * (x U_p)), y = h D_p, and the shared expert the same on all
// tokens.  x comes in 8 bits (the norm in front of the layer gives it so); a routed row reads its token's codes through src_of,
// so that dispatch need not copy rows.  Slots without rows produce no tile and their weights are never read.
#include <algorithm>

#include "ctx.hpp"
#include "mx8_stream.hpp"
#include "mx8_tile.hpp"

namespace revive {

namespace {

// Above so many rows per slot on average the tiles win, which read a slot's weights once per 256 rows and multiply faster, below it
// the streaming kernel: us of the two products, streaming (32 rows to a workgroup) and tiles, 288 slots, H = 7168, I = 2048: 14 rows
// 2040 and 2230, 28 rows 2470 and 2400, 57 rows 3520 and 2630; 72 slots, H = 2048, I = 1408: 21 rows 130 and 133, 43 rows 213 and
// 148, 84 rows 320 and 178.  The host knows no row counts: the average is over all slots, without rows or not.
// Fewer tiles than kMx8TileGrid leave too many CUs without one; 64 rows to a workgroup of the streaming kernel then.
constexpr int kMx8TileRowsPerSlot = 24, kMx8TileGrid = 96;
// The tiles' sums of gate and up are those of the 8-bit instruction (mx8_product.hpp), after which some 6 of 10 000 numbers of h are
// rounded to the neighbouring code: y's relative error is 0.0020 so, 0.0017 of it bf16's rounding, if there are many numbers to
// even that out; of 400 000 numbers it was up to 0.0027.  Fewer than 2^20 numbers are left to the streaming kernel, whose sums
// are exact, the shared expert's in a launch of their own if the routed ones are many.
constexpr int64_t kMx8ManyNumbers = 1 << 20;

struct Mx8Ffn {
  const uint8_t* x; const uint8_t* x_scales;
  const int32_t* src_of; const int32_t* slot_offsets; const void* const* w_gate_up; const void* const* w_down; void* y_perm;
  const void* w_sh_gate_up; const void* w_sh_down; void* y_shared;
  int N, T;  // routed rows, rows of the shared expert (0: none)
};

// One of the FFN's two products on the routed rows or on the shared expert's.
template <int EPI>
Mx8Problem mx8_problem(const revive_ctx* ctx, const Mx8Ffn& f, bool shared) {
  const revive_config& c = ctx->cfg;
  const Workspace& w = ctx->ws;
  const int I = shared ? c.I_shared : c.I, rows = shared ? f.T : f.N;
  uint8_t* h = ctx->d_ws + (shared ? w.off_mx8_h_shared : w.off_mx8_h);
  uint8_t* h_scales = ctx->d_ws + (shared ? w.off_mx8_h_shared_scales : w.off_mx8_h_scales);
  Mx8Problem p{};
  p.n_out = EPI == EPI8_H ? I : c.H;
  p.K = EPI == EPI8_H ? c.H : I;
  p.b_codes = mx8_packed_codes(p.n_out, p.K);
  p.a_row = p.K;
  if (EPI == EPI8_H) {
    p.A = f.x; p.A_scales = f.x_scales;
    p.src_of = shared ? nullptr : f.src_of; p.k = c.k;
    p.b_half = mx8_packed_bytes(I, c.H);
    p.H = h; p.H_scales = h_scales;
  } else {
    p.A = h; p.A_scales = h_scales;
    p.Y = static_cast<uint16_t*>(shared ? f.y_shared : f.y_perm);
  }
  if (shared) p.B_one = EPI == EPI8_H ? f.w_sh_gate_up : f.w_sh_down;
  else p.B_tab = EPI == EPI8_H ? f.w_gate_up : f.w_down;
  p.M = rows;
  return p;
}

// A product's arguments for tiles of tile_m rows and `width` columns; false: more than one launch takes.
template <int EPI>
bool mx8_args(const revive_ctx* ctx, const Mx8Ffn& f, int tile_m, int width, int threads, Mx8Args& a) {
  a = Mx8Args{};
  a.slot_offsets = f.slot_offsets;
  a.P = ctx->P;
  a.grouped = mx8_problem<EPI>(ctx, f, false);
  // as many row-tiles as the rows can make in the slots that can hold one
  bool fits = mx8_cut(a.grouped, f.N / tile_m + std::min(f.N, ctx->P), width, threads);
  if (f.T > 0) {
    a.dense = mx8_problem<EPI>(ctx, f, true);
    fits = mx8_cut(a.dense, ceil_div(f.T, tile_m), width, threads) && fits;
  }
  return fits;
}

int too_large(const revive_ctx* ctx) { return fail(ctx, REVIVE_EINVAL, "revive_mx_eight_expert_ffn: rows times columns are more than one launch takes"); }

template <int TMX, int W, int D, int EPI, bool WIDE = false>
int mx8_stream_product(revive_ctx* ctx, const Mx8Ffn& f, hipStream_t stream) {
  Mx8Args a;
  if (!mx8_args<EPI>(ctx, f, 16 * TMX, EPI == EPI8_H ? 32 : 16 * W, 256, a)) return too_large(ctx);
  return launch_mx8_stream<TMX, W, 4, D, EPI, WIDE>(ctx, a, stream);
}

template <int EPI>
int mx8_tile_product(revive_ctx* ctx, const Mx8Ffn& f, hipStream_t stream) {
  Mx8Args a;
  if (!mx8_args<EPI>(ctx, f, kMx8Tile, EPI == EPI8_H ? 128 : 256, 512, a)) return too_large(ctx);
  return launch_mx8_tile<4, EPI>(ctx, a, stream);
}

// One of the two products, in the form that suits its rows.
template <int EPI>
int mx8_product(revive_ctx* ctx, const Mx8Ffn& f, hipStream_t stream) {
  KernelTimer timer(ctx, EPI == EPI8_H ? REVIVE_K_MX8_GATE_UP : REVIVE_K_MX8_DOWN, stream);
  const revive_config& c = ctx->cfg;
  // All of x within 32 bits, as the tiles and the narrow form of the stream address it.
  const bool wide = EPI == EPI8_H && static_cast<int64_t>(c.T_max) * c.H >= (1ll << 32);
  if (wide) return mx8_stream_product<2, 4, 2, EPI, EPI == EPI8_H>(ctx, f, stream);
  if (f.N <= kMx8TileRowsPerSlot * static_cast<int64_t>(ctx->P)) return mx8_stream_product<2, 4, 2, EPI>(ctx, f, stream);
  const int columns = EPI == EPI8_H ? ceil_div(c.I, 128) : ceil_div(c.H, 256);
  const bool many = EPI != EPI8_H || static_cast<int64_t>(f.N) * c.I >= kMx8ManyNumbers;
  if (!many || static_cast<int64_t>(std::max(ctx->P, f.N / kMx8Tile)) * columns < kMx8TileGrid) return mx8_stream_product<4, 4, 1, EPI>(ctx, f, stream);
  if (EPI == EPI8_H && f.T > 0 && static_cast<int64_t>(f.T) * c.I_shared < kMx8ManyNumbers) {
    Mx8Ffn routed = f, shared = f;
    routed.T = 0;
    shared.N = 0;
    const int rc = mx8_tile_product<EPI>(ctx, routed, stream);
    return rc != REVIVE_OK ? rc : mx8_stream_product<4, 4, 1, EPI>(ctx, shared, stream);
  }
  return mx8_tile_product<EPI>(ctx, f, stream);
}

}  // namespace

int launch_mx8_expert_ffn(revive_ctx* ctx, const uint8_t* x, const uint8_t* x_scales, const int32_t* src_of, const int32_t* slot_offsets,
                          const void* const* w_gate_up, const void* const* w_down, void* y_perm, const void* w_sh_gate_up, const void* w_sh_down,
                          void* y_shared, int T, hipStream_t stream) {
  const Mx8Ffn f{x, x_scales, src_of, slot_offsets, w_gate_up, w_down, y_perm, w_sh_gate_up, w_sh_down, y_shared, T * ctx->cfg.k, y_shared ? T : 0};
  const int rc = mx8_product<EPI8_H>(ctx, f, stream);
  return rc != REVIVE_OK ? rc : mx8_product<EPI8_Y>(ctx, f, stream);
}

}  // namespace revive
