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
// the streaming kernel (64 rows to a workgroup).  us of both products, gate and up streamed and by tiles, down (gate and up streamed
// 32 rows at a time) streamed and by tiles: 288 slots, H = 7168, I = 2048: 7 rows 1881 1954, 1877 1950, 25 rows 2318 2343, 2366 2391, 39 rows
// 2700 2430, 2710 2660; 72 slots, H = 2048, I = 1408: 18 rows 127 124, 126 136, 27 rows 147 131, 147 155, 43 rows 172 139, 166 167, 84 rows 285
// 190, 275 254.  The host knows no row counts: the average is over all slots, without rows or not.  Fewer tiles than kMx8TileGrid
// leave too many CUs without one.  The shared expert takes the form of the routed rows, but for the case below: beside few of them all of its
// rows are streamed (288 slots, 2048 x 256, one slot a token, I_shared = 2816: 6000 tokens 378 us, 141 without the shared expert, 8000 tokens 319).
constexpr int kMx8TileRowsGateUp = 24, kMx8TileRowsDown = 36, kMx8TileGrid = 96;
// The tiles' sums of gate and up are those of the 8-bit instruction (mx8_product.hpp), after which some 17 of 10 000 numbers of h are
// rounded to another code (H = 256 to 2048; h is off by 0.0010 to 0.0012 of its size): y's relative error is 0.0020 so, 0.0017 of it bf16's
// rounding, if there are many numbers to even that out; of 400 000 numbers it was up to 0.0027.  Fewer than 2^20 numbers are left to the
// streaming kernel, whose sums are fp32 (of 500 000 numbers none is rounded to another code), the shared expert's in a launch of their own
// if the routed ones are many.
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

// 64 rows a workgroup: with 32, 64 tokens on 72 slots of 2048 x 1408 take 108 instead of 104 us, 700 of them 320 instead of 250, and a
// token on 288 slots of 7168 x 2048 75.7 instead of 77.4.  WIDE, 32: the wider addresses of 64 do not fit in the registers.
template <int EPI, bool WIDE = false>
int mx8_stream_product(revive_ctx* ctx, const Mx8Ffn& f, hipStream_t stream) {
  constexpr int TMX = WIDE ? 2 : 4, D = WIDE ? 2 : 1;
  Mx8Args a;
  if (!mx8_args<EPI>(ctx, f, 16 * TMX, EPI == EPI8_H ? 32 : 64, 256, a)) return too_large(ctx);
  return launch_mx8_stream<TMX, 4, 4, D, EPI, WIDE>(ctx, a, stream);
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
  if (EPI == EPI8_H && static_cast<int64_t>(c.T_max) * c.H >= (1ll << 32)) return mx8_stream_product<EPI, EPI == EPI8_H>(ctx, f, stream);
  const int columns = EPI == EPI8_H ? ceil_div(c.I, 128) : ceil_div(c.H, 256);
  const bool tiles = f.N > (EPI == EPI8_H ? kMx8TileRowsGateUp : kMx8TileRowsDown) * static_cast<int64_t>(ctx->P) &&
                     static_cast<int64_t>(std::max(ctx->P, f.N / kMx8Tile)) * columns >= kMx8TileGrid &&
                     (EPI != EPI8_H || static_cast<int64_t>(f.N) * c.I >= kMx8ManyNumbers);
  if (!tiles) return mx8_stream_product<EPI>(ctx, f, stream);
  if (EPI == EPI8_H && f.T > 0 && static_cast<int64_t>(f.T) * c.I_shared < kMx8ManyNumbers) {
    Mx8Ffn routed = f, shared = f;
    routed.T = 0;
    shared.N = 0;
    const int rc = mx8_tile_product<EPI>(ctx, routed, stream);
    return rc != REVIVE_OK ? rc : mx8_stream_product<EPI>(ctx, shared, stream);
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
