// Grouped SwiGLU expert FFN on microscaled 4-bit weights and activations.
//
// Paper: Sec. 2.1 (each expert acts as an FFN).  With Q the rounding of mx.hpp, every slot p with rows
// [slot_offsets[p], slot_offsets[p+1]) computes h = Q(silu(Q(x) G_p) * (Q(x) U_p)), y = h D_p, and the shared expert the same on
// all tokens.  x is quantised once per token, or where tokens are few by who multiplies it; a routed row reads its token's codes through src_of, so that dispatch need not
// copy rows.  Slots without rows produce no tile and their weights are never read.
#include <algorithm>

#include "ctx.hpp"
#include "mx_quant.hpp"
#include "mx_stream.hpp"
#include "mx_tile.hpp"

namespace revive {

namespace {

constexpr int kMxCus = 256;
// With few tokens each workgroup of the first product rounds its rows of x itself, 16 at most, which saves a launch.  us of the
// FFN, rounded on the way and by a launch of its own: 5 matrices of 1024 x 512 for a token 8.7 and 11.5, for 16 tokens 12.3 and
// 14.0; 2048 x 1408, a token 14.0 and 16.0, 16 tokens 49 and 45 to 51; 7168 x 2048, a token 39.5 and 42, 8 tokens 217 to 228 and
// 215, 16 tokens 373 and 357 to 377.  Of more tokens a slot may have several row-tiles, which a launch of some microseconds
// outweighs where there is little to stream in all: 40 slots of 1024 x 512, 32 tokens 13.1 and 14.8, 64 13.1 and 16.8, 128 14.5 and
// 16.0; 72 of 2048 x 1408, 32 tokens 53 and 57, 64 61 and 64, 128 66 and 64; 128 of 4096 x 256, 64 tokens 47 and 52; but 288 of
// 7168 x 2048 (6 GB), 32 tokens 620 and 588, 64 863 and 866.  (So the launch is as good or up to 4 % better from 8 to 16 tokens of
// the largest layers, which the line, drawn for the others, gives away.)
constexpr int kMxFewTokens = 16, kMxFewTokensSmall = 64;
constexpr int64_t kMxSmallBytes = 1ll << 30;
// Above so many rows per slot on average the tiles win, which read a slot's weights once per 256 rows and multiply faster, below
// it the streaming kernel, which starts sooner.  us, streaming and tiles: 288 slots, H = 7168, I = 2048: 14 rows 1146 and 1192,
// 28 rows 1276 and 1242, 57 rows 1426 and 1329; 72 slots, H = 2048, I = 1408: 21 rows 73 and 75, 43 rows 83 and 82; 40 slots, H =
// 1024, I = 512: 26 rows 18 and 22, 102 rows 26 and 24; 128 slots, H = 4096, I = 256: 8 rows 57 and 61, 32 rows 79 and 72.
// The host knows no row counts: the average is over all slots, without rows or not, so that a load on few slots crosses later.
constexpr int kMxTileRowsPerSlot = 32;

struct MxFfn {
  const int32_t* src_of; const int32_t* slot_offsets; const void* const* w_gate_up; const void* const* w_down; void* y_perm;
  const void* w_sh_gate_up; const void* w_sh_down; void* y_shared;
  int N, T;  // routed rows, rows of the shared expert (0: none)
};

// One of the FFN's two products on `rows` rows.
template <int EPI>
MxProblem mx_problem(const revive_ctx* ctx, const MxFfn& f, bool shared, int tile_m, int tile_n) {
  const revive_config& c = ctx->cfg;
  const Workspace& w = ctx->ws;
  const int I = shared ? c.I_shared : c.I, rows = shared ? f.T : f.N;
  uint8_t* h = ctx->d_ws + (shared ? w.off_mx_h_shared : w.off_mx_h);
  uint8_t* h_scales = ctx->d_ws + (shared ? w.off_mx_h_shared_scales : w.off_mx_h_scales);
  MxProblem p{};
  p.n_out = EPI == EPI_H ? I : c.H;
  p.K = EPI == EPI_H ? c.H : I;
  p.b_codes = mx_packed_codes(p.n_out, p.K);
  if (EPI == EPI_H) {
    p.A = ctx->d_ws + w.off_mx_x;
    p.a_row = mx_code_row(c.H); p.a_pair = kMxStep;
    p.A_scales = ctx->d_ws + w.off_mx_x_scales;
    p.src_of = shared ? nullptr : f.src_of; p.k = c.k;
    p.b_half = mx_packed_bytes(I, c.H);
    p.H = h; p.H_scales = h_scales; p.h_rows = rows;
  } else {
    p.A = h;
    p.a_row = kMxStep; p.a_pair = static_cast<int64_t>(rows) * kMxStep;
    p.A_scales = h_scales;
    p.Y = static_cast<uint16_t*>(shared ? f.y_shared : f.y_perm);
  }
  if (shared) p.B_one = EPI == EPI_H ? f.w_sh_gate_up : f.w_sh_down;
  else p.B_tab = EPI == EPI_H ? f.w_gate_up : f.w_down;
  p.n_col_tiles = ceil_div(EPI == EPI_H ? static_cast<int>(mx_up(I, kMxPanel)) : c.H, tile_n);
  const int used = f.N < ctx->P ? f.N : ctx->P;  // slots that can hold a row
  const int m_tiles = shared ? ceil_div(rows, tile_m) : rows / tile_m + used;
  p.blocks = m_tiles * p.n_col_tiles;
  p.blocks = ceil_div(p.blocks, 8) * 8;
  p.M = rows;
  return p;
}

template <int EPI>
MxArgs mx_args(const revive_ctx* ctx, const MxFfn& f, int tile_m, int tile_n) {
  MxArgs a{};
  a.slot_offsets = f.slot_offsets;
  a.P = ctx->P;
  a.grouped = mx_problem<EPI>(ctx, f, false, tile_m, tile_n);
  if (f.T > 0) a.dense = mx_problem<EPI>(ctx, f, true, tile_m, tile_n);
  return a;
}

template <int TMX, int NW, int EPI, bool BF16>
int mx_stream_as(revive_ctx* ctx, const MxFfn& f, const void* x, hipStream_t stream) {
  MxArgs a = mx_args<EPI>(ctx, f, 16 * TMX, NW * (EPI == EPI_H ? 32 : 64));
  if (BF16)
    for (MxProblem* p : {&a.dense, &a.grouped}) {
      p->A = static_cast<const uint8_t*>(x);
      p->a_row = static_cast<int64_t>(ctx->cfg.H) * 2;
    }
  KernelTimer timer(ctx, EPI == EPI_H ? REVIVE_K_MX_GATE_UP : REVIVE_K_MX_DOWN, stream);
  return launch_mx_stream<TMX, 4, NW, EPI, BF16>(ctx, a, stream);
}

// Workgroups of four wavefronts, or of two where that leaves the busiest CU less to stream.  us of the FFN, four and two: 9
// matrices of 7168 x 2048 (144 and 288 workgroups of gate/up: 4 and 4 wavefronts) 40 and 44, 33 (528 and 1056: 12 and 10) 138
// and 122, 7 of 2048 x 1408 (88 and 176: 4 and 2) 20.7 and 16.4.  Of one, whose lanes round four times as much, with few rows
// only; one and the better of the others: a token, 9 matrices of 7168 x 2048 39.5 and 41, 7 of 2048 x 1408 14.0 and 15.0, 5 of
// 1024 x 512 8.7 and 10.2; two tokens, 17 of 7168 x 2048 63 to 70 and 74, 13 of 2048 x 1408 17.5 and 19.4.
template <int TMX, int EPI, bool BF16>
int mx_stream_product(revive_ctx* ctx, const MxFfn& f, const void* x, hipStream_t stream) {
  auto busiest = [&](int nw) {  // wavefronts
    const MxArgs a = mx_args<EPI>(ctx, f, 16 * TMX, nw * (EPI == EPI_H ? 32 : 64));
    return nw * ceil_div(a.dense.blocks + a.grouped.blocks, kMxCus);
  };
  if (TMX == 1 && f.N <= kMxFewRows * ctx->cfg.k && busiest(1) < busiest(2) && busiest(1) < busiest(4))
    return mx_stream_as<TMX, TMX == 1 ? 1 : 2, EPI, BF16>(ctx, f, x, stream);  // of TMX > 1 there is none
  if (busiest(2) < busiest(4)) return mx_stream_as<TMX, 2, EPI, BF16>(ctx, f, x, stream);
  return mx_stream_as<TMX, 4, EPI, BF16>(ctx, f, x, stream);
}

int mx_tile_ffn(revive_ctx* ctx, const MxFfn& f, hipStream_t stream) {
  {
    KernelTimer timer(ctx, REVIVE_K_MX_GATE_UP, stream);
    const int rc = launch_mx_tile<EPI_H>(ctx, mx_args<EPI_H>(ctx, f, kMxTile, kMxPanel), stream);
    if (rc != REVIVE_OK) return rc;
  }
  KernelTimer timer(ctx, REVIVE_K_MX_DOWN, stream);
  return launch_mx_tile<EPI_Y>(ctx, mx_args<EPI_Y>(ctx, f, kMxTile, 2 * kMxPanel), stream);
}

}  // namespace

int launch_mx_expert_ffn(revive_ctx* ctx, const void* x, const int32_t* src_of, const int32_t* slot_offsets, const void* const* w_gate_up,
                         const void* const* w_down, void* y_perm, const void* w_sh_gate_up, const void* w_sh_down, void* y_shared, int T,
                         hipStream_t stream) {
  const revive_config& c = ctx->cfg;
  const Workspace& w = ctx->ws;
  const MxFfn f{src_of, slot_offsets, w_gate_up, w_down, y_perm, w_sh_gate_up, w_sh_down, y_shared, T * c.k, y_shared ? T : 0};
  const int64_t streamed = static_cast<int64_t>(std::min(f.N, ctx->P)) * (2 * mx_packed_bytes(c.I, c.H) + mx_packed_bytes(c.H, c.I));
  if (T <= kMxFewTokens || (T <= kMxFewTokensSmall && streamed <= kMxSmallBytes)) {
    const int rc = mx_stream_product<1, EPI_H, true>(ctx, f, x, stream);
    return rc != REVIVE_OK ? rc : mx_stream_product<1, EPI_Y, false>(ctx, f, nullptr, stream);
  }
  int rc = launch_mx_quantize_tiled(ctx, x, T, c.H, ctx->d_ws + w.off_mx_x, ctx->d_ws + w.off_mx_x_scales, stream);
  if (rc != REVIVE_OK) return rc;
  // The tiles address a row of x by 32 bits.
  if (f.N > kMxTileRowsPerSlot * static_cast<int64_t>(ctx->P) && static_cast<int64_t>(T) * mx_code_row(c.H) < (1ll << 32)) return mx_tile_ffn(ctx, f, stream);
  rc = mx_stream_product<4, EPI_H, false>(ctx, f, nullptr, stream);
  return rc != REVIVE_OK ? rc : mx_stream_product<4, EPI_Y, false>(ctx, f, nullptr, stream);
}

}  // namespace revive
