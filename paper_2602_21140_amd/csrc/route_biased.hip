// Gate with a bias for balance: experts are chosen by score + bias and weighted by the score alone.
//
//   s_e   = exp(z_e - max z) / sum exp(z - max z)  or  1 / (1 + exp(-z_e)), over all E experts
//   key_e = s_e + b_e; an expert without a live replica is out (paper Sec. 3.4 "Missing experts", Sec. 4.2)
//   a group's score is the sum of its two best keys above -inf (the one, if there is one); the topk_group best groups are kept
//   top-k by key, ties to the lower id;  weight_j = s_{e_j} [/ sum_j s_{e_j}] * route_scale
//
// All of it in fp32.  The keys are compared as integers whose order is that of the numbers, which gives what is no number a
// place: 0 = taken or in a dropped group, 1 = no live replica, 2 = NaN, from 3 on the numbers.
#include "ctx.hpp"

namespace revive {

namespace {

struct BiasedParams {
  const float* logits;
  const float* bias;
  const int32_t* l2p_count;
  const int32_t* l2p_table;
  int32_t* topk_logical;
  float* topk_weight;
  int32_t* topk_phys;
  int T, E, k, max_replicas, score_fn, n_group, topk_group, renormalise;
  long long t_offset;  // index of token 0 within the whole batch
  float route_scale;
};

constexpr uint32_t kTaken = 0, kLost = 1, kNaN = 2, kLowest = 0x007FFFFF;

// Order-preserving integer of a number: -inf is the lowest, kLowest.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v);
  return v != v ? kNaN : b ^ (static_cast<uint32_t>(static_cast<int>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t u) {  // of a key from 3 on
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// Cross-lane steps as operands of an ALU instruction: 0 to 3 combine lanes 1, 2, 4 and 8 apart inside rows of 16, after which
// every lane of a row has the row's result; 4 and 5 bring the rows' results to lanes 31 and 63, and then to lane 63; 6 and 7
// mirror halves of rows and rows, for disjoint sets of four and eight lanes that are alike by then.  Lanes that a step has nothing for get `other`.
template <int STEP>
__device__ __forceinline__ int dpp(int v, int other) {
  constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x124 : STEP == 3 ? 0x128 : STEP == 4 ? 0x142 : STEP == 5 ? 0x143 : STEP == 6 ? 0x141 : 0x140;
  constexpr int rows = STEP == 4 ? 0xA : STEP == 5 ? 0xC : 0xF;
  return __builtin_amdgcn_update_dpp(other, v, ctrl, rows, 0xF, false);
}
template <int STEP>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) { return static_cast<uint32_t>(dpp<STEP>(static_cast<int>(v), 0)); }
template <int STEP>
__device__ __forceinline__ float dpp_f(float v, float other) { return __int_as_float(dpp<STEP>(__float_as_int(v), __float_as_int(other))); }

__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, dpp_u<0>(v));
  v = max(v, dpp_u<1>(v));
  v = max(v, dpp_u<2>(v));
  return max(v, dpp_u<3>(v));
}
__device__ __forceinline__ int row_min(int v) {
  v = min(v, dpp<0>(v, 0));
  v = min(v, dpp<1>(v, 0));
  v = min(v, dpp<2>(v, 0));
  return min(v, dpp<3>(v, 0));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f<0>(v, 0.f));
  v = fmaxf(v, dpp_f<1>(v, 0.f));
  v = fmaxf(v, dpp_f<2>(v, 0.f));
  return fmaxf(v, dpp_f<3>(v, 0.f));
}
__device__ __forceinline__ float row_sum(float v) {  // by exchanges, so that every lane has the same bits
  v += dpp_f<0>(v, 0.f);
  v += dpp_f<1>(v, 0.f);
  v += dpp_f<6>(v, 0.f);
  return v + dpp_f<7>(v, 0.f);
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = row_max(v);
  v = max(v, dpp_u<4>(v));
  return static_cast<uint32_t>(last_lane(static_cast<int>(max(v, dpp_u<5>(v)))));
}
__device__ __forceinline__ float wave_max(float v) {
  const float NEG = -__builtin_inff();
  v = row_max(v);
  v = fmaxf(v, dpp_f<4>(v, NEG));
  return __int_as_float(last_lane(__float_as_int(fmaxf(v, dpp_f<5>(v, NEG)))));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum(v);
  v += dpp_f<4>(v, 0.f);
  return __int_as_float(last_lane(__float_as_int(v + dpp_f<5>(v, 0.f))));
}
// The two largest of two disjoint sets, each given by its two largest.
template <int STEP>
__device__ __forceinline__ void top2_step(uint32_t& m1, uint32_t& m2) {
  const uint32_t o1 = dpp_u<STEP>(m1), o2 = dpp_u<STEP>(m2);
  m2 = max(min(m1, o1), max(m2, o2));
  m1 = max(m1, o1);
}

// exp(x) for x in [-100, 88]: 2^p with p = x log2(e) rounded, times what the rounding left out.  Off by two units in the last
// place; __expf, which lacks the second factor, by as many as |x| says.  NaN stays.
__device__ __forceinline__ float exp_of(float x) {
  constexpr float kLog2e = 1.44269504f;
  const float p = x * kLog2e, rest = fmaf(x, kLog2e, -p) + x * 1.92596299e-8f;  // log2(e) = kLog2e + 1.92596299e-8
  const float e = __builtin_amdgcn_exp2f(p);
  return fmaf(e, rest * 0.693147181f, e);
}
// Softmax: the numerator, m the largest logit.  exp(-100) is zero in fp32.
__device__ __forceinline__ float exp_below(float z, float m) {
  const float d = z - m;
  return exp_of(d < -100.f ? -100.f : d);
}
__device__ __forceinline__ float sigmoid(float z) {
  const float x = z < -87.f ? -87.f : z > 87.f ? 87.f : z;
  return __builtin_amdgcn_rcpf(1.0f + exp_of(-x));
}

__device__ __forceinline__ void store_choice(const BiasedParams& p, int t, int j, int e, float weight) {
  const int64_t o = static_cast<int64_t>(t) * p.k + j;
  const int count = p.l2p_count[e];
  const unsigned long long b = static_cast<unsigned long long>(p.t_offset) + t;
  const int r = count <= 0 ? 0 : p.t_offset + p.T <= 0x7fffffffll ? static_cast<int>(static_cast<uint32_t>(b) % static_cast<uint32_t>(count)) : static_cast<int>(b % count);
  p.topk_logical[o] = e;
  p.topk_weight[o] = weight;
  p.topk_phys[o] = count > 0 ? p.l2p_table[e * p.max_replicas + r] : -1;
}

// 16 lanes, one DPP row, per token: four tokens to a wavefront, which takes several fours in turn and keeps bias and failure
// mask in registers.  A group of experts (all of them in a layer without groups) is a run of lg = 16 / n_group lanes, and a lane
// holds n = ceil(E / 16) <= V of its experts, dealt so that the run's loads are contiguous: lane j of the run holds the group's
// experts j, j + lg, ..., or with WIDE (E a multiple of 64, 16-byte loads) its words of four j, j + lg, ...
//
// Bound by the ALU.  What a choice costs is kept small by two levels: a lane has the best key of every four of its experts in
// registers and the keys in LDS; a round looks at the bests, and the four keys of the winning one are read, stripped of the
// winner and put back.
template <int V, bool GROUPED, bool WIDE>
__global__ __launch_bounds__(256) void route_biased_rows_kernel(BiasedParams p, int rounds) {
  constexpr int C = V / 4;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  __shared__ u32x4 keys[4][C][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane >> 4, li = lane & 15;
  const float NEG = -__builtin_inff();
  const int n = (p.E + 15) >> 4;
  const int lg = GROUPED ? 16 / p.n_group : 16, lj = li & (lg - 1);  // lanes of a group, this one's place among them
  const int e0 = GROUPED ? li / lg * (p.E / p.n_group) : 0;          // the group's first expert
  auto expert = [&](int i) { return e0 + (WIDE ? (i >> 2) * 4 * lg + lj * 4 + (i & 3) : i * lg + lj); };  // place i
  const bool sig = p.score_fn == REVIVE_SCORE_SIGMOID;
  float bias[V];
  bool live[V], is[V];  // is: there is an expert in this place
#pragma unroll
  for (int i = 0; i < V; ++i) {
    is[i] = i < n && expert(i) < p.E;
    const int e = min(expert(i), p.E - 1);
    bias[i] = p.bias[e];
    live[i] = p.l2p_count[e] > 0;
  }
  for (int r = 0; r < rounds; ++r) {
    const int t0 = ((r * gridDim.x + blockIdx.x) * 4 + wave) * 4, t = t0 + row;
    if (t0 >= p.T) return;  // whole wavefront leaves together
    const float* z = p.logits + static_cast<int64_t>(min(t, p.T - 1)) * p.E;
    float s[V];  // logits, then scores
#pragma unroll
    for (int i = 0; i < V; i += WIDE ? 4 : 1) {
      if (WIDE) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(z + (i < n ? expert(i) : 0));  // n is a multiple of 4
        s[i] = v[0]; s[i + 1] = v[1]; s[i + 2] = v[2]; s[i + 3] = v[3];
      } else {
        s[i] = z[min(expert(i), p.E - 1)];
      }
    }
    float shift = 0.f, scale = 1.f;
    if (sig) {
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] = sigmoid(s[i]);
    } else {
      shift = NEG;
#pragma unroll
      for (int i = 0; i < V; ++i) shift = is[i] ? fmaxf(shift, s[i]) : shift;
      shift = row_max(shift);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[i] = exp_below(s[i], shift);
        sum += is[i] ? s[i] : 0.f;
      }
      scale = 1.0f / row_sum(sum);
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= scale;
    }
    uint32_t best4[C];
    u32x4 u[C];
#pragma unroll
    for (int i = 0; i < V; ++i) u[i >> 2][i & 3] = !is[i] ? kTaken : live[i] ? ordered(s[i] + bias[i]) : kLost;
    if (GROUPED) {
      uint32_t m1 = 0, m2 = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        m2 = max(min(m1, u[i >> 2][i & 3]), m2);
        m1 = max(m1, u[i >> 2][i & 3]);
      }
      top2_step<0>(m1, m2);
      if (lg >= 4) top2_step<1>(m1, m2);
      if (lg >= 8) top2_step<6>(m1, m2);
      const float g = m1 <= kLowest ? NEG : m2 <= kLowest ? number(m1) : number(m1) + number(m2);
      // rank of my group among all groups of the token (better score first, ties to the lower group id)
      const uint32_t mine = ordered(g);
      int rank = 0;
      uint32_t o = mine;
      int h = li;
      for (int i = 1; i < p.n_group; ++i) {  // rotate the row by a group
        if (lg == 2) { o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(o), 0x122, 0xF, 0xF, false)); h = __builtin_amdgcn_mov_dpp(h, 0x122, 0xF, 0xF, false); }
        else if (lg == 4) { o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(o), 0x124, 0xF, 0xF, false)); h = __builtin_amdgcn_mov_dpp(h, 0x124, 0xF, 0xF, false); }
        else { o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(o), 0x128, 0xF, 0xF, false)); h = __builtin_amdgcn_mov_dpp(h, 0x128, 0xF, 0xF, false); }
        rank += o > mine || (o == mine && h < li);
      }
      const bool kept = rank < p.topk_group;
#pragma unroll
      for (int i = 0; i < V; ++i) u[i >> 2][i & 3] = kept ? u[i >> 2][i & 3] : kTaken;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      best4[c] = max(max(u[c][0], u[c][1]), max(u[c][2], u[c][3]));
      if (C > 1) keys[wave][c][lane] = u[c];
    }
    __builtin_amdgcn_wave_barrier();

    // k rounds of arg-max (largest key, ties to the lower expert id); lane j of the row keeps the j-th choice
    constexpr int kNone = 1 << 16;
    int my_e = 0;
#pragma unroll 1
    for (int j = 0; j < p.k; ++j) {
      uint32_t m = best4[0];
#pragma unroll
      for (int c = 1; c < C; ++c) m = max(m, best4[c]);
      const uint32_t best = row_max(m);
      int at = C - 1;
#pragma unroll
      for (int c = C - 2; c >= 0; --c) at = best4[c] == best ? c : at;
      u32x4 four = C > 1 ? keys[wave][at][lane] : u[0];
      const int pos = four[0] == best ? 0 : four[1] == best ? 1 : four[2] == best ? 2 : 3;
      const int mine = m == best ? expert(at * 4 + pos) : kNone, e = row_min(mine);
      const bool won = mine == e;
#pragma unroll
      for (int i = 0; i < 4; ++i) four[i] = won && pos == i ? kTaken : four[i];
      if (C > 1) keys[wave][at][lane] = four;
      else u[0] = four;
      const uint32_t left = max(max(four[0], four[1]), max(four[2], four[3]));
#pragma unroll
      for (int c = 0; c < C; ++c) best4[c] = won && at == c ? left : best4[c];
      my_e = li == j ? e : my_e;
    }
    my_e = min(my_e, p.E - 1);
    const float zc = z[my_e];
    const float sc = sig ? sigmoid(zc) : exp_below(zc, shift) * scale;
    const float total = p.renormalise ? row_sum(li < p.k ? sc : 0.f) : 1.f;
    if (li < p.k && t < p.T) store_choice(p, t, li, my_e, sc / total * p.route_scale);
  }
}

// A wavefront per token; lane l holds experts l, l + 64, ...
template <int V>
__global__ __launch_bounds__(256) void route_biased_kernel(BiasedParams p) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;  // whole wavefront leaves together
  const float NEG = -__builtin_inff();
  float score[V];
  uint32_t key[V];
  float m = NEG;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane + 64 * i;
    score[i] = e < p.E ? p.logits[static_cast<int64_t>(t) * p.E + e] : NEG;
    m = fmaxf(m, score[i]);
  }
  if (p.score_fn == REVIVE_SCORE_SIGMOID) {
#pragma unroll
    for (int i = 0; i < V; ++i) score[i] = sigmoid(score[i]);
  } else {
    m = wave_max(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      score[i] = lane + 64 * i < p.E ? exp_below(score[i], m) : 0.f;
      sum += score[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) score[i] /= sum;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane + 64 * i;
    key[i] = e >= p.E ? kTaken : p.l2p_count[e] > 0 ? ordered(score[i] + p.bias[e]) : kLost;
  }

  if (p.n_group > 1) {
    const int gsz = p.E / p.n_group;
    float mine = NEG;  // score of group `lane`
    for (int g = 0; g < p.n_group; ++g) {
      uint32_t m1 = 0, m2 = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = lane + 64 * i;
        const uint32_t u = e >= g * gsz && e < (g + 1) * gsz ? key[i] : 0;
        m2 = max(m2, min(m1, u));
        m1 = max(m1, u);
      }
      top2_step<0>(m1, m2);
      top2_step<1>(m1, m2);
      top2_step<6>(m1, m2);
      top2_step<7>(m1, m2);
      top2_step<4>(m1, m2);
      top2_step<5>(m1, m2);
      m1 = static_cast<uint32_t>(last_lane(static_cast<int>(m1)));
      m2 = static_cast<uint32_t>(last_lane(static_cast<int>(m2)));
      const float s = m1 <= kLowest ? NEG : m2 <= kLowest ? number(m1) : number(m1) + number(m2);
      if (lane == g) mine = s;
    }
    const uint32_t mine_u = lane < p.n_group ? ordered(mine) : 0;
    int rank = 0;
    for (int h = 0; h < p.n_group; ++h) {
      const uint32_t o = static_cast<uint32_t>(__shfl(static_cast<int>(mine_u), h));
      rank += o > mine_u || (o == mine_u && h < lane);
    }
    const unsigned long long kept = __ballot(lane < p.n_group && rank < p.topk_group);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int g = min((lane + 64 * i) / gsz, 63);
      if (!((kept >> g) & 1ull)) key[i] = kTaken;
    }
  }

  int my_e = 0;       // lane j: the j-th choice
  float my_s = 0.f;
  for (int j = 0; j < p.k; ++j) {
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) u = max(u, key[i]);
    const uint32_t best = wave_max(u);
    int wi = 0;
    unsigned long long holders = 1ull;
#pragma unroll
    for (int i = V - 1; i >= 0; --i) {
      const unsigned long long b = __ballot(key[i] == best);
      if (b) { holders = b; wi = i; }
    }
    const int w = __builtin_ctzll(holders);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (wi == i) {
        s = __shfl(score[i], w);
        if (lane == w) key[i] = kTaken;
      }
    if (lane == j) { my_e = min(wi * 64 + w, p.E - 1); my_s = s; }
  }

  const float sum = p.renormalise ? wave_sum(lane < p.k ? my_s : 0.f) : 1.f;
  if (lane < p.k) store_choice(p, t, lane, my_e, my_s / sum * p.route_scale);
}

}  // namespace

int launch_route_biased(revive_ctx* ctx, const float* logits, const float* bias, bool renormalise, int T, int32_t* topk_logical,
                        float* topk_weight, int32_t* topk_phys, hipStream_t stream) {
  const revive_config& c = ctx->cfg;
  BiasedParams p{};
  p.logits = logits; p.bias = bias;
  p.l2p_count = ctx->d_l2p_count(); p.l2p_table = ctx->d_l2p_table();
  p.topk_logical = topk_logical; p.topk_weight = topk_weight; p.topk_phys = topk_phys;
  p.T = T; p.E = c.E; p.k = c.k; p.max_replicas = c.max_replicas; p.score_fn = c.score_fn;
  p.n_group = c.n_group; p.topk_group = c.topk_group; p.renormalise = renormalise;
  p.t_offset = ctx->token_offset; p.route_scale = c.route_scale;
  KernelTimer timer(ctx, REVIVE_K_ROUTE_TOPK, stream);
  const dim3 block(256);
  const bool rows = c.k <= 16 && (c.n_group == 1 || (c.E % 16 == 0 && (c.n_group == 2 || c.n_group == 4 || c.n_group == 8)));
  if (rows) {
    const int fours = ceil_div(T, 16), workgroups = fours < 2048 ? fours : 2048, rounds = ceil_div(fours, workgroups);
    const int n = ceil_div(c.E, 16);
    const bool wide = c.E % 64 == 0 && reinterpret_cast<uintptr_t>(logits) % 16 == 0;
#define REVIVE_ROUTE_LAUNCH(V)                                                                                                             \
  do {                                                                                                                                     \
    if (c.n_group > 1 && wide) hipLaunchKernelGGL((route_biased_rows_kernel<V, true, true>), dim3(workgroups), block, 0, stream, p, rounds);  \
    else if (c.n_group > 1) hipLaunchKernelGGL((route_biased_rows_kernel<V, true, false>), dim3(workgroups), block, 0, stream, p, rounds);    \
    else if (wide) hipLaunchKernelGGL((route_biased_rows_kernel<V, false, true>), dim3(workgroups), block, 0, stream, p, rounds);             \
    else hipLaunchKernelGGL((route_biased_rows_kernel<V, false, false>), dim3(workgroups), block, 0, stream, p, rounds);                      \
  } while (0)
    if (n <= 4) REVIVE_ROUTE_LAUNCH(4);
    else if (n <= 8) REVIVE_ROUTE_LAUNCH(8);
    else if (n <= 16) REVIVE_ROUTE_LAUNCH(16);
    else if (n <= 24) REVIVE_ROUTE_LAUNCH(24);
    else REVIVE_ROUTE_LAUNCH(32);
#undef REVIVE_ROUTE_LAUNCH
    return check_hip(ctx, hipGetLastError(), "route_biased launch");
  }
  const dim3 grid(ceil_div(T, 4));
  switch (ceil_div(c.E, 64)) {
    case 1: hipLaunchKernelGGL(route_biased_kernel<1>, grid, block, 0, stream, p); break;
    case 2: hipLaunchKernelGGL(route_biased_kernel<2>, grid, block, 0, stream, p); break;
    case 3: case 4: hipLaunchKernelGGL(route_biased_kernel<4>, grid, block, 0, stream, p); break;
    case 5: case 6: hipLaunchKernelGGL(route_biased_kernel<6>, grid, block, 0, stream, p); break;
    default: hipLaunchKernelGGL(route_biased_kernel<8>, grid, block, 0, stream, p); break;
  }
  return check_hip(ctx, hipGetLastError(), "route_biased launch");
}

}  // namespace revive
