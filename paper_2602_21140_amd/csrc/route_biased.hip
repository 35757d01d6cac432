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

__device__ __forceinline__ uint32_t wave_max_u(uint32_t v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
  return v;
}
__device__ __forceinline__ float wave_max_f(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
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
    for (int i = 0; i < V; ++i) score[i] = 1.0f / (1.0f + expf(-score[i]));
  } else {
    m = wave_max_f(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      score[i] = lane + 64 * i < p.E ? expf(score[i] - m) : 0.f;
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
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t o1 = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m1), o)), o2 = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m2), o));
        m2 = max(min(m1, o1), max(m2, o2));
        m1 = max(m1, o1);
      }
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
    const uint32_t best = wave_max_u(u);
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
  if (lane < p.k) {
    const int64_t o = static_cast<int64_t>(t) * p.k + lane;
    const int count = p.l2p_count[my_e];
    const unsigned long long b = static_cast<unsigned long long>(p.t_offset) + t;
    p.topk_logical[o] = my_e;
    p.topk_weight[o] = my_s / sum * p.route_scale;
    p.topk_phys[o] = count > 0 ? p.l2p_table[my_e * p.max_replicas + static_cast<int>(b % count)] : -1;
  }
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
  const dim3 grid(ceil_div(T, 4)), block(256);
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
