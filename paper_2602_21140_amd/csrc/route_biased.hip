// Gate with a bias for balance: experts are chosen by score + bias and weighted by the score alone.
//
//   s_e   = exp(z_e - max z) / sum exp(z - max z)  or  1 / (1 + exp(-z_e)), over all E experts
//   key_e = s_e + b_e; an expert without a live replica is out (paper Sec. 3.4 "Missing experts", Sec. 4.2)
//   a group's score is the sum of its two best keys above -inf (the one, if there is one); the topk_group best groups are kept
//   top-k by key, ties to the lower id;  weight_j = s_{e_j} [/ sum_j s_{e_j}] * route_scale
//
// All of it in fp32.  What is no number has a place among the keys: NaN and -inf are kNone, behind every number and alike but for
// their ids; an expert that is lost, taken or in a dropped group is -inf.  kNone is fp32's lowest number, and keys that are numbers
// begin at the one above it, which a bias of the lowest number counts as.
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

constexpr float kNone = -0x1.fffffep127f, kLowest = -0x1.fffffcp127f;
constexpr float kOut = -__builtin_inff();

// Bias of an expert as key_of wants it: -inf without a live replica, kNone for a NaN or -inf, else a number from kLowest up or +inf.
__device__ __forceinline__ float bias_of(float b, int count) {
  const float number = b == kNone ? kLowest : b, place = fmaxf(number, kNone);
  return count > 0 ? place : kOut;
}
__device__ __forceinline__ float bias_of(const BiasedParams& p, int e, bool is) {
  e = min(e, p.E - 1);
  return bias_of(p.bias[e], is ? p.l2p_count[e] : 0);
}
// Scores are NaN or in [0, 1], so that a sum is no less than its bias; fmaxf passes a NaN over.
__device__ __forceinline__ float key_of(float score, float bias) { return fmaxf(score + bias, fminf(bias, kNone)); }
// Half the score of a group (which fp32 always holds) from its two best keys; kNone and -inf of groups without a number.
__device__ __forceinline__ float group_score(float m1, float m2) { return m2 > kNone ? fmaf(0.5f, m1, 0.5f * m2) : m1 > kNone ? 0.5f * m1 : m1; }

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
__device__ __forceinline__ float dpp_f(float v, float other) { return __int_as_float(dpp<STEP>(__float_as_int(v), __float_as_int(other))); }

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
__device__ __forceinline__ float wave_max(float v) {
  v = row_max(v);
  v = fmaxf(v, dpp_f<4>(v, kOut));
  return __int_as_float(last_lane(__float_as_int(fmaxf(v, dpp_f<5>(v, kOut)))));
}
constexpr int kLeast = -2147483647 - 1;  // changes no maximum, so that a step is one instruction
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, dpp<0>(v, kLeast));
  v = max(v, dpp<1>(v, kLeast));
  v = max(v, dpp<2>(v, kLeast));
  v = max(v, dpp<3>(v, kLeast));
  v = max(v, dpp<4>(v, kLeast));
  return last_lane(max(v, dpp<5>(v, kLeast)));
}
// An integer that is ordered as the float is (which is neither NaN nor -0).
__device__ __forceinline__ int ordered(float v) {
  const int b = __float_as_int(v);
  return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum(v);
  v += dpp_f<4>(v, 0.f);
  return __int_as_float(last_lane(__float_as_int(v + dpp_f<5>(v, 0.f))));
}
// The two largest of two disjoint sets, each given by its two largest.
template <int STEP>
__device__ __forceinline__ void top2_step(float& m1, float& m2) {
  const float o1 = dpp_f<STEP>(m1, kOut), o2 = dpp_f<STEP>(m2, kOut);
  m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
  m1 = fmaxf(m1, o1);
}

// The keys' scores.  exp by the hardware's 2^p with p = x log2(e) rounded is off by |x| units in its last place, which is less
// than one of the largest score; NaN stays, and infinities give what they should.
constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float near_exp(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }
__device__ __forceinline__ float near_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2e)); }
// The weights' scores, of the chosen experts: exp(x + more) for x in [-100, 88] and a small rest, with what the rounding of p left
// out.  The instruction has zero for what is below the least normal number, 2^-126.
__device__ __forceinline__ float exp_of(float x, float more) {
  const float p = x * kLog2e, rest = fmaf(x, kLog2e, -p) + x * 1.92596299e-8f;  // log2(e) = kLog2e + 1.92596299e-8
  const float e = __builtin_amdgcn_exp2f(p);
  return fmaf(e, fmaf(rest, 0.693147181f, more), e);
}
// exp(z - m), z <= m, of the difference and what its rounding left out; -100 stands for all that make zero.
__device__ __forceinline__ float exp_below(float z, float m) {
  const float d = z - m, t = d - z, more = (z - (d - t)) - (m + t);
  return d < -100.f ? exp_of(-100.f, 0.f) : exp_of(d, more);
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + exp_of(z > 87.f ? -87.f : -z, 0.f)); }

// Scores of the chosen experts of a token, which LANES lanes have, `mine` of them an expert; `shift` and `scale` are those of its
// softmax.  Where a score is too small for fp32, those of a renormalised token keep their shares: they are taken from the largest
// chosen logit, and what they have in common goes out.  (The token's largest may be lost, or kept back by the bias, and would
// leave nothing but zeros of scores 87 below it.  Below -30 a sigmoid is exp(z) to all bits of fp32.)  A token whose scores are
// NaN has `scale` NaN.  Hardly a call has such a score, and a wavefront without one passes that over.
template <int LANES>
__device__ __forceinline__ float chosen_score(float z, float shift, float scale, bool sig, bool renormalise, bool mine) {
  const float s = sig ? sigmoid(z) : exp_below(z, shift) * scale;
  const unsigned long long small = __ballot(mine && z - (sig ? 0.f : shift) < (sig ? -30.f : -80.f));
  if (small == 0) return s;
  const float top = LANES == 16 ? row_max(mine ? z : kOut) : wave_max(mine ? z : kOut);
  if (sig) return z < -30.f ? exp_below(z, renormalise && top < -30.f ? top : 0.f) : s;
  const bool here = LANES == 16 ? (small >> (threadIdx.x & 48) & 0xFFFFull) != 0 : true;
  return renormalise && here ? exp_below(z, top) * scale : s;
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
// Bound by the ALU where there are many tokens: 32 768 of 384 experts, k = 8, 20.8 us (2.5 TB/s), with vector instructions in 72 % of
// the cycles in which a CU is busy.  8192 of 256 experts in 8 groups 7.9 us (1.2 TB/s), 43 %: two wavefronts a SIMD, which wait for
// their loads and then for one choice after the other.  With a wavefront per token 33.1 and 12.6.  What a choice costs is kept
// small by two levels: a lane has the best key of every four of its experts in
// registers and the keys in LDS; a round looks at the bests, and the four keys of the winning one are read, stripped of the
// winner and put back.
template <int V, bool GROUPED, bool WIDE>
__global__ __launch_bounds__(256) void route_biased_rows_kernel(BiasedParams p, int rounds) {
  constexpr int C = V / 4;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  __shared__ f32x4 keys[4][C][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane >> 4, li = lane & 15;
  const int n = (p.E + 15) >> 4;
  const int lg = GROUPED ? 16 / p.n_group : 16, lj = li & (lg - 1);  // lanes of a group, this one's place among them
  const int e0 = GROUPED ? li / lg * (p.E / p.n_group) : 0;          // the group's first expert
  auto expert = [&](int i) { return e0 + (WIDE ? (i >> 2) * 4 * lg + lj * 4 + (i & 3) : i * lg + lj); };  // place i
  const bool sig = p.score_fn == REVIVE_SCORE_SIGMOID;
  float bias[V];
  if (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int e = c * 4 < n ? expert(c * 4) : 0;  // n is a multiple of 4
      const f32x4 b = *reinterpret_cast<const f32x4*>(p.bias + e);
      const int4 k = *reinterpret_cast<const int4*>(p.l2p_count + e);
      bias[c * 4] = bias_of(b[0], c * 4 < n ? k.x : 0);
      bias[c * 4 + 1] = bias_of(b[1], c * 4 < n ? k.y : 0);
      bias[c * 4 + 2] = bias_of(b[2], c * 4 < n ? k.z : 0);
      bias[c * 4 + 3] = bias_of(b[3], c * 4 < n ? k.w : 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = bias_of(p, expert(i), i < n && expert(i) < p.E);
  }
  for (int r = 0; r < rounds; ++r) {
    const int t0 = ((r * gridDim.x + blockIdx.x) * 4 + wave) * 4, t = t0 + row;
    if (t0 >= p.T) return;  // whole wavefront leaves together
    const float* z = p.logits + static_cast<int64_t>(min(t, p.T - 1)) * p.E;
    f32x4 s[C];  // logits, then scores, then keys
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (WIDE) {
        s[c] = *reinterpret_cast<const f32x4*>(z + (c * 4 < n ? expert(c * 4) : 0));
        if (c * 4 >= n) s[c] = f32x4{kOut, kOut, kOut, kOut};  // no experts in these places: scores of zero
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[c][i] = z[min(expert(c * 4 + i), p.E - 1)];
          if (c * 4 + i >= n || expert(c * 4 + i) >= p.E) s[c][i] = kOut;
        }
      }
    }
    float shift = kOut, scale = 1.f;
    if (sig) {
#pragma unroll
      for (int i = 0; i < V; ++i) s[i >> 2][i & 3] = near_sigmoid(s[i >> 2][i & 3]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) shift = fmaxf(shift, s[i >> 2][i & 3]);
      shift = row_max(shift);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) sum += s[i >> 2][i & 3] = near_exp(s[i >> 2][i & 3], shift);
      scale = 1.0f / row_sum(sum);
#pragma unroll
      for (int i = 0; i < V; ++i) s[i >> 2][i & 3] *= scale;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s[i >> 2][i & 3] = key_of(s[i >> 2][i & 3], bias[i]);
    if (GROUPED) {
      float m1 = kOut, m2 = kOut;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        m2 = fmaxf(fminf(m1, s[i >> 2][i & 3]), m2);
        m1 = fmaxf(m1, s[i >> 2][i & 3]);
      }
      top2_step<0>(m1, m2);
      if (lg >= 4) top2_step<1>(m1, m2);
      if (lg >= 8) top2_step<6>(m1, m2);
      // rank of my group among all groups of the token (better score first, ties to the lower group id)
      const float mine = group_score(m1, m2);
      int rank = 0, o = __float_as_int(mine), h = li;
      for (int i = 1; i < p.n_group; ++i) {  // rotate the row by a group
        if (lg == 2) { o = __builtin_amdgcn_mov_dpp(o, 0x122, 0xF, 0xF, false); h = __builtin_amdgcn_mov_dpp(h, 0x122, 0xF, 0xF, false); }
        else if (lg == 4) { o = __builtin_amdgcn_mov_dpp(o, 0x124, 0xF, 0xF, false); h = __builtin_amdgcn_mov_dpp(h, 0x124, 0xF, 0xF, false); }
        else { o = __builtin_amdgcn_mov_dpp(o, 0x128, 0xF, 0xF, false); h = __builtin_amdgcn_mov_dpp(h, 0x128, 0xF, 0xF, false); }
        rank += __int_as_float(o) > mine || (__int_as_float(o) == mine && h < li);
      }
      const bool kept = rank < p.topk_group;
#pragma unroll
      for (int i = 0; i < V; ++i) s[i >> 2][i & 3] = kept ? s[i >> 2][i & 3] : kOut;
    }
    float best4[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      best4[c] = fmaxf(fmaxf(s[c][0], s[c][1]), fmaxf(s[c][2], s[c][3]));
      if (C > 1) keys[wave][c][lane] = s[c];
    }

    // k rounds of arg-max (largest key, ties to the lower expert id); lane j of the row keeps the j-th choice
    constexpr int kNobody = 1 << 16;
    int my_e = 0;
#pragma unroll 1
    for (int j = 0; j < p.k; ++j) {
      float m = best4[0];
#pragma unroll
      for (int c = 1; c < C; ++c) m = fmaxf(m, best4[c]);
      const float best = row_max(m);
      int at = C - 1;
#pragma unroll
      for (int c = C - 2; c >= 0; --c) at = best4[c] == best ? c : at;
      f32x4 four = C > 1 ? keys[wave][at][lane] : s[0];
      const int pos = four[0] == best ? 0 : four[1] == best ? 1 : four[2] == best ? 2 : 3;
      const int mine = m == best ? expert(at * 4 + pos) : kNobody, e = row_min(mine);
      const bool won = mine == e;
#pragma unroll
      for (int i = 0; i < 4; ++i) four[i] = won && pos == i ? kOut : four[i];
      if (C > 1) keys[wave][at][lane] = four;
      else s[0] = four;
      const float left = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3]));
#pragma unroll
      for (int c = 0; c < C; ++c) best4[c] = won && at == c ? left : best4[c];
      my_e = li == j ? e : my_e;
    }
    my_e = min(my_e, p.E - 1);
    const float zc = z[my_e];
    const float sc = chosen_score<16>(zc, shift, scale, sig, p.renormalise, li < p.k);
    const float total = p.renormalise ? row_sum(li < p.k ? sc : 0.f) : 1.f;
    if (li < p.k && t < p.T) store_choice(p, t, li, my_e, sc / total * p.route_scale);
  }
}

// A wavefront per token; lane l holds experts l, l + 64, ...  Bound by latency: the choices follow one another, each a maximum over
// the wavefront (vector instructions in 20 % of the cycles).  64 tokens of 256 experts in 8 groups, k = 8, 5.8 us; 512 of 512
// experts, k = 16, 7.6.
template <int V>
__global__ __launch_bounds__(256) void route_biased_kernel(BiasedParams p) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;  // whole wavefront leaves together
  const float* z = p.logits + static_cast<int64_t>(t) * p.E;
  const bool sig = p.score_fn == REVIVE_SCORE_SIGMOID;
  float key[V], bias[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane + 64 * i;
    key[i] = e < p.E ? z[e] : kOut;
    bias[i] = bias_of(p, e, e < p.E);
  }
  float shift = kOut, scale = 1.f;
  if (sig) {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = near_sigmoid(key[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) shift = fmaxf(shift, key[i]);
    shift = wave_max(shift);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += key[i] = near_exp(key[i], shift);
    scale = 1.0f / wave_sum(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] *= scale;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] = key_of(key[i], bias[i]);

  if (p.n_group > 1) {
    const int gsz = p.E / p.n_group;
    float mine = kOut;  // score of group `lane`
    if (gsz >= 8 && (gsz & (gsz - 1)) == 0 && gsz <= 64) {  // groups are aligned runs of lanes: all of them at once
      const int per = 64 / gsz, src = (lane % per) * gsz;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float m1 = key[i], m2 = kOut;
        top2_step<0>(m1, m2);
        top2_step<1>(m1, m2);
        top2_step<6>(m1, m2);
        if (gsz >= 16) top2_step<7>(m1, m2);
        if (gsz >= 32) {
          const float o1 = __shfl_xor(m1, 16), o2 = __shfl_xor(m2, 16);
          m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
          m1 = fmaxf(m1, o1);
        }
        if (gsz >= 64) {
          const float o1 = __shfl_xor(m1, 32), o2 = __shfl_xor(m2, 32);
          m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
          m1 = fmaxf(m1, o1);
        }
        const float g = __shfl(group_score(m1, m2), src);
        if (lane / per == i && lane < p.n_group) mine = g;
      }
    } else {
      for (int g = 0; g < p.n_group; ++g) {
        float m1 = kOut, m2 = kOut;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = lane + 64 * i;
          const float u = e >= g * gsz && e < (g + 1) * gsz ? key[i] : kOut;
          m2 = fmaxf(m2, fminf(m1, u));
          m1 = fmaxf(m1, u);
        }
        top2_step<0>(m1, m2);
        top2_step<1>(m1, m2);
        top2_step<6>(m1, m2);
        top2_step<7>(m1, m2);
        top2_step<4>(m1, m2);
        top2_step<5>(m1, m2);
        const float s = __int_as_float(last_lane(__float_as_int(group_score(m1, m2))));
        if (lane == g) mine = s;
      }
    }
    int rank = 0;
    for (int h = 0; h < p.n_group; ++h) {
      const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), h));
      rank += o > mine || (o == mine && h < lane);
    }
    const unsigned long long kept = __ballot(lane < p.n_group && rank < p.topk_group);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // e / gsz: exact, e + 1/2 is never within 2^-11 of a multiple of gsz
      const int g = static_cast<int>((static_cast<float>(lane + 64 * i) + 0.5f) / static_cast<float>(gsz));
      if (!((static_cast<uint32_t>(kept) >> (g & 31)) & 1u)) key[i] = kOut;
    }
  }

  // k rounds of arg-max (largest key, ties to the lower expert id); lane j keeps the j-th choice.  Keys as integers of the same
  // order, whose maxima take the other lane's as an operand; a lane has its best, u, and which of its experts that is, so that
  // several lanes with the round's best are the only ones whose ids have to be compared.
  int place[V], u = 0, ui = 0, my_e = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) place[i] = ordered(key[i]);
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    u = place[0];
    ui = 0;
#pragma unroll
    for (int i = 1; i < V; ++i) {
      ui = place[i] > u ? i : ui;
      u = max(u, place[i]);
    }
    const int best = wave_max(u);
    const unsigned long long holders = __ballot(u == best);
    int w = __builtin_ctzll(holders);
    if (holders & (holders - 1)) w = -wave_max(u == best ? -(ui * 64 + lane) : -64 * V) & 63;
    const int e = __builtin_amdgcn_readlane(ui, w) * 64 + w;
    const int taken = lane == w ? ui : -1;
#pragma unroll
    for (int i = 0; i < V; ++i) place[i] = taken == i ? ordered(kOut) : place[i];
    if (lane == j) my_e = min(e, p.E - 1);
  }

  const float zc = z[my_e];
  const float sc = chosen_score<64>(zc, shift, scale, sig, p.renormalise, lane < p.k);
  const float sum = p.renormalise ? wave_sum(lane < p.k ? sc : 0.f) : 1.f;
  if (lane < p.k) store_choice(p, t, lane, my_e, sc / sum * p.route_scale);
}

}  // namespace

// Which kernel.  A row of lanes per token does a quarter of the work, but one after the other: it wins once a wavefront per token
// keeps the ALUs busy, later where experts are no multiple of 64 and its loads are of four bytes.  us in a graph, a row and a
// wavefront per token: 256 experts in 8 groups, k = 8, 1024 tokens 6.8 and 6.0, 2048 6.9 and 6.6, 3000 6.9 and 7.3, 8192 7.9 and
// 12.6; 384, k = 8, 2048 6.8 and 5.8, 3000 6.9 and 6.4, 8192 7.8 and 10.2; 512, k = 16, 2048 10.9 and 8.4, 3000 11.1 and 9.9, 4096
// 11.2 and 11.3; 64, k = 2, 3000 3.3 and 3.3, 4096 3.4 and 3.6; 100, k = 4, 4096 4.9 and 4.3, 8192 5.4 and 5.6; 500, k = 8, 6144
// 13.2 and 10.0, 8192 13.3 and 13.0.
constexpr int kRowsFrom = 3000, kNarrowRowsFrom = 8192;
// Workgroups of the rows' kernel at most; beyond them each takes its share of tokens.  32768 tokens of 384 experts: 512 26.6, 1024
// 20.6, 2048 20.5; of 256 in 8 groups 24.7, 18.7 and 18.6.
constexpr int kRowsWorkgroups = 1024;

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
  const bool wide = c.E % 64 == 0 && (reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(bias)) % 16 == 0;
  const bool rows = T >= (wide ? kRowsFrom : kNarrowRowsFrom) && c.k <= 16 &&
                    (c.n_group == 1 || (c.E % 16 == 0 && (c.n_group == 2 || c.n_group == 4 || c.n_group == 8)));
  if (rows) {
    const int fours = ceil_div(T, 16), workgroups = fours < kRowsWorkgroups ? fours : kRowsWorkgroups, rounds = ceil_div(fours, workgroups);
    const int n = ceil_div(c.E, 16);
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
