// The choice of a token's experts by the lanes of a warp.  The contract is that of asgd_route in include/asgd_experts.h; how it works and what it
// costs stands in asgd_route.cu.  The kernel of a whole layer (asgd_expert_layer.cu) takes the scores, the keys and the checks from here and has
// shorter code of its own around them; an order of sums that changes here changes there.
#pragma once

#include "asgd_experts_common.cuh"

namespace {

using namespace asgd::experts;

struct Choice {
  asgd_route_config c;
  int group_lanes;                           // log2 of the lanes a group's keys are shared by
  unsigned group_magic;                      // e / (experts of a group) = umulhi(e, group_magic); 0: groups of one
  int lanes;                                 // of a token: the softmax's sum is one of this many lanes' sums, whoever computes it
  const float* bias;
};

// floats as unsigned numbers of the same order; 0 stands for "not available" (below every number's image)
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v + 0.f);                         // -0 and +0 are equal
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(unsigned u) {
  return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u);
}
// The L lanes of a token: maxima (one instruction for a whole warp), votes, sums.  Every lane of the warp takes part.
template <int L> __device__ __forceinline__ unsigned lanes_max(unsigned v) {
  if (L == 32) return __reduce_max_sync(kAll, v);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
template <int L> __device__ __forceinline__ unsigned lanes_min(unsigned v) {
  if (L == 32) return __reduce_min_sync(kAll, v);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = min(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
template <int L> __device__ __forceinline__ unsigned lanes_ballot(bool p) {       // bit l: the token's lane l
  const unsigned b = __ballot_sync(kAll, p);
  return L == 32 ? b : (b >> (threadIdx.x & 31 & ~(L - 1))) & ((1u << (L & 31)) - 1u);
}
template <int L> __device__ __forceinline__ float lanes_max(float v) {            // NaNs are passed over
  if (L == 32) {
    const unsigned u = __reduce_max_sync(kAll, v == v ? ordered(v) : 0u);
    return u ? from_ordered(u) : v;
  }
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// sum over the lanes that hold a choice (those from top_k on hold zeros), known to the token's lanes
template <int L> __device__ __forceinline__ float choice_sum(float v, int K) {
  for (int o = 1; o < K; o <<= 1) v += __shfl_xor_sync(kAll, v, o);
  return __shfl_sync(kAll, v, 0, L);
}

__device__ __forceinline__ float sigmoid(float x) { return __frcp_rn(__fadd_rn(1.f, expf(-x))); }

// Softmax of the row in registers: its largest logit and the sum.  A logit equal to the largest counts exactly 1, so
// that rows of +inf have finite scores; entries beyond the row are -inf.
struct Softmax {
  float m, sum;
  __device__ __forceinline__ float part(float x) const { return x == m ? 1.f : expf(x - m); }
  __device__ __forceinline__ float score(float x) const { return __fdiv_rn(part(x), sum); }
};
template <int S, int L> __device__ __forceinline__ Softmax softmax(const float (&x)[S]) {
  Softmax f;
  float m = x[0];
#pragma unroll
  for (int j = 1; j < S; ++j) m = fmaxf(m, x[j]);
  f.m = lanes_max<L>(m);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < S; ++j) sum += f.part(x[j]);
  f.sum = lanes_sum<L>(sum);
  return f;
}

template <int S, int L, typename T> __device__ __forceinline__ void load_row(const T* row, int E, int lane, float (&x)[S]) {
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * L + lane;
    x[j] = (e < E) ? Elem<T>::to_f(row[e]) : -INFINITY;
  }
}

// a <-> b so that the larger key, of equal ones that of the lower slot, is in a
__device__ __forceinline__ void order2(unsigned& a, unsigned& b, int& ia, int& ib) {
  const bool swap = b > a || (b == a && ib < ia);
  const unsigned ka = a, kb = b;
  const int ja = ia, jb = ib;
  a = swap ? kb : ka; b = swap ? ka : kb;
  ia = swap ? jb : ja; ib = swap ? ja : jb;
}
// a lane's S keys, descending, with the slots they came from (odd-even merge sort)
template <int S> __device__ __forceinline__ void sort_keys(unsigned (&key)[S], int (&slot)[S]) {
#pragma unroll
  for (int p = 1; p < S; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < S; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < S && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order2(key[i + j], key[i + j + k], slot[i + j], slot[i + j + k]);
}

// Takes all experts but those of the best groups_kept groups out (their keys become 0).  A whole warp with room for its keys
// in shared memory gives each group the same number of lanes, and a lane an even share of the group's keys; else the groups
// take turns.
constexpr int kScratch = 256;                                          // numbers of shared memory per warp
template <int S, int L> __device__ __forceinline__ void keep_groups(const Choice& a, int lane, unsigned* scratch, unsigned (&key)[S]) {
  const asgd_route_config& c = a.c;
  int group[S];
#pragma unroll
  for (int j = 0; j < S; ++j) group[j] = a.group_magic ? (int)__umulhi((unsigned)(j * L + lane), a.group_magic) : j * L + lane;
  unsigned mine = 0;                                                   // lane g: the ordered score of group g (groups <= L)
  if (L == 32 && S * 32 <= kScratch) {
    const int per = c.experts / c.groups, shift = a.group_lanes;       // 2^shift lanes per group
    const int g = lane >> shift, sub = lane & ((1 << shift) - 1);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < S; ++j) scratch[j * 32 + lane] = key[j];
    __syncwarp();
    unsigned m1 = 0, m2 = 0;
    if (g < c.groups)
      for (int i = sub; i < per; i += 1 << shift) {
        const unsigned k = scratch[g * per + i];
        m2 = max(m2, min(m1, k));
        m1 = max(m1, k);
      }
    for (int o = 1; o < 1 << shift; o <<= 1) {                         // the two largest of two lanes' two largest
      const unsigned o1 = __shfl_xor_sync(kAll, m1, o), o2 = __shfl_xor_sync(kAll, m2, o);
      m2 = max(min(m1, o1), max(m2, o2));
      m1 = max(m1, o1);
    }
    if (c.group_top == 2 && m2) m1 = ordered(__fadd_rn(from_ordered(m1), from_ordered(m2)));
    const int from = (lane << shift) & 31;
    const unsigned got = __shfl_sync(kAll, m1, from);
    if (lane < c.groups) mine = got;
  } else {
    for (int g = 0; g < c.groups; ++g) {
      unsigned m1 = 0, m2 = 0;                                         // this lane's two largest keys of the group
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const unsigned k = group[j] == g ? key[j] : 0u;
        m2 = max(m2, min(m1, k));
        m1 = max(m1, k);
      }
      unsigned best = lanes_max<L>(m1);
      if (c.group_top == 2) {
        const unsigned holders = lanes_ballot<L>(m1 == best);
        const unsigned second = lanes_max<L>((lane == __ffs(holders) - 1) ? m2 : m1);
        if (second) best = ordered(__fadd_rn(from_ordered(best), from_ordered(second)));
      }
      if (lane == g) mine = best;
    }
  }
  unsigned kept = 0;
  for (int i = 0; i < c.groups_kept; ++i) {
    const bool taken = (kept >> lane) & 1u;
    const unsigned best = lanes_max<L>(taken ? 0u : mine);
    const unsigned holders = lanes_ballot<L>(best && mine == best && !taken);
    kept |= holders & (0u - holders);                                  // the lowest of them, if any
  }
#pragma unroll
  for (int j = 0; j < S; ++j) if (!((kept >> (group[j] & 31)) & 1u)) key[j] = 0u;
}

// The choice of one token.  Each lane returns a place among the top_k (or -1: it has none), the expert there (-1: nothing
// is available) and its weight.
template <int S, int L> __device__ __forceinline__ void choose(const Choice& a, const float (&x)[S], int lane, unsigned* scratch, int& place, int& id,
                                                               float& weight) {
  const asgd_route_config& c = a.c;
  const int E = c.experts, K = c.top_k;
  const bool by_logit = a.bias == nullptr && c.group_top == 1, sigmoid_scores = c.score == ASGD_SCORE_SIGMOID;
  Softmax f{0.f, 1.f};
  if (!sigmoid_scores) f = softmax<S, L>(x);
  unsigned key[S];
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * L + lane;
    float v = x[j];
    if (!by_logit) {
      v = sigmoid_scores ? sigmoid(x[j]) : f.score(x[j]);
      if (a.bias && e < E) v = __fadd_rn(v, a.bias[e]);
    }
    key[j] = (e < E && x[j] > -INFINITY && v > -INFINITY) ? ordered(v) : 0u;
  }
  if (c.groups_kept < c.groups) keep_groups<S, L>(a, lane, scratch, key);
  id = -1;
  place = lane < K ? lane : -1;
  float chosen = 0.f;                                                  // the choice's logit
  bool ranked = false;
  if constexpr (L == 32 && S <= 8) {
    // the bound: at least top_k keys reach it
    unsigned top = key[0], bound = 1u;
#pragma unroll
    for (int j = 1; j < S; ++j) top = max(top, key[j]);
    for (int i = 0; i < K; ++i) {
      bound = __reduce_max_sync(kAll, top);
      if (!bound) break;
      top = top == bound ? 0u : top;
    }
    bound = max(bound, 1u);
    unsigned votes[S];
    int n = 0;
#pragma unroll
    for (int j = 0; j < S; ++j) { votes[j] = __ballot_sync(kAll, key[j] >= bound); n += __popc(votes[j]); }
    if (n <= 32) {
      ranked = true;
      uint4* found = reinterpret_cast<uint4*>(scratch);                // (key, expert, logit), in the experts' order
      __syncwarp();
      int before = 0;
#pragma unroll
      for (int j = 0; j < S; ++j) {
        if (key[j] >= bound) found[before + __popc(votes[j] & ((1u << lane) - 1u))] = make_uint4(key[j], (unsigned)(j * 32 + lane), __float_as_uint(x[j]), 0u);
        before += __popc(votes[j]);
      }
      __syncwarp();
      const uint4 mine = lane < n ? found[lane] : make_uint4(0u, 0u, 0u, 0u);
      int rank = 0;
      for (int i = 0; i < n; ++i) {                                    // keys above, and equal ones of lower experts
        const unsigned k = __shfl_sync(kAll, mine.x, i);
        rank += i < lane ? k >= mine.x : k > mine.x;
      }
      if (lane < n) {
        place = rank < K ? rank : -1;
        if (rank < K) { id = (int)mine.y; chosen = __uint_as_float(mine.z); }
      }                                                                // places from n on have no key: their lanes hold none
    }
  }
  if (!ranked) {
    int slot[S];
#pragma unroll
    for (int j = 0; j < S; ++j) slot[j] = j;
    sort_keys<S>(key, slot);
    for (int i = 0; i < K; ++i) {
      const unsigned best = lanes_max<L>(key[0]);
      unsigned holders = lanes_ballot<L>(key[0] == best);
      // equal keys (of any of the warp's tokens): the lowest expert, so the first slot first
      if (__any_sync(kAll, (holders & (holders - 1)) && best)) {
        const unsigned mine = key[0] == best ? (unsigned)slot[0] : 32u, first = lanes_min<L>(mine);
        holders = lanes_ballot<L>(mine == first);
      }
      const int from = __ffs(holders) - 1, at = __shfl_sync(kAll, slot[0], from, L);
      if (lane == i && best) id = at * L + from;
      float v = from_ordered(best);
      if (!by_logit) {
        v = x[0];
#pragma unroll
        for (int j = 1; j < S; ++j) v = at == j ? x[j] : v;
        v = __shfl_sync(kAll, v, from, L);
      }
      if (lane == i) chosen = v;
      const bool pop = lane == from;
#pragma unroll
      for (int j = 0; j + 1 < S; ++j) { key[j] = pop ? key[j + 1] : key[j]; slot[j] = pop ? slot[j + 1] : slot[j]; }
      key[S - 1] = pop ? 0u : key[S - 1];
    }
  }
  const float s = id < 0 ? 0.f : sigmoid_scores ? sigmoid(chosen) : f.score(chosen);
  weight = 0.f;
  if (c.renormalise) {
    const float sum = lanes_sum<L>(s);                                 // lanes without a choice hold zeros
    if (id >= 0) weight = c.scale * s / (sum + 1e-20f);
  } else if (id >= 0) {
    weight = c.scale * s;
  }
}

inline bool config_ok(const asgd_route_config* c) {
  if (!c) return false;
  if (c->experts < 1 || c->top_k < 1 || c->groups < 1 || c->groups_kept < 1 || c->groups_kept > c->groups) return false;
  if (c->experts % c->groups) return false;
  if (c->score != ASGD_SCORE_SOFTMAX && c->score != ASGD_SCORE_SIGMOID) return false;
  if (c->group_top != 1 && c->group_top != 2) return false;
  if (c->renormalise != 0 && c->renormalise != 1) return false;
  if (c->align < 1) return false;
  if (c->top_k > c->groups_kept * (c->experts / c->groups)) return false;
  return true;
}
inline bool config_supported(const asgd_route_config* c) {
  return c->experts <= ASGD_MAX_EXPERTS && c->groups <= ASGD_MAX_EXPERT_GROUPS && c->top_k <= ASGD_MAX_TOP_K;
}
// Lanes of a token: 8 where they have room for the choices and the groups and hold eight numbers at most (see with_shape in asgd_route.cu).
inline int lanes_of(const asgd_route_config& c) {
  const int kept = c.groups_kept < c.groups ? c.groups : 1;
  return c.experts <= 64 && c.top_k <= 8 && kept <= 8 ? 8 : 32;
}
inline Choice choice_of(const asgd_route_config& c, const float* bias) {
  Choice a;
  a.c = c;
  a.group_lanes = 0;
  while ((c.groups << (a.group_lanes + 1)) <= 32) ++a.group_lanes;
  const unsigned per = (unsigned)(c.experts / c.groups);
  a.group_magic = per > 1 ? (unsigned)((1ull << 32) / per + 1) : 0;    // exact for numbers below 2^16
  a.lanes = lanes_of(c);
  a.bias = bias;
  return a;
}

}  // namespace
