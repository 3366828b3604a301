// Routing of tokens to experts: choice and weights, their gradient, and the plan that groups the assignments by expert.
// The contract is in include/asgd_experts.h.
//
// A warp, or with few experts 8 lanes of one, own a token: lane l holds the experts l, l + L, ... in registers, so the row
// is read once, coalesced at any stride.  Keys become unsigned numbers of the same order.  A whole warp prunes first: the
// top_k-th largest of the lanes' largest keys is a bound under every choice, and what reaches it (top_k to twice as many
// keys, as a rule) is gathered, one key per lane in the experts' order, and ranked by counting.  Where more than 32 keys
// reach the bound, and where 8 lanes own a token, each lane sorts its keys, and a choice is the largest of the lanes' first
// ones, a vote for the lane that has it, and a shift of that lane's list.  Only the chosen logits are turned into weights.
// Instructions and their latency are the bound, not the bytes: 16384 tokens among 128 experts 14 us (and 7 for the plan),
// 65536 among 256 in groups 115; each lane's keys sorted instead of pruned took 17 and 180.
//
// The plan is a stable counting sort by expert.  A block's tokens are a chunk (of 64 at most); inside a chunk each
// expert has a 64-bit word with a bit per token that chose it, so an assignment's rank among the chunk's is the
// population count below its bit.  Chunk counts are then summed along the chunks and the experts, and the ranks moved by
// those sums: integers only, so the plan does not depend on timing.
#include "asgd_experts_common.cuh"

#include <algorithm>
#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr int kMaxChunk = 64;                // tokens of a chunk (bits of an expert's word)
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kThreadsOne = 1024;            // the one block of a single chunk: two tokens per warp, latency counts
constexpr int kFillBlocks = 2 * kSMs;        // blocks at least that write the rows of nothing

struct RouteArgs {
  asgd_route_config c;
  long long T, ld, source_len;
  int chunk, chunks, stride;                 // tokens of a chunk, chunks, numbers of an expert in hist (a multiple of 4)
  int group_lanes;                           // log2 of the lanes a group's keys are shared by
  unsigned group_magic;                      // e / (experts of a group) = umulhi(e, group_magic); 0: groups of one
  const void* logits;
  const float* bias;
  int* ids;
  float* weights;
  int* offsets;
  int* rows;
  int* source;
  int* hist;                                 // [E][stride] assignments per expert and chunk, then those in the chunks before
  int* totals;                               // [E]
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
template <int S, int L> __device__ __forceinline__ void keep_groups(const RouteArgs& a, int lane, unsigned* scratch, unsigned (&key)[S]) {
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
template <int S, int L> __device__ __forceinline__ void choose(const RouteArgs& a, const float (&x)[S], int lane, unsigned* scratch, int& place, int& id,
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

// exclusive sums over the E padded counts of the block's shared array, in place; returns the total.  All threads.
__device__ int scan_padded(int* cnt, int E, int align, int* warp_part) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, nw = blockDim.x >> 5;
  const int per = (E + blockDim.x - 1) / blockDim.x;
  int mine = 0;
  for (int q = 0; q < per; ++q) {
    const int e = tid * per + q;
    if (e < E) mine += (cnt[e] + align - 1) / align * align;
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(kAll, inc, o); if (lane >= o) inc += v; }
  if (lane == 31) warp_part[wid] = inc;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < nw; ++w) { if (w < wid) before += warp_part[w]; total += warp_part[w]; }
  int run = before + inc - mine;
  for (int q = 0; q < per; ++q) {
    const int e = tid * per + q;
    if (e < E) { const int v = (cnt[e] + align - 1) / align * align; cnt[e] = run; run += v; }
  }
  __syncthreads();
  return total;
}

// -1 for the rows of nothing: the experts' padding, a warp each in turn, and the tail behind the last expert
__device__ void fill_nothing(const RouteArgs& a, const int* first_row, const int* count, int total, int block, int blocks) {
  const int E = a.c.experts, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
  if (a.c.align > 1)
    for (int e = block * nw + (int)(threadIdx.x >> 5); e < E; e += blocks * nw) {
      const int to = e + 1 < E ? first_row[e + 1] : total;
      for (int r = first_row[e] + count[e] + lane; r < to; r += 32) a.source[r] = -1;
    }
  for (long long r = total + (long long)block * blockDim.x + threadIdx.x; r < a.source_len; r += (long long)blocks * blockDim.x) a.source[r] = -1;
}

template <int S, int L, typename T> __global__ void __launch_bounds__(S <= 8 ? kThreadsOne : 512) route_kernel(const RouteArgs a) {
  wait_for_stream();
  if (a.chunks > 1) let_next_come();
  // 48 KB: the warps' scratch of the choices, then the plan's arrays in its place
  __shared__ unsigned long long word[ASGD_MAX_EXPERTS];
  __shared__ int ids[kMaxChunk * ASGD_MAX_TOP_K];
  __shared__ __align__(16) union Shared {
    unsigned scratch[32][kScratch];
    struct { int first_row[ASGD_MAX_EXPERTS], count[ASGD_MAX_EXPERTS], warp_part[32]; } after;
    __device__ Shared() {}
  } sh;
  int *first_row = sh.after.first_row, *count = sh.after.count, *warp_part = sh.after.warp_part;
  const int E = a.c.experts, K = a.c.top_k, lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool plan = a.offsets != nullptr;
  const long long t0 = (long long)blockIdx.x * a.chunk;
  const int nt = (int)min((long long)a.chunk, a.T - t0);
  if (plan) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) word[e] = 0;
    __syncthreads();
  }
  const int l = lane % L, sub = lane / L;                              // lane of the token, token of the warp
  for (int q0 = wid * (32 / L); q0 < nt; q0 += nw * (32 / L)) {
    const int q = q0 + sub;
    const bool there = q < nt;
    float x[S];
    load_row<S, L, T>(reinterpret_cast<const T*>(a.logits) + (t0 + q) * a.ld, there ? E : 0, l, x);
    int place, id;
    float w;
    choose<S, L>(a, x, l, sh.scratch[wid], place, id, w);
    if (there && place >= 0) {
      a.ids[(t0 + q) * K + place] = id;
      a.weights[(t0 + q) * K + place] = w;
      ids[q * K + place] = id;
      if (plan && id >= 0) atomicOr(&word[id], 1ull << q);
    }
  }
  if (!plan) return;
  __syncthreads();
  const bool one = a.chunks <= 1;
  int total = 0;
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    const int n = __popcll(word[e]);
    if (one) { count[e] = n; first_row[e] = n; }
    else a.hist[(long long)e * a.stride + blockIdx.x] = n;
  }
  if (one) {
    __syncthreads();
    total = scan_padded(first_row, E, a.c.align, warp_part);
    for (int e = threadIdx.x; e < E; e += blockDim.x) a.offsets[e] = first_row[e];
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
  for (int q = wid; q < nt; q += nw)
    if (lane < K) {
      const long long at = (t0 + q) * K + lane;
      const int id = ids[q * K + lane];
      int r = -1;
      if (id >= 0) {
        r = __popcll(word[id] & ((1ull << q) - 1ull));
        if (one) { r += first_row[id]; a.source[r] = (int)at; }
      }
      a.rows[at] = r;
    }
  if (one) fill_nothing(a, first_row, count, total, 0, 1);
}

// per expert (a warp each, a lane eight neighbouring chunks at a time): counts of the chunks before, and the total
__global__ void __launch_bounds__(128) chunk_sums_kernel(const RouteArgs a) {
  wait_for_stream();
  let_next_come();
  const int e = (int)(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)), lane = threadIdx.x & 31;
  if (e >= a.c.experts) return;
  int4* h = reinterpret_cast<int4*>(a.hist + (long long)e * a.stride);
  int run = 0;
  for (int c0 = 0; c0 < a.chunks; c0 += 256) {
    const int c = c0 + lane * 8;
    int n[8];
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const int4 v = c + i < a.stride ? h[(c + i) / 4] : make_int4(0, 0, 0, 0);
      n[i] = v.x; n[i + 1] = v.y; n[i + 2] = v.z; n[i + 3] = v.w;
    }
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { const int v = c + i < a.chunks ? n[i] : 0; n[i] = mine; mine += v; }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(kAll, inc, o); if (lane >= o) inc += v; }
    const int before = run + inc - mine;
#pragma unroll
    for (int i = 0; i < 8; i += 4)
      if (c + i < a.stride) h[(c + i) / 4] = make_int4(before + n[i], before + n[i + 1], before + n[i + 2], before + n[i + 3]);
    run += __shfl_sync(kAll, inc, 31);
  }
  if (lane == 0) a.totals[e] = run;
}

// ranks inside a chunk -> grouped rows, and the way back; more blocks than chunks where there is much to fill
__global__ void __launch_bounds__(kThreads) place_kernel(const RouteArgs a) {
  wait_for_stream();
  __shared__ int first_row[ASGD_MAX_EXPERTS], count[ASGD_MAX_EXPERTS], warp_part[32];
  const int E = a.c.experts, K = a.c.top_k;
  for (int e = threadIdx.x; e < E; e += blockDim.x) first_row[e] = count[e] = a.totals[e];
  __syncthreads();
  const int total = scan_padded(first_row, E, a.c.align, warp_part);
  if (blockIdx.x == 0) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) a.offsets[e] = first_row[e];
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
  if (blockIdx.x < a.chunks) {
    const long long from = (long long)blockIdx.x * a.chunk * K, to = min(from + (long long)a.chunk * K, a.T * K);
    for (long long at = from + threadIdx.x; at < to; at += blockDim.x) {
      const int id = a.ids[at];
      if (id < 0) continue;
      const int r = a.rows[at] + first_row[id] + a.hist[(long long)id * a.stride + blockIdx.x];
      a.rows[at] = r;
      a.source[r] = (int)at;
    }
  }
  fill_nothing(a, first_row, count, total, (int)blockIdx.x, (int)gridDim.x);
}

// nothing to route: an empty plan
__global__ void empty_plan_kernel(const RouteArgs a) {
  wait_for_stream();
  for (int e = threadIdx.x; e <= a.c.experts; e += blockDim.x) a.offsets[e] = 0;
  for (long long r = threadIdx.x; r < a.source_len; r += blockDim.x) a.source[r] = -1;
}

struct GradArgs {
  asgd_route_config c;
  long long T, ld, ld_out;
  const void* logits;
  const int* ids;
  const float* dweights;
  void* dlogits;
};

template <int S, int L, typename T> __global__ void __launch_bounds__(kThreads) route_grad_kernel(const GradArgs a) {
  wait_for_stream();
  const int K = a.c.top_k, lane = threadIdx.x % L;
  const bool sigmoid_scores = a.c.score == ASGD_SCORE_SIGMOID;
  const long long t = (long long)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const int E = t < a.T ? a.c.experts : 0;                             // lanes beyond the tokens go along with nothing
  const T* row = reinterpret_cast<const T*>(a.logits) + t * a.ld;
  T* out = reinterpret_cast<T*>(a.dlogits) + t * a.ld_out;
  // lane j: the j-th choice
  int id = -1;
  float dw = 0.f, chosen = 0.f;
  if (lane < K && t < a.T) { id = a.ids[t * K + lane]; dw = a.dweights[t * K + lane]; }
  const bool ok = id >= 0 && id < E;
  float x[S];
  load_row<S, L, T>(row, E, lane, x);
  if (ok) chosen = Elem<T>::to_f(row[id]);
  Softmax f{0.f, 1.f};
  if (!sigmoid_scores) f = softmax<S, L>(x);
  const float s = !ok ? 0.f : sigmoid_scores ? sigmoid(chosen) : f.score(chosen);
  float ds = 0.f;
  if (a.c.renormalise) {
    const float total = choice_sum<L>(s, K) + 1e-20f, dot = choice_sum<L>(ok ? dw * s : 0.f, K);
    if (ok) ds = a.c.scale * (dw - dot / total) / total;
  } else if (ok) {
    ds = a.c.scale * dw;
  }
  // every expert's gradient as of one that was not chosen, then the chosen ones' over it
  const float dot = sigmoid_scores ? 0.f : choice_sum<L>(ds * s, K), per = dot / f.sum;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * L + lane;
    if (e < E) out[e] = Elem<T>::from_f(sigmoid_scores ? 0.f : -f.part(x[j]) * per);
  }
  __syncwarp();
  // 1 - s as a sigmoid of its own: the difference loses all of it from logits of 17 on
  if (ok) out[id] = Elem<T>::from_f(sigmoid_scores ? ds * s * sigmoid(-chosen) : s * (ds - dot));
}

// Calls f with the numbers a lane holds and the lanes of a token, as compile-time numbers: 8 lanes where they have room
// for the choices and the groups and hold eight numbers at most, for most of the instructions are the same whatever the
// lanes hold (gradient of 32768 x 64 logits: 13 us with 32 lanes a token, 9.6 with 8).
template <int N> using Int = std::integral_constant<int, N>;
template <typename F> void with_shape(const asgd_route_config& c, F&& f) {
  const int E = c.experts, need = std::max(c.top_k, c.groups_kept < c.groups ? c.groups : 1);
  if (E <= 64 && need <= 8) {
    if (E <= 16) f(Int<2>(), Int<8>());
    else if (E <= 32) f(Int<4>(), Int<8>());
    else f(Int<8>(), Int<8>());
  } else if (E <= 64) f(Int<2>(), Int<32>());
  else if (E <= 128) f(Int<4>(), Int<32>());
  else if (E <= 256) f(Int<8>(), Int<32>());
  else if (E <= 512) f(Int<16>(), Int<32>());
  else f(Int<32>(), Int<32>());
}

bool config_ok(const asgd_route_config* c) {
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
bool config_supported(const asgd_route_config* c) {
  return c->experts <= ASGD_MAX_EXPERTS && c->groups <= ASGD_MAX_EXPERT_GROUPS && c->top_k <= ASGD_MAX_TOP_K;
}
// Tokens of a chunk: one block where it does all (few tokens, little to fill).  Else the number with the shortest way
// through: the waves of blocks (an SM holds four, of the widest instances two), by a block's turns of its eight warps and
// some one and a half more for its beginning and end; of equal ones the smallest, so that short batches spread over the GPU.
// (41270 tokens among 256 experts in groups: 74 us in chunks of 40, 90 in chunks of 64, which leave a half-empty wave.)
int chunk_of(const asgd_route_config* c, long long T) {
  if (T <= kMaxChunk && (long long)c->experts * (c->align - 1) <= 4096) return kMaxChunk;
  int at_once = 0;
  long long blocks = 0, least = 0;
  with_shape(*c, [&](auto s, auto l) {
    at_once = kWarps * (32 / decltype(l)::value);
    blocks = kSMs * (decltype(s)::value <= 8 ? 4 : 2);
  });
  int best = 0;
  for (int n = kWarps; n <= kMaxChunk; n += n < at_once ? n : at_once) {
    const long long cost = ceil_div(ceil_div(T, n), blocks) * (2 * ceil_div(n, at_once) + 3);
    if (!best || cost < least) { best = n; least = cost; }
  }
  return best;
}
bool one_block(const asgd_route_config* c, long long T) { return chunk_of(c, T) == kMaxChunk && T <= kMaxChunk; }
// (a plan that takes more than one block has two chunks at least, the second one empty if need be)
int chunks_of(const asgd_route_config* c, long long T) { return one_block(c, T) ? 1 : (int)std::max(2ll, ceil_div(T, chunk_of(c, T))); }
size_t workspace_bytes(const asgd_route_config* c, long long T) {
  return one_block(c, T) ? 0 : ((size_t)ceil_div(chunks_of(c, T), 4) * 4 + 1) * (size_t)c->experts * sizeof(int);
}

}  // namespace

extern "C" int asgd_route_workspace_bytes(const asgd_route_config* cfg, int64_t T, size_t* bytes) {
  if (!config_ok(cfg) || T < 0 || !bytes) return ASGD_EINVAL;
  if (!config_supported(cfg)) return ASGD_EUNSUPPORTED;
  *bytes = workspace_bytes(cfg, T);
  return ASGD_OK;
}

extern "C" int asgd_route(const asgd_route_config* cfg, int64_t T, const void* logits, int32_t type, int64_t ld, const float* bias,
                          int32_t* ids, float* weights, int32_t* offsets, int32_t* rows, int32_t* source, int64_t source_len,
                          void* workspace, size_t ws_bytes, void* stream) {
  if (!config_ok(cfg) || T < 0 || !float_type(type) || ld < cfg->experts) return ASGD_EINVAL;
  if (!config_supported(cfg)) return ASGD_EUNSUPPORTED;
  if (T > 0 && (!logits || !ids || !weights || !aligned(logits, type_bytes(type)))) return ASGD_EINVAL;
  if (!aligned_words(bias, ids, weights, offsets, rows, source)) return ASGD_EINVAL;
  const bool plan = offsets || rows || source;
  const long long need = (long long)T * cfg->top_k + (long long)cfg->experts * (cfg->align - 1);
  if (plan) {
    if (!offsets || (T > 0 && !rows) || (need > 0 && !source) || source_len < need) return ASGD_EINVAL;
    if (source_len > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  }
  if (T > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  const size_t want = plan ? workspace_bytes(cfg, T) : 0;
  if (want && (!workspace || ws_bytes < want)) return ASGD_ENOMEM;
  if (want && !aligned(workspace, 256)) return ASGD_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  RouteArgs a;
  a.c = *cfg;
  a.T = T; a.ld = ld; a.source_len = source_len;
  a.chunk = chunk_of(cfg, T);
  a.chunks = chunks_of(cfg, T);
  a.group_lanes = 0;
  while ((cfg->groups << (a.group_lanes + 1)) <= 32) ++a.group_lanes;
  const unsigned per = (unsigned)(cfg->experts / cfg->groups);
  a.group_magic = per > 1 ? (unsigned)((1ull << 32) / per + 1) : 0;    // exact for numbers below 2^16
  a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights;
  a.offsets = plan ? offsets : nullptr; a.rows = rows; a.source = source;
  a.hist = (int*)workspace;
  a.stride = (int)ceil_div(a.chunks, 4) * 4;
  a.totals = a.hist + (want ? (size_t)a.stride * cfg->experts : 0);
  if (T == 0) return !plan || launch_after(empty_plan_kernel, dim3(1), kThreads, 0, st, a) ? ASGD_OK : ASGD_ECUDA;
  const bool one = one_block(cfg, T);
  bool ok = false;
  with_shape(*cfg, [&](auto s, auto l) {
    with_type(type, [&](auto e) {
      // the widest instances need more registers than 1024 threads have
      const int threads = !one ? kThreads : decltype(s)::value > 8 ? 512 : kThreadsOne;
      ok = launch_after(route_kernel<decltype(s)::value, decltype(l)::value, decltype(e)>, dim3((unsigned)a.chunks), threads, 0, st, a);
    });
  });
  if (plan && !one) {
    ok = ok && launch_after(chunk_sums_kernel, dim3((unsigned)ceil_div(cfg->experts, 4)), 128, 0, st, a) &&
         launch_after(place_kernel, dim3((unsigned)std::max(a.chunks, cfg->align > 1 ? kFillBlocks : 1)), kThreads, 0, st, a);
  }
  return ok ? ASGD_OK : ASGD_ECUDA;
}

extern "C" int asgd_route_grad(const asgd_route_config* cfg, int64_t T, const void* logits, int32_t type, int64_t ld, const int32_t* ids,
                               const float* dweights, void* dlogits, int64_t ld_out, void* stream) {
  if (!config_ok(cfg) || T < 0 || !float_type(type) || ld < cfg->experts || ld_out < cfg->experts) return ASGD_EINVAL;
  if (!config_supported(cfg) || T > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  if (T == 0) return ASGD_OK;
  if (!logits || !ids || !dweights || !dlogits || !aligned(logits, type_bytes(type)) || !aligned(dlogits, type_bytes(type)) || !aligned_words(ids, dweights)) return ASGD_EINVAL;
  GradArgs a{*cfg, T, ld, ld_out, logits, ids, dweights, dlogits};
  asgd_route_config shape = *cfg;
  shape.groups = shape.groups_kept = 1;                                // groups have no part in the gradient
  bool ok = false;
  with_shape(shape, [&](auto s, auto l) {
    with_type(type, [&](auto e) {
      constexpr int L = decltype(l)::value;
      ok = launch_after(route_grad_kernel<decltype(s)::value, L, decltype(e)>, dim3((unsigned)ceil_div(T, kThreads / L)), kThreads, 0, (cudaStream_t)stream, a);
    });
  });
  return ok ? ASGD_OK : ASGD_ECUDA;
}
