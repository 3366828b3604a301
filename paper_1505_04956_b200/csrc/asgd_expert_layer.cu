// A whole layer of experts for a few tokens in one kernel.  The contract is in include/asgd_expert_layer.h.
//
// The bytes of the weights of the experts in use are the bound, so the design keeps them coming.  One block per SM, all at
// once.  The K blocks (128 columns of W by 128 rows) of all tiles of W1 that any token needs count as one run, and each block
// takes an equal stretch of it, wherever tiles begin and end; the same again with W2.  A block's copies of weights run ahead through
// a ring of slots, W2's behind W1's, whatever the tokens' side is waiting for: while blocks meet between the two
// products, some 150 KB of weights per SM are in flight or there already.
//
// The steps:
//   0  logits (with a router) and the tokens in 8 bits, by all warps of all blocks.   -- blocks meet
//   1  every block chooses the experts of all tokens for itself (more than 30 tokens are shared out, and the blocks meet once more), and lists
//      the rows by expert.  Then its stretch of W1: sums of partial tiles go to the workspace.  -- blocks meet
//   2  sums of a tile's stretches in the blocks' order, activation, 8 bits.   -- blocks meet (the copies of W2 went on)
//   3  its stretch of W2, sums to the workspace.   -- blocks meet
//   4  sums of the stretches and of a token's experts in their order, y.
// No sum depends on timing: every order is fixed by the sizes and the loads.
//
// A tile is 128 rows of W (the MMA's M) by BN tokens of one expert (its N; an expert with more has several chunks); a
// K block's products leave tensor memory and are added, scaled, in registers, as in asgd_product_few.cuh.
//
// What bounds it: one token of 128 experts (d 2048, h 768 gated, top 8) takes 29 us, of which its 39 MB need 6; the rest is a chain of
// steps that wait for one another (choice and plan 6, the meetings 5, activation 2, first bytes and last sums of either product 5, the launch 3).
// Eight tokens of 256 experts take 44 to 47 us, by the drawn choices (181 MB, 28 of them), 60 tokens 55 (186 MB): the weights come at 5 to 7 TB/s once they are on their
// way.  On the way there, 8 tokens: one warp that brings the tokens' rows 48, four 44.5; scales asked for before W1's copies are on their way
// 53; the sums of a token's eight choices one after another 6 of them, together 2.
//
// Warp roles after step 0: 0 issues the copies of weights; 1 and 3 issue the products, K blocks in turn; 2 and 12 to 14 bring the
// tokens' rows (gathered, 16-byte asynchronous copies into the swizzled layout that a tensor map would write) and the scales, K blocks in
// turn; 4 to 11 read the accumulators, and do steps 2 and 4.  Every wait is bounded, those of blocks for one another too.
#include <algorithm>

#include "../../include/asgd_expert_layer.h"
#include "asgd_choose.cuh"
#include "asgd_maps.cuh"
#include "asgd_product_few.cuh"

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kReaders = 8, kLoaders = 4;
constexpr int kMostRows = ASGD_LAYER_MAX_ASSIGNMENTS;
constexpr int kDry = kWarps - 1;                     // the warp that goes ahead, see the kernel
constexpr int kChoices = 2 * kDry;                   // tokens that every block chooses for itself; with more the blocks share them out and meet
constexpr int kTokenWords = ASGD_LAYER_MAX_TOKENS / 32;
enum { MEET_TOKENS, MEET_CHOICE, MEET_SUMS, MEET_HIDDEN, MEET_OUT, MEETINGS };

// What the blocks of a launch share, at the workspace's start; zeros before it.
struct Shared {
  struct { unsigned count, pad[31]; } meeting[MEETINGS];
  unsigned gave_up, pad[31];
};

struct Matrix {                                      // W1 or W2
  int tiles, kblocks;                                // of 128 rows, of 128 columns
  const float* scale;
  long long row, block, group;
  unsigned idesc;
};

struct LayerArgs : Choice {
  int T, d, h, rows1, gated, silu;
  const void* x;
  long long ldx;
  int type, x_wide;                                  // rows of x start at four numbers' alignment
  void* y;
  long long ldy;
  const void* logits;
  long long ld_logits;
  int logits_type;
  const void* router;
  long long ld_router;
  int router_type, router_wide;
  const float* shift;
  float temperature;
  Matrix w[2];
  int* ids;
  float* weights;
  // workspace
  Shared* shared;
  float* made_logits;                                // [T][E]
  int* made_ids;                                     // [T][top_k], where the blocks share the choices of many tokens
  float* made_weights;
  unsigned char* xq;                                 // [T][w[0].kblocks * 128]
  float* xs;                                         // [w[0].kblocks][T]: a K block's are neighbours
  unsigned char* hq;                                 // [rows][w[1].kblocks * 128]
  float* hs;                                         // [w[1].kblocks][T * top_k]
  float* sums;                                       // [rows of all tiles + BN per block][128]
  unsigned wait_limit;
  int withhold;
  int* status;
};

template <int BN> struct Layer {
  static constexpr int kSlots = BN == 64 ? 8 : 10;   // even: a slot always meets the same issuing thread
  static constexpr unsigned kWeights = kU * kKB, kTokens = BN * kKB, kSlotBytes = kWeights + kTokens;
  static constexpr int kScales = BN + 4;             // of a slot: the tokens', then the weights' one
  static constexpr int kRows = BN / 2;               // tokens of a tile that a reading thread has
  static constexpr unsigned kCols = kAccStages * BN;
  enum { FULL = 0, READY = kSlots, DONE = 2 * kSlots, SEMPTY = 3 * kSlots, ACCEMPTY = 4 * kSlots, DRAIN = ACCEMPTY + kAccStages, COUNT = DRAIN + 2 };
  static constexpr size_t kRing = (size_t)kSlots * kSlotBytes;
  static constexpr size_t kSmem = 1024 + kRing + (size_t)kSlots * kScales * 4 + COUNT * 8;
  static_assert(kSlots > kLoaders, "a loading warp meets every phase of what it waits for");
  static_assert(kSlots % 2 == 0 && kCols >= 32, "slots, tensor memory");
};

// The rows (assignments) in the experts' order.
struct Plan {
  short ids[kMostRows];                              // of an assignment
  float weights[kMostRows];
  short order[kMostRows];                            // the assignment of a row
  short row_of[kMostRows];                           // the row of an assignment, -1: none
  short chunk_of[kMostRows];                         // of a row
  short expert[kMostRows], first[kMostRows], rows[kMostRows];      // of a chunk
  int part[2][kWarps];
  int chunks, total_rows;
  unsigned per[2];                                   // K blocks of a block, of W1 and W2
};
// While the plan is made, where the ring will be.
struct Making {
  unsigned key[kWarps][ASGD_MAX_EXPERTS];            // of the choices
  float x[kWarps][ASGD_MAX_EXPERTS];
  unsigned mask[ASGD_MAX_EXPERTS][kTokenWords];      // the tokens of an expert
  int start[ASGD_MAX_EXPERTS], chunk[ASGD_MAX_EXPERTS];
  float bias[ASGD_MAX_EXPERTS];
  uint2 found[kWarps][32];                           // keys that reach a bound, and whose they are
  int place[kWarps][32];
};
constexpr size_t kMost = 227 * 1024 - sizeof(Plan) - 64;
static_assert(Layer<16>::kSmem <= kMost && Layer<32>::kSmem <= kMost && Layer<64>::kSmem <= kMost, "shared memory");
static_assert(sizeof(Making) <= Layer<16>::kRing, "the plan is made where the ring will be");

// ---- blocks that wait for one another ----

__device__ __forceinline__ void come(unsigned* count) { asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(count) : "memory"); }
__device__ __forceinline__ unsigned look(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// by one thread: all blocks have come
__device__ inline bool meet(Shared* sh, int which, unsigned limit, int* abort) {
  limit = max(limit, 1u << 10);                      // a drill that gives copies up after a few polls still lets blocks meet
  for (unsigned it = 0; it < limit; ++it) {
    if (look(&sh->meeting[which].count) >= gridDim.x) return true;
    if ((it & 15u) == 15u && (*reinterpret_cast<volatile int*>(abort) || look(&sh->gave_up))) break;
  }
  *reinterpret_cast<volatile int*>(abort) = 1;
  return false;
}

// A copy of weights, which are read once a step: the first to leave L2, so that they do not drive out what every step reads again
// (router, scales, and the kernel's own instructions, each of whose lines is otherwise fetched anew from HBM).
__device__ inline unsigned long long leaves_first() {
  unsigned long long p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ inline void load_weights(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar, unsigned long long policy) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
               ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)), "l"(policy) : "memory");
}

// ---- tokens ----

template <typename T> __device__ __forceinline__ float4 four(const T* at) {             // aligned
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float4*>(at);
  else {
    const uint2 u = *reinterpret_cast<const uint2*>(at);
    const T* e = reinterpret_cast<const T*>(&u);
    return make_float4(Elem<T>::to_f(e[0]), Elem<T>::to_f(e[1]), Elem<T>::to_f(e[2]), Elem<T>::to_f(e[3]));
  }
}
// four numbers from number `at` of a row on, zeros from `end` on
template <typename T> __device__ __forceinline__ float4 four(const T* row, int at, int end, bool wide) {
  if (wide && at + 4 <= end) return four(row + at);
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = at + i < end ? Elem<T>::to_f(row[at + i]) : 0.f;
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ float4 four(const void* base, int type, long long row, int at, int end, bool wide) {
  if (type == ASGD_F32) return four(reinterpret_cast<const float*>(base) + row, at, end, wide);
  if (type == ASGD_BF16) return four(reinterpret_cast<const __nv_bfloat16*>(base) + row, at, end, wide);
  return four(reinterpret_cast<const __half*>(base) + row, at, end, wide);
}

// A warp rounds a block of 128 numbers, four per lane, as asgd_quantize does (E4M3).
__device__ __forceinline__ void round_block(const float4& v, unsigned char* q, float* scale, int lane) {
  float m = fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w)));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
  m = fmaxf(m, 7.888609052210118e-31f);              // 2^-100
  const float inv = __fdiv_rn(448.f, m);
  const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(v.x * inv, v.y * inv), __NV_SATFINITE, __NV_E4M3);
  const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(v.z * inv, v.w * inv), __NV_SATFINITE, __NV_E4M3);
  reinterpret_cast<unsigned*>(q)[lane] = lo | hi << 16;
  if (lane == 0) *scale = __fmul_rn(m, 1.f / 448.f);
}

// Logits of a router: four warps share a row of it and kTok tokens; a block has three such groups.  (The types are the
// template's, so that a step's loads are all in flight at once: with a switch around each, 60 tokens took 16 us.)
constexpr int kLogitTokens = 8, kLogitWarps = 4, kLogitGroups = kDry / kLogitWarps;
template <typename X, typename R, int kTok> __device__ __forceinline__ void logit_sums(const LayerArgs& a, int e, int t0, int n, int first, float (&acc)[kLogitTokens]) {
  const R* r = reinterpret_cast<const R*>(a.router) + e * a.ld_router;
  const X* x[kTok];
#pragma unroll
  for (int t = 0; t < kTok; ++t) x[t] = reinterpret_cast<const X*>(a.x) + (t0 + min(t, n - 1)) * a.ldx;      // (places behind the last token repeat it)
  const bool wide = a.router_wide && a.x_wide;
  const int whole = wide ? a.d / 4 * 4 : 0;          // numbers read four at a time
#pragma unroll(kTok == 1 ? 4 : 2)
  for (int k = first; k < whole; k += kLogitWarps * 128) {
    const float4 m = four(r + k);
    float4 v[kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t) v[t] = four(x[t] + k);
#pragma unroll
    for (int t = 0; t < kTok; ++t) acc[t] = fmaf(v[t].x, m.x, fmaf(v[t].y, m.y, fmaf(v[t].z, m.z, fmaf(v[t].w, m.w, acc[t]))));
  }
#pragma unroll 1
  for (int k = whole + first / 4; k < a.d; k += kLogitWarps * 32) {
    const float m = Elem<R>::to_f(r[k]);
#pragma unroll
    for (int t = 0; t < kTok; ++t) acc[t] = fmaf(Elem<X>::to_f(x[t][k]), m, acc[t]);
  }
}
__device__ __forceinline__ void others_sync() { asm volatile("bar.sync 2, %0;" ::"n"(kDry * 32) : "memory"); }      // all warps but the one that goes ahead
template <int kTok> __device__ inline void make_logits(const LayerArgs& a, float (*part)[kLogitWarps][kLogitTokens], int lane, int wid) {
  const int E = a.c.experts, sets = (a.T + kTok - 1) / kTok, units = E * sets, group = wid / kLogitWarps, sub = wid % kLogitWarps;
  const int per = kLogitGroups * (int)gridDim.x, first = (sub * 32 + lane) * 4;
  for (int u0 = (int)blockIdx.x * kLogitGroups; u0 < units; u0 += per) {
    const int u = u0 + group, e = u / sets, t0 = u % sets * kTok, n = u < units && group < kLogitGroups ? min(kTok, a.T - t0) : 0;
    float acc[kLogitTokens];
#pragma unroll
    for (int t = 0; t < kLogitTokens; ++t) acc[t] = 0.f;
    if (n > 0) {
      auto of = [&](auto x) {
        using X = decltype(x);
        if (a.router_type == ASGD_F32) logit_sums<X, float, kTok>(a, e, t0, n, first, acc);
        else if (a.router_type == ASGD_BF16) logit_sums<X, __nv_bfloat16, kTok>(a, e, t0, n, first, acc);
        else logit_sums<X, __half, kTok>(a, e, t0, n, first, acc);
      };
      if (a.type == ASGD_F32) of(float());
      else if (a.type == ASGD_BF16) of(__nv_bfloat16());
      else of(__half());
    }
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[t] += __shfl_xor_sync(kAll, acc[t], o);
      if (lane == 0 && group < kLogitGroups) part[group][sub][t] = acc[t];
    }
    others_sync();
    if (sub == 0 && lane < n) {
      float s = part[group][0][lane];
#pragma unroll
      for (int w = 1; w < kLogitWarps; ++w) s += part[group][w][lane];
      a.made_logits[(long long)(t0 + lane) * E + e] = (s - (a.shift ? a.shift[e] : 0.f)) * a.temperature;
    }
    others_sync();
  }
}

// ---- the choice and the plan, by the whole block ----

// A warp chooses for one token from logits and keys in shared memory: lane l has the experts l, l + 32, ...  A kernel
// that runs once for a few tokens meets its instructions cold, so this code is short: loops over what a lane has, where asgd_route's is unrolled
// over registers (which took 10 us for a first token among 256 experts in groups, and 2 for every further one).  Choices and weights are asgd_route's to
// the last bit: every sum runs in its order (choose() in asgd_choose.cuh), the softmax's over the same number of lanes, the renormalising one over choices
// in the same places.  A lane returns a place among the top_k (-1: it has none), the expert there (-1: none) and its weight.
template <typename T> __device__ __forceinline__ void read_logits(const T* row, int E, int lane, float* x) {
#pragma unroll 4
  for (int e = lane; e < E; e += 32) x[e] = Elem<T>::to_f(__ldcg(row + e));
}
__device__ inline void choose_one(const LayerArgs& a, int t, const float* bias, float* x, unsigned* key, uint2* found, int* place, int lane, bool dry, int& at, int& id, float& weight) {
  const asgd_route_config& c = a.c;
  const int E = c.experts, K = c.top_k;
  const bool by_logit = a.bias == nullptr && c.group_top == 1, sigmoid_scores = c.score == ASGD_SCORE_SIGMOID;
  __syncwarp();
  if (dry)
    for (int e = lane; e < E; e += 32) x[e] = (float)e;
  else if (a.made_logits) read_logits(a.made_logits + (long long)t * E, E, lane, x);
  else if (a.logits_type == ASGD_F32) read_logits(reinterpret_cast<const float*>(a.logits) + t * a.ld_logits, E, lane, x);
  else if (a.logits_type == ASGD_BF16) read_logits(reinterpret_cast<const __nv_bfloat16*>(a.logits) + t * a.ld_logits, E, lane, x);
  else read_logits(reinterpret_cast<const __half*>(a.logits) + t * a.ld_logits, E, lane, x);
  Softmax f{0.f, 1.f};
  if (!sigmoid_scores) {
    float m = -INFINITY, sum = 0.f;
    for (int e = lane; e < E; e += 32) m = e == lane ? x[e] : fmaxf(m, x[e]);
    f.m = lanes_max<32>(m);
    __syncwarp();
#pragma unroll 1                                        // (short: instructions come cold; unrolled by four 1 token took 0.3 us more)
    for (int e = lane < a.lanes ? lane : E; e < E; e += a.lanes) sum += f.part(x[e]);
    f.sum = lanes_sum<32>(sum);                      // (lanes from a.lanes on add zeros)
  }
  unsigned best = 0;                                 // the lane's largest key, and whose it is
  int whose = -1;
#pragma unroll 4
  for (int e = lane; e < E; e += 32) {
    float v = x[e];
    const bool there = v > -INFINITY;
    if (!by_logit) {
      v = sigmoid_scores ? sigmoid(v) : f.score(v);
      if (a.bias) v = __fadd_rn(v, bias[e]);
    }
    const unsigned k = there && v > -INFINITY ? ordered(v) : 0u;
    key[e] = k;
    if (k > best) { best = k; whose = e; }
  }
  __syncwarp();
  if (c.groups_kept < c.groups) {                    // see keep_groups
    const int per = E / c.groups, shift = a.group_lanes, g = lane >> shift, sub = lane & ((1 << shift) - 1);
    unsigned m1 = 0, m2 = 0;
    if (g < c.groups)
#pragma unroll 4
      for (int i = sub; i < per; i += 1 << shift) {
        const unsigned k = key[g * per + i];
        m2 = max(m2, min(m1, k));
        m1 = max(m1, k);
      }
    for (int o = 1; o < 1 << shift; o <<= 1) {       // the two largest of two lanes' two largest
      const unsigned o1 = __shfl_xor_sync(kAll, m1, o), o2 = __shfl_xor_sync(kAll, m2, o);
      m2 = max(min(m1, o1), max(m2, o2));
      m1 = max(m1, o1);
    }
    if (c.group_top == 2 && m2) m1 = ordered(__fadd_rn(from_ordered(m1), from_ordered(m2)));
    const unsigned got = __shfl_sync(kAll, m1, (lane << shift) & 31);
    unsigned mine = lane < c.groups ? got : 0u, kept = 0;
    for (int i = 0; i < c.groups_kept; ++i) {
      const unsigned top = __reduce_max_sync(kAll, mine);
      const unsigned holders = __ballot_sync(kAll, top && mine == top), first = holders & (0u - holders);      // the lowest of them, if any
      kept |= first;
      if ((first >> lane) & 1u) mine = 0;
    }
    best = 0;
    whose = -1;
#pragma unroll 4
    for (int e = lane; e < E; e += 32) {
      const int of = a.group_magic ? (int)__umulhi((unsigned)e, a.group_magic) : e;
      const unsigned k = (kept >> of) & 1u ? key[e] : 0u;
      key[e] = k;
      if (k > best) { best = k; whose = e; }
    }
  }
  // What reaches the top_k-th largest of the lanes' largest keys (top_k keys at least) is gathered and ranked by counting.
  id = -1;
  at = lane < K ? lane : -1;
  unsigned top = best, bound = 1u;
  for (int i = 0; i < K; ++i) {
    const unsigned b = __reduce_max_sync(kAll, top);
    bound = max(b, 1u);
    if (!b) break;                                   // fewer lanes than that have a key: all of them
    top = top == b ? 0u : top;
  }
  int n = 0;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const unsigned k = e0 + lane < E ? key[e0 + lane] : 0u;
    const bool there = k >= bound;
    const unsigned votes = __ballot_sync(kAll, there);
    const int to = n + __popc(votes & ((1u << lane) - 1u));
    if (there && to < 32) found[to] = make_uint2(k, (unsigned)(e0 + lane));
    n += __popc(votes);
  }
  if (n <= 32) {
    __syncwarp();
    const uint2 mine = lane < n ? found[lane] : make_uint2(0u, 0u);
    int rank = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {                    // keys above, and equal ones of lower experts
      const unsigned k = __shfl_sync(kAll, mine.x, i);
      rank += i < lane ? k >= mine.x : k > mine.x;
    }
    if (a.lanes == 32 && E <= 256) {                 // asgd_route leaves choices where they were found
      if (lane < n) at = rank < K ? rank : -1;
      if (lane < n && rank < K) id = (int)mine.y;
    } else {
      if (lane < n && rank < K) place[rank] = (int)mine.y;
      __syncwarp();
      if (lane < min(n, K)) id = place[lane];
    }
  } else {                                           // one by one
    for (int i = 0; i < K; ++i) {
      const unsigned most = __reduce_max_sync(kAll, best);
      if (!most) break;                              // nothing is left
      const int first = (int)__reduce_min_sync(kAll, best == most ? (unsigned)whose : 0x7fffffffu);      // of equal keys the lowest expert's
      if (lane == i) id = first;
      if (whose == first) {
        key[first] = 0u;
        best = 0;
        whose = -1;
        for (int e = lane; e < E; e += 32) {
          const unsigned k = key[e];
          if (k > best) { best = k; whose = e; }
        }
      }
    }
  }
  const float chosen = id >= 0 ? x[id] : 0.f, s = id < 0 ? 0.f : sigmoid_scores ? sigmoid(chosen) : f.score(chosen);
  weight = 0.f;
  if (c.renormalise) {
    const float sum = lanes_sum<32>(s);
    if (id >= 0) weight = c.scale * s / (sum + 1e-20f);
  } else if (id >= 0) {
    weight = c.scale * s;
  }
}
// The choices of tokens first, first + step, ..., of a warp: to the workspace where the blocks share them out, or to the plan, with the
// tokens of each expert marked.  dry: as if for a token, without a result.
__device__ __forceinline__ void choose_some(const LayerArgs& a, int first, int step, Plan& plan, Making& m, int lane, int wid, bool share, bool dry) {
  const int K = a.c.top_k, end = dry ? 1 : a.T;
#pragma unroll 1
  for (int t = first; t < end; t += step) {
    int at, id;
    float w;
    choose_one(a, t, dry ? m.x[wid] : m.bias, m.x[wid], m.key[wid], m.found[wid], m.place[wid], lane, dry, at, id, w);
    if (at < 0 || dry) continue;
    if (share) {
      a.made_ids[t * K + at] = id;
      a.made_weights[t * K + at] = w;
    } else {
      plan.ids[t * K + at] = (short)id;
      plan.weights[t * K + at] = w;
      if (id >= 0) atomicOr(&m.mask[id][t >> 5], 1u << (t & 31));
    }
  }
}
// Rows by expert of 32 assignments at most, by a warp: lane i has assignment i; a row is the number of lanes before it by expert and place.
// (Two assignments a lane took longer than the whole block's way: 64 of them 3.5 us instead of 2.4.)
template <int BN> __device__ inline void make_small_plan(Plan& plan, int n, int lane) {
  const int e = lane < n ? plan.ids[lane] : -1;
  int row = 0, rank = 0;
  for (int i = 0; i < n; ++i) {
    const int o = __shfl_sync(kAll, e, i);
    const bool same = o == e && i < lane;
    row += (o >= 0 && o < e) || same;
    rank += same;
  }
  const unsigned there = __ballot_sync(kAll, e >= 0);
  // chunks begin where a rank is a multiple of BN; in the rows' order
  unsigned begins = e >= 0 && rank % BN == 0 ? 1u << row : 0u;
  begins = __reduce_or_sync(kAll, begins);
  if (lane < n) plan.row_of[lane] = (short)(e >= 0 ? row : -1);
  if (e >= 0) {
    const int chunk = __popc(begins & (2u << row) - 1u) - 1;
    plan.order[row] = (short)lane;
    plan.chunk_of[row] = (short)chunk;
    if ((begins >> row) & 1u) {
      const unsigned later = begins & ~((2u << row) - 1u);
      plan.expert[chunk] = (short)e;
      plan.first[chunk] = (short)row;
      plan.rows[chunk] = (short)((later ? __ffs(later) - 1 : __popc(there)) - row);
    }
  }
  if (lane == 0) { plan.total_rows = __popc(there); plan.chunks = __popc(begins); }
}
// Rows by expert from the choices in plan.ids and the marked tokens.  The whole block; dry: a warp, of no tokens.
template <int BN> __device__ inline void make_plan(const LayerArgs& a, Plan& plan, Making& m, int tid, int lane, int wid, bool dry) {
  const int E = a.c.experts, K = a.c.top_k, n = dry ? 0 : a.T * K;
  // rows and chunks before each expert
  constexpr int kPer = (ASGD_MAX_EXPERTS + kThreads - 1) / kThreads;
  int mine = 0, mine_chunks = 0, count[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int e = tid * kPer + q;
    count[q] = 0;
    if (e < E)
#pragma unroll
      for (int w = 0; w < kTokenWords; ++w) count[q] += dry ? 0 : __popc(m.mask[e][w]);
    mine += count[q];
    mine_chunks += (count[q] + BN - 1) / BN;
  }
  int inc = mine, inc_chunks = mine_chunks;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(kAll, inc, o), w = __shfl_up_sync(kAll, inc_chunks, o);
    if (lane >= o) { inc += v; inc_chunks += w; }
  }
  if (lane == 31) { plan.part[0][wid] = inc; plan.part[1][wid] = inc_chunks; }
  if (!dry) __syncthreads();
  int run = inc - mine, chunk = inc_chunks - mine_chunks;
  for (int w = 0; w < wid; ++w) { run += plan.part[0][w]; chunk += plan.part[1][w]; }
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int e = tid * kPer + q;
    if (e < E) { m.start[e] = run; m.chunk[e] = chunk; }
    for (int r = 0; r < count[q]; r += BN, ++chunk) {
      plan.expert[chunk] = (short)e;
      plan.first[chunk] = (short)(run + r);
      plan.rows[chunk] = (short)min(BN, count[q] - r);
    }
    run += count[q];
  }
  if (tid == kThreads - 1) { plan.total_rows = run; plan.chunks = chunk; }
  if (!dry) __syncthreads();
  for (int i = tid; i < n; i += kThreads) {
    const int e = plan.ids[i], t = i / K;
    int r = -1;
    if (e >= 0) {
      int rank = 0;
#pragma unroll
      for (int w = 0; w < kTokenWords; ++w) {
        const int b = t - 32 * w;
        rank += __popc(m.mask[e][w] & (b >= 32 ? kAll : b > 0 ? (1u << b) - 1u : 0u));
      }
      r = m.start[e] + rank;
      plan.order[r] = (short)i;
      plan.chunk_of[r] = (short)(m.chunk[e] + rank / BN);
    }
    plan.row_of[i] = (short)r;
  }
}

// ---- stretches ----

// A block's K blocks of all tiles of a matrix: `per` of them, the last blocks fewer or none.
struct Stretch {
  unsigned from, to;
  int chunk, tile, kb;                               // where it is
  __device__ __forceinline__ Stretch(const Matrix& w, int chunks, unsigned per) {
    const unsigned all = (unsigned)chunks * w.tiles * w.kblocks;
    from = min(all, blockIdx.x * per);
    to = min(all, from + per);
    const unsigned t = from / w.kblocks;
    kb = (int)(from - t * w.kblocks);
    chunk = (int)(t / w.tiles);
    tile = (int)(t - chunk * w.tiles);
  }
  __device__ __forceinline__ bool there() const { return from < to; }
  // K blocks of the tile it is in, and the next tile
  __device__ __forceinline__ int here(const Matrix& w) const { return (int)min((unsigned)(w.kblocks - kb), to - from); }
  __device__ __forceinline__ void next_tile(const Matrix& w) {
    from += here(w);
    kb = 0;
    if (++tile == w.tiles) { tile = 0; ++chunk; }
  }
};
// Sums of a tile's rows: in front of them those of all tiles before it, and BN for every block that ended a stretch before.
template <int BN> __device__ __forceinline__ long long sums_at(const Plan& plan, const Matrix& w, int chunk, int tile, int block) {
  return (long long)plan.first[chunk] * w.tiles + tile * plan.rows[chunk] + block * BN;
}
// Where the numbers of a row are, of one tile: the sums of every block that has a part in it, in order.
template <int BN> struct Parts {
  const float* at;
  int blocks;
  __device__ __forceinline__ Parts(const LayerArgs& a, const Plan& plan, int f, int row, int tile) {
    const Matrix& w = a.w[f];
    const int chunk = plan.chunk_of[row];
    const unsigned x = ((unsigned)chunk * w.tiles + tile) * w.kblocks, per = plan.per[f], lo = x / per;
    blocks = (int)((x + w.kblocks - 1) / per - lo) + 1;
    at = a.sums + (sums_at<BN>(plan, w, chunk, tile, (int)lo) + row - plan.first[chunk]) * 128;
  }
};
// Four neighbouring numbers of several results at once, each the sum of its parts in order; the loads of the results are in flight
// together.  (One after another each took L2's latency for every part: 6 us for a token's eight choices.)
template <int BN, int N> __device__ __forceinline__ void add_up(const float* const (&at)[N], const int (&blocks)[N], float4 (&sum)[N]) {
  int most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (blocks[i]) sum[i] = __ldcg(reinterpret_cast<const float4*>(at[i]));
    most = max(most, blocks[i]);
  }
#pragma unroll 1
  for (int b = 1; b < most; ++b) {
    float4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (b < blocks[i]) v[i] = __ldcg(reinterpret_cast<const float4*>(at[i] + b * (BN * 128)));
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (b < blocks[i]) { sum[i].x += v[i].x; sum[i].y += v[i].y; sum[i].z += v[i].z; sum[i].w += v[i].w; }
  }
}
// Where a lane's four numbers of u are, for four results at once: the blocks of 128 of units u, u + step, ..., or (gated) two units' and what gates
// them (h is a multiple of four).
template <int BN> struct HiddenAt {
  const float* at[4] = {};
  int blocks[4] = {};
  __device__ __forceinline__ HiddenAt() {}
  __device__ __forceinline__ HiddenAt(const LayerArgs& a, const Plan& plan, int u, int step, int units, int hb, int lane) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int unit = u + (a.gated ? r >> 1 : r) * step, j = unit % hb * 128 + lane * 4, first = a.gated && (r & 1) ? a.h : 0;
      if (unit >= units || j >= a.h) continue;
      const Parts<BN> p(a, plan, 0, unit / hb, (first + j) / 128);
      at[r] = p.at + (first + j) % 128;
      blocks[r] = p.blocks;
    }
  }
};
// Lane j: where a token's j-th choice's four numbers of a tile are (for lane 0), and its weight.
template <int BN> struct ChoiceAt {
  unsigned long long at = 0;
  int blocks = 0;
  float weight = 0.f;
  __device__ __forceinline__ ChoiceAt() {}
  __device__ __forceinline__ ChoiceAt(const LayerArgs& a, const Plan& plan, int t, int tile, int lane) {
    if (lane >= a.c.top_k) return;
    const int i = t * a.c.top_k + lane, row = plan.row_of[i];
    if (row < 0) return;
    const Parts<BN> p(a, plan, 1, row, tile);
    at = reinterpret_cast<unsigned long long>(p.at);
    blocks = p.blocks;
    weight = plan.weights[i];
  }
};
// four numbers of u from number j on of row `row`, one by one (h not a multiple of four)
template <int BN> __device__ inline float4 hidden_one_by_one(const LayerArgs& a, const Plan& plan, int row, int j, int end) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = 0.f;
    if (j + i < end) {
      const Parts<BN> p(a, plan, 0, row, (j + i) / 128);
      v[i] = __ldcg(p.at + (j + i) % 128);
      for (int b = 1; b < p.blocks; ++b) v[i] += __ldcg(p.at + b * (BN * 128) + (j + i) % 128);
    }
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ float activated(float u, bool silu) {
  if (silu) return u / (1.f + expf(-u));
  const float r = fmaxf(u, 0.f);
  return u != u ? u : r * r;                         // (the larger of a NaN and 0 would be 0)
}

// Whether a token has an infinity or a NaN, or a NaN among the logits made from it, by a warp.  Such a token gets no expert, and must not look like one
// that was left out on purpose.  (Asked for tokens without an expert alone.  Where y is x in place, tiles of it may be written already: with NaNs, if so.)
__device__ __noinline__ bool not_finite(const LayerArgs& a, int t, int lane) {
  bool bad = false;
  for (int e = lane; e < a.c.experts; e += 32) {
    const float v = __ldcg(a.made_logits + (long long)t * a.c.experts + e);
    bad = bad || v != v;
  }
  for (int k = lane * 4; k < a.d; k += 128) {
    const float4 v = four(a.x, a.type, t * a.ldx, k, a.d, a.x_wide);
    bad = bad || !(fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY && fabsf(v.z) < INFINITY && fabsf(v.w) < INFINITY);
  }
  return __any_sync(kAll, bad);
}

__device__ __forceinline__ void readers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kReaders * 32) : "memory"); }

__device__ __forceinline__ void tmem_load8(unsigned taddr, float* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(taddr) : "memory");
}

template <int BN> __global__ void __launch_bounds__(kThreads, 1)
expert_layer_kernel(const __grid_constant__ LayerArgs a, const __grid_constant__ CUtensorMap map_1, const __grid_constant__ CUtensorMap map_2) {
  using L = Layer<BN>;
  constexpr int S = L::kSlots;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  __shared__ Plan plan;
  __shared__ int misc[4];                            // [0] tensor memory, [1] abort, [2] K blocks whose copies were issued, [3] whether the readers go on
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  float* scales = reinterpret_cast<float*>(ring + L::kRing);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(scales + S * L::kScales);
  int* abort = misc + 1;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;

  if (tid == 0) {
    prefetch_map(&map_1);
    prefetch_map(&map_2);
    for (int q = 0; q < S; ++q) {
      mbar_init(bars + L::FULL + q, 1); mbar_init(bars + L::READY + q, 32); mbar_init(bars + L::DONE + q, 1); mbar_init(bars + L::SEMPTY + q, kReaders);
    }
    for (int q = 0; q < kAccStages; ++q) mbar_init(bars + L::ACCEMPTY + q, kReaders);
    for (int q = 0; q < 2; ++q) mbar_init(bars + L::DRAIN + q, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    misc[1] = misc[2] = 0;
  }
  if (wid == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "r"(L::kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  Making& making = *reinterpret_cast<Making*>(ring);
  const bool share = a.T > kChoices;
  const int assignments = a.T * a.c.top_k;
  // The last warp goes ahead: it walks through the choice and the plan once for nothing, while the others wait for the stream and do step 0, so
  // that their instructions are there when the others come (a line of them that no cache of the SM has costs some 500 cycles; without it
  // the two took 7 us for one token of 128 experts).  It takes part in nothing else until the choices are made.
#pragma unroll 1
  for (int dry = wid == kDry; dry >= 0; --dry) {
    const bool ahead = wid == kDry;                  // (its second time round it only meets the others)
    if (!ahead) {
      wait_for_stream();                             // what comes before reads nothing of the call's but its arguments
      // What is read soon comes now: from cold memory a first read takes 2 to 3 us.
      if (a.bias)
        for (int e = tid; e < a.c.experts; e += kDry * 32) copy4(making.bias + e, a.bias + e, true);
      if (a.logits) {
        const int t = share ? (int)blockIdx.x + wid * (int)gridDim.x : wid, size = a.logits_type == ASGD_F32 ? 4 : 2;
        const char* row = reinterpret_cast<const char*>(a.logits) + t * a.ld_logits * size;
        if (t < a.T)
          for (int at = lane * 128; at < a.c.experts * size; at += 32 * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + at));
      }
      for (int i = tid; i < a.c.experts * kTokenWords; i += kDry * 32) (&making.mask[0][0])[i] = 0;
      // step 0
      for (int u = (int)blockIdx.x * kDry + wid; u < a.T * a.w[0].kblocks; u += (int)gridDim.x * kDry) {
        const int t = u / a.w[0].kblocks, b = u % a.w[0].kblocks;
        round_block(four(a.x, a.type, t * a.ldx, b * 128 + lane * 4, a.d, a.x_wide), a.xq + (long long)u * 128, a.xs + b * a.T + t, lane);
      }
      if (a.router) {
        auto part = reinterpret_cast<float (*)[kLogitWarps][kLogitTokens]>(making.x);
        if (a.T == 1) make_logits<1>(a, part, lane, wid);
        else make_logits<kLogitTokens>(a, part, lane, wid);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      others_sync();
      if (a.router) {
        if (tid == 0) {
          come(&a.shared->meeting[MEET_TOKENS].count);
          meet(a.shared, MEET_TOKENS, a.wait_limit, abort);
        }
        others_sync();
      } else if (!share && tid == 0) {
        come(&a.shared->meeting[MEET_TOKENS].count);
      }
    } else if (!dry) {
      wait_for_stream();
    }
    if (!ahead || dry) choose_some(a, dry ? 0 : share ? (int)blockIdx.x + wid * (int)gridDim.x : wid, share ? (int)gridDim.x * kDry : kDry, plan, making, lane, wid, share, dry);
    if (!dry) {
      __syncthreads();
      if (share) {
        const int which = a.router ? MEET_CHOICE : MEET_TOKENS;
        if (tid == 0) {
          come(&a.shared->meeting[which].count);
          meet(a.shared, which, a.wait_limit, abort);
        }
        __syncthreads();
        for (int i = tid; i < assignments; i += kThreads) {
          // (what a block that gave up did not write could be anything)
          const int id = __ldcg(a.made_ids + i), t = i / a.c.top_k;
          const bool ok = id >= 0 && id < a.c.experts;
          plan.ids[i] = (short)(ok ? id : -1);
          plan.weights[i] = __ldcg(a.made_weights + i);
          if (ok) atomicOr(&making.mask[id][t >> 5], 1u << (t & 31));
        }
        __syncthreads();
      }
      if (blockIdx.x == 0)
        for (int i = tid; i < assignments; i += kThreads) {
          if (a.ids) a.ids[i] = plan.ids[i];
          if (a.weights) a.weights[i] = plan.weights[i];
        }
    }
    if (assignments > 32) make_plan<BN>(a, plan, making, tid, lane, wid, dry);
    else if (wid == (dry ? kDry : 0)) make_small_plan<BN>(plan, dry ? 0 : assignments, lane);
  }
  __syncthreads();
  if (tid < 2) plan.per[tid] = ((unsigned)plan.chunks * a.w[tid].tiles * a.w[tid].kblocks + gridDim.x - 1) / gridDim.x;
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // the ring was the plan's scratch until here
  fence_before();
  __syncthreads();
  fence_after();
  const unsigned tmem = (unsigned)misc[0];
  const int chunks = plan.chunks, rows = plan.total_rows;

  if (wid == 0) {
    if (lane == 0) {
      const unsigned long long policy = leaves_first();
      unsigned it = 0;
      bool ok = !*reinterpret_cast<volatile int*>(abort);
#pragma unroll
      for (int f = 0; f < 2 && ok && chunks; ++f) {
        const Matrix& w = a.w[f];
        for (Stretch s(w, chunks, plan.per[f]); s.there() && ok; s.next_tile(w)) {
          const int expert = plan.expert[s.chunk], end = s.kb + s.here(w);
          for (int kb = s.kb; kb < end; ++kb, ++it) {
            const unsigned q = it % S;
            if (it >= S && !(ok = wait(bars + L::DONE + q, (it / S - 1) & 1, a.wait_limit, abort))) break;
            mbar_expect_tx(bars + L::FULL + q, L::kWeights);
            if (!(a.withhold && it == 0)) load_weights(ring + (size_t)q * L::kSlotBytes, f ? &map_2 : &map_1, kb * kKB, s.tile * kU, expert, bars + L::FULL + q, policy);
          }
        }
      }
      misc[2] = (int)it;
    }
  } else if (wid == 1 || wid == 3) {
    const unsigned me = (unsigned)wid >> 1, at = __shfl_sync(kAll, tmem, 0);
    unsigned it = 0;
    bool ok = true;
#pragma unroll
    for (int f = 0; f < 2 && ok && chunks; ++f) {
      const unsigned idesc = a.w[f].idesc;
      for (Stretch s(a.w[f], chunks, plan.per[f]); s.there(); ++s.from, ++it) {
        if ((it & 1) != me) continue;
        const unsigned q = it % S, stage = it % kAccStages;
        ok = wait(bars + L::FULL + q, (it / S) & 1, a.wait_limit, abort) && wait(bars + L::READY + q, (it / S) & 1, a.wait_limit, abort);
        if (it >= kAccStages) ok = ok && wait(bars + L::ACCEMPTY + stage, (it / kAccStages - 1) & 1, a.wait_limit, abort);
        if (!(ok = __all_sync(kAll, ok))) break;
        fence_after();
        if (elect_one()) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the tokens' rows were written by ordinary copies
          const unsigned long long du = operand_desc(ring + (size_t)q * L::kSlotBytes), dv = operand_desc(ring + (size_t)q * L::kSlotBytes + L::kWeights);
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) mma_f8(at + stage * BN, du + 2 * k4, dv + 2 * k4, idesc, k4 != 0);
          commit(bars + L::DONE + q);
        }
        __syncwarp();
      }
    }
  } else if (wid == 2 || (wid >= 4 + kReaders && wid < 3 + kReaders + kLoaders)) {
    // Four warps, K blocks in turn: one took 700 cycles for a K block of 16 tokens, 1500 for 64, and set the pace.
    const int me = wid == 2 ? 0 : wid - (3 + kReaders);
    unsigned it = 0;                                 // K blocks before the tile
    bool ok = true;
#pragma unroll
    for (int f = 0; f < 2 && ok && chunks; ++f) {
      const Matrix& w = a.w[f];
      bool met = true;
      if (lane == 0 && (f || !(a.router || share))) met = meet(a.shared, f ? MEET_HIDDEN : MEET_TOKENS, a.wait_limit, abort);      // (the block has met for the tokens already, or not)
      if (!(ok = __all_sync(kAll, met))) break;
      __syncwarp();                                  // (a vote orders no memory: what lane 0 has met for is there for all lanes)
      const unsigned char* from = f ? a.hq : a.xq;
      const float* from_scales = f ? a.hs : a.xs;
      const int per_block = f ? a.T * a.c.top_k : a.T;
      constexpr int kCopies = BN * 8 / 32;           // 16-byte pieces of a lane
      for (Stretch s(w, chunks, plan.per[f]); s.there() && ok; s.next_tile(w)) {
        const int first = plan.first[s.chunk], n = plan.rows[s.chunk], here = s.here(w);
        auto row_at = [&](int r) { return f ? first + r : plan.order[first + r] / a.c.top_k; };
        const unsigned char* at[kCopies];            // its rows' first numbers, null: none
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int r = i * 4 + (lane >> 3);
          at[i] = r < n ? from + (long long)row_at(r) * (w.kblocks * 128) + (lane & 7) * 16 : nullptr;
        }
        const float* of_token[BN > 32 ? 2 : 1];
#pragma unroll
        for (int i = 0; i < (BN > 32 ? 2 : 1); ++i) of_token[i] = i * 32 + lane < n ? from_scales + row_at(i * 32 + lane) : nullptr;
        const float* of_weights = w.scale + plan.expert[s.chunk] * w.group + s.tile * w.row;
        for (int i0 = (me - it) & (kLoaders - 1); i0 < here; i0 += kLoaders) {
          const unsigned k = it + i0, q = k % S;
          const int kb = s.kb + i0;
          // (a slot's K block two rounds ago has been read: this warp has waited for a later one, kLoaders < S)
          if (k >= S && !(ok = __all_sync(kAll, wait(bars + L::SEMPTY + q, (k / S - 1) & 1, a.wait_limit, abort)))) break;
          unsigned char* to = ring + (size_t)q * L::kSlotBytes + L::kWeights;
#pragma unroll
          for (int i = 0; i < kCopies; ++i) {
            const int r = i * 4 + (lane >> 3);
            copy16(reinterpret_cast<float*>(to + r * kKB + (((lane & 7) ^ (r & 7)) << 4)), reinterpret_cast<const float*>(at[i] ? at[i] + kb * 128 : from), at[i] ? 16 : 0);
          }
          float* sc = scales + q * L::kScales;
#pragma unroll
          for (int i = 0; i < (BN > 32 ? 2 : 1); ++i)
            if (i * 32 + lane < BN) copy4(sc + i * 32 + lane, of_token[i] ? of_token[i] + kb * per_block : from_scales, of_token[i] != nullptr);
          if (lane == 0) copy4(sc + BN, of_weights + kb * w.block, true);
          arrive_after_copies(bars + L::READY + q);
        }
        it += here;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (wid >= 4 && wid < 4 + kReaders) {
    const int quarter = wid & 3, c_first = ((wid - 4) >> 2) * L::kRows;                 // the warp's rows of W and tokens
    const unsigned at_tmem = tmem + ((unsigned)(quarter * 32) << 16) + c_first;
    const int reader = (int)blockIdx.x * kReaders + wid - 4, readers = (int)gridDim.x * kReaders;
    unsigned it = 0;
    bool ok = true;                                  // (all readers go the same way, see below)
#pragma unroll
    for (int f = 0; f < 2 && ok; ++f) {
      const Matrix& w = a.w[f];
      if (chunks) {
        float acc[L::kRows];
        for (Stretch s(w, chunks, plan.per[f]); s.there();) {
#pragma unroll
          for (int c = 0; c < L::kRows; ++c) acc[c] = 0.f;
          const int chunk = s.chunk, tile = s.tile;
          const int n = s.here(w);
          for (int i = 0; i < n; ++i, ++it) {
            const unsigned q = it % S, stage = it % kAccStages;
            ok = wait(bars + L::READY + q, (it / S) & 1, a.wait_limit, abort) && wait(bars + L::DONE + q, (it / S) & 1, a.wait_limit, abort);
            if (!(ok = __all_sync(kAll, ok))) break;
            fence_after();
            const float* sc = scales + q * L::kScales;
            float v[L::kRows];
#pragma unroll
            for (int c = 0; c < L::kRows; c += 8) tmem_load8(at_tmem + stage * BN + c, v + c);
            const float of_weights = sc[BN];
            tmem_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) arrive(bars + L::ACCEMPTY + stage);
#pragma unroll
            for (int c = 0; c < L::kRows; c += 4) {
              const float4 t = *reinterpret_cast<const float4*>(sc + c_first + c);
              acc[c] = fmaf(v[c] * of_weights, t.x, acc[c]);
              acc[c + 1] = fmaf(v[c + 1] * of_weights, t.y, acc[c + 1]);
              acc[c + 2] = fmaf(v[c + 2] * of_weights, t.z, acc[c + 2]);
              acc[c + 3] = fmaf(v[c + 3] * of_weights, t.w, acc[c + 3]);
            }
            __syncwarp();
            if (lane == 0) arrive(bars + L::SEMPTY + q);
          }
          if (!ok) break;
          float* to = a.sums + (sums_at<BN>(plan, w, chunk, tile, (int)blockIdx.x) + c_first) * 128 + quarter * 32 + lane;
          const int left = plan.rows[chunk] - c_first;
#pragma unroll
          for (int c = 0; c < L::kRows; ++c) if (c < left) to[c * 128] = acc[c];
          s.next_tile(w);
        }
      }
      // what comes after the meeting, as far as it can be known before
      const int hb = a.w[1].kblocks;
      HiddenAt<BN> hidden;
      ChoiceAt<BN> choice;
      if (f == 0 && reader < rows * hb && a.h % 4 == 0) hidden = HiddenAt<BN>(a, plan, reader, readers, rows * hb, hb, lane);
      if (f == 1 && reader < a.T * w.tiles) choice = ChoiceAt<BN>(a, plan, reader / w.tiles, reader % w.tiles, lane);
      readers_sync();
      // (one thread decides for all readers: where a warp gave up, the block does not come, and the meeting fails)
      if (tid == 128) {
        const int which = f ? MEET_OUT : MEET_SUMS;
        if (!*reinterpret_cast<volatile int*>(abort)) come(&a.shared->meeting[which].count);
        misc[3] = meet(a.shared, which, a.wait_limit, abort);
      }
      readers_sync();
      ok = *reinterpret_cast<volatile int*>(misc + 3) != 0;
      if (!ok) break;
      if (f == 0) {
        auto finish = [&](int u, float4 v, const float4& up) {
          v = make_float4(activated(v.x, a.silu), activated(v.y, a.silu), activated(v.z, a.silu), activated(v.w, a.silu));
          if (a.gated) { v.x *= up.x; v.y *= up.y; v.z *= up.z; v.w *= up.w; }
          round_block(v, a.hq + (long long)u * 128, a.hs + u % hb * (a.T * a.c.top_k) + u / hb, lane);
        };
        const int units = rows * hb;
        if (a.h % 4 == 0) {
          const int many = a.gated ? 2 : 4;
#pragma unroll 1
          for (int u = reader; u < units; u += many * readers) {            // several at a time: their loads are in flight together
            if (u != reader) hidden = HiddenAt<BN>(a, plan, u, readers, units, hb, lane);
            float4 v[4];
            add_up<BN>(hidden.at, hidden.blocks, v);
            if (a.gated) {
              finish(u, v[0], v[1]);
              if (u + readers < units) finish(u + readers, v[2], v[3]);
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r) if (u + r * readers < units) finish(u + r * readers, v[r], v[r]);
            }
          }
        } else {
#pragma unroll 1
          for (int u = reader; u < units; u += readers) {
            const int row = u / hb, j = u % hb * 128 + lane * 4;
            const float4 v = hidden_one_by_one<BN>(a, plan, row, j, a.h);
            float4 up = v;
            if (a.gated) up = hidden_one_by_one<BN>(a, plan, row, a.h + min(j, a.h), 2 * a.h);
            finish(u, v, up);
          }
        }
        readers_sync();
        if (tid == 128) come(&a.shared->meeting[MEET_HIDDEN].count);
      } else {
        const int K = a.c.top_k;
        for (int u = reader; u < a.T * w.tiles; u += readers) {
          const int t = u / w.tiles, tile = u % w.tiles, c = tile * 128 + lane * 4;
          if (u != reader) choice = ChoiceAt<BN>(a, plan, t, tile, lane);
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          if (a.router && !__any_sync(kAll, choice.blocks != 0) && not_finite(a, t, lane)) y.x = y.y = y.z = y.w = __uint_as_float(0x7fffffffu);
          for (int j0 = 0; j0 < K; j0 += 8) {
            float4 z[8];
            const float* from[8];
            int n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int j = min(j0 + i, 31);
              from[i] = reinterpret_cast<const float*>(__shfl_sync(kAll, choice.at, j)) + lane * 4;
              n[i] = __shfl_sync(kAll, choice.blocks, j);            // (lanes from top_k on have none)
            }
            add_up<BN>(from, n, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float q = __shfl_sync(kAll, choice.weight, min(j0 + i, 31));
              if (j0 + i < K && n[i]) { y.x = fmaf(q, z[i].x, y.x); y.y = fmaf(q, z[i].y, y.y); y.z = fmaf(q, z[i].z, y.z); y.w = fmaf(q, z[i].w, y.w); }
            }
          }
          const float v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) if (c + i < a.d) store_c(a.y, a.type, t * a.ldy + c + i, v[i]);
        }
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  fence_after();
  if (*reinterpret_cast<volatile int*>(abort)) {     // a wait ran out: what is in flight ends first
    if (tid == 0) atomicExch(&a.shared->gave_up, 1u);
    if (wid == 0 && lane == 0) {
      const unsigned issued = (unsigned)misc[2];
      for (unsigned q = 0; q < S && q < issued; ++q) wait_in_flight(bars + L::FULL + q, ((issued - 1 - q) / S) & 1, a.wait_limit);      // a slot's last use
    } else if ((wid == 1 || wid == 3) && elect_one()) {                     // the lane that issued the products: a commit is of its own thread's
      commit(bars + L::DRAIN + (wid >> 1));
      wait_in_flight(bars + L::DRAIN + (wid >> 1), 0, a.wait_limit);
    }
    __syncthreads();
    fence_after();
  }
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kCols));
  if (tid == 0 && *reinterpret_cast<volatile int*>(abort)) atomicMin(a.status, ASGD_ETIMEOUT);
}

// The meetings' counts begin at zero.  (A kernel, so that the next one can come up beside it.)
__global__ void begin_kernel(Shared* sh) {
  wait_for_stream();
  let_next_come();
  for (unsigned i = threadIdx.x; i < sizeof(Shared) / 4; i += blockDim.x) reinterpret_cast<unsigned*>(sh)[i] = 0;
}

// ---- host ----

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Tokens of a tile, by the mean load of an expert: with even loads an expert's tokens fit into one chunk, and its weights are read once.  Uneven loads
// give popular experts several chunks, each of which reads the weights again: drawn loads with twice and three times the mean made the run of K blocks 10 % longer for
// 60 tokens of 32 experts (top 4), 12 % for 128 of 64 and 16 % for 128 of 128 (top 8), a fifth at most; up to 16 tokens of 64 experts none.
int tokens_of(long long assignments, int experts) {
  const double mean = (double)assignments / experts;
  return mean <= 8 ? 16 : mean <= 18 ? 32 : 64;
}
struct Places {
  size_t logits, ids, weights, xq, xs, hq, hs, sums, bytes;
};
Places places(const asgd_route_config& c, const asgd_expert_layer_args& a) {
  const size_t T = (size_t)a.T, rows = T * c.top_k, rows1 = (size_t)a.h * (a.gated ? 2 : 1);
  const size_t kb1 = (size_t)ceil_div(a.d, 128), kb2 = (size_t)ceil_div(a.h, 128), tiles = std::max((size_t)ceil_div((long long)rows1, 128), kb1);
  Places p;
  size_t at = up256(sizeof(Shared));
  auto take = [&](size_t n) { const size_t here = at; at += up256(n); return here; };
  p.logits = take(a.router ? T * c.experts * 4 : 0);
  p.ids = take(rows * 4);
  p.weights = take(rows * 4);
  p.xq = take(T * kb1 * 128);
  p.xs = take(T * kb1 * 4);
  p.hq = take(rows * kb2 * 128);
  p.hs = take(rows * kb2 * 4);
  p.sums = take((rows * tiles + (size_t)kSMs * tokens_of((long long)rows, c.experts)) * 512);
  p.bytes = at;
  return p;
}
// Sizes alone: ASGD_OK, or why not.
int sizes_ok(const asgd_route_config* c, const asgd_expert_layer_args* a) {
  if (!config_ok(c) || !a || a->T < 0 || a->d < 1 || a->h < 1 || (a->gated != 0 && a->gated != 1)) return ASGD_EINVAL;
  if (!config_supported(c) || a->T > ASGD_LAYER_MAX_TOKENS || a->T * c->top_k > ASGD_LAYER_MAX_ASSIGNMENTS) return ASGD_EUNSUPPORTED;
  if (a->d > ASGD_LAYER_MAX_WIDTH || a->h > ASGD_LAYER_MAX_WIDTH || a->h * (a->gated ? 2 : 1) > ASGD_LAYER_MAX_WIDTH) return ASGD_EUNSUPPORTED;
  // K blocks of all chunks (a row each at worst), times the blocks, in 32 bits
  const long long rows1 = a->h * (a->gated ? 2 : 1), most = std::max(ceil_div(rows1, 128) * ceil_div(a->d, 128), ceil_div(a->d, 128) * ceil_div(a->h, 128));
  if (most * (a->T * c->top_k) * (kSMs + 1) > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  return ASGD_OK;
}

template <int BN> int launch(const asgd_route_config& c, const asgd_expert_layer_args& a, const LayerArgs& p, cudaStream_t st) {
  CUtensorMap map_1{}, map_2{};
  if (!encode(&map_1, a.w1, a.d, p.rows1, c.experts, a.ldw1, a.w1_group, kU)) return ASGD_EINVAL;
  if (!encode(&map_2, a.w2, a.h, a.d, c.experts, a.ldw2, a.w2_group, kU)) return ASGD_EINVAL;
  static std::atomic<unsigned long long> done{0};
  if (!allow_smem(expert_layer_kernel<BN>, Layer<BN>::kSmem, done)) return ASGD_ECUDA;
  if (!launch_after(begin_kernel, dim3(1), 64, 0, st, p.shared)) return ASGD_ECUDA;
  cudaLaunchAttribute all[2];
  all[0].id = cudaLaunchAttributeCooperative;
  all[0].val.cooperative = 1;
  all[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // see launch_after
  all[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kSMs);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Layer<BN>::kSmem;
  cfg.stream = st;
  cfg.attrs = all;
  cfg.numAttrs = 2;
  return good(cudaLaunchKernelEx(&cfg, expert_layer_kernel<BN>, p, map_1, map_2)) ? ASGD_OK : ASGD_ECUDA;
}

unsigned instruction(int weights_type, int cols) {   // fp32 accumulators; weights by tokens (E4M3)
  return 1u << 4 | (weights_type == ASGD_E5M2 ? 1u : 0u) << 7 | (unsigned)(cols >> 3) << 17 | (unsigned)(kU >> 4) << 24;
}

}  // namespace

extern "C" int asgd_expert_layer_workspace_bytes(const asgd_route_config* cfg, const asgd_expert_layer_args* args, size_t* bytes) {
  if (!bytes) return ASGD_EINVAL;
  const int bad = sizes_ok(cfg, args);
  if (bad) return bad;
  *bytes = places(*cfg, *args).bytes;
  return ASGD_OK;
}

extern "C" int asgd_expert_layer(const asgd_route_config* cfg, const asgd_expert_layer_args* args, void* workspace, size_t workspace_bytes, void* stream) {
  const int bad = sizes_ok(cfg, args);
  if (bad) return bad;
  const asgd_expert_layer_args& a = *args;
  const asgd_route_config& c = *cfg;
  const long long rows1 = a.h * (a.gated ? 2 : 1), E = c.experts;
  if (!float_type(a.type) || !eight_bit_type(a.w1_type) || !eight_bit_type(a.w2_type)) return ASGD_EINVAL;
  if (a.activation != ASGD_ACT_RELU2 && a.activation != ASGD_ACT_SILU) return ASGD_EINVAL;
  if ((a.logits && a.router) || (a.shift && !a.router)) return ASGD_EINVAL;
  if (a.logits && (!float_type(a.logits_type) || a.ld_logits < E || !aligned(a.logits, type_bytes(a.logits_type)))) return ASGD_EINVAL;
  if (a.router && (!float_type(a.router_type) || a.ld_router < a.d || !aligned(a.router, type_bytes(a.router_type)))) return ASGD_EINVAL;
  if (a.ldx < a.d || a.ldy < a.d || a.ldw1 < a.d || a.ldw2 < a.h || a.ldw1 % 16 || a.ldw2 % 16) return ASGD_EINVAL;
  if (E > 1 && (a.w1_group < 0 || a.w2_group < 0 || a.w1_group % 16 || a.w2_group % 16)) return ASGD_EINVAL;
  if (!aligned_words(a.shift, a.bias, a.w1_scale, a.w2_scale, a.ids, a.weights)) return ASGD_EINVAL;
  if (a.T == 0) return ASGD_OK;
  if (!a.x || !a.y || (!a.logits && !a.router) || !aligned(a.x, type_bytes(a.type)) || !aligned(a.y, type_bytes(a.type))) return ASGD_EINVAL;
  if (!a.w1 || !a.w2 || !a.w1_scale || !a.w2_scale || !aligned(a.w1, 16) || !aligned(a.w2, 16)) return ASGD_EINVAL;
  const Places at = places(c, a);
  if (!workspace || workspace_bytes < at.bytes) return ASGD_ENOMEM;
  if (!aligned(workspace, 256)) return ASGD_EINVAL;

  const WaitDrill drill = wait_drill();
  const int bn = tokens_of(a.T * c.top_k, c.experts);
  unsigned char* base = reinterpret_cast<unsigned char*>(workspace);
  LayerArgs p{};
  static_cast<Choice&>(p) = choice_of(c, a.bias);
  p.T = (int)a.T; p.d = (int)a.d; p.h = (int)a.h; p.rows1 = (int)rows1; p.gated = a.gated; p.silu = a.activation == ASGD_ACT_SILU;
  p.x = a.x; p.ldx = a.ldx; p.type = a.type;
  p.x_wide = aligned(a.x, 4 * type_bytes(a.type)) && a.ldx % 4 == 0;
  p.y = a.y; p.ldy = a.ldy;
  p.logits = a.logits; p.ld_logits = a.ld_logits; p.logits_type = a.logits_type;
  p.router = a.router; p.ld_router = a.ld_router; p.router_type = a.router_type;
  p.router_wide = a.router && aligned(a.router, 4 * type_bytes(a.router_type)) && a.ld_router % 4 == 0;
  p.shift = a.shift; p.temperature = a.temperature;
  p.w[0] = {(int)ceil_div(rows1, 128), (int)ceil_div(a.d, 128), a.w1_scale, a.w1_scale_row, a.w1_scale_block, a.w1_scale_group, instruction(a.w1_type, bn)};
  p.w[1] = {(int)ceil_div(a.d, 128), (int)ceil_div(a.h, 128), a.w2_scale, a.w2_scale_row, a.w2_scale_block, a.w2_scale_group, instruction(a.w2_type, bn)};
  p.ids = a.ids; p.weights = a.weights;
  p.shared = reinterpret_cast<Shared*>(base);
  p.made_logits = a.router ? reinterpret_cast<float*>(base + at.logits) : nullptr;
  p.made_ids = reinterpret_cast<int*>(base + at.ids);
  p.made_weights = reinterpret_cast<float*>(base + at.weights);
  p.xq = base + at.xq;
  p.xs = reinterpret_cast<float*>(base + at.xs);
  p.hq = base + at.hq;
  p.hs = reinterpret_cast<float*>(base + at.hs);
  p.sums = reinterpret_cast<float*>(base + at.sums);
  p.wait_limit = drill.limit;
  p.withhold = drill.withhold;
  p.status = status_word();
  if (!p.status) return ASGD_ECUDA;
  const cudaStream_t st = (cudaStream_t)stream;
  return bn == 16 ? launch<16>(c, a, p, st) : bn == 32 ? launch<32>(c, a, p, st) : launch<64>(c, a, p, st);
}
