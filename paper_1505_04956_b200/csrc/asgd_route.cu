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
#include "asgd_choose.cuh"

#include <algorithm>
#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr int kMaxChunk = 64;                // tokens of a chunk (bits of an expert's word)
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kThreadsOne = 1024;            // the one block of a single chunk: two tokens per warp, latency counts
constexpr int kFillBlocks = 2 * kSMs;        // blocks at least that write the rows of nothing

struct RouteArgs : Choice {
  long long T, ld, source_len;
  int chunk, chunks, stride;                 // tokens of a chunk, chunks, numbers of an expert in hist (a multiple of 4)
  const void* logits;
  int* ids;
  float* weights;
  int* offsets;
  int* rows;
  int* source;
  int* hist;                                 // [E][stride] assignments per expert and chunk, then those in the chunks before
  int* totals;                               // [E]
};

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
  const int E = c.experts;
  if (lanes_of(c) == 8) {
    if (E <= 16) f(Int<2>(), Int<8>());
    else if (E <= 32) f(Int<4>(), Int<8>());
    else f(Int<8>(), Int<8>());
  } else if (E <= 64) f(Int<2>(), Int<32>());
  else if (E <= 128) f(Int<4>(), Int<32>());
  else if (E <= 256) f(Int<8>(), Int<32>());
  else if (E <= 512) f(Int<16>(), Int<32>());
  else f(Int<32>(), Int<32>());
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
  static_cast<Choice&>(a) = choice_of(*cfg, bias);
  a.T = T; a.ld = ld; a.source_len = source_len;
  a.chunk = chunk_of(cfg, T);
  a.chunks = chunks_of(cfg, T);
  a.logits = logits; a.ids = ids; a.weights = weights;
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
