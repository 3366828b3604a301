// Routing of tokens to experts: choice and weights, their gradient, and the plan that groups the assignments by expert.
// The contract is in include/asgd_experts.h.
//
// A warp owns a token: lane l holds the experts l, l + 32, ... in registers, so the row is read once, coalesced at any
// stride.  Keys become unsigned numbers of the same order, and each choice is two warp-wide integer reductions (the
// largest key, then the lowest index that has it).  The plan is a stable counting sort by expert.  A block's tokens are
// a chunk of 64; inside a chunk each expert has a 64-bit word with a bit per token that chose it, so an assignment's
// rank among the chunk's is the population count below its bit.  Chunk counts are then summed along the chunks and the
// experts, and the ranks moved by those sums: integers only, so the plan does not depend on timing.
#include "asgd_experts_common.cuh"

namespace {

using namespace asgd::experts;

constexpr int kChunk = 64;                   // tokens of a chunk (bits of an expert's word)
constexpr int kThreads = 256;                // threads of a block when there are many chunks
constexpr int kThreadsOne = 1024;            // the one block of a single chunk: two tokens per warp, latency counts

struct RouteArgs {
  asgd_route_config c;
  long long T, ld, chunks, source_len;
  const void* logits;
  const float* bias;
  int* ids;
  float* weights;
  int* offsets;
  int* rows;
  int* source;
  int* hist;                                 // [E][chunks] assignments per expert and chunk, then those in the chunks before
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
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// Scores of the row in registers.  Softmax over all E (entries beyond E are -inf logits); a logit equal to the largest
// counts exactly 1, so that rows of +inf have finite scores.
template <int S> __device__ __forceinline__ void scores(const float (&x)[S], float (&p)[S], int score) {
  if (score == ASGD_SCORE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < S; ++j) p[j] = __fdiv_rn(1.f, __fadd_rn(1.f, expf(-x[j])));
    return;
  }
  float m = x[0];
#pragma unroll
  for (int j = 1; j < S; ++j) m = fmaxf(m, x[j]);
  m = warp_max(m);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < S; ++j) { p[j] = (x[j] == m) ? 1.f : expf(x[j] - m); sum += p[j]; }
  sum = warp_sum(sum);
#pragma unroll
  for (int j = 0; j < S; ++j) p[j] = __fdiv_rn(p[j], sum);
}

// p[e] of the row, known to every lane
template <int S> __device__ __forceinline__ float pick(const float (&p)[S], int e) {
  float v = 0.f;
#pragma unroll
  for (int j = 0; j < S; ++j) v = (e >> 5) == j ? p[j] : v;
  return __shfl_sync(kAll, v, e & 31);
}

template <int S, typename T> __device__ __forceinline__ void load_row(const T* row, int E, int lane, float (&x)[S]) {
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * 32 + lane;
    x[j] = (e < E) ? Elem<T>::to_f(row[e]) : -INFINITY;
  }
}

// The choice of one token: lane j < top_k returns its j-th expert (or -1) and weight.
template <int S> __device__ __forceinline__ void choose(const asgd_route_config& c, const float (&x)[S], const float* bias, int lane, int& id, float& weight) {
  const int E = c.experts;
  float p[S];
  scores<S>(x, p, c.score);
  const bool by_logit = bias == nullptr && c.group_top == 1;
  unsigned key[S];
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * 32 + lane;
    const float v = by_logit ? x[j] : (bias && e < E) ? __fadd_rn(p[j], bias[e]) : p[j];
    key[j] = (e < E && x[j] > -INFINITY && v > -INFINITY) ? ordered(v) : 0u;
  }
  if (c.groups_kept < c.groups) {
    const int per = E / c.groups;
    unsigned mine = 0;                                                 // lane g: the ordered score of group g
    for (int g = 0; g < c.groups; ++g) {
      unsigned m1 = 0, m2 = 0;                                         // this lane's two largest keys of the group
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const int e = j * 32 + lane;
        const unsigned k = (e >= g * per && e < (g + 1) * per) ? key[j] : 0u;
        m2 = max(m2, min(m1, k));
        m1 = max(m1, k);
      }
      unsigned best = __reduce_max_sync(kAll, m1);
      if (c.group_top == 2 && best) {
        const unsigned holders = __ballot_sync(kAll, m1 == best);
        const unsigned second = __reduce_max_sync(kAll, (lane == __ffs(holders) - 1) ? m2 : m1);
        if (second) best = ordered(__fadd_rn(from_ordered(best), from_ordered(second)));
      }
      if (lane == g) mine = best;
    }
    unsigned kept = 0;
    for (int i = 0; i < c.groups_kept; ++i) {
      const unsigned best = __reduce_max_sync(kAll, (kept >> lane) & 1u ? 0u : mine);
      if (!best) break;
      kept |= 1u << (__ffs(__ballot_sync(kAll, mine == best && !((kept >> lane) & 1u))) - 1);
    }
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const int e = j * 32 + lane;
      if (e < E && !((kept >> (e / per)) & 1u)) key[j] = 0u;
    }
  }
  id = -1;
  weight = 0.f;
  float sum = 0.f;
  for (int i = 0; i < c.top_k; ++i) {
    unsigned m = key[0];
#pragma unroll
    for (int j = 1; j < S; ++j) m = max(m, key[j]);
    const unsigned best = __reduce_max_sync(kAll, m);
    if (!best) break;
    unsigned at = 0xffffffffu;
#pragma unroll
    for (int j = S - 1; j >= 0; --j) at = key[j] == best ? (unsigned)(j * 32 + lane) : at;
    const int e = (int)__reduce_min_sync(kAll, at);
#pragma unroll
    for (int j = 0; j < S; ++j) if (e == j * 32 + lane) key[j] = 0u;
    const float s = pick<S>(p, e);
    sum += s;
    if (lane == i) { id = e; weight = s; }
  }
  if (id >= 0) weight = c.renormalise ? c.scale * weight / (sum + 1e-20f) : c.scale * weight;
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

// -1 for the rows of nothing: experts e = first, first + step, ... and the tail behind the last expert
__device__ void fill_nothing(const RouteArgs& a, const int* first_row, const int* count, int total, int first, int step) {
  const int E = a.c.experts;
  if (a.c.align > 1)
    for (int e = first; e < E; e += step) {
      const int to = e + 1 < E ? first_row[e + 1] : total;
      for (int r = first_row[e] + count[e] + (int)threadIdx.x; r < to; r += blockDim.x) a.source[r] = -1;
    }
  for (long long r = total + (long long)first * blockDim.x + threadIdx.x; r < a.source_len; r += (long long)step * blockDim.x) a.source[r] = -1;
}

template <int S, typename T> __global__ void route_kernel(const RouteArgs a) {
  __shared__ unsigned long long word[ASGD_MAX_EXPERTS];
  __shared__ int first_row[ASGD_MAX_EXPERTS], count[ASGD_MAX_EXPERTS], warp_part[32];
  const int E = a.c.experts, K = a.c.top_k, lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const bool plan = a.offsets != nullptr;
  const long long t0 = (long long)blockIdx.x * kChunk;
  const int nt = (int)min((long long)kChunk, a.T - t0);
  if (plan) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) word[e] = 0;
    __syncthreads();
  }
  for (int q = wid; q < nt; q += nw) {
    float x[S];
    load_row<S, T>(reinterpret_cast<const T*>(a.logits) + (t0 + q) * a.ld, E, lane, x);
    int id;
    float w;
    choose<S>(a.c, x, a.bias, lane, id, w);
    if (lane < K) {
      a.ids[(t0 + q) * K + lane] = id;
      a.weights[(t0 + q) * K + lane] = w;
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
    else a.hist[(long long)e * a.chunks + blockIdx.x] = n;
  }
  if (one) {
    __syncthreads();
    total = scan_padded(first_row, E, a.c.align, warp_part);
    for (int e = threadIdx.x; e < E; e += blockDim.x) a.offsets[e] = first_row[e];
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
  for (int i = threadIdx.x; i < nt * K; i += blockDim.x) {
    const long long at = t0 * K + i;
    const int id = a.ids[at], q = i / K;                               // written by this block before the barrier above
    int r = -1;
    if (id >= 0) {
      r = __popcll(word[id] & ((1ull << q) - 1ull));
      if (one) { r += first_row[id]; a.source[r] = (int)at; }
    }
    a.rows[at] = r;
  }
  if (one) fill_nothing(a, first_row, count, total, 0, 1);
}

// per expert (a warp each): counts of the chunks before, and the total
__global__ void chunk_sums_kernel(const RouteArgs a) {
  const int e = (int)(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)), lane = threadIdx.x & 31;
  if (e >= a.c.experts) return;
  int* h = a.hist + (long long)e * a.chunks;
  int run = 0;
  for (long long c0 = 0; c0 < a.chunks; c0 += 32) {
    const int n = c0 + lane < a.chunks ? h[c0 + lane] : 0;
    int inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(kAll, inc, o); if (lane >= o) inc += v; }
    if (c0 + lane < a.chunks) h[c0 + lane] = run + inc - n;
    run += __shfl_sync(kAll, inc, 31);
  }
  if (lane == 0) a.totals[e] = run;
}

// ranks inside a chunk -> grouped rows, and the way back
__global__ void place_kernel(const RouteArgs a) {
  __shared__ int first_row[ASGD_MAX_EXPERTS], count[ASGD_MAX_EXPERTS], warp_part[32];
  const int E = a.c.experts, K = a.c.top_k;
  for (int e = threadIdx.x; e < E; e += blockDim.x) first_row[e] = count[e] = a.totals[e];
  __syncthreads();
  const int total = scan_padded(first_row, E, a.c.align, warp_part);
  if (blockIdx.x == 0) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) a.offsets[e] = first_row[e];
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
  const long long t0 = (long long)blockIdx.x * kChunk;
  const int nt = (int)min((long long)kChunk, a.T - t0);
  for (int i = threadIdx.x; i < nt * K; i += blockDim.x) {
    const long long at = t0 * K + i;
    const int id = a.ids[at];
    if (id < 0) continue;
    const int r = a.rows[at] + first_row[id] + a.hist[(long long)id * a.chunks + blockIdx.x];
    a.rows[at] = r;
    a.source[r] = (int)at;
  }
  fill_nothing(a, first_row, count, total, (int)blockIdx.x, (int)gridDim.x);
}

// nothing to route: an empty plan
__global__ void empty_plan_kernel(const RouteArgs a) {
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

template <int S, typename T> __global__ void __launch_bounds__(kThreads) route_grad_kernel(const GradArgs a) {
  const int E = a.c.experts, K = a.c.top_k, lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  float x[S], p[S];
  load_row<S, T>(reinterpret_cast<const T*>(a.logits) + t * a.ld, E, lane, x);
  int id = -1;
  float dw = 0.f;
  if (lane < K) { id = a.ids[t * K + lane]; dw = a.dweights[t * K + lane]; }
  const bool ok = id >= 0 && id < E;
  scores<S>(x, p, a.c.score);
  // lane j: score of the j-th choice
  float s = 0.f;
  for (int i = 0; i < K; ++i) {
    const int e = __shfl_sync(kAll, ok ? id : 0, i);
    const float v = pick<S>(p, e);
    if (lane == i) s = v;
  }
  if (!ok) { s = 0.f; dw = 0.f; }
  float ds;
  if (a.c.renormalise) {
    const float total = warp_sum(s) + 1e-20f;
    ds = a.c.scale * (dw - warp_sum(dw * s) / total) / total;
  } else {
    ds = a.c.scale * dw;
  }
  if (!ok) ds = 0.f;
  const float dot = warp_sum(ds * s);
  float g[S];
#pragma unroll
  for (int j = 0; j < S; ++j) g[j] = 0.f;
  for (int i = 0; i < K; ++i) {
    const int e = __shfl_sync(kAll, ok ? id : -1, i);
    const float v = __shfl_sync(kAll, ds, i);
#pragma unroll
    for (int j = 0; j < S; ++j) if (e == j * 32 + lane) g[j] += v;
  }
  T* out = reinterpret_cast<T*>(a.dlogits) + t * a.ld_out;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int e = j * 32 + lane;
    if (e < E) out[e] = Elem<T>::from_f(a.c.score == ASGD_SCORE_SIGMOID ? g[j] * p[j] * (1.f - p[j]) : p[j] * (g[j] - dot));
  }
}

// Calls f with the registers a lane needs for E experts, as a compile-time number.
template <typename F> void with_slots(int E, F&& f) {
  if (E <= 32) f(std::integral_constant<int, 1>());
  else if (E <= 64) f(std::integral_constant<int, 2>());
  else if (E <= 128) f(std::integral_constant<int, 4>());
  else if (E <= 256) f(std::integral_constant<int, 8>());
  else if (E <= 512) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
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
size_t workspace_bytes(const asgd_route_config* c, long long T) {
  if (T <= kChunk) return 0;
  return ((size_t)ceil_div(T, kChunk) + 1) * (size_t)c->experts * sizeof(int);
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
  a.T = T; a.ld = ld; a.chunks = ceil_div(T, kChunk); a.source_len = source_len;
  a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights;
  a.offsets = plan ? offsets : nullptr; a.rows = rows; a.source = source;
  a.hist = (int*)workspace;
  a.totals = a.hist + (want ? (size_t)a.chunks * cfg->experts : 0);
  if (T == 0) {
    if (plan) empty_plan_kernel<<<1, kThreads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
  }
  with_slots(cfg->experts, [&](auto s) {
    with_type(type, [&](auto e) {
      // the widest instance needs more registers than 1024 threads have
      const int threads = a.chunks > 1 ? kThreads : decltype(s)::value > 8 ? 512 : kThreadsOne;
      route_kernel<decltype(s)::value, decltype(e)><<<(unsigned)a.chunks, threads, 0, st>>>(a);
    });
  });
  if (plan && a.chunks > 1) {
    chunk_sums_kernel<<<(unsigned)ceil_div(cfg->experts, 4), 128, 0, st>>>(a);
    place_kernel<<<(unsigned)a.chunks, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}

extern "C" int asgd_route_grad(const asgd_route_config* cfg, int64_t T, const void* logits, int32_t type, int64_t ld, const int32_t* ids,
                               const float* dweights, void* dlogits, int64_t ld_out, void* stream) {
  if (!config_ok(cfg) || T < 0 || !float_type(type) || ld < cfg->experts || ld_out < cfg->experts) return ASGD_EINVAL;
  if (!config_supported(cfg) || T > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  if (T == 0) return ASGD_OK;
  if (!logits || !ids || !dweights || !dlogits || !aligned(logits, type_bytes(type)) || !aligned(dlogits, type_bytes(type))) return ASGD_EINVAL;
  GradArgs a{*cfg, T, ld, ld_out, logits, ids, dweights, dlogits};
  with_slots(cfg->experts, [&](auto s) {
    with_type(type, [&](auto e) {
      route_grad_kernel<decltype(s)::value, decltype(e)><<<(unsigned)ceil_div(T, kThreads / 32), kThreads, 0, (cudaStream_t)stream>>>(a);
    });
  });
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}
