// The norm of many tensors together, and clipping by it.  The contract is in include/asgd_gradients.h.
//
// norm^2 is a sum over everything, so there are two passes: partial sums, then (a kernel that every block of begins with
// adding up the same partial sums in the same order) the factor and the scaling.  The bytes are the bound: the list of
// tensors counts as one run of 32-byte pieces, and every block takes an equal stretch of it, whatever tensors it meets there.
// The second pass walks each stretch from its end, where the first one's last bytes are still in L2.
// Loads and stores of 32 bytes a thread, two of them in flight, with 1024 threads an SM: 344 M bf16 numbers of 56 tensors 355 us
// (three passes at HBM's rate would be 316); 16 bytes, four in flight, 465; eight 434; two with 2048 threads 413.  The norm alone of 87 M numbers of
// 512 tensors 42.5 us (5.5 TB/s) where 16 bytes took 65.
// Squares are added in fp64: a number of fp32 squared passes fp32's range from 2^64 on, and long sums in fp32 lose digits;
// the conversions and multiply-adds (two instructions a number) hide behind the loads (sums by eight in fp32 gained nothing).
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/asgd_gradients.h"
#include "asgd_experts_common.cuh"

namespace {

using namespace asgd::experts;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBlocks = 2 * kSMs;                    // partial sums of a launch
constexpr int kFlight = 2;                           // pieces a thread has in flight
constexpr int kPiece = 32;                           // bytes: the widest load and store there is

// The tensors of a launch, by value: N at most.
template <int N> struct List {
  const void* x[N];
  void* out[N];
  long long n[N];
  long long first[N + 1];                            // pieces of the tensors before
  unsigned char type[N];
  int count;
};
constexpr int kFew = 64, kMany = 640;                // tensors that a launch's parameters hold (21.1 KB of 32 at most)
static_assert(sizeof(List<kMany>) < 32000, "kernel parameters");

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[kWarps];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  if (lane == 0) part[wid] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += part[w];
  return s;
}

struct __align__(32) Piece { unsigned w[8]; };
template <typename T> constexpr int kPer = kPiece / (int)sizeof(T);
template <typename T> __device__ __forceinline__ void unpack(const Piece& p, float (&v)[kPer<T>]) {
  const T* e = reinterpret_cast<const T*>(p.w);
#pragma unroll
  for (int i = 0; i < kPer<T>; ++i) v[i] = Elem<T>::to_f(e[i]);
}
// Pieces are those of memory, 32 bytes from a multiple of 32 on, so that a view that begins anywhere is read whole piece by whole piece;
// its first and last ones may have numbers that are not its own.  (So which numbers a thread adds up depends on where the view begins in a piece.)
template <typename T> __device__ __forceinline__ int skipped(const T* x) { return (int)(reinterpret_cast<unsigned long long>(x) & (kPiece - 1)) / (int)sizeof(T); }
// Piece u of a tensor of n numbers behind `skip`; zeros for numbers that are not its own.
template <typename T> __device__ __forceinline__ Piece load_piece(const T* x, long long n, long long u, int skip) {
  constexpr int V = kPer<T>;
  const long long at = u * V - skip;
  Piece p;
  if (at >= 0 && at + V <= n) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[2]), "=r"(p.w[3]), "=r"(p.w[4]), "=r"(p.w[5]), "=r"(p.w[6]), "=r"(p.w[7]) : "l"(x + at) : "memory");
    return p;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) p.w[i] = 0;
  T* e = reinterpret_cast<T*>(p.w);
#pragma unroll
  for (int i = 0; i < V; ++i) if (at + i >= 0 && at + i < n) e[i] = x[at + i];
  return p;
}
__device__ __forceinline__ void store_piece(void* to, const Piece& p) {              // read again by nobody here
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(to), "r"(p.w[0]), "r"(p.w[1]), "r"(p.w[2]), "r"(p.w[3]), "r"(p.w[4]), "r"(p.w[5]), "r"(p.w[6]), "r"(p.w[7]) : "memory");
}
template <typename T> __device__ __forceinline__ double squares(const T* x, long long n, long long from, long long to) {
  constexpr int V = kPer<T>;
  const int skip = skipped(x);
  double sum[2] = {0.0, 0.0};
  auto add = [&](const Piece& w) {
    float v[V];
    unpack<T>(w, v);
#pragma unroll
    for (int i = 0; i < V; ++i) { const double d = v[i]; sum[i & 1] = fma(d, d, sum[i & 1]); }
  };
  long long u = from + threadIdx.x;
  for (; u + (kFlight - 1) * kThreads < to; u += kFlight * kThreads) {
    Piece w[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) w[k] = load_piece<T>(x, n, u + k * kThreads, skip);
#pragma unroll
    for (int k = 0; k < kFlight; ++k) add(w[k]);
  }
  for (; u < to; u += kThreads) add(load_piece<T>(x, n, u, skip));
  return sum[0] + sum[1];
}
template <typename T> __device__ __forceinline__ void scale_pieces(const T* x, T* out, long long n, long long from, long long to, float f) {
  constexpr int V = kPer<T>;
  const int skip = skipped(x);
  const bool alike = skipped(out) == skip;           // else the results are written one by one
  auto put = [&](long long u, const Piece& w) {
    float v[V];
    unpack<T>(w, v);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= f;
    const long long at = u * V - skip;
    if (alike && at >= 0 && at + V <= n) {
      Piece to;
      T* e = reinterpret_cast<T*>(to.w);
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = Elem<T>::from_f(v[i]);
      store_piece(out + at, to);
    } else
#pragma unroll
      for (int i = 0; i < V; ++i) if (at + i >= 0 && at + i < n) out[at + i] = Elem<T>::from_f(v[i]);
  };
  long long u = to - 1 - threadIdx.x;
  for (; u - (kFlight - 1) * kThreads >= from; u -= kFlight * kThreads) {
    Piece w[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) w[k] = load_piece<T>(x, n, u - k * kThreads, skip);
#pragma unroll
    for (int k = 0; k < kFlight; ++k) put(u - k * kThreads, w[k]);
  }
  for (; u >= from; u -= kThreads) put(u, load_piece<T>(x, n, u, skip));
}

// the tensor that holds piece u
template <int N> __device__ __forceinline__ int tensor_of(const List<N>& l, long long u) {
  int a = 0, b = l.count;
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (l.first[m] <= u) a = m; else b = m;
  }
  return a;
}
template <int N> __device__ __forceinline__ void stretch(const List<N>& l, long long& from, long long& to) {
  const long long all = l.first[l.count];
  from = all * blockIdx.x / gridDim.x;               // below 2^55: 640 tensors of 2^37 pieces and one (2^40 numbers of fp32) by 296 blocks
  to = all * (blockIdx.x + 1ll) / gridDim.x;
}

template <int N> __global__ void __launch_bounds__(kThreads, 2) squares_kernel(const __grid_constant__ List<N> l, double* part) {
  wait_for_stream();
  let_next_come();
  long long from, to;
  stretch(l, from, to);
  double sum = 0.0;
  if (from < to)
    for (int t = tensor_of(l, from); t < l.count && l.first[t] < to; ++t) {
      const long long a = max(from - l.first[t], 0ll), b = min(to, l.first[t + 1]) - l.first[t];
      if (l.type[t] == ASGD_F32) sum += squares(reinterpret_cast<const float*>(l.x[t]), l.n[t], a, b);
      else if (l.type[t] == ASGD_BF16) sum += squares(reinterpret_cast<const __nv_bfloat16*>(l.x[t]), l.n[t], a, b);
      else sum += squares(reinterpret_cast<const __half*>(l.x[t]), l.n[t], a, b);
    }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// every block adds the same sums up in the same order
__device__ __forceinline__ float norm_of(const double* part, int parts) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) sum += part[i];
  return (float)sqrt(block_sum(sum));
}
__global__ void __launch_bounds__(kThreads) norm_kernel(const double* part, int parts, float* norm) {
  wait_for_stream();
  const float v = norm_of(part, parts);
  if (threadIdx.x == 0) *norm = v;
}
template <int N> __global__ void __launch_bounds__(kThreads, 2) scale_kernel(const __grid_constant__ List<N> l, const double* part, int parts, float max_norm, float* norm) {
  wait_for_stream();
  const float v = norm_of(part, parts);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
  const float q = __fdiv_rn(max_norm, v + 1e-6f), f = q > 1.f || max_norm == INFINITY ? 1.f : q;       // a NaN stays
  long long from, to;
  stretch(l, from, to);
  if (from >= to) return;
  for (int t = tensor_of(l, to - 1); t >= 0 && l.first[t + 1] > from; --t) {
    if (f == 1.f && l.x[t] == l.out[t]) continue;
    const long long a = max(from - l.first[t], 0ll), b = min(to, l.first[t + 1]) - l.first[t];
    if (a >= b) continue;
    if (l.type[t] == ASGD_F32) scale_pieces(reinterpret_cast<const float*>(l.x[t]), reinterpret_cast<float*>(l.out[t]), l.n[t], a, b, f);
    else if (l.type[t] == ASGD_BF16) scale_pieces(reinterpret_cast<const __nv_bfloat16*>(l.x[t]), reinterpret_cast<__nv_bfloat16*>(l.out[t]), l.n[t], a, b, f);
    else scale_pieces(reinterpret_cast<const __half*>(l.x[t]), reinterpret_cast<__half*>(l.out[t]), l.n[t], a, b, f);
  }
}

// ---- host ----

// The next tensors that have numbers, N at most.
template <int N> void fill(List<N>& l, const asgd_gradient* list, long long count, long long& at) {
  l.count = 0;
  l.first[0] = 0;
  for (; at < count && l.count < N; ++at) {
    const asgd_gradient& g = list[at];
    if (g.n == 0) continue;
    const int i = l.count++;
    l.x[i] = g.x; l.out[i] = g.out; l.n[i] = g.n; l.type[i] = (unsigned char)g.type;
    const long long size = (long long)type_bytes(g.type), skip = (long long)((uintptr_t)g.x & (kPiece - 1)) / size;
    l.first[i + 1] = l.first[i] + ceil_div(g.n + skip, kPiece / size);
  }
}
// Blocks: two pieces a thread at least, so that few numbers take few blocks (and few partial sums).
unsigned blocks_of(long long pieces) { return (unsigned)std::min<long long>(kBlocks, std::max(1ll, ceil_div(pieces, 2 * kThreads))); }

template <int N> int norm_launches(const asgd_gradient* list, long long count, double* part, int& parts, cudaStream_t st) {
  static thread_local List<N> l;
  for (long long at = 0; at < count;) {
    fill(l, list, count, at);
    if (!l.count) continue;
    const unsigned blocks = blocks_of(l.first[l.count]);
    if (!launch_after(squares_kernel<N>, dim3(blocks), kThreads, 0, st, l, part + parts)) return ASGD_ECUDA;
    parts += (int)blocks;
  }
  return ASGD_OK;
}
template <int N> int scale_launches(const asgd_gradient* list, long long count, const double* part, int parts, float max_norm, float* norm, cudaStream_t st) {
  static thread_local List<N> l;
  for (long long at = 0; at < count;) {
    fill(l, list, count, at);
    if (!l.count) continue;
    if (!launch_after(scale_kernel<N>, dim3(blocks_of(l.first[l.count])), kThreads, 0, st, l, part, parts, max_norm, norm)) return ASGD_ECUDA;
    norm = nullptr;                                  // written once
  }
  return ASGD_OK;
}

constexpr long long kMostTensors = 1ll << 20;

// Whether what a clipping call writes meets anything else of the call's: ranges by where they begin, against the furthest end so far.
bool overlaps(const asgd_gradient* list, int64_t count) {
  struct Range { uintptr_t from, to; bool written; };
  std::vector<Range> all;
  all.reserve((size_t)count * 2);
  for (int64_t i = 0; i < count; ++i) {
    const asgd_gradient& g = list[i];
    const size_t bytes = (size_t)g.n * type_bytes(g.type);
    if (!bytes) continue;
    all.push_back({(uintptr_t)g.out, (uintptr_t)g.out + bytes, true});
    if (g.x != g.out) all.push_back({(uintptr_t)g.x, (uintptr_t)g.x + bytes, false});
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t read = 0, written = 0;                   // ends
  for (const Range& r : all) {
    if (r.from < written || (r.written && r.from < read)) return true;
    uintptr_t& end = r.written ? written : read;
    end = std::max(end, r.to);
  }
  return false;
}

size_t bytes_of(long long count) { return (size_t)(ceil_div(std::max(count, 1ll), kMany) * kBlocks) * sizeof(double); }

int check(const asgd_gradient* list, int64_t count, bool scaled, const float* norm, const void* workspace, size_t bytes) {
  if (count < 0 || (count > 0 && !list) || !norm || !aligned_words(norm)) return ASGD_EINVAL;
  if (count > kMostTensors) return ASGD_EUNSUPPORTED;
  for (int64_t i = 0; i < count; ++i) {
    const asgd_gradient& g = list[i];
    if (g.n < 0 || !float_type(g.type) || g.reserved != 0) return ASGD_EINVAL;
    if (g.n > ASGD_GRADIENT_MAX) return ASGD_EUNSUPPORTED;
    if (g.n > 0 && (!g.x || !aligned(g.x, type_bytes(g.type)))) return ASGD_EINVAL;
    if (scaled && g.n > 0 && (!g.out || !aligned(g.out, type_bytes(g.type)))) return ASGD_EINVAL;
  }
  if (!workspace || bytes < bytes_of(count)) return ASGD_ENOMEM;
  if (!aligned(workspace, 16)) return ASGD_EINVAL;
  if (scaled && count > 0) try {
    if (overlaps(list, count)) return ASGD_EINVAL;
  } catch (const std::bad_alloc&) {                  // of the host's memory
    return ASGD_ENOMEM;
  }
  return ASGD_OK;
}

}  // namespace

extern "C" int asgd_gradients_workspace_bytes(int64_t count, size_t* bytes) {
  if (!bytes || count < 0) return ASGD_EINVAL;
  if (count > kMostTensors) return ASGD_EUNSUPPORTED;
  *bytes = bytes_of(count);
  return ASGD_OK;
}

extern "C" int asgd_grad_norm(const asgd_gradient* list, int64_t count, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  const int bad = check(list, count, false, norm, workspace, workspace_bytes);
  if (bad) return bad;
  const cudaStream_t st = (cudaStream_t)stream;
  double* part = reinterpret_cast<double*>(workspace);
  int parts = 0;
  const int rc = count <= kFew ? norm_launches<kFew>(list, count, part, parts, st) : norm_launches<kMany>(list, count, part, parts, st);
  if (rc) return rc;
  return launch_after(norm_kernel, dim3(1), kThreads, 0, st, part, parts, norm) ? ASGD_OK : ASGD_ECUDA;
}

extern "C" int asgd_clip_grads(const asgd_gradient* list, int64_t count, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  const int bad = check(list, count, true, norm, workspace, workspace_bytes);
  if (bad) return bad;
  if (!(max_norm > 0.f)) return ASGD_EINVAL;
  const cudaStream_t st = (cudaStream_t)stream;
  double* part = reinterpret_cast<double*>(workspace);
  int parts = 0;
  int rc = count <= kFew ? norm_launches<kFew>(list, count, part, parts, st) : norm_launches<kMany>(list, count, part, parts, st);
  if (rc) return rc;
  if (!parts) return launch_after(norm_kernel, dim3(1), kThreads, 0, st, part, 0, norm) ? ASGD_OK : ASGD_ECUDA;
  return count <= kFew ? scale_launches<kFew>(list, count, part, parts, max_norm, norm, st) : scale_launches<kMany>(list, count, part, parts, max_norm, norm, st);
}
