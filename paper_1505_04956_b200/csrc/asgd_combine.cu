// The experts' rows back into token order, and the gradient.  The contract is in include/asgd_experts.h.
//
// HBM is the bound: every row of z is read once (and written once in the gradient), a token's row of y or dy once.  In
// the sum a thread block takes a stretch of a token's row, a thread 16-byte pieces of it, and the rows of z are met in
// ascending place; in the gradient a warp takes an assignment.  Every sum has one order.  8192 tokens of four rows of 4096 bf16 numbers:
// 55 us, 6.1 TB/s; with the numbers unpacked as they came, eight rows always, 153.
#include "asgd_experts_common.cuh"

#include <algorithm>
#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr int kGradThreads = 128, kGradWarps = kGradThreads / 32;
constexpr int kFillRows = 4;                               // grouped rows a warp looks at for those of nothing
constexpr int kMaxRows = 8;                                // rows of z a thread has in flight

struct Args {
  long long T, D, R, ldz, ldy, ld_dy, ld_dz;
  int top_k;
  const void *z, *dy;
  const int *rows, *source;
  const float* weights;
  void *y, *dz;
  float* dweights;
};

// A piece of a row as it is in memory: 16 bytes where all rows start at 16-byte boundaries, else one number.
template <typename T, bool kVec> struct Piece {
  using Word = typename std::conditional<kVec, uint4, T>::type;
  static constexpr int kN = kVec ? kPer16<T> : 1;
  static __device__ __forceinline__ void unpack(const Word& w, float (&v)[kN]) {
    if constexpr (kVec) unpack16<T>(w, v);
    else v[0] = Elem<T>::to_f(w);
  }
  static __device__ __forceinline__ Word pack(const float (&v)[kN]) {
    if constexpr (kVec) return pack16<T>(v);
    else return Elem<T>::from_f(v[0]);
  }
  static __device__ __forceinline__ Word load(const T* p) { return *reinterpret_cast<const Word*>(p); }
  static __device__ __forceinline__ void store(T* p, const Word& w) { *reinterpret_cast<Word*>(p) = w; }
};

// The row of z that an assignment takes, and its factor; row -1: no part
__device__ __forceinline__ void assignment(const Args& a, long long t, int j, int& row, float& w) {
  row = -1;
  w = 0.f;
  if (j >= a.top_k) return;
  const int r = a.rows[t * a.top_k + j];
  if (r < 0 || r >= a.R) return;
  row = r;
  w = a.weights ? a.weights[t * a.top_k + j] : 1.f;
}

// N: rows met at a time; U: pieces per thread, blockDim apart (what is in flight is N * U pieces).  Small blocks, that are
// through soon and make room for the next ones' loads: 64 threads with four pieces each (32 with eight, where eight rows
// are met; 32 narrow ones).  8192 tokens, 4096 bf16 numbers, of 1, 2, 4 and 8 rows: 26, 35, 55 and 92 us; with 128 threads
// and eight pieces 31, 41, 61 and 103; 32 threads with four pieces 36, 36, 70, for then blocks come up too slowly.
template <bool kVec, int N> struct Shape {
  static constexpr int kThreads = kVec && N == 8 ? 32 : 64, U = (kVec ? (N == 8 ? 8 : 4) : 32) / N;
};
template <typename T, bool kVec, int N> __global__ void __launch_bounds__(Shape<kVec, N>::kThreads) combine_kernel(const Args a) {
  constexpr int kThreads = Shape<kVec, N>::kThreads, U = Shape<kVec, N>::U;
  wait_for_stream();
  using P = Piece<T, kVec>;
  const long long t = blockIdx.x, c0 = ((long long)blockIdx.y * U * kThreads + threadIdx.x) * P::kN;
  const T* z = reinterpret_cast<const T*>(a.z);
  float acc[U][P::kN];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < P::kN; ++i) acc[u][i] = 0.f;
  for (int j0 = 0; j0 < a.top_k; j0 += N) {
    int row[N];
    float w[N];
#pragma unroll
    for (int j = 0; j < N; ++j) assignment(a, t, j0 + j, row[j], w[j]);
    typename P::Word raw[N][U];
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long c = c0 + (long long)u * kThreads * P::kN;
        raw[j][u] = typename P::Word{};
        if (row[j] >= 0 && c < a.D) raw[j][u] = P::load(z + row[j] * a.ldz + c);
      }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[P::kN];
        P::unpack(raw[j][u], v);
#pragma unroll
        for (int i = 0; i < P::kN; ++i) acc[u][i] = fmaf(w[j], v[i], acc[u][i]);
      }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long c = c0 + (long long)u * kThreads * P::kN;
    if (c < a.D) P::store(reinterpret_cast<T*>(a.y) + t * a.ldy + c, P::pack(acc[u]));
  }
}

// W warps take an assignment (one where there are many): its row of z and its token's row of dy, U pieces of each in
// flight per thread.  A token's assignments are neighbours, so its row of dy comes from HBM once and from the caches after
// that; what a thread holds is small, and it is the bytes in flight that the rate needs (a token per block with all its rows
// in registers: 91 us where this takes 54, 6.2 TB/s, on 5003 x 6 rows of 2560 bf16 numbers).  The warps behind the assignments'
// take four grouped rows each, for those of nothing become zeros: a block with 128 rows, one after the other, was a tail of
// some 12 us in every call (64 assignments 10 us, now 2.3).
template <typename T, bool kVec, int W> __global__ void __launch_bounds__(kGradThreads, kVec ? 10 : 6) combine_grad_kernel(const Args a, long long fill_from) {
  wait_for_stream();
  using P = Piece<T, kVec>;
  constexpr int U = kVec ? 2 : 8, kAcross = 32 * W;
  T* dz = reinterpret_cast<T*>(a.dz);
  if (blockIdx.x >= fill_from) {
    const int lane = threadIdx.x & 31;
    const long long r0 = (((long long)blockIdx.x - fill_from) * kGradWarps + (threadIdx.x >> 5)) * kFillRows, mine = r0 + lane;
    unsigned nothing = __ballot_sync(kAll, lane < kFillRows && mine < a.R && a.source[mine] < 0);
    for (; nothing; nothing &= nothing - 1) {
      T* out = dz + (r0 + __ffs(nothing) - 1) * a.ld_dz;
      for (long long c = (long long)lane * P::kN; c < a.D; c += 32 * P::kN) P::store(out + c, typename P::Word{});
    }
    return;
  }
  __shared__ float part[kGradWarps];
  const int of = threadIdx.x / kAcross, at = threadIdx.x % kAcross;      // assignment of the block, thread of the assignment
  const long long i = (long long)blockIdx.x * (kGradThreads / kAcross) + of, t = i / a.top_k;
  int row = -1;
  float w = 0.f, dot = 0.f;
  if (t < a.T) assignment(a, t, (int)(i - t * a.top_k), row, w);
  if (row >= 0) {
    const T* dy = reinterpret_cast<const T*>(a.dy) + t * a.ld_dy;
    const T* z = reinterpret_cast<const T*>(a.z) + row * a.ldz;
    T* out = dz + row * a.ld_dz;
    for (long long c0 = at * P::kN; c0 < a.D; c0 += U * kAcross * P::kN) {
      typename P::Word g[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long c = c0 + u * kAcross * P::kN;
        g[u] = v[u] = typename P::Word{};
        if (c < a.D) {
          g[u] = P::load(dy + c);
          if (a.dweights) v[u] = P::load(z + c);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long c = c0 + u * kAcross * P::kN;
        float x[P::kN], y[P::kN];
        P::unpack(g[u], x);
        P::unpack(v[u], y);
        if (c < a.D) {
#pragma unroll
          for (int e = 0; e < P::kN; ++e) { dot = fmaf(x[e], y[e], dot); y[e] = w * x[e]; }
          if (a.dz) P::store(out + c, P::pack(y));
        }
      }
    }
  }
  if (!a.dweights) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(kAll, dot, o);
  if (W > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = dot;
    __syncthreads();
    dot = 0.f;
#pragma unroll
    for (int q = 0; q < W; ++q) dot += part[of * W + q];
  }
  if (at == 0 && t < a.T) a.dweights[i] = dot;
}

template <typename T> bool whole(const void* p, long long ld) { return aligned(p, 16) && ld % kPer16<T> == 0; }

// Calls f with the kind of pieces and the rows met at a time, as compile-time constants.
template <typename F> void with_rows(int top_k, bool vec, F&& f) {
  auto rows = [&](auto v) {
    if (top_k <= 2) f(v, std::integral_constant<int, 2>());
    else if (top_k <= 4) f(v, std::integral_constant<int, 4>());
    else f(v, std::integral_constant<int, kMaxRows>());
  };
  if (vec) rows(std::true_type());
  else rows(std::false_type());
}

}  // namespace

extern "C" int asgd_combine(int64_t T, int64_t D, int32_t top_k, const void* z, int32_t type, int64_t R, int64_t ldz, const int32_t* rows,
                            const float* weights, void* y, int64_t ldy, void* stream) {
  if (T < 0 || D < 0 || R < 0 || top_k < 1 || !float_type(type) || ldz < D || ldy < D) return ASGD_EINVAL;
  if (T > 0x7fffffffll || R > 0x7fffffffll || top_k > ASGD_MAX_TOP_K) return ASGD_EUNSUPPORTED;
  if (T == 0 || D == 0) return ASGD_OK;
  if ((R > 0 && !z) || !rows || !y || !aligned(z, type_bytes(type)) || !aligned(y, type_bytes(type)) || !aligned_words(rows, weights)) return ASGD_EINVAL;
  Args a{};
  a.T = T; a.D = D; a.R = R; a.ldz = ldz; a.ldy = ldy; a.top_k = top_k;
  a.z = z; a.rows = rows; a.weights = weights; a.y = y;
  int rc = ASGD_OK;
  with_type(type, [&](auto e) {
    using E = decltype(e);
    const bool vec = whole<E>(z, ldz) && whole<E>(y, ldy) && D % kPer16<E> == 0;
    with_rows(top_k, vec, [&](auto v, auto n) {
      constexpr bool kVec = decltype(v)::value;
      constexpr int N = decltype(n)::value, kThreads = Shape<kVec, N>::kThreads;
      const long long stretches = ceil_div(D, (long long)kThreads * Shape<kVec, N>::U * (kVec ? kPer16<E> : 1));
      if (stretches > 65535) { rc = ASGD_EUNSUPPORTED; return; }
      if (!launch_after(combine_kernel<E, kVec, N>, dim3((unsigned)T, (unsigned)stretches), kThreads, 0, (cudaStream_t)stream, a)) rc = ASGD_ECUDA;
    });
  });
  return rc;
}

extern "C" int asgd_combine_grad(int64_t T, int64_t D, int32_t top_k, const void* dy, int32_t type, int64_t ld_dy, const void* z, int64_t R,
                                 int64_t ldz, const int32_t* rows, const float* weights, const int32_t* source, void* dz, int64_t ld_dz,
                                 float* dweights, void* stream) {
  if (T < 0 || D < 0 || R < 0 || top_k < 1 || !float_type(type) || ld_dy < D || (dweights && ldz < D) || (dz && ld_dz < D)) return ASGD_EINVAL;
  if (T > 0x7fffffffll || R > 0x7fffffffll || top_k > ASGD_MAX_TOP_K) return ASGD_EUNSUPPORTED;
  if (!dz && !dweights) return ASGD_OK;
  if (T > 0 && (!rows || (D > 0 && !dy) || (D > 0 && R > 0 && dweights && !z))) return ASGD_EINVAL;
  if (!aligned(dy, type_bytes(type)) || !aligned(z, type_bytes(type)) || !aligned(dz, type_bytes(type))) return ASGD_EINVAL;
  if (!aligned_words(rows, weights, source, dweights)) return ASGD_EINVAL;
  Args a{};
  a.T = T; a.D = D; a.R = R; a.ldz = ldz; a.ld_dy = ld_dy; a.ld_dz = ld_dz; a.top_k = top_k;
  a.z = z; a.dy = dy; a.rows = rows; a.weights = weights; a.source = source; a.dz = dz; a.dweights = dweights;
  // a warp per assignment where that keeps the SMs full, else four
  const long long assignments = T * top_k;
  const int warps = assignments >= kSMs * 32 ? 1 : 4;
  const long long fill_from = ceil_div(assignments * warps, kGradWarps), blocks = fill_from + (dz && source ? ceil_div(R, kGradWarps * kFillRows) : 0);
  if (blocks > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  if (blocks == 0) return ASGD_OK;
  bool ok = false;
  with_type(type, [&](auto e) {
    using E = decltype(e);
    const bool vec = whole<E>(dy, ld_dy) && (!dweights || whole<E>(z, ldz)) && (!dz || whole<E>(dz, ld_dz)) && D % kPer16<E> == 0;
    const auto kernel = vec ? (warps == 1 ? combine_grad_kernel<E, true, 1> : combine_grad_kernel<E, true, 4>)
                            : (warps == 1 ? combine_grad_kernel<E, false, 1> : combine_grad_kernel<E, false, 4>);
    ok = launch_after(kernel, dim3((unsigned)blocks), kGradThreads, 0, (cudaStream_t)stream, a, fill_from);
  });
  return ok ? ASGD_OK : ASGD_ECUDA;
}
