// The experts' rows back into token order, and the gradient.  The contract is in include/asgd_experts.h.
//
// HBM is the bound: every row of z is read once (and written once in the gradient), a token's row of y or dy once.  A
// thread block takes a token (the sum: a stretch of a token's row), threads take 16-byte pieces; the rows of z are met
// in ascending place, so a sum has one order.
#include "asgd_experts_common.cuh"

#include <algorithm>
#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr int kThreads = 128;                              // the sum; the gradient takes what fits the row
constexpr int kMaxThreads = 256;
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

// N: rows met at a time; U: pieces per thread, blockDim apart (what is in flight is N * U pieces)
template <typename T, bool kVec, int N, int U> __global__ void __launch_bounds__(kThreads) combine_kernel(const Args a) {
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

// Blocks 0..T-1: a token each.  The blocks behind them: 128 grouped rows each, those of nothing become zeros.
template <typename T, bool kVec, int N> __global__ void __launch_bounds__(kMaxThreads) combine_grad_kernel(const Args a) {
  using P = Piece<T, kVec>;
  T* dz = reinterpret_cast<T*>(a.dz);
  if (blockIdx.x >= a.T) {
    const long long r0 = ((long long)blockIdx.x - a.T) * 128;
    for (int q = 0; q < 128; ++q) {
      const long long r = r0 + q;
      if (r >= a.R || a.source[r] >= 0) continue;
      for (long long c = (long long)threadIdx.x * P::kN; c < a.D; c += (long long)blockDim.x * P::kN) P::store(dz + r * a.ld_dz + c, typename P::Word{});
    }
    return;
  }
  __shared__ float part[kMaxThreads / 32][N];
  const T* z = reinterpret_cast<const T*>(a.z);
  const long long t = blockIdx.x;
  const T* dy = reinterpret_cast<const T*>(a.dy) + t * a.ld_dy;
  for (int j0 = 0; j0 < a.top_k; j0 += N) {
    int row[N];
    float w[N], dot[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { assignment(a, t, j0 + j, row[j], w[j]); dot[j] = 0.f; }
    for (long long c = (long long)threadIdx.x * P::kN; c < a.D; c += (long long)blockDim.x * P::kN) {
      typename P::Word raw[N];
      const typename P::Word raw_g = P::load(dy + c);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        raw[j] = typename P::Word{};
        if (a.dweights && row[j] >= 0) raw[j] = P::load(z + row[j] * a.ldz + c);
      }
      float g[P::kN];
      P::unpack(raw_g, g);
      if (a.dz)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (row[j] < 0) continue;
          float o[P::kN];
#pragma unroll
          for (int i = 0; i < P::kN; ++i) o[i] = w[j] * g[i];
          P::store(dz + row[j] * a.ld_dz + c, P::pack(o));
        }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float v[P::kN];
        P::unpack(raw[j], v);
        if (row[j] >= 0)                             // a row that takes no part adds nothing, whatever dy holds
#pragma unroll
          for (int i = 0; i < P::kN; ++i) dot[j] = fmaf(g[i], v[i], dot[j]);
      }
    }
    if (!a.dweights) continue;
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(kAll, dot[j], o);
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < N && j0 + (int)threadIdx.x < a.top_k) {
      float s = 0.f;
      for (int v = 0; v < (int)blockDim.x / 32; ++v) s += part[v][threadIdx.x];
      a.dweights[t * a.top_k + j0 + threadIdx.x] = s;
    }
    __syncthreads();
  }
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
  if ((R > 0 && !z) || !rows || !y || !aligned(z, type_bytes(type)) || !aligned(y, type_bytes(type))) return ASGD_EINVAL;
  Args a{};
  a.T = T; a.D = D; a.R = R; a.ldz = ldz; a.ldy = ldy; a.top_k = top_k;
  a.z = z; a.rows = rows; a.weights = weights; a.y = y;
  int rc = ASGD_OK;
  with_type(type, [&](auto e) {
    using E = decltype(e);
    const bool vec = whole<E>(z, ldz) && whole<E>(y, ldy) && D % kPer16<E> == 0;
    with_rows(top_k, vec, [&](auto v, auto n) {
      constexpr bool kVec = decltype(v)::value;
      constexpr int N = decltype(n)::value, U = 8 / N;
      const long long stretches = ceil_div(D, (long long)kThreads * U * (kVec ? kPer16<E> : 1));
      if (stretches > 65535) { rc = ASGD_EUNSUPPORTED; return; }
      combine_kernel<E, kVec, N, U><<<dim3((unsigned)T, (unsigned)stretches), kThreads, 0, (cudaStream_t)stream>>>(a);
    });
  });
  if (rc != ASGD_OK) return rc;
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}

extern "C" int asgd_combine_grad(int64_t T, int64_t D, int32_t top_k, const void* dy, int32_t type, int64_t ld_dy, const void* z, int64_t R,
                                 int64_t ldz, const int32_t* rows, const float* weights, const int32_t* source, void* dz, int64_t ld_dz,
                                 float* dweights, void* stream) {
  if (T < 0 || D < 0 || R < 0 || top_k < 1 || !float_type(type) || ld_dy < D || (dweights && ldz < D) || (dz && ld_dz < D)) return ASGD_EINVAL;
  if (T > 0x7fffffffll || R > 0x7fffffffll || top_k > ASGD_MAX_TOP_K) return ASGD_EUNSUPPORTED;
  if (!dz && !dweights) return ASGD_OK;
  if (T > 0 && (!rows || (D > 0 && !dy) || (D > 0 && R > 0 && dweights && !z))) return ASGD_EINVAL;
  if (!aligned(dy, type_bytes(type)) || !aligned(z, type_bytes(type)) || !aligned(dz, type_bytes(type))) return ASGD_EINVAL;
  Args a{};
  a.T = T; a.D = D; a.R = R; a.ldz = ldz; a.ld_dy = ld_dy; a.ld_dz = ld_dz; a.top_k = top_k;
  a.z = z; a.dy = dy; a.rows = rows; a.weights = weights; a.source = source; a.dz = dz; a.dweights = dweights;
  const long long blocks = T + (dz && source ? ceil_div(R, 128) : 0);
  if (blocks > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  if (blocks == 0) return ASGD_OK;
  with_type(type, [&](auto e) {
    using E = decltype(e);
    const bool vec = whole<E>(dy, ld_dy) && (!dweights || whole<E>(z, ldz)) && (!dz || whole<E>(dz, ld_dz)) && D % kPer16<E> == 0;
    // threads that share the row's pieces evenly: as many turns as 256 threads would take
    const long long pieces = std::max(1ll, ceil_div(D, vec ? kPer16<E> : 1)), turns = ceil_div(pieces, kMaxThreads);
    const unsigned threads = (unsigned)ceil_div(ceil_div(pieces, turns), 32) * 32;
    with_rows(top_k, vec, [&](auto v, auto n) {
      combine_grad_kernel<E, decltype(v)::value, decltype(n)::value><<<(unsigned)blocks, threads, 0, (cudaStream_t)stream>>>(a);
    });
  });
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}
