// The experts' rows back into token order, and the gradient.  The contract is in include/asgd_experts.h.
//
// HBM is the bound: every row of z is read once (and written once in the gradient), a token's row of y or dy once.  A
// thread block takes a token (the sum: a stretch of a token's row), threads take 16-byte pieces; the rows of z are met
// in ascending place, so a sum has one order.
#include "asgd_experts_common.cuh"

namespace {

using namespace asgd::experts;

constexpr int kThreads = 128;
constexpr int kRows = 8;                                   // rows of z a thread has in flight

struct Args {
  long long T, D, R, ldz, ldy, ld_dy, ld_dz;
  int top_k;
  const void *z, *dy;
  const int *rows, *source;
  const float* weights;
  void *y, *dz;
  float* dweights;
};

// V numbers from column c of a row (c < D); the vector form only where whole vectors are aligned
template <typename T, int V> __device__ __forceinline__ void load(const T* p, float (&v)[V]) {
  if constexpr (V == 1) v[0] = Elem<T>::to_f(*p);
  else unpack16<T>(*reinterpret_cast<const uint4*>(p), v);
}
template <typename T, int V> __device__ __forceinline__ void store(T* p, const float (&v)[V]) {
  if constexpr (V == 1) *p = Elem<T>::from_f(v[0]);
  else *reinterpret_cast<uint4*>(p) = pack16<T>(v);
}

template <typename T, int V> __global__ void __launch_bounds__(kThreads) combine_kernel(const Args a, int stretches) {
  const long long t = blockIdx.x / stretches, c = ((long long)(blockIdx.x % stretches) * kThreads + threadIdx.x) * V;
  if (c >= a.D) return;
  const T* z = reinterpret_cast<const T*>(a.z) + c;
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  for (int j0 = 0; j0 < a.top_k; j0 += kRows) {
    float v[kRows][V], w[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int r = j0 + j < a.top_k ? a.rows[t * a.top_k + j0 + j] : -1;
      const bool ok = r >= 0 && r < a.R;
      w[j] = !ok ? 0.f : a.weights ? a.weights[t * a.top_k + j0 + j] : 1.f;
      if (ok) load<T, V>(z + (long long)r * a.ldz, v[j]);
      else
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = fmaf(w[j], v[j][i], acc[i]);
  }
  store<T, V>(reinterpret_cast<T*>(a.y) + t * a.ldy + c, acc);
}

// Blocks 0..T-1: a token each.  The blocks behind them: 128 grouped rows each, those of nothing become zeros.
template <typename T, int V> __global__ void __launch_bounds__(kThreads) combine_grad_kernel(const Args a) {
  if (blockIdx.x >= a.T) {
    const long long r0 = ((long long)blockIdx.x - a.T) * 128;
    for (int q = 0; q < 128; ++q) {
      const long long r = r0 + q;
      if (r >= a.R || a.source[r] >= 0) continue;
      T* dz = reinterpret_cast<T*>(a.dz) + r * a.ld_dz;
      for (long long c = threadIdx.x; c < a.D; c += kThreads) dz[c] = Elem<T>::from_f(0.f);
    }
    return;
  }
  __shared__ float part[kThreads / 32][kRows];
  const long long t = blockIdx.x;
  const T* dy = reinterpret_cast<const T*>(a.dy) + t * a.ld_dy;
  for (int j0 = 0; j0 < a.top_k; j0 += kRows) {
    long long at[kRows];
    float w[kRows], dot[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int r = j0 + j < a.top_k ? a.rows[t * a.top_k + j0 + j] : -1;
      at[j] = (r >= 0 && r < a.R) ? r : -1;
      w[j] = at[j] < 0 ? 0.f : a.weights ? a.weights[t * a.top_k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    for (long long c = (long long)threadIdx.x * V; c < a.D; c += (long long)kThreads * V) {
      float g[V];
      load<T, V>(dy + c, g);
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        if (at[j] < 0) continue;
        if (a.dweights) {
          float v[V];
          load<T, V>(reinterpret_cast<const T*>(a.z) + at[j] * a.ldz + c, v);
#pragma unroll
          for (int i = 0; i < V; ++i) dot[j] = fmaf(g[i], v[i], dot[j]);
        }
        if (a.dz) {
          float o[V];
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = w[j] * g[i];
          store<T, V>(reinterpret_cast<T*>(a.dz) + at[j] * a.ld_dz + c, o);
        }
      }
    }
    if (!a.dweights) continue;
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(kAll, dot[j], o);
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < kRows && j0 + (int)threadIdx.x < a.top_k) {
      float s = 0.f;
#pragma unroll
      for (int w2 = 0; w2 < kThreads / 32; ++w2) s += part[w2][threadIdx.x];
      a.dweights[t * a.top_k + j0 + threadIdx.x] = s;
    }
    __syncthreads();
  }
}

template <typename T> bool whole(const void* p, long long ld) { return aligned(p, 16) && ld % kPer16<T> == 0; }

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
    const long long stretches = ceil_div(D, (long long)kThreads * (vec ? kPer16<E> : 1));
    if (stretches * T > 0x7fffffffll) { rc = ASGD_EUNSUPPORTED; return; }
    if (vec) combine_kernel<E, kPer16<E>><<<(unsigned)(stretches * T), kThreads, 0, (cudaStream_t)stream>>>(a, (int)stretches);
    else combine_kernel<E, 1><<<(unsigned)(stretches * T), kThreads, 0, (cudaStream_t)stream>>>(a, (int)stretches);
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
    if (vec) combine_grad_kernel<E, kPer16<E>><<<(unsigned)blocks, kThreads, 0, (cudaStream_t)stream>>>(a);
    else combine_grad_kernel<E, 1><<<(unsigned)blocks, kThreads, 0, (cudaStream_t)stream>>>(a);
  });
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}
