// Shared by the operators of a layer of experts: element types, conversions, and host-side checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/asgd_experts.h"

namespace asgd {
namespace experts {

constexpr int kSMs = 148;                    // B200
constexpr unsigned kAll = 0xffffffffu;

inline bool float_type(int t) { return t == ASGD_F32 || t == ASGD_BF16 || t == ASGD_F16; }
inline bool eight_bit_type(int t) { return t == ASGD_E4M3 || t == ASGD_E5M2; }
inline size_t type_bytes(int t) { return t == ASGD_F32 ? 4 : (t == ASGD_BF16 || t == ASGD_F16) ? 2 : 1; }
inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
template <typename... P> inline bool aligned_words(const P*... p) { return (aligned(p, 4) && ...); }       // 32-bit arrays (null is fine)
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ float to_f(float v) { return v; }
  static __device__ __forceinline__ float from_f(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
  static __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
};

// 16 bytes as 4 or 8 numbers
template <typename T> constexpr int kPer16 = 16 / (int)sizeof(T);
template <typename T> __device__ __forceinline__ void unpack16(const uint4& u, float (&v)[kPer16<T>]) {
  const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
  for (int i = 0; i < kPer16<T>; ++i) v[i] = Elem<T>::to_f(e[i]);
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float (&v)[kPer16<T>]) {
  uint4 u;
  T* e = reinterpret_cast<T*>(&u);
#pragma unroll
  for (int i = 0; i < kPer16<T>; ++i) e[i] = Elem<T>::from_f(v[i]);
  return u;
}

// Whether a CUDA call went well; the error of one that did not is this call's, and left to no later one.
inline bool good(cudaError_t e) {
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess;
}

// A launch that may begin while the kernel before it in the stream ends: blocks come up as SMs fall free, and wait (first
// thing, wait_for_stream) until all that was before is complete and visible.
template <typename... P, typename... A> inline bool launch_after(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return good(cudaLaunchKernelEx(&cfg, kernel, P(args)...));
}
// (in a kernel that another one of the same call follows) the next kernel's blocks may come up as soon as there is room
__device__ __forceinline__ void let_next_come() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Calls f with a value of the C++ type of a floating element type.
template <typename F> inline void with_type(int type, F&& f) {
  if (type == ASGD_F32) f(float());
  else if (type == ASGD_BF16) f(__nv_bfloat16());
  else f(__half());
}

}  // namespace experts
}  // namespace asgd
