// Rounding to 4-bit floating point with a power of two for each 32 neighbours of a row, and the way back.  The contract is in
// include/asgd_fp4.h.
//
// A number is read once and stays in registers from the search for its block's largest magnitude to the rounding; the bytes
// are the bound.  A lane takes 16-byte pieces of a row, so that a warp's loads are neighbours; 4 lanes (16-bit numbers) or 8
// (fp32) have a block together and find its maximum by exchanges.  Magnitudes are compared as integers: floats of one sign
// are ordered like their bits, and infinities and NaNs come out on top.  The power of two comes from the largest one's
// exponent and one comparison of its mantissa (a <= 6 s with a = m 2^k: s = 2^(k - 2) up to m = 1.5, else 2^(k - 1)), and
// scaling by it is exact, so the one rounding is that of the conversion.
#include <cuda_fp4.h>

#include "../../include/asgd_fp4.h"
#include "asgd_rows.cuh"

namespace {

using namespace asgd::experts;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr unsigned kTinyBits = (127u - 100u) << 23;  // 2^-100: smallest magnitude a block is scaled by
constexpr unsigned kInfBits = 0x7f800000u;

struct Args {
  asgd_quantize4_args a;
  unsigned per_magic;                                // s / per_token = umulhi(s, per_magic) >> per_shift; 0: per_token 1
  int per_shift;
  const char *lo, *hi;                               // where x begins and ends
  int q_wide;                                        // rows of q start at whole pieces
};

// bits of the largest magnitude among a piece's numbers, as fp32
template <typename T> __device__ __forceinline__ unsigned largest(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    return max(max(w.x & 0x7fffffffu, w.y & 0x7fffffffu), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
  } else {                                           // two at a time
    const unsigned m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
    const unsigned short h = (unsigned short)max(m & 0xffffu, m >> 16);
    return __float_as_uint(Elem<T>::to_f(*reinterpret_cast<const T*>(&h))) & 0x7fffffffu;
  }
}

// A warp takes a stretch of a row: U pieces per lane, all loaded before the first is used.
template <typename T, bool kVec, bool kWeights, int U> __global__ void __launch_bounds__(kThreads) rows4_kernel(const Args p) {
  wait_for_stream();
  constexpr int V = kPer16<T>, LB = ASGD_BLOCK4 / V;                     // numbers per piece, lanes per block
  const asgd_quantize4_args& a = p.a;
  const int lane = threadIdx.x & 31, K = (int)a.K;
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V;
  if (r >= a.M) return;
  float factor;
  const long long from = input_row(p, r, factor);
  const T* row = reinterpret_cast<const T*>(a.x) + from * a.ldx;
  uint4 raw[U];
  if constexpr (kVec || sizeof(T) == 4) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 32 * V;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (from >= 0 && c < K) raw[u] = load<T, uint4, kVec>(row, c, K);
    }
  } else {
    Unaligned<T, uint4> two[U];
#pragma unroll
    for (int u = 0; u < U; ++u) two[u].start(p, row, c0 + u * 32 * V, from >= 0 && c0 + u * 32 * V < K);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = two[u].get(row, c0 + u * 32 * V, K, from >= 0 && c0 + u * 32 * V < K);
  }
  unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r * a.ldq;
  unsigned char* scale = reinterpret_cast<unsigned char*>(a.scale) + r * a.scale_row;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    float v[V];
    unpack16<T>(raw[u], v);
    unsigned m = 0;
    if (kWeights) {
#pragma unroll
      for (int i = 0; i < V; ++i) { v[i] = __fmul_rn(v[i], factor); m = max(m, __float_as_uint(v[i]) & 0x7fffffffu); }
    } else {
      m = largest<T>(raw[u]);
    }
#pragma unroll
    for (int o = 1; o < LB; o <<= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
    const bool none = m >= kInfBits;
    m = max(m, kTinyBits);
    const unsigned code = none ? 255u : (m >> 23) - 2u + ((m & 0x7fffffu) > 0x400000u ? 1u : 0u);       // 25 .. 253
    const float inv = none ? 0.f : __uint_as_float((254u - code) << 23);                                // 2^(127 - code)
    if (lane % LB == 0 && c < K) scale[c / ASGD_BLOCK4] = (unsigned char)code;
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < V; i += 2)
      w |= (unsigned)__nv_cvt_float2_to_fp4x2(make_float2(v[i] * inv, v[i + 1] * inv), __NV_E2M1, cudaRoundNearest) << (4 * i);
    if (none) w = 0;                                 // an infinity times 0
    if (c >= K) continue;
    if (p.q_wide && c + V <= K) {
      if constexpr (V == 8) *reinterpret_cast<unsigned*>(q + c / 2) = w;
      else *reinterpret_cast<unsigned short*>(q + c / 2) = (unsigned short)w;
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) if (c + i < K) q[(c + i) / 2] = (unsigned char)((w >> (4 * i)) & (c + i + 1 < K ? 255u : 15u));    // (a factor may make a zero behind the row -0)
    }
  }
}

// A lane takes the numbers of 16 bytes of the result.
template <typename T, int U> __global__ void __launch_bounds__(kThreads)
values4_kernel(int M, int K, const unsigned char* q, long long ldq, const unsigned char* scale, long long scale_row, T* out, long long ld_out, bool q_wide, bool out_wide) {
  wait_for_stream();
  constexpr int V = kPer16<T>;
  const int lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V;
  if (r >= M) return;
  q += r * ldq;
  scale += r * scale_row;
  out += r * ld_out;
  unsigned w[U], code[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    w[u] = code[u] = 0;
    if (c >= K) continue;
    code[u] = scale[c / ASGD_BLOCK4];
    if (q_wide && c + V <= K) {
      if constexpr (V == 8) w[u] = *reinterpret_cast<const unsigned*>(q + c / 2);
      else w[u] = *reinterpret_cast<const unsigned short*>(q + c / 2);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) if (c + i < K) w[u] |= (unsigned)q[(c + i) / 2] << (4 * i);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    if (c >= K) continue;
    const float s = code[u] == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(code[u] ? code[u] << 23 : 0x00400000u);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 f = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)((w[u] >> (4 * i)) & 0xffu), __NV_E2M1)));
      v[i] = f.x * s;
      v[i + 1] = f.y * s;
    }
    if (out_wide && c + V <= K) *reinterpret_cast<uint4*>(out + c) = pack16<T>(v);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) if (c + i < K) out[c + i] = Elem<T>::from_f(v[i]);
  }
}

// Calls f with the pieces per lane: no more than a row has.
template <typename F> bool with_pieces(long long K, int V, F&& f) {
  if (K <= 32 * V) return f(std::integral_constant<int, 1>());
  if (K <= 64 * V) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 4>());
}
template <typename T> bool launch(Args p, cudaStream_t st) {
  constexpr int V = kPer16<T>;
  const asgd_quantize4_args& a = p.a;
  const bool vec = aligned(a.x, 16) && a.ldx % V == 0;
  p.q_wide = aligned(a.q, V / 2) && a.ldq % (V / 2) == 0;
  p.lo = reinterpret_cast<const char*>(a.x);
  p.hi = a.rows_x > 0 ? p.lo + ((a.rows_x - 1) * a.ldx + a.K) * (long long)sizeof(T) : p.lo;
  return with_pieces(a.K, V, [&](auto u) {
    constexpr int U = decltype(u)::value;
    const dim3 grid((unsigned)ceil_div(a.M, kWarps), (unsigned)ceil_div(a.K, 32 * V * U));
    if (vec) return a.weights ? launch_after(rows4_kernel<T, true, true, U>, grid, kThreads, 0, st, p) : launch_after(rows4_kernel<T, true, false, U>, grid, kThreads, 0, st, p);
    return a.weights ? launch_after(rows4_kernel<T, false, true, U>, grid, kThreads, 0, st, p) : launch_after(rows4_kernel<T, false, false, U>, grid, kThreads, 0, st, p);
  });
}

bool sizes_fit(long long M, long long K) {                // rows and columns of a call stay inside 32 bits, and the grid inside its limits
  return M <= 0x7fffffffll && K <= ASGD_QUANTIZE_MAX && ceil_div(K, 512) <= 65535;
}

}  // namespace

extern "C" int asgd_quantize4(const asgd_quantize4_args* args, void* stream) {
  if (!args) return ASGD_EINVAL;
  const asgd_quantize4_args& a = *args;
  if (a.M < 0 || a.K < 0 || !float_type(a.x_type) || a.per_token < 1) return ASGD_EINVAL;
  if ((a.weights && !a.source) || a.rows_x < 0 || (!a.source && a.rows_x != a.M)) return ASGD_EINVAL;
  if (a.ldx < a.K || a.ldq < ceil_div(a.K, 2) || a.scale_row < ceil_div(a.K, ASGD_BLOCK4)) return ASGD_EINVAL;
  if (!sizes_fit(a.M, a.K)) return ASGD_EUNSUPPORTED;
  if (a.M == 0 || a.K == 0) return ASGD_OK;
  if (!a.q || !a.scale || (a.rows_x > 0 && !a.x) || !aligned(a.x, type_bytes(a.x_type)) || !aligned_words(a.source, a.weights)) return ASGD_EINVAL;
  Args p{};
  p.a = a;
  per_token_magic(a.per_token, p.per_magic, p.per_shift);
  bool ok = false;
  with_type(a.x_type, [&](auto e) { ok = launch<decltype(e)>(p, (cudaStream_t)stream); });
  return ok ? ASGD_OK : ASGD_ECUDA;
}

extern "C" int asgd_dequantize4(int64_t M, int64_t K, const void* q, int64_t ldq, const void* scale, int64_t scale_row, void* out, int32_t type, int64_t ld_out,
                                void* stream) {
  if (M < 0 || K < 0 || !float_type(type)) return ASGD_EINVAL;
  if (ldq < ceil_div(K, 2) || scale_row < ceil_div(K, ASGD_BLOCK4) || ld_out < K) return ASGD_EINVAL;
  if (!sizes_fit(M, K)) return ASGD_EUNSUPPORTED;
  if (M == 0 || K == 0) return ASGD_OK;
  if (!q || !scale || !out || !aligned(out, type_bytes(type))) return ASGD_EINVAL;
  bool ok = false;
  with_type(type, [&](auto e) {
    using T = decltype(e);
    constexpr int V = kPer16<T>;
    const bool q_wide = aligned(q, V / 2) && ldq % (V / 2) == 0, out_wide = aligned(out, 16) && ld_out % V == 0;
    ok = with_pieces(K, V, [&](auto u) {
      constexpr int U = decltype(u)::value;
      const dim3 grid((unsigned)ceil_div(M, kWarps), (unsigned)ceil_div(K, 32 * V * U));
      return launch_after(values4_kernel<T, U>, grid, kThreads, 0, (cudaStream_t)stream, (int)M, (int)K, reinterpret_cast<const unsigned char*>(q), ldq,
                          reinterpret_cast<const unsigned char*>(scale), scale_row, reinterpret_cast<T*>(out), ld_out, q_wide, out_wide);
    });
  });
  return ok ? ASGD_OK : ASGD_ECUDA;
}
