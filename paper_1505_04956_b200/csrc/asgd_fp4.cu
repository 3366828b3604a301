// Rounding to 4-bit floating point with a power of two for each 32 neighbours of a row, and the way back.  The contract is in
// include/asgd_fp4.h.
//
// A number is read once and stays in registers from the search for its block's largest magnitude to the rounding; the bytes
// are the bound.  A lane takes pieces of a row of 32 bytes (16 where rows do not start at 32), two or four of them in flight,
// so that a warp's loads are neighbours; 2 lanes (16-bit numbers) or 4 (fp32) have a block together and find its maximum by
// exchanges.  8192 x 4096 bf16 numbers 13.3 us (6.3 TB/s; with 16-byte pieces 19), back 12.5; gathered four times 38.5, where the
// instructions are the bound (widened and scaled by one instruction instead of by one and a half, compared as floats instead of as integers: 44 before),
// back 57 (6.0 TB/s).  Magnitudes of fp32 are compared as integers: floats of one
// sign are ordered like their bits, and infinities and NaNs come out on top.  The power of two comes from the largest one's
// exponent and one comparison of its mantissa (a <= 6 s with a = m 2^k: s = 2^(k - 2) up to m = 1.5, else 2^(k - 1)), and
// scaling by it is exact, so the one rounding is that of the conversion.
#include <cuda_fp4.h>

#include <type_traits>

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

// What a lane takes of a row at a time: 16 bytes, or 32 where rows start at multiples of that.
template <int kBytes> struct __align__(kBytes) Piece { unsigned w[kBytes / 4]; };
template <int kAlign> __device__ __forceinline__ void read_piece(const void* at, Piece<32>& p) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[2]), "=r"(p.w[3]), "=r"(p.w[4]), "=r"(p.w[5]), "=r"(p.w[6]), "=r"(p.w[7]) : "l"(at) : "memory");
}
template <int kAlign> __device__ __forceinline__ void read_piece(const void* at, Piece<16>& p) {
  if constexpr (kAlign == 8) {
    const uint2* from = reinterpret_cast<const uint2*>(at);
    const uint2 a = from[0], b = from[1];
    p.w[0] = a.x; p.w[1] = a.y; p.w[2] = b.x; p.w[3] = b.y;
  } else {
    p = *reinterpret_cast<const Piece<16>*>(at);
  }
}
template <int kAlign> __device__ __forceinline__ void write_piece(void* at, const Piece<32>& p) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(at), "r"(p.w[0]), "r"(p.w[1]), "r"(p.w[2]), "r"(p.w[3]), "r"(p.w[4]), "r"(p.w[5]), "r"(p.w[6]), "r"(p.w[7]) : "memory");
}
template <int kAlign> __device__ __forceinline__ void write_piece(void* at, const Piece<16>& p) {
  if constexpr (kAlign == 8) {
    uint2* to = reinterpret_cast<uint2*>(at);
    to[0] = make_uint2(p.w[0], p.w[1]);
    to[1] = make_uint2(p.w[2], p.w[3]);
  } else {
    *reinterpret_cast<Piece<16>*>(at) = p;
  }
}

// bits of the largest magnitude among a piece's numbers, as fp32
template <typename T, int kBytes> __device__ __forceinline__ unsigned largest(const Piece<kBytes>& p) {
  constexpr unsigned kMask = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
  unsigned m = p.w[0] & kMask;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 1; i < kBytes / 4; ++i) m = max(m, p.w[i] & kMask);
    return m;
  } else {                                           // two at a time; a NaN stays the largest
#pragma unroll
    for (int i = 1; i < kBytes / 4; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) asm("{\n .reg .b32 t;\n abs.bf16x2 t, %1;\n max.NaN.bf16x2 %0, %0, t;\n}" : "+r"(m) : "r"(p.w[i]));
      else asm("{\n .reg .b32 t;\n abs.f16x2 t, %1;\n max.NaN.f16x2 %0, %0, t;\n}" : "+r"(m) : "r"(p.w[i]));
    }
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return max(m << 16, m & 0xffff0000u);
    const unsigned short h = (unsigned short)max(m & 0xffffu, m >> 16);
    return __float_as_uint(Elem<T>::to_f(*reinterpret_cast<const T*>(&h))) & 0x7fffffffu;
  }
}
// eight numbers as 4-bit ones, the first in the lowest bits
__device__ __forceinline__ unsigned eight_codes(const float* v) {
  unsigned w;
  asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      " cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return w;
}
// V 4-bit numbers (V / 2 bytes) as one store
template <int V> __device__ __forceinline__ void store_codes(unsigned char* to, const unsigned (&w)[V > 8 ? 2 : 1]) {
  if constexpr (V == 16) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  else if constexpr (V == 8) *reinterpret_cast<unsigned*>(to) = w[0];
  else *reinterpret_cast<unsigned short*>(to) = (unsigned short)w[0];
}

// A warp takes a stretch of a row: U pieces per lane, all loaded before the first is used.
// kAlign: bytes that rows of x start at multiples of, 32, 16 or (fp32) 8; 0: anywhere.
template <typename T, int kAlign, bool kWeights, int U> __global__ void __launch_bounds__(kThreads) rows4_kernel(const Args p) {
  wait_for_stream();
  constexpr int kBytes = kAlign == 32 ? 32 : 16, V = kBytes / (int)sizeof(T), LB = ASGD_BLOCK4 / V;     // numbers per piece, lanes per block
  using P = Piece<kBytes>;
  const asgd_quantize4_args& a = p.a;
  const int lane = threadIdx.x & 31, K = (int)a.K;
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V;
  if (r >= a.M) return;
  float factor;
  const long long from = input_row(p, r, factor);
  const T* row = reinterpret_cast<const T*>(a.x) + from * a.ldx;
  P raw[U];
  if constexpr (kAlign || sizeof(T) == 4) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 32 * V;
#pragma unroll
      for (int i = 0; i < kBytes / 4; ++i) raw[u].w[i] = 0;
      if (from < 0 || c >= K) continue;
      if (kAlign && c + V <= K) read_piece<kAlign>(row + c, raw[u]);
      else {
        T* e = reinterpret_cast<T*>(raw[u].w);
#pragma unroll
        for (int i = 0; i < V; ++i) if (c + i < K) e[i] = row[c + i];
      }
    }
  } else {
    Unaligned<T, uint4> two[U];
#pragma unroll
    for (int u = 0; u < U; ++u) two[u].start(p, row, c0 + u * 32 * V, from >= 0 && c0 + u * 32 * V < K);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint4 w = two[u].get(row, c0 + u * 32 * V, K, from >= 0 && c0 + u * 32 * V < K);
      raw[u].w[0] = w.x; raw[u].w[1] = w.y; raw[u].w[2] = w.z; raw[u].w[3] = w.w;
    }
  }
  unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r * a.ldq;
  unsigned char* scale = reinterpret_cast<unsigned char*>(a.scale) + r * a.scale_row;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    T* e = reinterpret_cast<T*>(raw[u].w);
    float v[V];
    unsigned m = 0;
    if (kWeights) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = Elem<T>::to_f(e[i]);
#pragma unroll
      for (int i = 0; i < V; ++i) { v[i] = __fmul_rn(v[i], factor); m = max(m, __float_as_uint(v[i]) & 0x7fffffffu); }
    } else {
      m = largest<T>(raw[u]);
    }
#pragma unroll
    for (int o = 1; o < LB; o <<= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
    const bool none = m >= kInfBits;
    m = max(m, kTinyBits);
    const unsigned code = none ? 255u : ((m + 0x3fffffu) >> 23) - 2u;        // one more from a mantissa above 1.5 on; 25 .. 253
    const float inv = none ? 0.f : __uint_as_float((254u - code) << 23);                                // 2^(127 - code)
    if (lane % LB == 0 && c < K) scale[c / ASGD_BLOCK4] = (unsigned char)code;
    // bf16 numbers are widened and scaled by one instruction (-0 added keeps the sign of a zero)
    if constexpr (std::is_same<T, __nv_bfloat16>::value && !kWeights) {
      const unsigned short by = (unsigned short)(__float_as_uint(inv) >> 16);
#pragma unroll
      for (int i = 0; i < V; ++i) asm("fma.rn.f32.bf16 %0, %1, %2, %3;" : "=f"(v[i]) : "h"(reinterpret_cast<const unsigned short*>(e)[i]), "h"(by), "f"(-0.f));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (kWeights ? v[i] : Elem<T>::to_f(e[i])) * inv;
    }
    unsigned w[V > 8 ? 2 : 1] = {};
    if constexpr (V >= 8) {
#pragma unroll
      for (int i = 0; i < V; i += 8) w[i / 8] = eight_codes(v + i);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2)
        w[0] |= (unsigned)__nv_cvt_float2_to_fp4x2(make_float2(v[i], v[i + 1]), __NV_E2M1, cudaRoundNearest) << (4 * i);
    }
    if (none) {                                      // an infinity times 0
#pragma unroll
      for (int i = 0; i < (V > 8 ? 2 : 1); ++i) w[i] = 0;
    }
    if (c >= K) continue;
    if (p.q_wide && c + V <= K) store_codes<V>(q + c / 2, w);
    else
#pragma unroll
      for (int i = 0; i < V; i += 2) if (c + i < K) q[(c + i) / 2] = (unsigned char)((w[i / 8] >> (4 * (i & 7))) & (c + i + 1 < K ? 255u : 15u));    // (a factor may make a zero behind the row -0)
  }
}

// Numbers c .. c + 7 of a 4-bit row, at any c: from the two words that hold them.
__device__ __forceinline__ unsigned codes_at(const unsigned char* q, int c, int bytes, bool words) {
  const int at = (c >> 3) * 4;                       // (down, for a c below zero too)
  unsigned w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int b = at + 4 * i;
    w[i] = 0;
    if (words && b >= 0 && b + 4 <= bytes) w[i] = *reinterpret_cast<const unsigned*>(q + b);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) if (b + j >= 0 && b + j < bytes) w[i] |= (unsigned)q[b + j] << (8 * j);
  }
  return __funnelshift_r(w[0], w[1], 4 * (c & 7));
}
__device__ __forceinline__ float power_of(unsigned code) {
  return code == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(code ? code << 23 : 0x00400000u);
}

// A lane takes the numbers of a piece of the result.  Its rows start at multiples of kAlign bytes, or (0) anywhere: then the pieces of 16-bit results are
// those of memory, so that all but a row's first and last are whole stores, and a piece's numbers begin anywhere in the row of q.
// (8192 rows of 4095 bf16 numbers: 28.5 us, stored one by one 98; fp32 numbers stored one by one 34, this way 43.)
template <typename T, int kAlign, int U> __global__ void __launch_bounds__(kThreads)
values4_kernel(int M, int K, const unsigned char* q, long long ldq, const unsigned char* scale, long long scale_row, T* out, long long ld_out, bool q_wide) {
  wait_for_stream();
  constexpr int kBytes = kAlign == 32 ? 32 : 16, V = kBytes / (int)sizeof(T), W = V > 8 ? 2 : 1;
  constexpr bool kShift = kAlign == 0 && sizeof(T) == 2;
  const int lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (r >= M) return;
  q += r * ldq;
  scale += r * scale_row;
  out += r * ld_out;
  const int skip = !kShift ? 0 : (int)(reinterpret_cast<unsigned long long>(out) & (kBytes - 1)) / (int)sizeof(T);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V - skip;
  unsigned w[U][W], code[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    code[u][0] = code[u][1] = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) w[u][i] = 0;
    if (c >= K || c + V <= 0) continue;
    code[u][0] = scale[max(c, 0) / ASGD_BLOCK4];
    if constexpr (!kShift) {
      if (q_wide && c + V <= K) {
        if constexpr (V == 16) { const uint2 x = *reinterpret_cast<const uint2*>(q + c / 2); w[u][0] = x.x; w[u][W - 1] = x.y; }
        else if constexpr (V == 8) w[u][0] = *reinterpret_cast<const unsigned*>(q + c / 2);
        else w[u][0] = *reinterpret_cast<const unsigned short*>(q + c / 2);
      } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) if (c + i < K) w[u][i / 8] |= (unsigned)q[(c + i) / 2] << (4 * (i & 7));
      }
    } else {
      code[u][1] = scale[min(c + V - 1, K - 1) / ASGD_BLOCK4];
      w[u][0] = codes_at(q, c, (K + 1) / 2, q_wide);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    if (c >= K || c + V <= 0) continue;
    const float s = power_of(code[u][0]), s2 = !kShift ? s : power_of(code[u][1]);
    const int border = (max(c, 0) / ASGD_BLOCK4 + 1) * ASGD_BLOCK4 - c;             // numbers from there on have the second scale
    Piece<kBytes> p;
    T* e = reinterpret_cast<T*>(p.w);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 f = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)((w[u][i / 8] >> (4 * (i & 7))) & 0xffu), __NV_E2M1)));
      e[i] = Elem<T>::from_f(f.x * (!kShift || i < border ? s : s2));
      e[i + 1] = Elem<T>::from_f(f.y * (!kShift || i + 1 < border ? s : s2));
    }
    if ((kAlign || kShift) && c >= 0 && c + V <= K) write_piece<kAlign>(out + c, p);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) if (c + i >= 0 && c + i < K) out[c + i] = e[i];
  }
}

// Calls f with the pieces per lane: no more than a row has.
template <typename F> bool with_pieces(long long K, int V, F&& f) {
  if (K <= 32 * V) return f(std::integral_constant<int, 1>());
  if (K <= 64 * V || V > 8) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 4>());
}
// Calls f with what rows of `bytes` from `base` on start at multiples of.  (8 for fp32: 4001 rows of 2058 numbers 9.6 us, back 8.0;
// one by one 9.9 and 9.9.)
template <typename T, typename F> bool with_align(const void* base, long long bytes, F&& f) {
  if (aligned(base, 32) && bytes % 32 == 0) return f(std::integral_constant<int, 32>());
  if (aligned(base, 16) && bytes % 16 == 0) return f(std::integral_constant<int, 16>());
  if constexpr (sizeof(T) == 4)
    if (aligned(base, 8) && bytes % 8 == 0) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, 0>());
}
template <typename T> bool launch(Args p, cudaStream_t st) {
  const asgd_quantize4_args& a = p.a;
  p.lo = reinterpret_cast<const char*>(a.x);
  p.hi = a.rows_x > 0 ? p.lo + ((a.rows_x - 1) * a.ldx + a.K) * (long long)sizeof(T) : p.lo;
  return with_align<T>(a.x, a.ldx * (long long)sizeof(T), [&](auto align) {
    constexpr int A = decltype(align)::value, V = (A == 32 ? 32 : 16) / (int)sizeof(T);
    p.q_wide = aligned(a.q, V / 2) && a.ldq % (V / 2) == 0;
    return with_pieces(a.K, V, [&](auto u) {
      constexpr int U = decltype(u)::value;
      const dim3 grid((unsigned)ceil_div(a.M, kWarps), (unsigned)ceil_div(a.K, 32 * V * U));
      return a.weights ? launch_after(rows4_kernel<T, A, true, U>, grid, kThreads, 0, st, p) : launch_after(rows4_kernel<T, A, false, U>, grid, kThreads, 0, st, p);
    });
  });
}

bool sizes_fit(long long M, long long K) {                // rows and columns of a call stay inside 32 bits, and the grid inside its limits
  return M <= 0x7fffffffll && K <= ASGD_QUANTIZE_MAX && ceil_div(K + 7, 512) <= 65535;
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
    ok = with_align<T>(out, ld_out * (long long)sizeof(T), [&](auto align) {
      constexpr int A = decltype(align)::value, V = (A == 32 ? 32 : 16) / (int)sizeof(T);
      constexpr bool kShift = A == 0 && sizeof(T) == 2;
      constexpr int N = kShift ? 4 : V / 2;          // bytes of q that are read together
      const bool q_wide = aligned(q, N) && ldq % N == 0;
      const long long span = kShift ? K + V - 1 : K;      // from a piece's beginning before the row's first number
      return with_pieces(span, V, [&](auto u) {
        constexpr int U = decltype(u)::value;
        const dim3 grid((unsigned)ceil_div(M, kWarps), (unsigned)ceil_div(span, 32 * V * U));
        return launch_after(values4_kernel<T, A, U>, grid, kThreads, 0, (cudaStream_t)stream, (int)M, (int)K, reinterpret_cast<const unsigned char*>(q), ldq,
                            reinterpret_cast<const unsigned char*>(scale), scale_row, reinterpret_cast<T*>(out), ld_out, q_wide);
      });
    });
  });
  return ok ? ASGD_OK : ASGD_ECUDA;
}
