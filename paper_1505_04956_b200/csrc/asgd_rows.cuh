// Rows that a quantiser reads: in order or gathered, at any alignment.  `Args` has the call's arguments in `a`, the magic
// number of a.per_token (per_magic, per_shift), and where x begins and ends (lo, hi).
#pragma once

#include "asgd_experts_common.cuh"

namespace {

using namespace asgd::experts;

// The input row that result row r takes (-1: none, its numbers are zeros), and its factor.
template <typename Args> __device__ __forceinline__ long long input_row(const Args& p, long long r, float& factor) {
  const auto& a = p.a;
  factor = 1.f;
  if (r >= a.M) return -1;
  if (!a.source) return r;
  const int s = a.source[r];
  if (s < 0) return -1;
  const int t = p.per_magic ? (int)(__umulhi((unsigned)s, p.per_magic) >> p.per_shift) : s;
  if (t >= a.rows_x) return -1;
  if (a.weights) factor = a.weights[s];
  return t;
}

// 16 or 8 bytes of a row from column c, as they are in memory; numbers beyond K are zeros
template <typename T, typename Word, bool kVec> __device__ __forceinline__ Word load(const T* row, int c, int K) {
  constexpr int V = (int)(sizeof(Word) / sizeof(T));
  if (kVec && c + V <= K) return *reinterpret_cast<const Word*>(row + c);
  Word w{};
  T* e = reinterpret_cast<T*>(&w);
#pragma unroll
  for (int i = 0; i < V; ++i) if (c + i < K) e[i] = row[c + i];
  return w;
}

// Rows of 16-bit numbers that do not start at vectors: the two aligned vectors that hold the numbers from column c on, put
// together.  (8192 rows of 4095 bf16 numbers: 25 us; number by number 56; 4096 numbers at vectors 17.  fp32 numbers are read
// one by one: 47 us both ways where this took 64.)  Vectors that reach beyond x, at its very ends, are not read.
__device__ __forceinline__ uint2 join(const uint2& a, const uint2& b, unsigned skip) {      // bytes skip.. of the two
  const unsigned w0 = skip & 4 ? a.y : a.x, w1 = skip & 4 ? b.x : a.y, w2 = skip & 4 ? b.y : b.x, bits = (skip & 3) * 8;
  return make_uint2(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits));
}
__device__ __forceinline__ uint4 join(const uint4& a, const uint4& b, unsigned skip) {
  unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = skip & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = skip & 4 ? w[i + 1] : w[i];
  const unsigned bits = (skip & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}
template <typename T, typename Word> struct Unaligned {
  Word a, b;
  bool ok;
  template <typename Args> __device__ __forceinline__ void start(const Args& p, const T* row, int c, bool there) {
    const char* at = reinterpret_cast<const char*>(row + c);
    const unsigned skip = (unsigned)reinterpret_cast<unsigned long long>(at) & (sizeof(Word) - 1);
    const Word* from = reinterpret_cast<const Word*>(at - skip);
    ok = there && at - skip >= p.lo && at - skip + (skip ? 2 : 1) * sizeof(Word) <= p.hi;
    a = b = Word{};
    if (ok) {
      a = from[0];
      if (skip) b = from[1];
    }
  }
  __device__ __forceinline__ Word get(const T* row, int c, int K, bool there) const {
    constexpr int V = (int)(sizeof(Word) / sizeof(T));
    if (!there) return Word{};
    if (!ok) return load<T, Word, false>(row, c, K);
    Word w = join(a, b, (unsigned)reinterpret_cast<unsigned long long>(row + c) & (sizeof(Word) - 1));
    if (c + V > K) {
      T* e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int i = 0; i < V; ++i) if (c + i >= K) e[i] = Elem<T>::from_f(0.f);
    }
    return w;
  }
};
// s / per_token for 0 <= s < 2^31 by a multiplication: a magic number of 32 bits and a shift (0 and 0: per_token 1)
inline void per_token_magic(int per_token, unsigned& magic, int& shift) {
  magic = 0;
  shift = 0;
  if (per_token > 1) {
    while ((1ll << shift) < per_token) ++shift;           // 2^shift >= per_token > 2^(shift - 1)
    shift -= 1;
    magic = (unsigned)(((1ull << (32 + shift)) + per_token - 1) / per_token);
  }
}

}  // namespace
