// Rounding to 8-bit floating point with a scale for each block of 128, of rows taken in order or gathered, as they are
// and transposed.  The contract is in include/asgd_experts.h.
//
// Both kernels read a number once and keep it in registers from the search for the block's largest magnitude to the
// rounding; HBM is the bound.  A row's blocks alone (rows_kernel): a warp takes a stretch of a row, its loads all in
// flight before the first is used.  The transposed matrix too, or 128 x 128 blocks (tile_kernel): a thread block takes
// a 128 x 128 tile, a thread 16 neighbouring rows of 4 columns, so that 16 rounded numbers of a column are one 16-byte
// store into the transposed tile in shared memory.
#include "asgd_rows.cuh"

#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr float kTiny = 7.888609052210118e-31f;      // 2^-100: smallest magnitude a block is scaled by
constexpr int kThreads = 256, kWarps = kThreads / 32;

struct Args {
  asgd_quantize_args a;
  unsigned per_magic;                                // s / per_token = umulhi(s, per_magic) >> per_shift; 0: per_token 1
  int per_shift;
  int row_blocks, col_blocks;                        // blocks of 128 along K and along M
  float fmax, inv_fmax;
  const char *lo, *hi;                               // where x begins and ends
  int q_wide;                                        // rows of q start at vectors (for rows of x that do not)
};

template <bool kE5M2> __device__ __forceinline__ unsigned short round2(float x, float y) {
  return __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, kE5M2 ? __NV_E5M2 : __NV_E4M3);
}
template <bool kE5M2> __device__ __forceinline__ unsigned round4(float x, float y, float z, float w) {
  return (unsigned)round2<kE5M2>(x, y) | ((unsigned)round2<kE5M2>(z, w) << 16);
}

template <typename T, typename Word> __device__ __forceinline__ float element(const Word& w, int i) {
  return Elem<T>::to_f(reinterpret_cast<const T*>(&w)[i]);
}

// largest magnitude of the numbers in 16 bytes (a NaN is passed over)
template <typename T> __device__ __forceinline__ float largest(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    const float* v = reinterpret_cast<const float*>(&w);
    return fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
  } else {                                               // two at a time
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    const T2* v = reinterpret_cast<const T2*>(&w);
    const T2 m = __hmax2(__hmax2(__habs2(v[0]), __habs2(v[1])), __hmax2(__habs2(v[2]), __habs2(v[3])));
    return fmaxf(Elem<T>::to_f(m.x), Elem<T>::to_f(m.y));
  }
}

// A warp takes a stretch of a row: U 16-byte pieces per lane, all loaded before the first is used.  The blocks a lane has a
// part in are reduced together: each exchange between lanes folds half of the maxima onto half of the lanes, so that a
// lane ends with one block's maximum, divides once, and hands the result round (with eight pieces 16 exchanges and one
// division where eight separate reductions take 32 to 40 and eight).  The instructions issued are the bound for gathered
// rows that come from L2: 8192 x 4096 numbers gathered four times took 107 us with separate reductions.
template <typename T, bool kVec, bool kE5M2, bool kWeights, int U> __global__ void __launch_bounds__(kThreads) rows_kernel(const Args p) {
  wait_for_stream();
  constexpr int V = kPer16<T>, LB = 128 / V;             // numbers per piece, lanes per block
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, K = (int)a.K;
  // the block's warps take neighbouring rows of the same stretch: their scales are neighbours in memory
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V;
  if (r >= a.M) return;
  float factor;
  const long long from = input_row(p, r, factor);
  const T* row = reinterpret_cast<const T*>(a.x) + from * a.ldx;
  const bool whole = kVec && ((int)blockIdx.y + 1) * (U * 32 * V) <= K;
  uint4 raw[U];
  if constexpr (kVec || sizeof(T) == 4) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 32 * V;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (from >= 0) {
        if (whole) raw[u] = *reinterpret_cast<const uint4*>(row + c);
        else if (c < K) raw[u] = load<T, uint4, kVec>(row, c, K);
      }
    }
  } else {
    Unaligned<T, uint4> two[U];
#pragma unroll
    for (int u = 0; u < U; ++u) two[u].start(p, row, c0 + u * 32 * V, from >= 0 && c0 + u * 32 * V < K);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = two[u].get(row, c0 + u * 32 * V, K, from >= 0 && c0 + u * 32 * V < K);
  }
  float m[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (kWeights) {
      float v[V];
      unpack16<T>(raw[u], v);
      m[u] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) m[u] = fmaxf(m[u], fabsf(__fmul_rn(v[i], factor)));
    } else {
      m[u] = largest<T>(raw[u]);
    }
  }
  constexpr int OL = LB / U;                             // lanes that end with the same block
#pragma unroll
  for (int n = U / 2, o = LB / 2; n > 0; n /= 2, o /= 2)
#pragma unroll
    for (int u = 0; u < n; ++u) {
      const bool high = lane & o;
      const float got = __shfl_xor_sync(kAll, high ? m[u] : m[u + n], o);
      m[u] = fmaxf(high ? m[u + n] : m[u], got);
    }
#pragma unroll
  for (int o = OL / 2; o > 0; o /= 2) m[0] = fmaxf(m[0], __shfl_xor_sync(kAll, m[0], o));
  const float best = fmaxf(m[0], kTiny), mine = __fdiv_rn(p.fmax, best);
  if (lane % OL == 0) {                                  // the block this lane ended with
    const int c = ((int)blockIdx.y * U + lane % LB / OL) * 32 * V + lane / LB * 128;
    if (c < K) a.scale[r * a.scale_row + (c >> 7) * a.scale_block] = __fmul_rn(best, p.inv_fmax);
  }
  unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r * a.ldq;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    const float inv = __shfl_sync(kAll, mine, lane / LB * LB + u * OL);
    float v[V];
    unpack16<T>(raw[u], v);
    unsigned w[V / 4];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (kWeights ? __fmul_rn(v[i], factor) : v[i]) * inv;
#pragma unroll
    for (int i = 0; i < V; i += 4) w[i / 4] = round4<kE5M2>(v[i], v[i + 1], v[i + 2], v[i + 3]);
    if (whole || ((kVec || p.q_wide) && c + V <= K)) {
      if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<unsigned*>(q + c) = w[0];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) if (c + i < K) q[c + i] = (unsigned char)(w[i / 4] >> (8 * (i & 3)));
    }
  }
}

// Four neighbouring numbers of a row: magnitudes' maxima over several rows, per column
template <typename T> struct ColMax;
template <> struct ColMax<float> {
  float4 m;
  __device__ __forceinline__ void start(const uint4& w) { m = make_float4(0.f, 0.f, 0.f, 0.f); add(w); }
  __device__ __forceinline__ void add(const uint4& w) {
    m.x = fmaxf(m.x, fabsf(__uint_as_float(w.x))); m.y = fmaxf(m.y, fabsf(__uint_as_float(w.y)));
    m.z = fmaxf(m.z, fabsf(__uint_as_float(w.z))); m.w = fmaxf(m.w, fabsf(__uint_as_float(w.w)));
  }
  __device__ __forceinline__ float4 get() const { return m; }
};
template <typename T, typename T2> struct ColMax16 {                    // two at a time
  T2 a, b;
  __device__ __forceinline__ void start(const uint2& w) { a = __habs2(reinterpret_cast<const T2*>(&w)[0]); b = __habs2(reinterpret_cast<const T2*>(&w)[1]); }
  __device__ __forceinline__ void add(const uint2& w) {
    a = __hmax2(a, __habs2(reinterpret_cast<const T2*>(&w)[0]));
    b = __hmax2(b, __habs2(reinterpret_cast<const T2*>(&w)[1]));
  }
  __device__ __forceinline__ float4 get() const { return make_float4(Elem<T>::to_f(a.x), Elem<T>::to_f(a.y), Elem<T>::to_f(b.x), Elem<T>::to_f(b.y)); }
};
template <> struct ColMax<__half> : ColMax16<__half, __half2> {};
template <> struct ColMax<__nv_bfloat16> : ColMax16<__nv_bfloat16, __nv_bfloat162> {};
__device__ __forceinline__ float4 max4(float4 a, float4 b) { return make_float4(fmaxf(a.x, b.x), fmaxf(a.y, b.y), fmaxf(a.z, b.z), fmaxf(a.w, b.w)); }

// The numbers stay in registers as they came (16-bit ones packed), and are taken apart once for the rows' rounding and
// once for the columns': more blocks per SM are worth more than the second unpacking (loads' latency is the bound).  Blocks
// per SM: as many as spill nothing to speak of (8192 x 4096 both ways: bf16 30 us with four, 33 with three; fp32 42 with two,
// 45 with three).
template <typename T, bool kVec, bool kE5M2, bool kWeights> __global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : kVec && !kWeights ? 4 : 3) tile_kernel(const Args p) {
  wait_for_stream();
  using Word = typename std::conditional<sizeof(T) == 4, uint4, uint2>::type;      // 4 numbers
  constexpr int kAtOnce = 8;                                    // rows in flight where they do not start at vectors (four: 50 us, eight: 48)
  __shared__ __align__(16) unsigned char tile[128 * 128];       // [column][row], 16-byte pieces exchanged by column / 4
  __shared__ float4 col_max[kWarps][32];
  __shared__ float whole_max[kWarps];
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, K = (int)a.K;
  const long long m0 = (long long)blockIdx.y * 128;
  const int k0 = (int)blockIdx.x * 128;
  const long long r0 = m0 + 16 * wid;
  const int c = k0 + 4 * lane;
  const T* x = reinterpret_cast<const T*>(a.x);
  // lane i < 16: where row i of the warp's comes from
  float factor_of = 1.f;
  long long from = lane < 16 ? input_row(p, r0 + lane, factor_of) : -1;
  const unsigned there = __ballot_sync(kAll, from >= 0);
  Word raw[16];
  if (kVec && k0 + 128 <= K) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const long long t = a.source ? __shfl_sync(kAll, from, i) : r0 + i;
      raw[i] = Word{};
      if ((there >> i) & 1u) raw[i] = *reinterpret_cast<const Word*>(x + t * a.ldx + c);
    }
  } else if constexpr (kVec || sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const long long t = __shfl_sync(kAll, from, i);
      raw[i] = Word{};
      if (((there >> i) & 1u) && c < K) raw[i] = load<T, Word, kVec>(x + t * a.ldx, c, K);
    }
  } else {
#pragma unroll
    for (int i0 = 0; i0 < 16; i0 += kAtOnce) {
      Unaligned<T, Word> two[kAtOnce];
      const T* row[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        row[i] = x + __shfl_sync(kAll, from, i0 + i) * a.ldx;
        two[i].start(p, row[i], c, ((there >> (i0 + i)) & 1u) && c < K);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) raw[i0 + i] = two[i].get(row[i], c, K, ((there >> (i0 + i)) & 1u) && c < K);
    }
  }
  float factor[kWeights ? 16 : 1];
  if (kWeights)
#pragma unroll
    for (int i = 0; i < 16; ++i) factor[kWeights ? i : 0] = __shfl_sync(kAll, factor_of, i);
  auto value = [&](int i, int j) {
    const float v = element<T>(raw[i], j);
    return kWeights ? __fmul_rn(v, factor[kWeights ? i : 0]) : v;
  };
  auto row_max = [&](int i) {
    if constexpr (kWeights || sizeof(T) == 4) {
      return fmaxf(fmaxf(fabsf(value(i, 0)), fabsf(value(i, 1))), fmaxf(fabsf(value(i, 2)), fabsf(value(i, 3))));
    } else {
      ColMax<T> m;
      m.start(raw[i]);
      const auto w = __hmax2(m.a, m.b);
      return fmaxf(Elem<T>::to_f(w.x), Elem<T>::to_f(w.y));
    }
  };
  float one = kTiny;
  if (a.square) {
#pragma unroll
    for (int i = 0; i < 16; ++i) one = fmaxf(one, row_max(i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) one = fmaxf(one, __shfl_xor_sync(kAll, one, o));
    if (lane == 0) whole_max[wid] = one;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) one = fmaxf(one, whole_max[w]);
    if (threadIdx.x == 0) a.scale[blockIdx.y * a.scale_row + blockIdx.x * a.scale_block] = __fmul_rn(one, p.inv_fmax);
  }
  if (a.q) {
    float m[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) m[i] = a.square ? one : row_max(i);
    if (!a.square) {
      // 16 rows' maxima over 32 lanes by halving: each step folds half of the rows onto the other half of the lanes, so
      // that lane l ends with row l / 2 (16 exchanges instead of 80), and the rows' inverses come from 16 lanes at once
#pragma unroll
      for (int n = 8, o = 16; n > 0; n >>= 1, o >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const bool high = lane & o;
          const float got = __shfl_xor_sync(kAll, high ? m[i] : m[i + n], o);
          m[i] = fmaxf(high ? m[i + n] : m[i], got);
        }
      m[0] = fmaxf(fmaxf(m[0], __shfl_xor_sync(kAll, m[0], 1)), kTiny);
      const long long r = r0 + (lane >> 1);
      if (!(lane & 1) && r < a.M) a.scale[r * a.scale_row + blockIdx.x * a.scale_block] = __fmul_rn(m[0], p.inv_fmax);
    }
    const float mine = __fdiv_rn(p.fmax, m[0]);
    unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r0 * a.ldq + c;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float inv = __shfl_sync(kAll, mine, 2 * i);
      const unsigned w = round4<kE5M2>(value(i, 0) * inv, value(i, 1) * inv, value(i, 2) * inv, value(i, 3) * inv);
      if (r0 + i < a.M) {
        if ((kVec || p.q_wide) && c + 4 <= K) *reinterpret_cast<unsigned*>(q) = w;
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) if (c + j < K) q[j] = (unsigned char)(w >> (8 * j));
      }
      q += a.ldq;
    }
  }
  if (!a.qt) return;
  float4 inv;
  if (a.square) {
    inv.x = inv.y = inv.z = inv.w = __fdiv_rn(p.fmax, one);
  } else {
    float4 m;
    if constexpr (kWeights) {
      m = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 16; ++i) m = max4(m, make_float4(fabsf(value(i, 0)), fabsf(value(i, 1)), fabsf(value(i, 2)), fabsf(value(i, 3))));
    } else {
      ColMax<T> cm;
      cm.start(raw[0]);
#pragma unroll
      for (int i = 1; i < 16; ++i) cm.add(raw[i]);
      m = cm.get();
    }
    col_max[wid][lane] = m;
    __syncthreads();
    m = make_float4(kTiny, kTiny, kTiny, kTiny);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = max4(m, col_max[w][lane]);
    inv = make_float4(__fdiv_rn(p.fmax, m.x), __fdiv_rn(p.fmax, m.y), __fdiv_rn(p.fmax, m.z), __fdiv_rn(p.fmax, m.w));
    const float best[4] = {m.x, m.y, m.z, m.w};
    if (wid == 0)
#pragma unroll
      for (int j = 0; j < 4; ++j) if (c + j < K) a.scale_t[(c + j) * a.scale_t_row + blockIdx.y * a.scale_t_block] = __fmul_rn(best[j], p.inv_fmax);
  }
  const float inv_of[4] = {inv.x, inv.y, inv.z, inv.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    unsigned u[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      u[g] = round4<kE5M2>(value(4 * g, j) * inv_of[j], value(4 * g + 1, j) * inv_of[j], value(4 * g + 2, j) * inv_of[j], value(4 * g + 3, j) * inv_of[j]);
    *reinterpret_cast<uint4*>(tile + (4 * lane + j) * 128 + ((wid ^ (lane & 7)) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
  }
  __syncthreads();
  unsigned char* qt = reinterpret_cast<unsigned char*>(a.qt);
  const bool wide = ((reinterpret_cast<unsigned long long>(qt) | (unsigned long long)a.ldqt) & 15) == 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = (int)(threadIdx.x >> 3) + 32 * i, piece = threadIdx.x & 7;
    if (k0 + col >= K) continue;
    const uint4 u = *reinterpret_cast<const uint4*>(tile + col * 128 + ((piece ^ ((col >> 2) & 7)) << 4));
    const long long r = m0 + 16 * piece;
    unsigned char* to = qt + (k0 + col) * a.ldqt + r;
    if (wide && r + 16 <= a.M) *reinterpret_cast<uint4*>(to) = u;
    else {
      const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int b = 0; b < 16; ++b) if (r + b < a.M) to[b] = (unsigned char)(w[b >> 2] >> (8 * (b & 3)));
    }
  }
}

// Calls f with three flags as compile-time constants.
template <typename F> void with_flags(bool vec, bool e5m2, bool weights, F&& f) {
  auto third = [&](auto v, auto e) { if (weights) f(v, e, std::true_type()); else f(v, e, std::false_type()); };
  auto second = [&](auto v) { if (e5m2) third(v, std::true_type()); else third(v, std::false_type()); };
  if (vec) second(std::true_type());
  else second(std::false_type());
}
template <typename T, int U> bool launch_rows(const Args& p, bool vec, cudaStream_t st) {
  const dim3 grid((unsigned)ceil_div(p.a.M, kWarps), (unsigned)ceil_div(p.a.K, 32 * kPer16<T> * U));
  bool ok = false;
  with_flags(vec, p.a.q_type == ASGD_E5M2, p.a.weights != nullptr, [&](auto kv, auto ke, auto kw) {
    if constexpr (decltype(kv)::value || U <= 4)         // eight pieces for whole vectors alone
      ok = launch_after(rows_kernel<T, decltype(kv)::value, decltype(ke)::value, decltype(kw)::value, U>, grid, kThreads, 0, st, p);
  });
  return ok;
}
template <typename T> bool launch(const Args& given, cudaStream_t st) {
  const asgd_quantize_args& a = given.a;
  const bool e5m2 = a.q_type == ASGD_E5M2, w = a.weights != nullptr;
  const bool rows_only = !a.qt && !a.square;
  const int V = rows_only ? kPer16<T> : 4;
  // vector accesses need every row of the input and of the result to start at a whole vector
  const bool q_wide = !a.q || (aligned(a.q, V) && a.ldq % V == 0), vec = aligned(a.x, V * sizeof(T)) && a.ldx % V == 0 && q_wide;
  Args p = given;
  p.q_wide = q_wide;
  p.lo = reinterpret_cast<const char*>(a.x);
  p.hi = a.rows_x > 0 ? p.lo + ((a.rows_x - 1) * a.ldx + a.K) * (long long)sizeof(T) : p.lo;
  if (rows_only) {
    // eight pieces per lane for gathered rows, which L2 feeds faster than they are rounded (8192 x 4096 bf16 numbers four
    // times: 53 us, with four pieces 57), where they leave enough warps, a row is that long and pieces are loaded whole; rows
    // in order come from HBM and are faster with more warps (once: 17.2 us with four pieces, 18.3 with eight)
    if (vec && a.source && a.K >= 32 * V * 8 && a.M >= 4 * kSMs) return launch_rows<T, 8>(p, vec, st);
    // short rows: no more pieces than there are (27008 gathered rows of 384 bf16 numbers: 9 us, with four pieces 15)
    if (a.K <= 32 * V) return launch_rows<T, 1>(p, vec, st);
    if (a.K <= 64 * V) return launch_rows<T, 2>(p, vec, st);
    return launch_rows<T, 4>(p, vec, st);
  } else {
    const dim3 grid((unsigned)p.row_blocks, (unsigned)p.col_blocks);
    bool ok = false;
    with_flags(vec, e5m2, w, [&](auto kv, auto ke, auto kw) {
      ok = launch_after(tile_kernel<T, decltype(kv)::value, decltype(ke)::value, decltype(kw)::value>, grid, kThreads, 0, st, p);
    });
    return ok;
  }
}

}  // namespace

extern "C" int asgd_quantize(const asgd_quantize_args* args, void* stream) {
  if (!args) return ASGD_EINVAL;
  const asgd_quantize_args& a = *args;
  if (a.M < 0 || a.K < 0 || !float_type(a.x_type) || !eight_bit_type(a.q_type)) return ASGD_EINVAL;
  if ((a.square != 0 && a.square != 1) || a.per_token < 1) return ASGD_EINVAL;
  if ((a.square && a.source) || (a.weights && !a.source) || a.rows_x < 0 || (!a.source && a.rows_x != a.M)) return ASGD_EINVAL;
  if (a.ldx < a.K || (a.q && a.ldq < a.K) || (a.qt && a.ldqt < a.M)) return ASGD_EINVAL;
  if (a.M > 0x7fffffffll || a.K > ASGD_QUANTIZE_MAX) return ASGD_EUNSUPPORTED;   // column numbers stay inside 32 bits
  if (a.M == 0 || a.K == 0) return ASGD_OK;
  if ((!a.q && !a.qt) || (a.rows_x > 0 && !a.x) || !aligned(a.x, type_bytes(a.x_type))) return ASGD_EINVAL;
  if (!aligned_words(a.source, a.weights, a.scale, a.scale_t)) return ASGD_EINVAL;
  if (((a.q || a.square) && !a.scale) || (a.qt && !a.square && !a.scale_t)) return ASGD_EINVAL;
  Args p;
  p.a = a;
  const long long rb = ceil_div(a.K, 128), cb = ceil_div(a.M, 128);
  p.row_blocks = (int)rb;
  p.col_blocks = (int)cb;
  per_token_magic(a.per_token, p.per_magic, p.per_shift);
  p.fmax = a.q_type == ASGD_E4M3 ? 448.f : 57344.f;
  p.inv_fmax = a.q_type == ASGD_E4M3 ? 1.f / 448.f : 1.f / 57344.f;
  // limits of the grid: 65535 tiles along M, or 65535 stretches of a row
  if ((a.qt || a.square) ? cb > 65535 : ceil_div(a.K, 512) > 65535) return ASGD_EUNSUPPORTED;
  bool ok = false;
  with_type(a.x_type, [&](auto e) { ok = launch<decltype(e)>(p, (cudaStream_t)stream); });
  return ok ? ASGD_OK : ASGD_ECUDA;
}
