// Rounding to 8-bit floating point with a scale for each block of 128, of rows taken in order or gathered, as they are
// and transposed.  The contract is in include/asgd_experts.h.
//
// Both kernels read a number once and keep it in registers from the search for the block's largest magnitude to the
// rounding; HBM is the bound.  A row's blocks alone (rows_kernel): a warp takes a stretch of a row, its loads all in
// flight before the first is used.  The transposed matrix too, or 128 x 128 blocks (tile_kernel): a thread block takes
// a 128 x 128 tile, a thread 16 neighbouring rows of 4 columns, so that 16 rounded numbers of a column are one 16-byte
// store into the transposed tile in shared memory.
#include "asgd_experts_common.cuh"

#include <type_traits>

namespace {

using namespace asgd::experts;

constexpr float kTiny = 7.888609052210118e-31f;      // 2^-100: smallest magnitude a block is scaled by
constexpr int kThreads = 256, kWarps = kThreads / 32;

struct Args {
  asgd_quantize_args a;
  int row_blocks, col_blocks;                        // blocks of 128 along K and along M
  float fmax, inv_fmax;
};

template <bool kE5M2> __device__ __forceinline__ unsigned short round2(float x, float y) {
  return __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, kE5M2 ? __NV_E5M2 : __NV_E4M3);
}
template <bool kE5M2> __device__ __forceinline__ unsigned round4(float x, float y, float z, float w) {
  return (unsigned)round2<kE5M2>(x, y) | ((unsigned)round2<kE5M2>(z, w) << 16);
}

// the input row of result row r, its factor, and whether there is one
template <typename T> __device__ __forceinline__ const T* input_row(const asgd_quantize_args& a, long long r, float& factor) {
  factor = 1.f;
  if (r >= a.M) return nullptr;
  long long t = r;
  if (a.source) {
    const int s = a.source[r];
    if (s < 0) return nullptr;
    t = s / a.per_token;
    if (t >= a.rows_x) return nullptr;
    if (a.weights) factor = a.weights[s];
  }
  return reinterpret_cast<const T*>(a.x) + t * a.ldx;
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

// A warp takes a stretch of a row: four 16-byte pieces per lane, all loaded before the first is used.  The four blocks a
// lane has a part in are reduced together: each exchange between lanes folds half of the maxima onto half of the lanes,
// so that a lane ends with one block's maximum, divides once, and hands the result round (9 exchanges and one division
// where four separate reductions take 16 to 20 and four).
template <typename T, bool kVec, bool kE5M2, bool kWeights> __global__ void __launch_bounds__(kThreads) rows_kernel(const Args p) {
  constexpr int V = kPer16<T>, LB = 128 / V, U = 4;      // numbers per piece, lanes per block, pieces per lane
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, K = (int)a.K;
  // the block's warps take neighbouring rows of the same stretch: their scales are neighbours in memory
  const long long r = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int c0 = ((int)blockIdx.y * U * 32 + lane) * V;
  if (r >= a.M) return;
  float factor;
  const T* row = input_row<T>(a, r, factor);
  const bool whole = kVec && ((int)blockIdx.y + 1) * (U * 32 * V) <= K;
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    raw[u] = make_uint4(0, 0, 0, 0);
    if (row) {
      if (whole) raw[u] = *reinterpret_cast<const uint4*>(row + c);
      else if (c < K) raw[u] = load<T, uint4, kVec>(row, c, K);
    }
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
  constexpr int O1 = LB / 2, O2 = LB / 4;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const bool high = lane & O1;
    const float got = __shfl_xor_sync(kAll, high ? m[u] : m[u + 2], O1);
    m[u] = fmaxf(high ? m[u + 2] : m[u], got);
  }
  {
    const bool high = lane & O2;
    const float got = __shfl_xor_sync(kAll, high ? m[0] : m[1], O2);
    m[0] = fmaxf(high ? m[1] : m[0], got);
  }
#pragma unroll
  for (int o = O2 / 2; o > 0; o >>= 1) m[0] = fmaxf(m[0], __shfl_xor_sync(kAll, m[0], o));
  const float best = fmaxf(m[0], kTiny), mine = __fdiv_rn(p.fmax, best);
  if ((lane & (O2 - 1)) == 0) {                          // the block this lane ended with
    const int c = (int)blockIdx.y * U * 32 * V + (((lane & O1) ? 2 : 0) + ((lane & O2) ? 1 : 0)) * 32 * V + (LB == 16 ? (lane & 16) * V : 0);
    if (c < K) a.scale[r * a.scale_row + (c >> 7) * a.scale_block] = __fmul_rn(best, p.inv_fmax);
  }
  unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r * a.ldq;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 32 * V;
    const float inv = __shfl_sync(kAll, mine, (LB == 16 ? lane & 16 : 0) | ((u & 2) ? O1 : 0) | ((u & 1) ? O2 : 0));
    float v[V];
    unpack16<T>(raw[u], v);
    unsigned w[V / 4];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (kWeights ? __fmul_rn(v[i], factor) : v[i]) * inv;
#pragma unroll
    for (int i = 0; i < V; i += 4) w[i / 4] = round4<kE5M2>(v[i], v[i + 1], v[i + 2], v[i + 3]);
    if (whole || (kVec && c + V <= K)) {
      if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<unsigned*>(q + c) = w[0];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) if (c + i < K) q[c + i] = (unsigned char)(w[i / 4] >> (8 * (i & 3)));
    }
  }
}

template <typename T, bool kVec, bool kE5M2> __global__ void __launch_bounds__(kThreads) tile_kernel(const Args p) {
  using Word = typename std::conditional<sizeof(T) == 4, uint4, uint2>::type;      // 4 numbers
  __shared__ __align__(16) unsigned char tile[128 * 128];       // [column][row], 16-byte pieces exchanged by column / 4
  __shared__ float col_max[kWarps][128];
  __shared__ float whole[kWarps];
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, K = (int)a.K;
  const long long m0 = (long long)blockIdx.y * 128;
  const int k0 = (int)blockIdx.x * 128;
  const long long r0 = m0 + 16 * wid;
  const int c = k0 + 4 * lane;
  Word raw[16];
  float factor[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const T* row = input_row<T>(a, r0 + i, factor[i]);
    raw[i] = Word{};
    if (row && c < K) raw[i] = load<T, Word, kVec>(row, c, K);
  }
  float v[16][4];
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[i][j] = element<T>(raw[i], j);
      if (a.weights) v[i][j] = __fmul_rn(v[i][j], factor[i]);
    }
  float one = kTiny;
  if (a.square) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) one = fmaxf(one, fabsf(v[i][j]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) one = fmaxf(one, __shfl_xor_sync(kAll, one, o));
    if (lane == 0) whole[wid] = one;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) one = fmaxf(one, whole[w]);
    if (threadIdx.x == 0) a.scale[blockIdx.y * a.scale_row + blockIdx.x * a.scale_block] = __fmul_rn(one, p.inv_fmax);
  }
  if (a.q) {
    float m[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      m[i] = one;
      if (!a.square)
#pragma unroll
        for (int j = 0; j < 4; ++j) m[i] = fmaxf(m[i], fabsf(v[i][j]));
    }
    if (!a.square) {
      // 16 rows' maxima over 32 lanes by halving: each step folds half of the rows onto the other half of the lanes, so
      // that lane l ends with row l / 2 (16 exchanges instead of 80), and the rows' inverses come from 16 lanes at once
#pragma unroll
      for (int n = 8, o = 16; n > 0; n >>= 1, o >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const bool high = lane & o;
          const float send = high ? m[i] : m[i + n], keep = high ? m[i + n] : m[i];
          m[i] = fmaxf(keep, __shfl_xor_sync(kAll, send, o));
        }
      m[0] = fmaxf(m[0], __shfl_xor_sync(kAll, m[0], 1));
      const long long r = r0 + (lane >> 1);
      if (!(lane & 1) && r < a.M) a.scale[r * a.scale_row + blockIdx.x * a.scale_block] = __fmul_rn(m[0], p.inv_fmax);
    }
    const float mine = __fdiv_rn(p.fmax, m[0]);
    unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r0 * a.ldq + c;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float inv = __shfl_sync(kAll, mine, 2 * i);
      const unsigned w = round4<kE5M2>(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
      if (r0 + i < a.M) {
        if (kVec && c + 4 <= K) *reinterpret_cast<unsigned*>(q + i * a.ldq) = w;
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) if (c + j < K) q[i * a.ldq + j] = (unsigned char)(w >> (8 * j));
      }
    }
  }
  if (!a.qt) return;
  float inv[4];
  if (a.square) {
    inv[0] = inv[1] = inv[2] = inv[3] = __fdiv_rn(p.fmax, one);
  } else {
    float4 m = make_float4(kTiny, kTiny, kTiny, kTiny);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      m.x = fmaxf(m.x, fabsf(v[i][0])); m.y = fmaxf(m.y, fabsf(v[i][1]));
      m.z = fmaxf(m.z, fabsf(v[i][2])); m.w = fmaxf(m.w, fabsf(v[i][3]));
    }
    *reinterpret_cast<float4*>(&col_max[wid][4 * lane]) = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 o = *reinterpret_cast<const float4*>(&col_max[w][4 * lane]);
      m.x = fmaxf(m.x, o.x); m.y = fmaxf(m.y, o.y); m.z = fmaxf(m.z, o.z); m.w = fmaxf(m.w, o.w);
    }
    const float best[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      inv[j] = __fdiv_rn(p.fmax, best[j]);
      if (wid == 0 && c + j < K) a.scale_t[(c + j) * a.scale_t_row + blockIdx.y * a.scale_t_block] = __fmul_rn(best[j], p.inv_fmax);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4 u;
    u.x = round4<kE5M2>(v[0][j] * inv[j], v[1][j] * inv[j], v[2][j] * inv[j], v[3][j] * inv[j]);
    u.y = round4<kE5M2>(v[4][j] * inv[j], v[5][j] * inv[j], v[6][j] * inv[j], v[7][j] * inv[j]);
    u.z = round4<kE5M2>(v[8][j] * inv[j], v[9][j] * inv[j], v[10][j] * inv[j], v[11][j] * inv[j]);
    u.w = round4<kE5M2>(v[12][j] * inv[j], v[13][j] * inv[j], v[14][j] * inv[j], v[15][j] * inv[j]);
    *reinterpret_cast<uint4*>(tile + (4 * lane + j) * 128 + ((wid ^ (lane & 7)) << 4)) = u;
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

template <typename T> void launch(const Args& p, cudaStream_t st) {
  const asgd_quantize_args& a = p.a;
  const bool e5m2 = a.q_type == ASGD_E5M2;
  const bool rows_only = !a.qt && !a.square;
  const int V = rows_only ? kPer16<T> : 4;
  // vector accesses need every row of the input and of the result to start at a whole vector
  const bool vec = aligned(a.x, V * sizeof(T)) && a.ldx % V == 0 && (!a.q || (aligned(a.q, V) && a.ldq % V == 0));
  if (rows_only) {
    const dim3 grid((unsigned)ceil_div(a.M, kWarps), (unsigned)ceil_div(a.K, 32 * V * 4));
    const bool w = a.weights != nullptr;
    const auto k = vec ? (e5m2 ? (w ? rows_kernel<T, true, true, true> : rows_kernel<T, true, true, false>) : (w ? rows_kernel<T, true, false, true> : rows_kernel<T, true, false, false>))
                       : (e5m2 ? (w ? rows_kernel<T, false, true, true> : rows_kernel<T, false, true, false>) : (w ? rows_kernel<T, false, false, true> : rows_kernel<T, false, false, false>));
    k<<<grid, kThreads, 0, st>>>(p);
  } else {
    const auto k = vec ? (e5m2 ? tile_kernel<T, true, true> : tile_kernel<T, true, false>) : (e5m2 ? tile_kernel<T, false, true> : tile_kernel<T, false, false>);
    k<<<dim3((unsigned)p.row_blocks, (unsigned)p.col_blocks), kThreads, 0, st>>>(p);
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
  if (a.M > 0x7fffffffll || a.K > 0x7fff0000ll) return ASGD_EUNSUPPORTED;   // column numbers stay inside 32 bits
  if (a.M == 0 || a.K == 0) return ASGD_OK;
  if ((!a.q && !a.qt) || (a.rows_x > 0 && !a.x) || !aligned(a.x, type_bytes(a.x_type))) return ASGD_EINVAL;
  if (((a.q || a.square) && !a.scale) || (a.qt && !a.square && !a.scale_t)) return ASGD_EINVAL;
  Args p;
  p.a = a;
  const long long rb = ceil_div(a.K, 128), cb = ceil_div(a.M, 128);
  p.row_blocks = (int)rb;
  p.col_blocks = (int)cb;
  p.fmax = a.q_type == ASGD_E4M3 ? 448.f : 57344.f;
  p.inv_fmax = a.q_type == ASGD_E4M3 ? 1.f / 448.f : 1.f / 57344.f;
  // limits of the grid: 65535 tiles along M, or 65535 stretches of a row
  if ((a.qt || a.square) ? cb > 65535 : ceil_div(a.K, 512) > 65535) return ASGD_EUNSUPPORTED;
  with_type(a.x_type, [&](auto e) { launch<decltype(e)>(p, (cudaStream_t)stream); });
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}
