// Rounding to 8-bit floating point with a scale for each block of 128, of rows taken in order or gathered, as they are
// and transposed.  The contract is in include/asgd_experts.h.
//
// Both kernels read a number once and keep it in registers from the search for the block's largest magnitude to the
// rounding; HBM is the bound.  A row's blocks alone (rows_kernel): a warp takes a stretch of a row, its loads all in
// flight before the first is used.  The transposed matrix too, or 128 x 128 blocks (tile_kernel): a thread block takes
// a 128 x 128 tile, a thread 16 neighbouring rows of 4 columns, so that 16 rounded numbers of a column are one 16-byte
// store into the transposed tile in shared memory.
#include "asgd_experts_common.cuh"

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

// V numbers of a row from column c; numbers beyond K are zeros
template <typename T, int V, bool kVec> __device__ __forceinline__ void load(const T* row, long long c, long long K, float (&v)[V]) {
  if (kVec && c + V <= K) {
    if constexpr (sizeof(T) * V == 16) {
      unpack16<T>(*reinterpret_cast<const uint4*>(row + c), v);
    } else {
      static_assert(sizeof(T) * V == 8, "8 or 16 bytes");
      const uint2 u = *reinterpret_cast<const uint2*>(row + c);
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = Elem<T>::to_f(e[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = c + i < K ? Elem<T>::to_f(row[c + i]) : 0.f;
  }
}

template <typename T, bool kVec, bool kE5M2> __global__ void __launch_bounds__(kThreads) rows_kernel(const Args p) {
  constexpr int V = kPer16<T>, LB = 128 / V, U = 4;      // numbers per lane, lanes per block, loads in flight per lane
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const long long span = 32 * V * U, segs = (a.K + span - 1) / span;
  // the block's warps take neighbouring rows of the same stretch: their scales are neighbours in memory
  const long long r = (long long)blockIdx.x / segs * kWarps + wid, c0 = (long long)blockIdx.x % segs * span;
  if (r >= a.M) return;
  float factor;
  const T* row = input_row<T>(a, r, factor);
  float v[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long c = c0 + (u * 32 + lane) * V;
    if (row && c < a.K) load<T, V, kVec>(row, c, a.K, v[u]);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) v[u][i] = 0.f;
  }
  unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + r * a.ldq;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long c = c0 + (u * 32 + lane) * V;
    float m = kTiny;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (a.weights) v[u][i] = __fmul_rn(v[u][i], factor);
      m = fmaxf(m, fabsf(v[u][i]));
    }
#pragma unroll
    for (int o = LB / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
    const float inv = __fdiv_rn(p.fmax, m);
    if (c < a.K) {
      if ((lane & (LB - 1)) == 0) a.scale[r * a.scale_row + (c >> 7) * a.scale_block] = __fmul_rn(m, p.inv_fmax);
      unsigned w[V / 4];
#pragma unroll
      for (int i = 0; i < V; i += 4) w[i / 4] = round4<kE5M2>(v[u][i] * inv, v[u][i + 1] * inv, v[u][i + 2] * inv, v[u][i + 3] * inv);
      if (kVec && c + V <= a.K) {
        if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<unsigned*>(q + c) = w[0];
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) if (c + i < a.K) q[c + i] = (unsigned char)(w[i / 4] >> (8 * (i & 3)));
      }
    }
  }
}

template <typename T, bool kVec, bool kE5M2> __global__ void __launch_bounds__(kThreads) tile_kernel(const Args p) {
  __shared__ __align__(16) unsigned char tile[128 * 128];       // [column][row], 16-byte pieces exchanged by column / 4
  __shared__ float col_max[kWarps][128];
  __shared__ float whole[kWarps];
  const asgd_quantize_args& a = p.a;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  const long long m0 = (long long)blockIdx.y * 128, k0 = (long long)blockIdx.x * 128;
  const long long r0 = m0 + 16 * wid, c = k0 + 4 * lane;
  float v[16][4];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float factor;
    const T* row = input_row<T>(a, r0 + i, factor);
    if (row) load<T, 4, kVec>(row, c, a.K, v[i]);
    else { v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0.f; }
    if (a.weights)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = __fmul_rn(v[i][j], factor);
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
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float m = one;
      if (!a.square) {
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, fabsf(v[i][j]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
      }
      const float inv = __fdiv_rn(p.fmax, m);
      if (r0 + i < a.M) {
        if (!a.square && lane == 0) a.scale[(r0 + i) * a.scale_row + blockIdx.x * a.scale_block] = __fmul_rn(m, p.inv_fmax);
        unsigned char* q = reinterpret_cast<unsigned char*>(a.q) + (r0 + i) * a.ldq;
        const unsigned w = round4<kE5M2>(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
        if (kVec && c + 4 <= a.K) *reinterpret_cast<unsigned*>(q + c) = w;
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) if (c + j < a.K) q[c + j] = (unsigned char)(w >> (8 * j));
      }
    }
  }
  if (!a.qt) return;
  float inv[4];
  if (a.square) {
    inv[0] = inv[1] = inv[2] = inv[3] = __fdiv_rn(p.fmax, one);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float m = kTiny;
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(v[i][j]));
      col_max[wid][4 * lane + j] = m;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float m = kTiny;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, col_max[w][4 * lane + j]);
      inv[j] = __fdiv_rn(p.fmax, m);
      if (wid == 0 && c + j < a.K) a.scale_t[(c + j) * a.scale_t_row + blockIdx.y * a.scale_t_block] = __fmul_rn(m, p.inv_fmax);
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
    if (k0 + col >= a.K) continue;
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
    const long long span = 32 * V * 4, blocks = ceil_div(a.K, span) * ceil_div(a.M, kWarps);
    const auto k = vec ? (e5m2 ? rows_kernel<T, true, true> : rows_kernel<T, true, false>) : (e5m2 ? rows_kernel<T, false, true> : rows_kernel<T, false, false>);
    k<<<(unsigned)blocks, kThreads, 0, st>>>(p);
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
  if (a.M > 0x7fffffffll || a.K > 0x7fffffffll) return ASGD_EUNSUPPORTED;
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
  // limits of the grid: 65535 tiles along M, 2^31 - 1 blocks of rows
  if ((a.qt || a.square) ? cb > 65535 : ceil_div(a.K, 512) * ceil_div(a.M, kWarps) > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  with_type(a.x_type, [&](auto e) { launch<decltype(e)>(p, (cudaStream_t)stream); });
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}
