// Product of 8-bit matrices with block scales on the tensor cores: dense, grouped over rows, grouped over the inner
// dimension.  The contract is in include/asgd_experts.h.
//
// A scale belongs to 128 neighbours along K, so the products of one K block go into a fresh accumulator in tensor
// memory (four tcgen05.mma of K = 32), and threads add them, scaled, to sums they keep in registers while the tensor
// cores fill the other accumulator stage.
//
// Here a tile is 128 columns of C (rows of B, the weights: the MMA's M, one per epilogue thread) by BN rows of C (rows
// of A, the tokens: the MMA's N).  Few tokens then cost few columns of the tensor core's tile, and a warp writes 32
// neighbouring numbers of a row of C.
//
// Warp roles: 0 issues the TMA loads (128-byte K blocks of both operands, swizzled, through a ring of slots); 1 issues
// the products; 2 brings the tokens' scales (asynchronous 4-byte copies into the same ring); 4 to 7 read the
// accumulators (tcgen05.ld: one column of C per thread) and keep the sums.  Blocks are persistent and take tiles in
// turn.  Every wait is bounded.
#include "asgd_experts_common.cuh"

#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "asgd_stream.cuh"   // mbarrier helpers

namespace {

using namespace asgd::experts;
using asgd::mbar_expect_tx;
using asgd::mbar_init;
using asgd::mbar_try_wait;
using asgd::smem_u32;

__device__ int g_status;                             // what asgd_experts_sync reports: the smallest (worst) code seen
std::atomic<unsigned> g_wait_limit{asgd::DEFAULT_WAIT_LIMIT};
std::atomic<int> g_withhold{0};

constexpr int kKB = 128;                             // numbers (bytes) of a K block: a 128-byte swizzled row
constexpr int kU = 128;                              // columns of C per tile
constexpr int kThreads = 256;
constexpr size_t kSmemLimit = 227 * 1024;

struct Params {
  int M, N, K, groups, inner, tiles_u, kblocks;
  const float *sa, *sb;
  long long sa_row, sa_block, sb_row, sb_block, sb_group;
  int sb_shift;
  void* c;
  long long ldc, c_group;
  int c_type;
  const int* offsets;
  unsigned idesc, wait_limit;
  int withhold;
};

// ---- tensor-core and copy wrappers ----

__device__ inline void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
// K-major rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 bytes apart
__device__ inline unsigned long long operand_desc(const void* smem) {
  return (unsigned long long)((smem_u32(smem) & 0x3FFFFu) >> 4) | 1ull << 16 | (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ inline void mma_f8(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, bool acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
               ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc) : "memory");
}
__device__ inline void commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ inline void arrive(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ inline void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ inline void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ inline void copy4(float* dst, const float* src, bool there) {       // asynchronous; zero where not there
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ inline void arrive_after_copies(unsigned long long* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 16 columns of the warp's 32 accumulator rows
__device__ inline void tmem_load16(unsigned taddr, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                 "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(taddr) : "memory");
}
__device__ inline void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// A bounded wait that also ends when another warp of the block gave up.
__device__ inline bool wait(unsigned long long* bar, unsigned parity, unsigned limit, int* abort) {
  for (unsigned it = 0; it < limit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 63u && *reinterpret_cast<volatile int*>(abort)) return false;
  }
  *reinterpret_cast<volatile int*>(abort) = 1;
  return false;
}

__device__ inline void store_c(void* c, int type, long long at, float v) {
  if (type == ASGD_F32) reinterpret_cast<float*>(c)[at] = v;
  else if (type == ASGD_BF16) reinterpret_cast<__nv_bfloat16*>(c)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(c)[at] = __float2half_rn(v);
}

// ---- tiles ----

struct Tile {
  int g, u0, v0, v_end, kb0, kb1;
  bool bad;                                          // inner groups whose bounds cut a block
};

__device__ inline void group_bounds(const Params& p, int g, int limit, int& lo, int& hi) {
  lo = 0; hi = limit;
  if (p.offsets) {
    lo = min(max(p.offsets[g], 0), limit);
    hi = min(max(p.offsets[g + 1], lo), limit);
  }
}

// prefix[g]: tiles of the groups before g.  All threads of the block; ends with a barrier.
__device__ inline void count_tiles(const Params& p, int bn, int* prefix, int* warp_part) {
  const int G = max(p.groups, 1), tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, nw = blockDim.x >> 5;
  const int per = (G + blockDim.x - 1) / blockDim.x;
  int mine = 0;
  for (int q = 0; q < per; ++q) {
    const int g = tid * per + q;
    if (g >= G) break;
    int lo = 0, hi = p.M;
    if (p.groups && !p.inner) group_bounds(p, g, p.M, lo, hi);
    const int n = (hi - lo + bn - 1) / bn * p.tiles_u;
    prefix[g] = n;
    mine += n;
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(kAll, inc, o); if (lane >= o) inc += v; }
  if (lane == 31) warp_part[wid] = inc;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wid && w < nw; ++w) before += warp_part[w];
  int run = before + inc - mine;
  for (int q = 0; q < per; ++q) {
    const int g = tid * per + q;
    if (g >= G) break;
    const int n = prefix[g];
    prefix[g] = run;
    run += n;
    if (g == G - 1) prefix[G] = run;
  }
  __syncthreads();
}

__device__ inline Tile find_tile(const Params& p, int bn, const int* prefix, int tile) {
  Tile t;
  int a = 0, b = max(p.groups, 1);
  while (b - a > 1) {                                // the last group that starts at or before the tile
    const int m = (a + b) >> 1;
    if (prefix[m] <= tile) a = m; else b = m;
  }
  t.g = a;
  int lo = 0, hi = p.M;
  if (p.groups && !p.inner) group_bounds(p, a, p.M, lo, hi);
  const int nv = (hi - lo + bn - 1) / bn, at = tile - prefix[a];
  t.u0 = at / nv * kU;                               // neighbouring blocks share a tile of B
  t.v0 = lo + at % nv * bn;
  t.v_end = hi;
  t.kb0 = 0; t.kb1 = p.kblocks;
  t.bad = false;
  if (p.inner) {
    group_bounds(p, a, p.K, lo, hi);
    t.kb0 = lo / kKB;
    t.kb1 = hi > lo ? (hi + kKB - 1) / kKB : t.kb0;
    t.bad = hi > lo && (lo % kKB || (hi % kKB && hi != p.K));
    if (t.bad) t.kb1 = t.kb0;
  }
  return t;
}

// ---- the kernel ----

template <int BN> __host__ __device__ constexpr int slots() { return BN == 128 ? 6 : BN == 64 ? 8 : 10; }
template <int BN> __host__ __device__ constexpr unsigned slot_bytes() { return (kU + BN) * kKB; }
enum { kMaxSlots = 10, B_FULL = 0, B_EMPTY = kMaxSlots, B_SFULL = 2 * kMaxSlots, B_SEMPTY = 3 * kMaxSlots, B_ACCFULL = 4 * kMaxSlots,
       B_ACCEMPTY = B_ACCFULL + 2, B_DRAIN = B_ACCEMPTY + 2, B_COUNT };
template <int BN> __host__ __device__ constexpr size_t smem_bytes() {
  return 1024 + (size_t)slots<BN>() * slot_bytes<BN>() + (size_t)slots<BN>() * BN * 4 + (ASGD_MAX_EXPERTS + 1 + 32) * 4 + B_COUNT * 8 + 64;
}

template <int BN> __global__ void __launch_bounds__(kThreads, 1)
product_kernel(const Params p, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_v) {
  constexpr int S = slots<BN>();
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  float* sv = reinterpret_cast<float*>(ring + (size_t)S * slot_bytes<BN>());           // [slot][BN] scales of the tokens
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(sv + S * BN);
  int* prefix = reinterpret_cast<int*>(bars + B_COUNT);
  int* warp_part = prefix + ASGD_MAX_EXPERTS + 1;
  int* misc = warp_part + 32;                                                            // [0] tensor memory, [1] abort
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  constexpr unsigned kCols = 2 * BN < 32 ? 32 : 2 * BN;

  if (tid == 0) {
    for (int q = 0; q < S; ++q) { mbar_init(bars + B_FULL + q, 1); mbar_init(bars + B_EMPTY + q, 1); mbar_init(bars + B_SFULL + q, 32); mbar_init(bars + B_SEMPTY + q, 4); }
    for (int q = 0; q < 2; ++q) { mbar_init(bars + B_ACCFULL + q, 1); mbar_init(bars + B_ACCEMPTY + q, 4); }
    mbar_init(bars + B_DRAIN, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    misc[1] = 0;
  }
  if (wid == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  count_tiles(p, BN, prefix, warp_part);
  fence_before();
  __syncthreads();
  fence_after();
  const unsigned tmem = (unsigned)misc[0];
  const int tiles = prefix[max(p.groups, 1)];
  int* abort = misc + 1;

  if (wid == 0) {
    if (lane == 0) {
      unsigned it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        const Tile t = find_tile(p, BN, prefix, tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S;
          if (it >= S && !(ok = wait(bars + B_EMPTY + q, (it / S - 1) & 1, p.wait_limit, abort))) break;
          unsigned char* to = ring + (size_t)q * slot_bytes<BN>();
          mbar_expect_tx(bars + B_FULL + q, slot_bytes<BN>());
          if (!(p.withhold && it == 0)) {
            tma_load_3d(to, &map_u, kb * kKB, t.u0, p.inner ? 0 : t.g, bars + B_FULL + q);
            tma_load_3d(to + kU * kKB, &map_v, kb * kKB, t.v0, 0, bars + B_FULL + q);
          }
        }
      }
      if (!ok)                                       // copies in flight land before the block leaves
        for (unsigned q = 0; q < S && q < it; ++q) {
          const unsigned last = (it - 1 - q) / S;    // the slot's last use
          for (unsigned n = 0; n < p.wait_limit && !mbar_try_wait(bars + B_FULL + q, last & 1); ++n) {}
        }
    }
  } else if (wid == 1) {
    if (lane == 0) {
      unsigned it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        const Tile t = find_tile(p, BN, prefix, tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S, stage = it & 1;
          if (it >= 2 && !(ok = wait(bars + B_ACCEMPTY + stage, (it / 2 - 1) & 1, p.wait_limit, abort))) break;
          if (!(ok = wait(bars + B_FULL + q, (it / S) & 1, p.wait_limit, abort))) break;
          fence_after();
          const unsigned long long du = operand_desc(ring + (size_t)q * slot_bytes<BN>()), dv = operand_desc(ring + (size_t)q * slot_bytes<BN>() + kU * kKB);
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) mma_f8(tmem + stage * BN, du + 2 * k4, dv + 2 * k4, p.idesc, k4 != 0);
          commit(bars + B_EMPTY + q);
          commit(bars + B_ACCFULL + stage);
        }
      }
      if (!ok && it) {                               // products in flight end before the tensor memory is freed
        commit(bars + B_DRAIN);
        for (unsigned n = 0; n < p.wait_limit && !mbar_try_wait(bars + B_DRAIN, 0); ++n) {}
      }
    }
  } else if (wid == 2) {
    unsigned it = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      const Tile t = find_tile(p, BN, prefix, tile);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S;
        if (it >= S && !(ok = __all_sync(kAll, wait(bars + B_SEMPTY + q, (it / S - 1) & 1, p.wait_limit, abort)))) break;
#pragma unroll
        for (int c = 0; c < BN; c += 32) {
          const int r = t.v0 + c + lane;
          if (c + lane < BN) copy4(sv + q * BN + c + lane, r < t.v_end ? p.sa + r * p.sa_row + kb * p.sa_block : p.sa, r < t.v_end);
        }
        arrive_after_copies(bars + B_SFULL + q);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (wid >= 4) {
    const int quarter = wid & 3;
    unsigned it = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      const Tile t = find_tile(p, BN, prefix, tile);
      const int u = t.u0 + quarter * 32 + lane;
      const float* su_at = p.sb + (p.inner ? 0 : t.g * p.sb_group) + (long long)(min(u, p.N - 1) >> p.sb_shift) * p.sb_row;
      float acc[BN];
#pragma unroll
      for (int c = 0; c < BN; ++c) acc[c] = 0.f;
      float su_next = t.kb0 < t.kb1 ? __ldg(su_at + t.kb0 * p.sb_block) : 0.f;
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S, stage = it & 1;
        const float su = su_next;
        if (kb + 1 < t.kb1) su_next = __ldg(su_at + (kb + 1) * p.sb_block);
        ok = wait(bars + B_SFULL + q, (it / S) & 1, p.wait_limit, abort) && wait(bars + B_ACCFULL + stage, (it / 2) & 1, p.wait_limit, abort);
        if (!(ok = __all_sync(kAll, ok))) break;
        fence_after();
#pragma unroll
        for (int c0 = 0; c0 < BN; c0 += 16) {
          float v[16];
          tmem_load16(tmem + ((unsigned)(quarter * 32) << 16) + stage * BN + c0, v);
          tmem_wait();
#pragma unroll
          for (int c = 0; c < 16; ++c) acc[c0 + c] = fmaf(v[c] * su, sv[q * BN + c0 + c], acc[c0 + c]);
        }
        fence_before();
        __syncwarp();
        if (lane == 0) { arrive(bars + B_ACCEMPTY + stage); arrive(bars + B_SEMPTY + q); }
      }
      if (!ok) break;
      if (t.bad && lane == 0) atomicMin(&g_status, ASGD_EINVAL);
      if (u < p.N) {
        const long long base = (p.inner ? t.g * p.c_group : 0) + u;
#pragma unroll
        for (int c = 0; c < BN; ++c)
          if (t.v0 + c < t.v_end) store_c(p.c, p.c_type, base + (long long)(t.v0 + c) * p.ldc, t.bad ? __int_as_float(0x7fffffff) : acc[c]);
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
  if (tid == 0 && *reinterpret_cast<volatile int*>(abort)) atomicMin(&g_status, ASGD_ETIMEOUT);
}

// ---- host ----

// rows of 128-byte K blocks of an 8-bit matrix [outer][rows][cols]; what lies beyond is read as zeros
bool encode(CUtensorMap* map, const void* base, long long cols, long long rows, long long outer, long long ld, long long outer_stride, unsigned box_rows) {
  static std::atomic<PFN_cuTensorMapEncodeTiled> known{nullptr};
  PFN_cuTensorMapEncodeTiled f = known.load();
  if (!f) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || !fn) return false;
    f = (PFN_cuTensorMapEncodeTiled)fn;
    known.store(f);
  }
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)outer};
  cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)(outer > 1 ? outer_stride : ld)};
  cuuint32_t box[3] = {kKB, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN> int launch(const asgd_product_args& a, Params p, cudaStream_t st) {
  CUtensorMap map_u{}, map_v{};
  if (p.K > 0) {
    if (!encode(&map_u, a.b, p.K, p.N, p.inner ? 1 : max(p.groups, 1), a.ldb, a.b_group, kU)) return ASGD_EINVAL;
    if (!encode(&map_v, a.a, p.K, p.M, 1, a.lda, 0, BN)) return ASGD_EINVAL;
  }
  p.idesc |= (unsigned)(BN >> 3) << 17 | (unsigned)(kU >> 4) << 24;
  const long long most = (ceil_div(p.M, BN) * (p.inner ? max(p.groups, 1) : 1) + (p.inner ? 0 : p.groups)) * p.tiles_u;
  if (most > 0x7fffffffll) return ASGD_EUNSUPPORTED;
  static_assert(smem_bytes<BN>() <= kSmemLimit, "shared memory");
  if (cudaFuncSetAttribute(product_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<BN>()) != cudaSuccess) return ASGD_ECUDA;
  product_kernel<BN><<<(unsigned)min(most, (long long)kSMs), kThreads, smem_bytes<BN>(), st>>>(p, map_u, map_v);
  return cudaGetLastError() == cudaSuccess ? ASGD_OK : ASGD_ECUDA;
}

}  // namespace

extern "C" int asgd_product(const asgd_product_args* args, void* stream) {
  if (!args) return ASGD_EINVAL;
  const asgd_product_args& a = *args;
  if (a.M < 0 || a.N < 0 || a.K < 0 || a.groups < 0 || (a.inner != 0 && a.inner != 1) || (a.b_square != 0 && a.b_square != 1)) return ASGD_EINVAL;
  if (!eight_bit_type(a.a_type) || !eight_bit_type(a.b_type) || !float_type(a.c_type)) return ASGD_EINVAL;
  if ((a.groups > 0) != (a.offsets != nullptr) || (a.inner && !a.groups)) return ASGD_EINVAL;
  if (a.lda < a.K || a.ldb < a.K || a.ldc < a.N || (a.K > 0 && (a.lda % 16 || a.ldb % 16))) return ASGD_EINVAL;
  if (a.M > 0x7fffffffll || a.N > 0x7fffffffll || a.K > 0x7fffff00ll || a.groups > ASGD_MAX_EXPERTS) return ASGD_EUNSUPPORTED;
  if (a.M == 0 || a.N == 0) return ASGD_OK;
  if (!a.c || !aligned(a.c, type_bytes(a.c_type))) return ASGD_EINVAL;
  if (a.K > 0 && (!a.a || !a.b || !a.a_scale || !a.b_scale || !aligned(a.a, 16) || !aligned(a.b, 16) || !aligned(a.a_scale, 4) || !aligned(a.b_scale, 4))) return ASGD_EINVAL;
  if (a.groups > 1 && !a.inner && (a.b_group % 16 || a.b_group < 0)) return ASGD_EINVAL;
  Params p;
  p.M = (int)a.M; p.N = (int)a.N; p.K = (int)a.K; p.groups = a.groups; p.inner = a.inner;
  p.tiles_u = (int)ceil_div(a.N, kU);
  p.kblocks = (int)ceil_div(a.K, kKB);
  p.sa = a.a_scale; p.sa_row = a.a_scale_row; p.sa_block = a.a_scale_block;
  p.sb = a.b_scale; p.sb_row = a.b_scale_row; p.sb_block = a.b_scale_block; p.sb_group = a.b_scale_group;
  p.sb_shift = a.b_square ? 7 : 0;
  p.c = a.c; p.ldc = a.ldc; p.c_group = a.c_group; p.c_type = a.c_type;
  p.offsets = a.offsets;
  // fp32 accumulators; formats of the MMA's first operand (B) and second (A): 0 = E4M3, 1 = E5M2
  p.idesc = 1u << 4 | (a.b_type == ASGD_E5M2 ? 1u : 0u) << 7 | (a.a_type == ASGD_E5M2 ? 1u : 0u) << 10;
  p.wait_limit = g_wait_limit.load();
  p.withhold = g_withhold.load();
  cudaStream_t st = (cudaStream_t)stream;
  const long long rows = a.groups && !a.inner ? ceil_div(a.M, a.groups) : a.M;     // rows of a group, on average
  if (rows <= 16) return launch<16>(a, p, st);
  if (rows <= 32) return launch<32>(a, p, st);
  if (rows <= 64) return launch<64>(a, p, st);
  return launch<128>(a, p, st);
}

extern "C" int asgd_experts_sync(void* stream) {
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return ASGD_ECUDA;
  int status = 0;
  const int none = 0;
  if (cudaMemcpyFromSymbol(&status, g_status, sizeof(int)) != cudaSuccess) return ASGD_ECUDA;
  if (status && cudaMemcpyToSymbol(g_status, &none, sizeof(int)) != cudaSuccess) return ASGD_ECUDA;
  return status;
}

extern "C" int asgd_product_set_wait_drill(uint32_t wait_limit, int32_t withhold) {
  if (wait_limit == 0) return ASGD_EINVAL;
  g_wait_limit.store(wait_limit);
  g_withhold.store(withhold != 0);
  return ASGD_OK;
}
