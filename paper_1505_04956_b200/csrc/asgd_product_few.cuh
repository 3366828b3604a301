// The kernel of asgd_product for few rows of A (per group).
//
// A tile is 128 columns of C (rows of B, the weights: the MMA's M, one per epilogue thread) by BN rows of C (rows of
// A, the tokens: the MMA's N).  Few tokens then cost few columns of the tensor core's tile, and a warp writes 32
// neighbouring numbers of a row of C.
//
// Warp roles: 0 issues the TMA loads (128-byte K blocks of both operands, swizzled, through a ring of slots); 1 issues
// the products; 2 brings the tokens' scales (asynchronous 4-byte copies into the same ring); 4 to 7 read the
// accumulators (tcgen05.ld: one column of C per thread) and keep the sums.  Blocks are persistent and take tiles in
// turn.  Every wait is bounded.
#pragma once

#include "asgd_product_common.cuh"

namespace {

constexpr int kU = 128;                              // columns of C per tile
constexpr int kThreads = 256;
constexpr int kNoBand = 1 << 30;

template <int BN> __host__ __device__ constexpr int slots() { return BN == 128 ? 6 : BN == 64 ? 8 : 10; }
template <int BN> __host__ __device__ constexpr unsigned slot_bytes() { return (kU + BN) * kKB; }
enum { kMaxSlots = 10, B_FULL = 0, B_EMPTY = kMaxSlots, B_SFULL = 2 * kMaxSlots, B_SEMPTY = 3 * kMaxSlots, B_ACCFULL = 4 * kMaxSlots,
       B_ACCEMPTY = B_ACCFULL + 2, B_DRAIN = B_ACCEMPTY + 2, B_COUNT };
template <int BN> __host__ __device__ constexpr size_t smem_bytes() {
  return 1024 + (size_t)slots<BN>() * slot_bytes<BN>() + (size_t)slots<BN>() * BN * 4 + (ASGD_MAX_EXPERTS + 1 + 32) * 4 + B_COUNT * 8 + 64;
}

template <int BN> __global__ void __launch_bounds__(kThreads, 1)
product_few_kernel(const Params p, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_v) {
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
        const Tile t = find_tile(p, BN, kU, kNoBand, prefix, tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S;
          if (it >= S && !(ok = wait(bars + B_EMPTY + q, (it / S - 1) & 1, p.wait_limit, abort))) break;
          unsigned char* to = ring + (size_t)q * slot_bytes<BN>();
          mbar_expect_tx(bars + B_FULL + q, slot_bytes<BN>());
          if (!(p.withhold && it == 0)) {
            tma_load_3d(to, &map_u, kb * kKB, t.n0, p.inner ? 0 : t.g, bars + B_FULL + q);
            tma_load_3d(to + kU * kKB, &map_v, kb * kKB, t.m0, 0, bars + B_FULL + q);
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
        const Tile t = find_tile(p, BN, kU, kNoBand, prefix, tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S, stage = it & 1;
          if (it >= 2 && !(ok = wait(bars + B_ACCEMPTY + stage, (it / 2 - 1) & 1, p.wait_limit, abort))) break;
          if (!(ok = wait(bars + B_FULL + q, (it / S) & 1, p.wait_limit, abort))) break;
          fence_after();
          const unsigned long long du = operand_desc(ring + (size_t)q * slot_bytes<BN>()), dv = operand_desc(ring + (size_t)q * slot_bytes<BN>() + kU * kKB);
          const int steps = steps_of(t, kb);
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) if (k4 < steps) mma_f8(tmem + stage * BN, du + 2 * k4, dv + 2 * k4, p.idesc, k4 != 0);
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
      const Tile t = find_tile(p, BN, kU, kNoBand, prefix, tile);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S;
        if (it >= S && !(ok = __all_sync(kAll, wait(bars + B_SEMPTY + q, (it / S - 1) & 1, p.wait_limit, abort)))) break;
#pragma unroll
        for (int c = 0; c < BN; c += 32) {
          const int r = t.m0 + c + lane;
          if (c + lane < BN) copy4(sv + q * BN + c + lane, r < t.m_end ? p.sa + r * p.sa_row + kb * p.sa_block : p.sa, r < t.m_end);
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
      const Tile t = find_tile(p, BN, kU, kNoBand, prefix, tile);
      const int u = t.n0 + quarter * 32 + lane;
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
          if (t.m0 + c < t.m_end) store_c(p.c, p.c_type, base + (long long)(t.m0 + c) * p.ldc, t.bad ? __int_as_float(0x7fffffff) : acc[c]);
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols));
  if (tid == 0 && *reinterpret_cast<volatile int*>(abort)) atomicMin(&g_status, ASGD_ETIMEOUT);
}

}  // namespace
