// The kernel of asgd_product for few rows of A (per group), or few tiles of C.
//
// A tile is 128 columns of C (rows of B, the weights: the MMA's M, one per epilogue thread) by BN rows of C (rows of
// A, the tokens: the MMA's N).  Few tokens then cost few columns of the tensor core's tile, and a warp writes 32
// neighbouring numbers of a row of C.  The weights' bytes are the bound; a tile's products alternate between four
// accumulator stages, so that the copies never wait for the sums (256 rows over 64 experts of 2048 x 2048, some 55 of them
// with rows: 43 us, about 5.5 TB/s of weights; with two stages and two commits a K block 60).
//
// With fewer tiles than SMs a cluster of blocks shares a tile: each takes a stretch of the K blocks, leaves its sums in
// its shared memory (where the ring was), and adds up its share of the tile's rows from all the cluster's, in the
// blocks' order, so that the result does not depend on timing (5 rows by 4096 x 4096: 8.5 us
// in clusters of four; an earlier form with a block per tile took 22).
//
// Warp roles: 0 issues the TMA loads (128-byte K blocks of both operands, swizzled, through a ring of slots); 1 and 3
// issue the products, K blocks in turn (a commit holds its thread for several hundred cycles), one commit per K block,
// which says "the slot is free" and "the accumulator is full"; 2 brings the scales (asynchronous copies of 16 or 4 bytes; a load
// into registers would hold the reading warps); the warps from 4 on read the accumulators (tcgen05.ld: one column of C per thread; with 64 or
// more tokens two warps share a column's rows) and keep the sums.  Blocks are persistent and take tiles in turn.  Every
// wait is bounded.
#pragma once

#include "asgd_product_common.cuh"

namespace {

constexpr int kU = 128;                              // columns of C per tile
constexpr int kNoBand = 1 << 30;
constexpr int kAccStages = 4;
constexpr int kMaxSplit = 8;                         // blocks that share a tile

template <int BN> struct Few {
  static constexpr int kSlots = BN == 128 ? 6 : BN == 64 ? 8 : 10;     // even: a slot always meets the same issuing thread
  static constexpr unsigned kSlotBytes = (kU + BN) * kKB;
  static constexpr int kShare = BN >= 64 ? 2 : 1;                       // warps that share a column's rows of C
  static constexpr int kRows = BN / kShare;
  static constexpr int kThreads = 128 + 128 * kShare;
  static constexpr unsigned kCols = kAccStages * BN < 32 ? 32 : kAccStages * BN;
  enum { FULL = 0, DONE = kSlots, SFULL = 2 * kSlots, SEMPTY = 3 * kSlots, ACCEMPTY = 4 * kSlots, DRAIN = ACCEMPTY + kAccStages, COUNT = DRAIN + 2 };
  static constexpr int kScales = BN + kU;                               // of a slot: the tokens', then the columns'
  static constexpr size_t kSmem = 1024 + (size_t)kSlots * kSlotBytes + (size_t)kSlots * kScales * 4 + COUNT * 8 + sizeof(Groups) + 64;
  static_assert(kSmem <= kSmemLimit, "shared memory");
  static_assert((size_t)BN * kU * 4 <= (size_t)kSlots * kSlotBytes, "a block's sums fit where the ring was");
};

__device__ inline unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ inline unsigned cluster_size() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ inline void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ inline float4 load_cluster4(unsigned addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// kSplit: launched in clusters, a tile per cluster
template <int BN, bool kSplit> __global__ void __launch_bounds__(Few<BN>::kThreads, 1)
product_few_kernel(const Params p, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_v) {
  using F = Few<BN>;
  constexpr int S = F::kSlots;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  float* scales = reinterpret_cast<float*>(ring + (size_t)S * F::kSlotBytes);          // [slot][kScales]
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(scales + S * F::kScales);
  Groups& gs = *reinterpret_cast<Groups*>(bars + F::COUNT);
  int* misc = reinterpret_cast<int*>(&gs + 1);                                          // [0] tensor memory, [1] abort, [2] copies issued
  int* abort = misc + 1;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = kSplit ? (int)cluster_rank() : 0, share = kSplit ? (int)cluster_size() : 1;
  const int first = (int)blockIdx.x / share, step = (int)gridDim.x / share;

  if (tid == 0) {
    prefetch_map(&map_u);
    prefetch_map(&map_v);
    for (int q = 0; q < S; ++q) {
      mbar_init(bars + F::FULL + q, 1); mbar_init(bars + F::DONE + q, 1);
      mbar_init(bars + F::SFULL + q, 32); mbar_init(bars + F::SEMPTY + q, 4 * F::kShare);
    }
    for (int q = 0; q < kAccStages; ++q) mbar_init(bars + F::ACCEMPTY + q, 4 * F::kShare);
    for (int q = 0; q < 2; ++q) mbar_init(bars + F::DRAIN + q, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    misc[1] = 0;
  }
  if (wid == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "r"(F::kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  wait_for_stream();                                 // what comes before reads nothing of the call's but its arguments
  count_tiles(p, BN, gs);
  fence_before();
  __syncthreads();
  fence_after();
  const unsigned tmem = (unsigned)misc[0];
  const int tiles = gs.prefix[max(p.groups, 1)];
  // a tile's K blocks, or the block's stretch of them
  auto tile_at = [&](int tile) {
    Tile t = find_tile(p, BN, kU, kNoBand, gs, tile);
    if (kSplit) {
      const int n = t.kb1 - t.kb0, from = t.kb0;
      t.kb0 = from + n * rank / share;
      t.kb1 = from + n * (rank + 1) / share;
    }
    return t;
  };

  if (wid == 0) {
    if (lane == 0) {
      unsigned it = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += step) {
        const Tile t = tile_at(tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S;
          if (it >= S && !(ok = wait(bars + F::DONE + q, (it / S - 1) & 1, p.wait_limit, abort))) break;
          unsigned char* to = ring + (size_t)q * F::kSlotBytes;
          mbar_expect_tx(bars + F::FULL + q, F::kSlotBytes);
          if (!(p.withhold && it == 0)) {
            tma_load_3d(to, &map_u, kb * kKB, t.n0, p.inner ? 0 : t.g, bars + F::FULL + q);
            tma_load_3d(to + kU * kKB, &map_v, kb * kKB, t.m0, 0, bars + F::FULL + q);
          }
        }
      }
      misc[2] = (int)it;                             // K blocks whose copies were issued
    }
  } else if (wid == 1 || wid == 3) {
    if (lane == 0) {
      const unsigned me = (unsigned)wid >> 1;
      unsigned it = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += step) {
        const Tile t = tile_at(tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          if ((it & 1) != me) continue;
          const unsigned q = it % S, stage = it % kAccStages;
          if (!(ok = wait(bars + F::FULL + q, (it / S) & 1, p.wait_limit, abort))) break;
          const unsigned long long du = operand_desc(ring + (size_t)q * F::kSlotBytes), dv = operand_desc(ring + (size_t)q * F::kSlotBytes + kU * kKB);
          const int steps = steps_of(t, kb);
          if (it >= kAccStages && !(ok = wait(bars + F::ACCEMPTY + stage, (it / kAccStages - 1) & 1, p.wait_limit, abort))) break;
          fence_after();
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) if (k4 < steps) mma_f8(tmem + stage * BN, du + 2 * k4, dv + 2 * k4, p.idesc, k4 != 0);
          commit(bars + F::DONE + q);
        }
      }
    }
  } else if (wid == 2) {
    unsigned it = 0;
    bool ok = true;
    for (int tile = first; tile < tiles && ok; tile += step) {
      const Tile t = tile_at(tile);
      const float* from = p.sb + (p.inner ? 0 : t.g * p.sb_group);
      ScaleRows<kU> cols;
      ScaleRows<BN> rows;
      cols.start(from + (t.n0 >> p.sb_shift) * p.sb_row, p.sb_shift ? 0 : p.sb_row, p.sb_block, t.kb0, 0, p.sb_shift ? kU : p.N - t.n0, lane);
      rows.start(p.sa, p.sa_row, p.sa_block, t.kb0, t.m0, t.m_end, lane);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S;
        if (it >= S && !(ok = __all_sync(kAll, wait(bars + F::SEMPTY + q, (it / S - 1) & 1, p.wait_limit, abort)))) break;
        float* to = scales + q * F::kScales;
        cols.copy(to + BN, lane);
        rows.copy(to, lane);
        arrive_after_copies(bars + F::SFULL + q);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    const int quarter = wid & 3, c_first = ((wid - 4) >> 2) * F::kRows;                  // the warp's columns and rows of C
    const unsigned at_tmem = tmem + ((unsigned)(quarter * 32) << 16) + c_first;
    unsigned it = 0;
    bool ok = true;
    for (int tile = first; tile < tiles && ok; tile += step) {
      const Tile t = tile_at(tile);
      const int u = t.n0 + quarter * 32 + lane;
      float acc[F::kRows];
#pragma unroll
      for (int c = 0; c < F::kRows; ++c) acc[c] = 0.f;
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S, stage = it % kAccStages;
        ok = wait(bars + F::SFULL + q, (it / S) & 1, p.wait_limit, abort) && wait(bars + F::DONE + q, (it / S) & 1, p.wait_limit, abort);
        if (!(ok = __all_sync(kAll, ok))) break;
        fence_after();
        const float su = scales[q * F::kScales + BN + quarter * 32 + lane];
        const float4* scale = reinterpret_cast<const float4*>(scales + q * F::kScales + c_first);
        float v[2][16];
        tmem_load16(at_tmem + stage * BN, v[0]);
#pragma unroll
        for (int c0 = 0; c0 < F::kRows; c0 += 16) {
          tmem_wait();
          if (c0 + 16 < F::kRows) tmem_load16(at_tmem + stage * BN + c0 + 16, v[(c0 / 16 + 1) & 1]);
          else {
            fence_before();
            __syncwarp();
            if (lane == 0) arrive(bars + F::ACCEMPTY + stage);
          }
#pragma unroll
          for (int c = 0; c < 16; c += 4) {
            const float4 f = scale[(c0 + c) / 4];
            const float* w = v[(c0 / 16) & 1] + c;
            acc[c0 + c] = fmaf(w[0] * su, f.x, acc[c0 + c]);
            acc[c0 + c + 1] = fmaf(w[1] * su, f.y, acc[c0 + c + 1]);
            acc[c0 + c + 2] = fmaf(w[2] * su, f.z, acc[c0 + c + 2]);
            acc[c0 + c + 3] = fmaf(w[3] * su, f.w, acc[c0 + c + 3]);
          }
        }
        __syncwarp();
        if (lane == 0) arrive(bars + F::SEMPTY + q);
      }
      if (!ok) break;
      if (t.bad && lane == 0) atomicMin(&g_status, ASGD_EINVAL);
      if (kSplit) {
        // every copy into the ring has been read: the products that read them are complete
        float* sums = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int c = 0; c < F::kRows; ++c) sums[(c_first + c) * kU + quarter * 32 + lane] = t.bad ? __int_as_float(0x7fffffff) : acc[c];
      } else if (u < p.N) {
        const long long base = (p.inner ? t.g * p.c_group : 0) + u;
#pragma unroll
        for (int c = 0; c < F::kRows; ++c) {
          const int m = t.m0 + c_first + c;
          if (m < t.m_end) store_c(p.c, p.c_type, base + (long long)m * p.ldc, t.bad ? __int_as_float(0x7fffffff) : acc[c]);
        }
      }
    }
  }
  __syncwarp();
  fence_before();
  if (kSplit) {
    cluster_sync();
    if (first < tiles && !*reinterpret_cast<volatile int*>(abort)) {
      const Tile t = find_tile(p, BN, kU, kNoBand, gs, first);
      const int rows = min(BN, t.m_end - t.m0), cols = min(kU, p.N - t.n0);
      const long long base = (p.inner ? t.g * p.c_group : 0) + t.n0;
      unsigned from[kMaxSplit];
#pragma unroll
      for (int r = 0; r < kMaxSplit; ++r) from[r] = in_block(ring, r < share ? r : 0);
      // four neighbouring columns per thread and turn
      for (int e = rows * rank / share * (kU / 4) + tid; e < rows * (rank + 1) / share * (kU / 4); e += F::kThreads) {
        float4 s[kMaxSplit];
#pragma unroll
        for (int r = 0; r < kMaxSplit; ++r) if (r < share) s[r] = load_cluster4(from[r] + e * 16);
        float4 sum = s[0];
#pragma unroll
        for (int r = 1; r < kMaxSplit; ++r) if (r < share) { sum.x += s[r].x; sum.y += s[r].y; sum.z += s[r].z; sum.w += s[r].w; }
        const int u = e % (kU / 4) * 4;
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
        const long long at = base + (long long)(t.m0 + e / (kU / 4)) * p.ldc + u;
#pragma unroll
        for (int i = 0; i < 4; ++i) if (u + i < cols) store_c(p.c, p.c_type, at + i, v[i]);
      }
    }
    cluster_sync();                                  // no block leaves while another reads its sums
  } else {
    __syncthreads();
  }
  fence_after();
  if (*reinterpret_cast<volatile int*>(abort)) {     // a wait ran out: what is in flight ends first
    if (wid == 0 && lane == 0) {
      const unsigned issued = (unsigned)misc[2];
      for (unsigned q = 0; q < S && q < issued; ++q) wait_in_flight(bars + F::FULL + q, ((issued - 1 - q) / S) & 1, p.wait_limit);      // a slot's last use
    } else if ((wid == 1 || wid == 3) && lane == 0) {
      commit(bars + F::DRAIN + (wid >> 1));
      wait_in_flight(bars + F::DRAIN + (wid >> 1), 0, p.wait_limit);
    }
    __syncthreads();
    fence_after();
  }
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::kCols));
  if (tid == 0 && *reinterpret_cast<volatile int*>(abort)) atomicMin(&g_status, ASGD_ETIMEOUT);
}

}  // namespace
