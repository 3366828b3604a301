// The kernel of asgd_product4 for many rows of A (per group): a pair of thread blocks on neighbouring SMs takes a tile of 256
// rows by NT columns of C.
//
// tcgen05.mma of a pair (cta_group::2, kind::mxf4) multiplies 256 rows of A by NT rows of B; each SM holds half of either
// operand and the scales of its rows of A and of all of the tile's rows of B.  The sums of a tile stay in tensor memory until
// its last K block.  Scales come and are turned as in asgd_product4_few.cuh, 512 numbers of K at a time, through slots of their own.
//
// What bounds it: a K block of 256 numbers is 35 KB per SM out of L2 for 2 x 256 x 128 x 256 operations, and L2 gives some 9 TB/s in all: 8192^3 takes
// 250 us (4.4 PFLOP/s), without its copies 162, without its stores 217.  So a tile is as wide as it can be: NT = 256 leaves no room for a second tile's
// sums, and the readers take a tile's sums into registers at once so that the next tile's products begin; NT = 224 with two tiles' sums, whose
// way out is hidden whole, takes 278 (16384 rows over 32 of 2744 x 2080: 94 us, this way 87).  Five slots of operands and one piece of a warp's stage (four
// slots and two pieces: 251 and 89); other orders of the tiles (bands of 4 to 16 rows of them) are within 2 %.
//
// Warp roles in each block: 0 issues the copies (the halves of the operands report to the first block's barrier, the scales to
// the block's own); 1, in the first block, issues the products and the scales' copies into both SMs' tensor memory; 2 and 3 turn the
// scales; 4 to 11 take C out, a row per thread and half of the columns per warp, through shared memory (store_rows).
#pragma once

#include "asgd_product4_few.cuh"
#include "asgd_product_pair.cuh"

namespace {

constexpr int kPair4Slots = 5, kScaleSlots = 4;      // K blocks of operands, units of scales
constexpr int kPair4Pieces = 1;                      // of a warp's stage on the way to C
constexpr unsigned kScaleSlotBytes = 3 * kTurned;    // the block's rows of A, the first 128 rows of B, the others
enum { Q_FULL = 0, Q_DONE = kPair4Slots, Q_SFULL = 2 * kPair4Slots, Q_TURNED = Q_SFULL + kScaleSlots, Q_SDONE = Q_TURNED + kScaleSlots, Q_ACCFULL = Q_SDONE + kScaleSlots,
       Q_ACCEMPTY = Q_ACCFULL + 2, Q_DRAIN = Q_ACCEMPTY + 2, Q_COUNT = Q_DRAIN + 1 };

template <int NT> struct Pair4 {
  static constexpr int kHalfCols = NT / 2;           // rows of B per block
  static constexpr unsigned kSlotBytes = (kHalf + kHalfCols) * kKB;
  static constexpr unsigned kScalesCopied = (kHalf + NT) * 16;
  static constexpr int kStages = 2 * NT + 48 <= 512 ? 2 : 1;
  static constexpr unsigned kScaleCols = kStages * NT;
  static constexpr size_t kSmem = 1024 + (size_t)kPair4Slots * kSlotBytes + kScaleSlots * kScaleSlotBytes + 8 * kPair4Pieces * kPieceBytes + Q_COUNT * 8 + sizeof(Groups) + 64;
  static_assert(kScaleCols + 48 <= 512 && NT % 32 == 0 && NT > 128 && NT <= 256 && kHalfCols % 8 == 0, "tile");
  static_assert(kSmem <= kSmemLimit, "shared memory");
};

__device__ inline void copy_scales_pair(unsigned tmem, unsigned long long desc) {          // in both blocks, from the same place of each
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ inline void mma_f4_pair(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sa, unsigned sb, bool acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
               ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)acc) : "memory");
}
// what the warp has written to shared memory is known to whoever waits for the barrier in the other block
__device__ inline void arrive_release_cluster(unsigned bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ inline bool try_wait_cluster(unsigned long long* bar, unsigned parity) {
  unsigned ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ inline bool wait_cluster(unsigned long long* bar, unsigned parity, unsigned limit, int* abort) {      // as wait()
  for (unsigned it = 0; it < limit; ++it) {
    if (try_wait_cluster(bar, parity)) return true;
    if ((it & 63u) == 63u && *reinterpret_cast<volatile int*>(abort)) return false;
  }
  *reinterpret_cast<volatile int*>(abort) = 1;
  return false;
}

template <int NT> __global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
product4_pair_kernel(const Params4 p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                     const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb, const __grid_constant__ CUtensorMap map_c) {
  using P4 = Pair4<NT>;
  constexpr int S = kPair4Slots;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned char* scales = ring + (size_t)S * P4::kSlotBytes;
  unsigned char* stages = scales + kScaleSlots * kScaleSlotBytes;
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(stages + 8 * kPair4Pieces * kPieceBytes);
  Groups& gs = *reinterpret_cast<Groups*>(bars + Q_COUNT);
  int* misc = reinterpret_cast<int*>(&gs + 1);       // [0] tensor memory, [1] abort, [2, 3] K blocks whose copies each block has issued, [4] one of the blocks gave up, [5] units of scales this one has asked for
  int* abort = misc + 1;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const unsigned rank = rank_in_pair();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int blocks = (p.K + kKB - 1) / kKB;          // of 128 bytes; a unit has two, the last one of a row one or two

  if (tid == 0) {
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    prefetch_map(&map_sa);
    prefetch_map(&map_sb);
    if (p.c_by_map) prefetch_map(&map_c);
    for (int q = 0; q < S; ++q) { mbar_init(bars + Q_FULL + q, 1); mbar_init(bars + Q_DONE + q, 1); }
    for (int q = 0; q < kScaleSlots; ++q) { mbar_init(bars + Q_SFULL + q, 1); mbar_init(bars + Q_TURNED + q, rank ? 2 : 3); mbar_init(bars + Q_SDONE + q, 1); }
    for (int q = 0; q < 2; ++q) { mbar_init(bars + Q_ACCFULL + q, 1); mbar_init(bars + Q_ACCEMPTY + q, 16); }
    mbar_init(bars + Q_DRAIN, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int q = 1; q < 6; ++q) misc[q] = 0;
  }
  if (wid == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  wait_for_stream();                                 // what comes before reads nothing of the call's but its arguments
  count_tiles(p, kPairRows, gs);
  fence_before();
  __syncthreads();
  pair_sync();
  fence_after();
  const unsigned tmem = (unsigned)misc[0];
  const int tiles = gs.prefix[max(p.groups, 1)];

  if (wid < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (wid == 0 && lane == 0) {
      const unsigned bars0 = in_block(bars, 0);
      unsigned it = 0, su = 0, asked = 0;            // K blocks, units; units whose scales were asked for
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        const Tile t = find_tile(p, kPairRows, NT, kPairBand, gs, tile);
        for (int u = 0; u < p.kblocks && ok; ++u, ++su) {
          const unsigned sq = su % kScaleSlots;
          // (a barrier of its own: the K block that a slot of scales was last used with may be two rounds of its slot ago)
          if (su >= kScaleSlots && !(ok = wait(bars + Q_SDONE + sq, (su / kScaleSlots - 1) & 1, p.wait_limit, abort))) break;
          unsigned char* to = scales + sq * kScaleSlotBytes;
          mbar_expect_tx(bars + Q_SFULL + sq, P4::kScalesCopied);
          tma_load_3d(to, &map_sa, u * 16, t.m0 + (int)rank * kHalf, 0, bars + Q_SFULL + sq);
          tma_load_3d(to + kTurned, &map_sb, u * 16, t.n0, t.g, bars + Q_SFULL + sq);
          asked = su + 1;
          for (int kb = 2 * u; kb < min(2 * u + 2, blocks); ++kb, ++it) {
            const unsigned q = it % S;
            if (it >= S && !(ok = wait(bars + Q_DONE + q, (it / S - 1) & 1, p.wait_limit, abort))) break;
            unsigned char* data = ring + (size_t)q * P4::kSlotBytes;
            if (rank == 0) mbar_expect_tx(bars + Q_FULL + q, 2 * P4::kSlotBytes);
            const unsigned full = bars0 + (Q_FULL + q) * 8;
            if (!(p.withhold && it == 0)) {
              tma_load_pair(data, &map_a, kb * kKB, t.m0 + (int)rank * kHalf, 0, full);
              tma_load_pair(data + kHalfBytes, &map_b, kb * kKB, t.n0 + (int)rank * P4::kHalfCols, t.g, full);
            }
          }
        }
      }
      misc[5] = (int)asked;
      store_cluster(in_block(misc + 2 + rank, 0), it);
    } else if (wid == 1 && rank == 0) {
      const unsigned at = __shfl_sync(kAll, tmem, 0);
      unsigned it = 0, su = 0, n = 0;                // K blocks, units, tiles
      bool ok = true;
      for (int tile = pair; tile < tiles && ok && blocks > 0; tile += pairs, ++n) {
        const unsigned stage = n % P4::kStages, d = at + stage * NT;
        for (int u = 0; u < p.kblocks; ++u, ++su) {
          const unsigned sq = su % kScaleSlots;
          ok = wait_cluster(bars + Q_TURNED + sq, (su / kScaleSlots) & 1, p.wait_limit, abort);
          if (u == 0 && n >= P4::kStages) ok = ok && wait(bars + Q_ACCEMPTY + stage, (n / P4::kStages - 1) & 1, p.wait_limit, abort);
          const bool last = u + 1 == p.kblocks;
          const int here = last && (blocks & 1) ? 1 : 2;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if (b >= here) break;
            const unsigned q = it % S;
            ok = ok && wait(bars + Q_FULL + q, (it / S) & 1, p.wait_limit, abort);
            if (!(ok = __all_sync(kAll, ok))) break;
            fence_after();
            if (elect_one()) {
              const unsigned cols = at + P4::kScaleCols + b * 24;                       // A's: 2 x 4 columns, B's: 2 x 8
              const unsigned char* atom = scales + sq * kScaleSlotBytes + 2 * b * kAtom;
              const int steps = steps4(p.K - (2 * u + b) * kKB, 4);
#pragma unroll
              for (int a = 0; a < 2; ++a)
                if (2 * a < steps) {
                  copy_scales_pair(cols + 4 * a, scale_desc(atom + a * kAtom));
                  copy_scales_pair(cols + 8 + 8 * a, scale_desc(atom + a * kAtom + kTurned));
                  copy_scales_pair(cols + 12 + 8 * a, scale_desc(atom + a * kAtom + 2 * kTurned));
                }
              const unsigned long long da = operand_desc(ring + (size_t)q * P4::kSlotBytes), db = operand_desc(ring + (size_t)q * P4::kSlotBytes + kHalfBytes);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (k < steps)
                  mma_f4_pair(d, da + 2 * k, db + 2 * k, with_scales(p.idesc, k), cols + 4 * (k >> 1), cols + 8 + 8 * (k >> 1), k != 0 || b != 0 || u != 0);
              commit_pair(bars + Q_DONE + q);
              if (b + 1 == here) commit_pair(bars + Q_SDONE + sq);
              if (last && b + 1 == here) commit_pair(bars + Q_ACCFULL + stage);
            }
            __syncwarp();
            ++it;
          }
          if (!ok) break;
        }
      }
    } else if (wid == 1 && lane == 0) {
      // The second block's word that its scales are turned.  (A release for the whole cluster waits for what its thread has in
      // flight, 1400 cycles in the warps that turn them: 8192^3 285 us.)
      unsigned su = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs)
        for (int u = 0; u < p.kblocks && ok; ++u, ++su) {
          const unsigned sq = su % kScaleSlots;
          ok = wait(bars + Q_TURNED + sq, (su / kScaleSlots) & 1, p.wait_limit, abort);
          if (ok) arrive_release_cluster(in_block(bars + Q_TURNED + sq, 0));
        }
    } else if (wid >= 2) {
      unsigned su = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs)
        for (int u = 0; u < p.kblocks; ++u, ++su) {
          const unsigned sq = su % kScaleSlots;
          if (!(ok = __all_sync(kAll, wait(bars + Q_SFULL + sq, (su / kScaleSlots) & 1, p.wait_limit, abort)))) break;
          unsigned char* at = scales + sq * kScaleSlotBytes + (wid - 2) * (2 * kTurned);
          ScaleRows4 one, two;
          one.read(at, 16, wid == 2 ? kHalf : NT - 128, lane);
          if (wid == 2) two.read(at + kTurned, 16, 128, lane);
          __syncwarp();
          one.write(at, lane);
          if (wid == 2) two.write(at + kTurned, lane);
          turned();
          if (lane == 0) arrive(bars + Q_TURNED + sq);
        }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int quarter = wid & 3, half = (wid - 4) >> 2;
    const unsigned free0 = in_block(bars + Q_ACCEMPTY, 0);
    const unsigned at_tmem = tmem + ((unsigned)(quarter * 32) << 16) + half * 128;
    unsigned char* stage_smem = stages + (wid - 4) * (kPair4Pieces * kPieceBytes);
    const LaneGroups lg(p, gs, lane);
    unsigned n_tile = 0;
    for (int tile = pair; tile < tiles; tile += pairs, ++n_tile) {
      const Tile t = lg.find(p, kPairRows, NT, kPairBand, gs, tile, lane);
      const int m = t.m0 + (int)rank * kHalf + quarter * 32, n = t.n0 + half * 128;      // the warp's corner
      const unsigned stage = n_tile % P4::kStages;
      float acc[128];
#pragma unroll
      for (int c = 0; c < 128; ++c) acc[c] = 0.f;
      if (blocks > 0) {
        if (!__all_sync(kAll, wait(bars + Q_ACCFULL + stage, (n_tile / P4::kStages) & 1, p.wait_limit, abort))) break;
        fence_after();
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (half == 0 || i * 32 < NT - 128) tmem_load32(at_tmem + stage * NT + i * 32, *reinterpret_cast<float(*)[32]>(acc + i * 32));
        tmem_wait();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(free0 + stage * 8);
      }
      Out o;
      o.map = &map_c;
      o.rows = min(32, t.m_end - m); o.cols = min(half ? NT - 128 : 128, p.N - n);
      o.n = n; o.m = m; o.z = 0;
      o.ldc = p.ldc;
      o.at = m * p.ldc + n;
      o.by_map = p.c_by_map && o.rows == 32;
      if (o.rows > 0 && o.cols > 0) {
        if (p.c_type == ASGD_F32) store_rows<float, false, kPair4Pieces>(acc, stage_smem, reinterpret_cast<float*>(p.c), o, lane);
        else if (p.c_type == ASGD_BF16) store_rows<__nv_bfloat16, false, kPair4Pieces>(acc, stage_smem, reinterpret_cast<__nv_bfloat16*>(p.c), o, lane);
        else store_rows<__half, false, kPair4Pieces>(acc, stage_smem, reinterpret_cast<__half*>(p.c), o, lane);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  // Both blocks are through; where one gave up, what is in flight ends first (as in product_pair_kernel).
  if (*reinterpret_cast<volatile int*>(abort) && lane == 0) {
    store_cluster(in_block(misc + 4, 0), 1);
    store_cluster(in_block(misc + 4, 1), 1);
  }
  fence_before();
  pair_sync();
  fence_after();
  const bool gave_up = *reinterpret_cast<volatile int*>(misc + 4) != 0;
  if (gave_up && tid == 0) {
    for (unsigned su = misc[5] > kScaleSlots ? misc[5] - kScaleSlots : 0; su < (unsigned)misc[5]; ++su)      // this block's scales
      wait_in_flight(bars + Q_SFULL + su % kScaleSlots, (su / kScaleSlots) & 1, p.wait_limit);
    if (rank == 0) {
      const unsigned mine = (unsigned)misc[2], other = (unsigned)misc[3], end = max(mine, other);
      for (unsigned i = min(mine, other); i < end; ++i) {
        if (i < mine) complete_tx(bars + Q_FULL + i % S, P4::kSlotBytes);
        else mbar_expect_tx(bars + Q_FULL + i % S, P4::kSlotBytes);
      }
      if (p.withhold && end) complete_tx(bars + Q_FULL, ((mine > 0) + (other > 0)) * P4::kSlotBytes);
      for (unsigned i = end > S ? end - S : 0; i < end; ++i)                   // every barrier's last use
        wait_in_flight(bars + Q_FULL + i % S, (i / S) & 1, p.wait_limit);
      atomicMin(p.status, ASGD_ETIMEOUT);
    }
  } else if (gave_up && wid == 1 && elect_one()) {   // the lane that issued the products: a commit is of its own thread's
    if (rank == 0) commit_pair(bars + Q_DRAIN);
    wait_in_flight(bars + Q_DRAIN, 0, p.wait_limit);
  }
  __syncwarp();
  pair_sync();
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

}  // namespace
