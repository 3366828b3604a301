// The kernel of asgd_product4 for few rows of A (per group), or few tiles of C.
//
// As in the 8-bit kernel (asgd_product_few.cuh) a tile is 128 columns of C (rows of B, the weights: the MMA's M) by BN rows of C
// (rows of A, the tokens: the MMA's N), and with fewer tiles than SMs a cluster of blocks shares a tile's K units and adds up
// through distributed shared memory, in the blocks' order.  What differs: the tensor cores apply the powers of two themselves
// (kind::mxf4, block scales), so that the sums of a whole row stay in tensor memory until the tile is through, and nothing is
// read out on the way.  The weights' bytes are the bound.  256 rows over 64 matrices of 2048 x 2048: 26 us (4.3 TB/s; the last turn of tiles is a
// third of them), 5 rows by 4096 x 4096: 6.2 us, the chain of launch, maps, first copies and the cluster's sum.  Every instruction of the tensor pipe
// is issued by an elected thread: behind `lane == 0` the compiler walks the warp's lanes one by one, some 80 cycles each (8.7 and 36 us).
//
// A unit is 512 numbers of K: two 128-byte swizzled pieces of either operand, and 16 bytes of scales a row, which is what a
// tensor map can copy.  The tensor cores want scales in tensor memory, where one 32-bit column of a lane holds four scales of one row,
// rows l, l + 32, l + 64 and l + 96 side by side; a warp per operand therefore turns a unit's scales round in place: a
// lane reads the 16 bytes of its four rows and writes, for each 128 numbers of K, their four words together.
//
// Warp roles: 0 issues the copies, 1 the products (and the scales' way into tensor memory, which the tensor pipe keeps in
// order with them), 2 and 3 turn the scales of the weights and the tokens, the warps from 4 on take C out.
#pragma once

#include "asgd_product_few.cuh"

namespace {

constexpr int kUnit = 256;                           // bytes of a row in a unit
constexpr int kAtom = 512;                           // bytes: scales of 128 rows, 128 numbers of K
constexpr int kTurned = 4 * kAtom;                   // of a unit

struct Params4 : Params {                            // K and the leading dimensions in bytes, kblocks in units
  int* status;
};

// scales of 128 rows by 128 numbers of K, 32 lanes of 16 bytes, into four columns of tensor memory (and the same in each quarter of its lanes)
__device__ inline unsigned long long scale_desc(const void* smem) {
  return (unsigned long long)((smem_u32(smem) & 0x3FFFFu) >> 4) | (unsigned long long)(128 >> 4) << 32 | 1ull << 46;
}
__device__ inline void copy_scales(unsigned tmem, unsigned long long desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ inline void mma_f4(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sa, unsigned sb, bool acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
               ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)acc) : "memory");
}
// the instruction of the k-th 64 numbers: which two of a column's four scales it takes
__device__ inline unsigned with_scales(unsigned idesc, int k) { return idesc | (k & 1 ? 2u << 4 | 2u << 29 : 0u); }
// instructions of 64 numbers (32 bytes) that `bytes` of a row take, n at most
__device__ inline int steps4(int bytes, int n) { return min(n, (bytes + 31) >> 5); }

// A warp turns the scales of `rows` rows (16 bytes each, `pitch` bytes apart) into four atoms, in place or elsewhere; rows from there to
// 128 have zeros.  What it has read, and (whole warp between) what it writes; a fence for the tensor pipe's reads afterwards.
struct ScaleRows4 {
  uint4 r[4];
  __device__ __forceinline__ void read(const unsigned char* from, int pitch, int rows, int lane) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      r[c] = make_uint4(0, 0, 0, 0);
      if (32 * c + lane < rows) r[c] = *reinterpret_cast<const uint4*>(from + (32 * c + lane) * pitch);
    }
  }
  __device__ __forceinline__ void write(unsigned char* at, int lane) const {
    uint4* to = reinterpret_cast<uint4*>(at) + lane;
    to[0] = make_uint4(r[0].x, r[1].x, r[2].x, r[3].x);
    to[kAtom / 16] = make_uint4(r[0].y, r[1].y, r[2].y, r[3].y);
    to[2 * kAtom / 16] = make_uint4(r[0].z, r[1].z, r[2].z, r[3].z);
    to[3 * kAtom / 16] = make_uint4(r[0].w, r[1].w, r[2].w, r[3].w);
  }
};
__device__ inline void turned() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

template <int BN> struct Few4 {
  static constexpr int kSlots = BN == 16 ? 5 : BN == 128 ? 3 : 4;
  static constexpr unsigned kPiece = BN * kKB;                          // of the tokens
  static constexpr unsigned kScalesAt = 2 * (kU * kKB + kPiece), kSlotBytes = kScalesAt + 2 * kTurned;
  static constexpr unsigned kCopied = kScalesAt + (kU + BN) * 16;
  static constexpr int kShare = BN >= 64 ? 2 : 1;                       // warps that share a column's rows of C
  static constexpr int kRows = BN / kShare;
  static constexpr int kThreads = 128 + 128 * kShare;
  static constexpr unsigned kScaleCols = 2 * BN;                        // behind two stages of sums: two units' scales, 32 columns each
  static constexpr unsigned kCols = BN == 128 ? 512 : BN == 64 ? 256 : 128;
  enum { FULL = 0, TURNED = kSlots, DONE = 2 * kSlots, ACCFULL = 3 * kSlots, ACCEMPTY = ACCFULL + 2, DRAIN = ACCEMPTY + 2, COUNT = DRAIN + 1 };
  static constexpr size_t kSmem = 1024 + (size_t)kSlots * kSlotBytes + COUNT * 8 + sizeof(Groups) + 64;
  static_assert(kScaleCols + 64 <= kCols, "tensor memory");
  static_assert(kSmem <= kSmemLimit, "shared memory");
  static_assert((size_t)BN * kU * 4 <= (size_t)kSlots * kSlotBytes, "a block's sums fit where the ring was");
};

// kSplit: launched in clusters, a tile per cluster
template <int BN, bool kSplit> __global__ void __launch_bounds__(Few4<BN>::kThreads, 1)
product4_few_kernel(const Params4 p, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_su, const __grid_constant__ CUtensorMap map_sv) {
  using F = Few4<BN>;
  constexpr int S = F::kSlots;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(ring + (size_t)S * F::kSlotBytes);
  Groups& gs = *reinterpret_cast<Groups*>(bars + F::COUNT);
  int* misc = reinterpret_cast<int*>(&gs + 1);                          // [0] tensor memory, [1] abort, [2] units whose copies were issued
  int* abort = misc + 1;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = kSplit ? (int)cluster_rank() : 0, share = kSplit ? (int)cluster_size() : 1;
  const int first = (int)blockIdx.x / share, step = (int)gridDim.x / share;

  if (tid == 0) {
    prefetch_map(&map_u);
    prefetch_map(&map_v);
    prefetch_map(&map_su);
    prefetch_map(&map_sv);
    for (int q = 0; q < S; ++q) { mbar_init(bars + F::FULL + q, 1); mbar_init(bars + F::TURNED + q, 2); mbar_init(bars + F::DONE + q, 1); }
    for (int q = 0; q < 2; ++q) { mbar_init(bars + F::ACCFULL + q, 1); mbar_init(bars + F::ACCEMPTY + q, 4 * F::kShare); }
    mbar_init(bars + F::DRAIN, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    misc[1] = misc[2] = 0;
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
  // a tile's units, or the block's stretch of them
  auto tile_at = [&](int tile) {
    Tile t = find_tile(p, BN, kU, kNoBand, gs, tile);
    if (kSplit) {
      const int n = t.kb1;
      t.kb0 = n * rank / share;
      t.kb1 = n * (rank + 1) / share;
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
          unsigned long long* full = bars + F::FULL + q;
          mbar_expect_tx(full, F::kCopied);
          if (!(p.withhold && it == 0)) {
            tma_load_3d(to, &map_u, kb * kUnit, t.n0, t.g, full);
            tma_load_3d(to + kU * kKB, &map_u, kb * kUnit + kKB, t.n0, t.g, full);
            tma_load_3d(to + 2 * kU * kKB, &map_v, kb * kUnit, t.m0, 0, full);
            tma_load_3d(to + 2 * kU * kKB + F::kPiece, &map_v, kb * kUnit + kKB, t.m0, 0, full);
            tma_load_3d(to + F::kScalesAt, &map_su, kb * 16, t.n0, t.g, full);
            tma_load_3d(to + F::kScalesAt + kTurned, &map_sv, kb * 16, t.m0, 0, full);
          }
        }
      }
      misc[2] = (int)it;
    }
  } else if (wid == 1) {
    const unsigned at = __shfl_sync(kAll, tmem, 0);
    // a tile's units are the same for every tile
    const int units = kSplit ? p.kblocks * (rank + 1) / share - p.kblocks * rank / share : p.kblocks, from = kSplit ? p.kblocks * rank / share : 0;
    unsigned it = 0, n = 0;                          // units, tiles
    bool ok = true;
    for (int tile = first; tile < tiles && units && ok; tile += step, ++n) {
      const unsigned stage = n & 1, d = at + stage * BN;
      for (int u = 0; u < units; ++u, ++it) {
        const unsigned q = it % S;
        ok = wait(bars + F::FULL + q, (it / S) & 1, p.wait_limit, abort) && wait(bars + F::TURNED + q, (it / S) & 1, p.wait_limit, abort);
        if (u == 0 && n >= 2) ok = ok && wait(bars + F::ACCEMPTY + stage, (n / 2 - 1) & 1, p.wait_limit, abort);
        if (!(ok = __all_sync(kAll, ok))) break;
        fence_after();
        if (elect_one()) {
          const unsigned char* slot = ring + (size_t)q * F::kSlotBytes;
          const unsigned scales = at + F::kScaleCols + (it & 1) * 32;
          const int steps = steps4(p.K - (from + u) * kUnit, 8);
#pragma unroll
          for (int a = 0; a < 4; ++a)
            if (2 * a < steps) {
              copy_scales(scales + 4 * a, scale_desc(slot + F::kScalesAt + a * kAtom));
              copy_scales(scales + 16 + 4 * a, scale_desc(slot + F::kScalesAt + kTurned + a * kAtom));
            }
          const unsigned long long du = operand_desc(slot), dv = operand_desc(slot + 2 * kU * kKB);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (k < steps)
              mma_f4(d, du + (k >> 2) * (kU * kKB >> 4) + 2 * (k & 3), dv + (k >> 2) * (F::kPiece >> 4) + 2 * (k & 3), with_scales(p.idesc, k),
                     scales + 4 * (k >> 1), scales + 16 + 4 * (k >> 1), k != 0 || u != 0);
          commit(bars + F::DONE + q);
          if (u + 1 == units) commit(bars + F::ACCFULL + stage);
        }
        __syncwarp();
      }
    }
  } else if (wid < 4) {
    unsigned it = 0;
    bool ok = true;
    for (int tile = first; tile < tiles && ok; tile += step) {
      const Tile t = tile_at(tile);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S;
        if (!(ok = __all_sync(kAll, wait(bars + F::FULL + q, (it / S) & 1, p.wait_limit, abort)))) break;
        unsigned char* at = ring + (size_t)q * F::kSlotBytes + F::kScalesAt + (wid - 2) * kTurned;
        ScaleRows4 rows;
        rows.read(at, 16, wid == 2 ? kU : BN, lane);
        __syncwarp();
        rows.write(at, lane);
        turned();
        if (lane == 0) arrive(bars + F::TURNED + q);
      }
    }
  } else {
    const int quarter = wid & 3, c_first = ((wid - 4) >> 2) * F::kRows;                 // the warp's columns and rows of C
    const unsigned at_tmem = tmem + ((unsigned)(quarter * 32) << 16) + c_first;
    unsigned n = 0;
    for (int tile = first; tile < tiles; tile += step) {
      const Tile t = tile_at(tile);
      const int u = t.n0 + quarter * 32 + lane;
      const unsigned stage = n & 1;
      float acc[F::kRows];
#pragma unroll
      for (int c = 0; c < F::kRows; ++c) acc[c] = 0.f;
      if (t.kb0 < t.kb1) {
        if (!__all_sync(kAll, wait(bars + F::ACCFULL + stage, (n / 2) & 1, p.wait_limit, abort))) break;
        fence_after();
#pragma unroll
        for (int c0 = 0; c0 < F::kRows; c0 += 16) tmem_load16(at_tmem + stage * BN + c0, *reinterpret_cast<float(*)[16]>(acc + c0));
        tmem_wait();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(bars + F::ACCEMPTY + stage);
        ++n;
      }
      if (kSplit) {
        // every copy into the ring has been read: the products that read them are complete
        float* sums = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int c = 0; c < F::kRows; ++c) sums[(c_first + c) * kU + quarter * 32 + lane] = acc[c];
      } else if (u < p.N) {
#pragma unroll
        for (int c = 0; c < F::kRows; ++c) {
          const int m = t.m0 + c_first + c;
          if (m < t.m_end) store_c(p.c, p.c_type, u + (long long)m * p.ldc, acc[c]);
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
        const long long at = t.n0 + (long long)(t.m0 + e / (kU / 4)) * p.ldc + u;
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
    } else if (wid == 1 && elect_one()) {            // the lane that issued the products: a commit is of its own thread's
      commit(bars + F::DRAIN);
      wait_in_flight(bars + F::DRAIN, 0, p.wait_limit);
    }
    __syncthreads();
    fence_after();
  }
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::kCols));
  if (tid == 0 && *reinterpret_cast<volatile int*>(abort)) atomicMin(p.status, ASGD_ETIMEOUT);
}

}  // namespace
