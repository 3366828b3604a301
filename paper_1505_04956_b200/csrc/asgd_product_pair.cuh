// The kernel of asgd_product for many rows of A (per group): a pair of thread blocks on neighbouring SMs takes a tile of
// 256 x 256 numbers of C.
//
// tcgen05.mma of a pair (cta_group::2) multiplies 256 rows of A by 256 rows of B; each SM holds half of either operand
// (128 rows of A, its rows of C; 128 rows of B, of which both SMs' tensor cores read both halves), so a K block of 128
// costs an SM 32 KB of shared memory and of L2 traffic where a single SM's 128 x 256 tile would cost 48 KB.
//
// Warp roles in each block: 0 issues the TMA loads of the block's halves, which all report to the first block's barrier;
// 1 and 3, in the first block, issue the products and commit each K block to a barrier in both blocks, which says "the slot
// is free" to the copies and "the accumulator is full" to the readers; 2 brings the scales (asynchronous copies of 16 or 4 bytes; a
// load into registers would hold the reading warps); 4 to 11 read the accumulators, a row of C per thread and 128 columns
// per warp, and add them, scaled, to sums in registers.  Warps 0 to 3 hand most of their registers to these (56 and 224 a
// thread; with 40 and 232 8192^3 takes 538 us instead of 515, with 72 and 216 a sixth more).  A row's scale and, with
// 128 x 128 blocks of B, the columns' scale are one number per thread, so that a product of the K block costs one multiply-add.
//
// What bounds it: a K block's way round, and the readers' multiply-adds in it.  Its products take the tensor cores 512
// cycles, and about 1000 from their issue until the readers see them; reading them out, with half of the adds, takes 300 to
// 380, and the word back to the issuing thread 300.  Tensor memory holds two stages of 256 columns, so a K block takes half of
// that, some 950 cycles, where 512 would be the tensor cores' own rate (readers that only hand the accumulator back: 564;
// that load it and do not add: 619; that add without a load: 940; four stages of 128 columns: 1250, since halves of the columns
// read the rows of A twice and shared memory is then the bound).  On the device: 8192 x 8192 x 8192 510 us (2.16 PFLOP/s; in a
// user's loop of calls, where the power limit holds the clock near 1.4 GHz, 590 to 609), 32 groups of 16384 rows by 2744 x 2064
// 145 to 155 us (174 to 186), of which a fifth is rows of tiles that no group fills and a sixth the way of C through shared
// memory.  With a scale per column the readers' arithmetic
// is the pace, some 1500 cycles a K block (870 without it): weight gradients of 16 groups, 16384 rows, 2048 x 2048, 131 us.
// C straight from registers, 32 bytes a thread, took 541 us where the way through shared memory took 525 (8192^3), and
// 166 where that took 149 (weight gradient).
#pragma once

#include "asgd_product_common.cuh"

namespace {

constexpr int kPairRows = 256, kPairCols = 256;      // of C, per pair
constexpr int kHalf = 128;                           // rows of either operand per block
constexpr int kPairThreads = 384;
constexpr int kPairSlots = 5;
constexpr int kPairBand = 8;                         // tile rows that neighbouring pairs run down before the next column
constexpr unsigned kHalfBytes = kHalf * kKB, kPairBytes = 2 * kHalfBytes;      // per block: one operand, a slot
constexpr int kPieceBytes = 32 * 64;                 // per warp, on the way to C: 64 bytes of each of its 32 rows
constexpr int kStagePieces = 2, kStageBytes = kStagePieces * kPieceBytes;
constexpr int kScales = kHalf + kPairCols;           // of a slot: the block's rows', then the columns' (256, or two blocks')
enum { P_FULL = 0 /* [issuing thread][slot] */, P_DONE = 2 * kPairSlots, P_SFULL = 3 * kPairSlots, P_SEMPTY = 4 * kPairSlots, P_ACCEMPTY = 5 * kPairSlots,
       P_DRAIN = P_ACCEMPTY + 2, P_COUNT = P_DRAIN + 2 };
constexpr size_t kPairSmem = 1024 + (size_t)kPairSlots * kPairBytes + 8 * kStageBytes + (size_t)kPairSlots * kScales * 4 +
                             P_COUNT * 8 + sizeof(Groups) + 64;
static_assert(kPairSmem <= kSmemLimit, "shared memory");

// K block number `it` of a block's work: its full barrier (each issuing thread has its own, so that it meets every phase of
// what it waits on: a wait on a parity cannot tell a phase from the one two before) and the phase
__device__ inline unsigned full_of(unsigned it) { return P_FULL + (it & 1) * kPairSlots + it % kPairSlots; }
__device__ inline unsigned full_phase(unsigned it) { return it / (2 * kPairSlots) & 1; }
static_assert(kPairSlots % 2 == 1, "a slot meets the issuing threads in turn");

__device__ inline unsigned rank_in_pair() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ inline void pair_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// the block's own half; the bytes are counted at a barrier of the pair's first block
__device__ inline void tma_load_pair(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ inline void mma_f8_pair(unsigned d_tmem, unsigned long long a, unsigned long long b, unsigned idesc, bool acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
               ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc) : "memory");
}
__device__ inline void commit_pair(unsigned long long* bar) {                  // at the same place in both blocks
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_u32(bar)), "h"((unsigned short)3) : "memory");
}
// No release at cluster scope: what is handed over is tensor memory (ordered by the tcgen05 fence before), and such a
// release would wait for the warp's loads in flight, about 1000 cycles of every K block.
__device__ inline void arrive_cluster(unsigned bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ inline void complete_tx(unsigned long long* bar, unsigned bytes) {  // bytes that will not come
  asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ inline void store_cluster(unsigned addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// 32 columns of the warp's 32 accumulator rows
__device__ inline void tmem_load32(unsigned taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
        "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
        "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}

// 16 columns of 32 accumulator rows, a thread's share: rows lane / 4 + 8 i, columns 8 g + 2 (lane % 4) + e as v[(g * 4 + i) * 2 + e]
__device__ inline void tmem_load_fragments(unsigned taddr, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]) : "r"(taddr) : "memory");
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(taddr + (16u << 16)) : "memory");
}
__device__ inline void tma_store_3d(const CUtensorMap* map, int x, int y, int z, const void* src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(src)) : "memory");
}

// Two sums at a time: x * s + acc, x * (a * f) + acc.  The packed form takes the multiply-add pipe for as long as two
// scalar ones and half of the issue slots: with scalar ones the reading warps kept the issuing threads of the products
// (same schedulers) from theirs.
__device__ __forceinline__ unsigned long long pair_of(float x, float y) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void fma2(float& acc0, float& acc1, float x0, float x1, unsigned long long s) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_of(x0, x1)), "l"(s), "l"(pair_of(acc0, acc1)));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(acc0), "=f"(acc1) : "l"(r));
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <typename T> __device__ __forceinline__ unsigned pack32(float a, float b) {       // two 16-bit numbers
  const T v[2] = {Elem<T>::from_f(a), Elem<T>::from_f(b)};
  return *reinterpret_cast<const unsigned*>(v);
}

// Where a warp's 32 rows x 128 columns go.  map: the copies out of shared memory run on while the warp goes on, for
// whole warps' rows and where C's rows start at 16-byte boundaries; else the warp writes C itself.
struct Out {
  const CUtensorMap* map;
  bool by_map;
  int n, m, z;                                       // the corner, the group
  long long ldc, at;                                 // elements from C to the corner
  int rows, cols;                                    // how many there are
};

// 64 bytes of every row make a piece of the warp's stage, with parts of 16 bytes exchanged by row (the 64-byte swizzle),
// so that no access meets a bank more than twice.
template <typename T, bool kFragments> __device__ __forceinline__ void store_rows(const float (&acc)[128], unsigned char* stage, T* c, const Out& o, int lane) {
  constexpr int per = 64 / (int)sizeof(T), part = 16 / (int)sizeof(T);         // numbers of a row in a piece, in a part
  T* corner = c + o.at;
  const bool whole = ((reinterpret_cast<unsigned long long>(corner) | ((unsigned long long)o.ldc * sizeof(T))) & 15) == 0;
  // Rows that the warp writes itself add no groups of copies, so the count below says nothing of the tile before: all of
  // its copies have read the stage first.
  if (!o.by_map) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
  }
#pragma unroll
  for (int first = 0; first < 128; first += per) {
    unsigned char* piece = stage + first / per % kStagePieces * kPieceBytes;
    // the copy before last, out of the same place, has read it (a piece that is copied is a group of its own)
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kStagePieces - 1) : "memory");
    __syncwarp();
    if constexpr (!kFragments) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[part];
#pragma unroll
        for (int i = 0; i < part; ++i) v[i] = acc[first + q * part + i];
        *reinterpret_cast<uint4*>(piece + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = pack16<T>(v);
      }
    } else {
#pragma unroll
      for (int g = 0; g < per / 8; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = acc[((first / 8 + g) * 4 + i) * 2], y = acc[((first / 8 + g) * 4 + i) * 2 + 1];
          const int r = (lane >> 2) + 8 * i, byte = (8 * g + 2 * (lane & 3)) * (int)sizeof(T);
          unsigned char* at = piece + r * 64 + (((byte >> 4) ^ ((r >> 1) & 3)) << 4) + (byte & 15);
          if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(at) = make_float2(x, y);
          else *reinterpret_cast<unsigned*>(at) = pack32<T>(x, y);
        }
    }
    if (o.by_map) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        if (first < o.cols) tma_store_3d(o.map, o.n + first, o.m, o.z, piece);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
    } else {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 2), q = lane & 3, at = first + q * part;
        if (r < o.rows && at < o.cols) {
          const unsigned char* from = piece + r * 64 + ((q ^ ((r >> 1) & 3)) << 4);
          T* to = corner + (long long)r * o.ldc + at;
          if (whole && at + part <= o.cols) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
          else
            for (int b = 0; b < part && at + b < o.cols; ++b) to[b] = reinterpret_cast<const T*>(from)[b];
        }
      }
      __syncwarp();
    }
  }
}

// kColumns: the columns have a scale each (rows of B scaled by blocks of 128 along K alone)
template <bool kColumns> __global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
product_pair_kernel(const Params p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                    const __grid_constant__ CUtensorMap map_c) {
  constexpr int S = kPairSlots;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char* ring = smem_dyn + ((1024u - (smem_u32(smem_dyn) & 1023u)) & 1023u);
  unsigned char* stages = ring + (size_t)S * kPairBytes;
  float* scales = reinterpret_cast<float*>(stages + 8 * kStageBytes);                   // [slot][kScales]
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(scales + S * kScales);
  Groups& gs = *reinterpret_cast<Groups*>(bars + P_COUNT);
  int* misc = reinterpret_cast<int*>(&gs + 1);        // [0] tensor memory, [1] abort, [2, 3] K blocks whose copies each block has issued, [4] one of the blocks gave up
  int* abort = misc + 1;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const unsigned rank = rank_in_pair();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (tid == 0) {
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    if (p.c_by_map) prefetch_map(&map_c);
    for (int q = 0; q < 2 * S; ++q) mbar_init(bars + P_FULL + q, 1);
    for (int q = 0; q < S; ++q) { mbar_init(bars + P_DONE + q, 1); mbar_init(bars + P_SFULL + q, 32); mbar_init(bars + P_SEMPTY + q, 8); }
    for (int q = 0; q < 2; ++q) { mbar_init(bars + P_ACCEMPTY + q, 16); mbar_init(bars + P_DRAIN + q, 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int q = 1; q < 5; ++q) misc[q] = 0;
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
      unsigned it = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        const Tile t = find_tile(p, kPairRows, kPairCols, kPairBand, gs, tile);
        const int za = 0, zb = p.inner ? 0 : t.g;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S;
          if (it >= S && !(ok = wait(bars + P_DONE + q, (it / S - 1) & 1, p.wait_limit, abort))) break;
          unsigned char* to = ring + (size_t)q * kPairBytes;
          if (rank == 0) mbar_expect_tx(bars + full_of(it), 2 * kPairBytes);
          const unsigned full = bars0 + full_of(it) * 8;
          if (!(p.withhold && it == 0)) {
            tma_load_pair(to, &map_a, kb * kKB, t.m0 + (int)rank * kHalf, za, full);
            tma_load_pair(to + kHalfBytes, &map_b, kb * kKB, t.n0 + (int)rank * kHalf, zb, full);
          }
        }
      }
      store_cluster(in_block(misc + 2 + rank, 0), it);
    } else if ((wid == 1 || wid == 3) && lane == 0 && rank == 0) {
      // Two issuing threads, one per accumulator stage, K blocks in turn: a commit holds the thread that issues it for
      // several hundred cycles, and the other thread's products fill the gap.
      const unsigned me = (unsigned)wid >> 1;
      unsigned it = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        Tile t;                                      // the K blocks alone
        t.kb0 = 0; t.kb1 = p.kblocks; t.k_end = p.K;
        if (p.inner) t = find_tile(p, kPairRows, kPairCols, kPairBand, gs, tile);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S, stage = it & 1;
          if (stage != me) continue;
          // the operands are there long before the accumulator is free: what can be done is done before that wait
          if (!(ok = wait(bars + full_of(it), full_phase(it), p.wait_limit, abort))) break;
          const unsigned long long da = operand_desc(ring + (size_t)q * kPairBytes), db = operand_desc(ring + (size_t)q * kPairBytes + kHalfBytes);
          const int steps = steps_of(t, kb);
          if (it >= 2 && !(ok = wait(bars + P_ACCEMPTY + stage, (it / 2 - 1) & 1, p.wait_limit, abort))) break;
          fence_after();
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) if (k4 < steps) mma_f8_pair(tmem + stage * kPairCols, da + 2 * k4, db + 2 * k4, p.idesc, k4 != 0);
          commit_pair(bars + P_DONE + q);
        }
      }
    } else if (wid == 2) {
      const LaneGroups lg(p, gs, lane);
      unsigned it = 0;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        const Tile t = lg.find(p, kPairRows, kPairCols, kPairBand, gs, tile, lane);
        const float* from = p.sb + (p.inner ? 0 : t.g * p.sb_group);
        ScaleRows<kHalf> rows;
        ScaleRows<kPairCols> cols;
        rows.start(p.sa, p.sa_row, p.sa_block, t.kb0, t.m0 + (int)rank * kHalf, t.m_end, lane);
        if (kColumns) cols.start(from, p.sb_row, p.sb_block, t.kb0, t.n0, p.N, lane);
        const int n = t.n0 + 128 * min(lane, 1);     // two blocks of columns
        const bool there = n < p.N;
        const float* of_block = there ? from + (n >> 7) * p.sb_row + t.kb0 * p.sb_block : p.sb;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const unsigned q = it % S;
          if (it >= S && !(ok = __all_sync(kAll, wait(bars + P_SEMPTY + q, (it / S - 1) & 1, p.wait_limit, abort)))) break;
          float* to = scales + q * kScales;
          rows.copy(to, lane);
          if (kColumns) {
            cols.copy(to + kHalf, lane);
          } else {
            if (lane < 2) copy4(to + kHalf + lane, of_block, there);
            if (there) of_block += p.sb_block;
          }
          arrive_after_copies(bars + P_SFULL + q);
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const int quarter = wid & 3, half = (wid - 4) >> 2;
    const unsigned free0 = in_block(bars + P_ACCEMPTY, 0);
    const unsigned at_tmem = tmem + ((unsigned)(quarter * 32) << 16) + half * 128;
    unsigned char* stage_smem = stages + (wid - 4) * kStageBytes;
    const LaneGroups lg(p, gs, lane);
    unsigned it = 0;
    bool ok = true;
    for (int tile = pair; tile < tiles && ok; tile += pairs) {
      const Tile t = lg.find(p, kPairRows, kPairCols, kPairBand, gs, tile, lane);
      const int m = t.m0 + (int)rank * kHalf + quarter * 32, n = t.n0 + half * 128;      // the warp's corner
      float acc[128];
#pragma unroll
      for (int c = 0; c < 128; ++c) acc[c] = 0.f;
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const unsigned q = it % S, stage = it & 1;
        ok = wait(bars + P_SFULL + q, (it / S) & 1, p.wait_limit, abort) && wait(bars + P_DONE + q, (it / S) & 1, p.wait_limit, abort);
        if (!(ok = __all_sync(kAll, ok))) break;
        fence_after();
        const float* of_rows = scales + q * kScales + quarter * 32;
        const float* of_cols = scales + q * kScales + kHalf;
        const unsigned from = at_tmem + stage * kPairCols;
        auto hand_back = [&]() {                     // the warp's part of the accumulator has been read
          fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster(free0 + stage * 8);
        };
        if constexpr (!kColumns) {
          float s0, v[2][32];
          auto add = [&](int i) {
#pragma unroll
            for (int c = 0; c < 32; ++c) acc[i * 32 + c] = fmaf(v[i & 1][c], s0, acc[i * 32 + c]);
          };
          // the reads as early as the registers allow: the accumulator goes back before the last two adds
          tmem_load32(from, v[0]);
          tmem_load32(from + 32, v[1]);
          s0 = of_rows[lane] * of_cols[half];
          tmem_wait();
          add(0);
          tmem_load32(from + 64, v[0]);
          add(1);
          tmem_load32(from + 96, v[1]);
          tmem_wait();
          hand_back();
          add(2);
          add(3);
        } else {
          // fragments of 32 rows x 16 columns: a thread needs 32 columns' scales of a K block where a row per thread
          // would need 128 (every broadcast read of 16 bytes takes four cycles of the shared memory's path)
          float v[2][16], a0[4];
          float2 f[2][2];                            // the columns' scales, read one step ahead
          const float* cols = of_cols + half * 128 + 2 * (lane & 3);
          f[0][0] = *reinterpret_cast<const float2*>(cols);
          f[0][1] = *reinterpret_cast<const float2*>(cols + 8);
          tmem_load_fragments(from, v[0]);
#pragma unroll
          for (int i = 0; i < 4; ++i) a0[i] = of_rows[(lane >> 2) + 8 * i];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            tmem_wait();
            if (j < 7) {
              tmem_load_fragments(from + (j + 1) * 16, v[(j + 1) & 1]);
              f[(j + 1) & 1][0] = *reinterpret_cast<const float2*>(cols + (j + 1) * 16);
              f[(j + 1) & 1][1] = *reinterpret_cast<const float2*>(cols + (j + 1) * 16 + 8);
            } else hand_back();
#pragma unroll
            for (int g = 0; g < 2; ++g) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int e = (g * 4 + i) * 2;
                fma2(acc[j * 16 + e], acc[j * 16 + e + 1], v[j & 1][e], v[j & 1][e + 1], mul2(pair_of(a0[i], a0[i]), pair_of(f[j & 1][g].x, f[j & 1][g].y)));
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) arrive(bars + P_SEMPTY + q);
      }
      if (!ok) break;
      if (t.bad) {
        if (lane == 0) atomicMin(&g_status, ASGD_EINVAL);
#pragma unroll
        for (int c = 0; c < 128; ++c) acc[c] = __int_as_float(0x7fffffff);
      }
      Out o;
      o.map = &map_c;
      o.rows = min(32, t.m_end - m); o.cols = min(128, p.N - n);
      o.n = n; o.m = m; o.z = p.inner ? t.g : 0;
      o.ldc = p.ldc;
      o.at = o.z * p.c_group + m * p.ldc + n;
      o.by_map = p.c_by_map && o.rows == 32;
      if (o.rows > 0 && o.cols > 0) {
        if (p.c_type == ASGD_F32) store_rows<float, kColumns>(acc, stage_smem, reinterpret_cast<float*>(p.c), o, lane);
        else if (p.c_type == ASGD_BF16) store_rows<__nv_bfloat16, kColumns>(acc, stage_smem, reinterpret_cast<__nv_bfloat16*>(p.c), o, lane);
        else store_rows<__half, kColumns>(acc, stage_smem, reinterpret_cast<__half*>(p.c), o, lane);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  // Both blocks are through.  Where one gave up, the first block settles its barriers: bytes announced that nobody will
  // send, copies issued that nobody announced; then every copy in flight has landed when the last phases are complete.  The
  // products, and the word of them in both blocks, end as well.
  if (*reinterpret_cast<volatile int*>(abort) && lane == 0) {
    store_cluster(in_block(misc + 4, 0), 1);
    store_cluster(in_block(misc + 4, 1), 1);
  }
  fence_before();
  pair_sync();
  fence_after();
  if (rank == 0 && tid == 0 && *reinterpret_cast<volatile int*>(misc + 4)) {
    const unsigned mine = (unsigned)misc[2], other = (unsigned)misc[3], last = max(mine, other);
    for (unsigned i = min(mine, other); i < last; ++i) {
      if (i < mine) complete_tx(bars + full_of(i), kPairBytes);
      else mbar_expect_tx(bars + full_of(i), kPairBytes);
    }
    if (p.withhold && last) complete_tx(bars + full_of(0), ((mine > 0) + (other > 0)) * kPairBytes);
    for (unsigned i = last > 2 * S ? last - 2 * S : 0; i < last; ++i)          // every barrier's last use
      wait_in_flight(bars + full_of(i), full_phase(i), p.wait_limit);
    atomicMin(&g_status, ASGD_ETIMEOUT);
  } else if ((wid == 1 || wid == 3) && lane == 0 && *reinterpret_cast<volatile int*>(misc + 4)) {
    if (rank == 0) commit_pair(bars + P_DRAIN + (wid >> 1));
    wait_in_flight(bars + P_DRAIN + (wid >> 1), 0, p.wait_limit);
  }
  __syncwarp();
  pair_sync();
  if (wid == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

}  // namespace
