// Shared by the two kernels of asgd_product: parameters, wrappers of the tensor-core and copy instructions, bounded
// waits, and the tiles of C that persistent blocks take in turn.
#pragma once

#include "asgd_experts_common.cuh"

#include <cuda.h>

#include "asgd_stream.cuh"   // mbarrier helpers

namespace {

using namespace asgd::experts;
using asgd::mbar_expect_tx;
using asgd::mbar_init;
using asgd::mbar_try_wait;
using asgd::smem_u32;

__device__ int g_status;                             // what asgd_experts_sync reports: the smallest (worst) code seen
constexpr int kKB = 128;                             // numbers (bytes) of a K block: a 128-byte swizzled row
constexpr size_t kSmemLimit = 227 * 1024;

struct Params {
  int M, N, K, groups, inner, kblocks;
  int tiles_n;                                       // tiles of C along a row
  const float *sa, *sb;
  long long sa_row, sa_block, sb_row, sb_block, sb_group;
  int sb_shift;
  void* c;
  long long ldc, c_group;
  int c_type, c_by_map;                              // c_by_map: a tensor map of C is there
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
__device__ inline unsigned in_block(const void* smem, unsigned rank) {         // the same place in another block of the cluster
  unsigned a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(smem)), "r"(rank));
  return a;
}
__device__ inline void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ inline void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ inline void copy4(float* dst, const float* src, bool there) {       // asynchronous; zero where not there
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ inline void copy16(float* dst, const float* src, int bytes) {       // the first `bytes` of 16, zeros for the others
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ inline void arrive_after_copies(unsigned long long* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ inline void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
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

// A block in which a wait ran out leaves when its copies and products in flight have ended, whichever thread issued them and
// whether or not that thread knew.  This wait is bounded as well, by the limit given and by 2^14 polls at
// least (1.3 ms; a copy or a product takes microseconds).
__device__ inline void wait_in_flight(unsigned long long* bar, unsigned parity, unsigned limit) {
  limit = max(limit, 1u << 14);
  for (unsigned n = 0; n < limit && !mbar_try_wait(bar, parity); ++n) {}
}

__device__ inline void store_c(void* c, int type, long long at, float v) {
  if (type == ASGD_F32) reinterpret_cast<float*>(c)[at] = v;
  else if (type == ASGD_BF16) reinterpret_cast<__nv_bfloat16*>(c)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(c)[at] = __float2half_rn(v);
}

// ---- scales ----

// The scales of kRows rows, K block after K block, brought by a warp: zeros from row `end` on.  Where neighbouring rows'
// scales are neighbours in memory and start at 16-byte boundaries, a lane takes four at a time; addresses are worked out
// once a tile.  (One copy and one address per scale held up the products: a gradient of 2048 x 2048 over 16384 rows, with
// 384 scales a K block, took 125 us.)
template <int kRows> struct ScaleRows {
  const float *at, *any;                             // any: for copies of no bytes, which need an aligned address too
  long long part, block;                             // from a lane's copy to its next one, from a K block to the next
  int left;                                          // rows from the lane's first on
  bool wide;
  __device__ __forceinline__ void start(const float* scales, long long row, long long block_, int kb, int first, int end, int lane) {
    const float* from = scales + first * row + kb * block_;
    any = reinterpret_cast<const float*>(reinterpret_cast<unsigned long long>(scales) & ~15ull);
    block = block_;
    wide = row == 1 && ((reinterpret_cast<unsigned long long>(from) | (unsigned long long)block * 4) & 15) == 0;
    const int unit = wide ? 4 : 1;
    at = from + lane * unit * row;
    part = 32 * unit * row;
    left = min(end - first, kRows) - lane * unit;
  }
  __device__ __forceinline__ void copy(float* to, int lane) {
    if (wide) {
#pragma unroll
      for (int c = 0; c < kRows; c += 128)
        if (c + 128 <= kRows || c + 4 * lane < kRows) {
          const int n = min(max(left - c, 0), 4);
          copy16(to + c + 4 * lane, n ? at + c / 128 * part : any, 4 * n);
        }
    } else {
#pragma unroll
      for (int c = 0; c < kRows; c += 32)
        if (c + 32 <= kRows || c + lane < kRows) copy4(to + c + lane, left > c ? at + c / 32 * part : any, left > c);
    }
    at += block;
  }
};

// ---- tiles ----

struct Tile {
  int g, n0, m0, m_end, kb0, kb1;                    // group, first column and row of C, end of the group's rows, K blocks
  int k_end;                                         // end of the inner dimension
  bool bad;                                          // inner groups whose bounds cut a block
};

// What the blocks know of the groups, in shared memory: prefix[g], the tiles (of bm rows) of the groups before g, and
// start[g], the first row (or K number) of group g.  All threads of the block; ends with a barrier.  (Offsets by plain loads:
// the kernel that writes them may still run when this one comes up, so they are not constant for its life.)
struct Groups {
  int prefix[ASGD_MAX_EXPERTS + 1], start[ASGD_MAX_EXPERTS + 1], warp_part[32];
};
__device__ inline void count_tiles(const Params& p, int bm, Groups& gs) {
  const int G = max(p.groups, 1), tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int limit = p.inner ? p.K : p.M;
  if (p.groups)
    for (int g = tid; g <= G; g += blockDim.x) gs.start[g] = min(max(p.offsets[g], 0), limit);
  else if (tid <= 1) gs.start[tid] = tid ? limit : 0;
  __syncthreads();
  const int per = (G + blockDim.x - 1) / blockDim.x;
  int mine = 0;
  for (int q = 0; q < per; ++q) {
    const int g = tid * per + q;
    if (g >= G) break;
    const int rows = p.inner ? p.M : max(gs.start[g + 1] - gs.start[g], 0);
    const int n = (rows + bm - 1) / bm * p.tiles_n;
    gs.prefix[g] = n;
    mine += n;
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(kAll, inc, o); if (lane >= o) inc += v; }
  if (lane == 31) gs.warp_part[wid] = inc;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wid; ++w) before += gs.warp_part[w];
  int run = before + inc - mine;
  for (int q = 0; q < per; ++q) {
    const int g = tid * per + q;
    if (g >= G) break;
    const int n = gs.prefix[g];
    gs.prefix[g] = run;
    run += n;
    if (g == G - 1) gs.prefix[G] = run;
  }
  __syncthreads();
}

// Tile number `tile` of tiles of bm x bn, of group g that has `before` tiles before it and the rows (or K numbers) lo to
// hi.  Inside a group the tiles run down bands of `band` tile rows, column after column: neighbouring blocks share
// operands in L2.
__device__ inline Tile make_tile(const Params& p, int bm, int bn, int band, int g, int before, int lo, int hi, int tile) {
  Tile t;
  t.g = g;
  hi = max(hi, lo);
  const int first_row = p.inner ? 0 : lo;
  t.m_end = p.inner ? p.M : hi;
  const int rows = (t.m_end - first_row + bm - 1) / bm;
  int at = tile - before, first = 0, high = rows;
  if (rows > band) {
    first = at / (band * p.tiles_n) * band;
    at -= first * p.tiles_n;
    high = min(band, rows - first);
  }
  t.n0 = at / high * bn;
  t.m0 = first_row + (first + at % high) * bm;
  t.kb0 = 0; t.kb1 = p.kblocks;
  t.k_end = p.K;
  t.bad = false;
  if (p.inner) {
    t.kb0 = lo / kKB;
    t.kb1 = hi > lo ? (hi + kKB - 1) / kKB : t.kb0;
    t.k_end = hi;
    t.bad = hi > lo && (lo % kKB || (hi % kKB && hi != p.K));
    if (t.bad) t.kb1 = t.kb0;
  }
  return t;
}
// by one thread: the last group that starts at or before the tile
__device__ inline Tile find_tile(const Params& p, int bm, int bn, int band, const Groups& gs, int tile) {
  int a = 0, b = max(p.groups, 1);
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (gs.prefix[m] <= tile) a = m; else b = m;
  }
  return make_tile(p, bm, bn, band, a, gs.prefix[a], gs.start[a], gs.start[a + 1], tile);
}
// By a whole warp, 32 groups at a look: a search step by step through shared memory that the tensor cores keep busy takes
// some 250 cycles a step.  With at most 32 groups the lanes keep them in registers.
struct LaneGroups {
  int prefix, start, next;
  __device__ inline LaneGroups(const Params& p, const Groups& gs, int lane) {
    const int G = max(p.groups, 1), g = min(lane, G - 1);
    prefix = lane < G ? gs.prefix[g] : 0x7fffffff;
    start = gs.start[g];
    next = gs.start[g + 1];
  }
  __device__ inline Tile find(const Params& p, int bm, int bn, int band, const Groups& gs, int tile, int lane) const {
    const int G = max(p.groups, 1);
    if (G <= 32) {
      const int a = 31 - __clz(__ballot_sync(kAll, prefix <= tile));
      return make_tile(p, bm, bn, band, a, __shfl_sync(kAll, prefix, a), __shfl_sync(kAll, start, a), __shfl_sync(kAll, next, a), tile);
    }
    int a = -1;
    for (int g = 0; g < G; g += 32) a += __popc(__ballot_sync(kAll, g + lane < G && gs.prefix[min(g + lane, G - 1)] <= tile));
    return make_tile(p, bm, bn, band, a, gs.prefix[a], gs.start[a], gs.start[a + 1], tile);
  }
};

// instructions of 32 numbers that K block kb takes (the last block of the inner dimension may be short)
__device__ inline int steps_of(const Tile& t, int kb) { return min(4, (t.k_end - kb * kKB + 31) >> 5); }

}  // namespace
