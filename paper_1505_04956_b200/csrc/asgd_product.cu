// Product of 8-bit matrices with block scales on the tensor cores: dense, grouped over rows, grouped over the inner
// dimension.  The contract is in include/asgd_experts.h.
//
// A scale belongs to 128 neighbours along K, so the products of one K block go into a fresh accumulator in tensor
// memory (four tcgen05.mma of K = 32), and threads add them, scaled, to sums they keep in registers while the tensor
// cores fill the other accumulator stage.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <mutex>

#include "asgd_maps.cuh"
#include "asgd_product_few.cuh"
#include "asgd_product_pair.cuh"

namespace {

std::atomic<unsigned> g_wait_limit{asgd::DEFAULT_WAIT_LIMIT};
std::atomic<int> g_withhold{0};

// What has been reported becomes the answer, in one exchange: a report that comes while it is taken is for the next one.
__device__ int g_taken;
__global__ void take_status_kernel() {
  wait_for_stream();
  g_taken = atomicExch(&g_status, 0);
}

// ---- host ----

constexpr long long kMostTiles = 0x7fffffffll - 2 * kSMs;    // a block's next tile number stays inside 32 bits

// the most tiles of bm x bn there can be: what the offsets say is known on the device alone
long long most_tiles(const Params& p, int bm, int bn) {
  const long long rows = p.inner ? ceil_div(p.M, bm) * p.groups : ceil_div(p.M, bm) + p.groups;
  return rows * ceil_div(p.N, bn);
}
// fp32 accumulators; formats of the MMA's first and second operand (0 = E4M3, 1 = E5M2); its columns and rows
unsigned instruction(int type0, int type1, int cols, int rows) {
  return 1u << 4 | (type0 == ASGD_E5M2 ? 1u : 0u) << 7 | (type1 == ASGD_E5M2 ? 1u : 0u) << 10 | (unsigned)(cols >> 3) << 17 | (unsigned)(rows >> 4) << 24;
}

// `split` blocks share a tile (1: a block takes whole tiles in turn)
template <int BN, bool kSplit> int launch_few(const asgd_product_args& a, Params p, int split, cudaStream_t st) {
  CUtensorMap map_u{}, map_v{};
  if (p.K > 0) {
    if (!encode(&map_u, a.b, p.K, p.N, p.inner ? 1 : max(p.groups, 1), a.ldb, a.b_group, kU)) return ASGD_EINVAL;
    if (!encode(&map_v, a.a, p.K, p.M, 1, a.lda, 0, BN)) return ASGD_EINVAL;
  }
  p.idesc = instruction(a.b_type, a.a_type, BN, kU);
  p.tiles_n = (int)ceil_div(p.N, kU);
  const long long most = most_tiles(p, BN, kU);
  if (most > kMostTiles) return ASGD_EUNSUPPORTED;
  static std::atomic<unsigned long long> done{0};
  if (!allow_smem(product_few_kernel<BN, kSplit>, Few<BN>::kSmem, done)) return ASGD_ECUDA;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;    // see launch_after
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (unsigned)split;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(kSplit ? (unsigned)(most * split) : (unsigned)min(most, (long long)kSMs));
  cfg.blockDim = dim3(Few<BN>::kThreads);
  cfg.dynamicSmemBytes = Few<BN>::kSmem;
  cfg.stream = st;
  cfg.attrs = attrs;
  cfg.numAttrs = kSplit ? 2 : 1;
  return good(cudaLaunchKernelEx(&cfg, product_few_kernel<BN, kSplit>, p, map_u, map_v)) ? ASGD_OK : ASGD_ECUDA;
}

// Blocks per tile of the few-rows kernel: a power of two, with two K blocks each at least, whose clusters are on the SMs
// all at once: of 8 blocks with an SM each 14 fit for certain (a cluster stays inside one of the GPU's partitions; two
// more and 1024 x 4096 with 200 rows takes 17.5 us instead of 11), of 4 blocks 32, of 2 blocks 74.
int split_of(const Params& p, int bn) {
  const long long most = most_tiles(p, bn, kU);
  for (const int split : {8, 4, 2})
    if (most <= (split == 8 ? 14 : split == 4 ? 32 : kSMs / 2) && p.kblocks >= split * 2) return split;
  return 1;
}
template <int BN> int launch_few(const asgd_product_args& a, const Params& p, cudaStream_t st) {
  const int split = split_of(p, BN);
  return split > 1 ? launch_few<BN, true>(a, p, split, st) : launch_few<BN, false>(a, p, 1, st);
}

int launch_pair(const asgd_product_args& a, Params p, cudaStream_t st) {
  CUtensorMap map_a{}, map_b{};
  if (p.K > 0) {
    if (!encode(&map_a, a.a, p.K, p.M, 1, a.lda, 0, kHalf)) return ASGD_EINVAL;
    if (!encode(&map_b, a.b, p.K, p.N, p.inner ? 1 : max(p.groups, 1), a.ldb, a.b_group, kHalf)) return ASGD_EINVAL;
  }
  p.idesc = instruction(a.a_type, a.b_type, kPairCols, kPairRows);
  p.tiles_n = (int)ceil_div(p.N, kPairCols);
  const long long most = most_tiles(p, kPairRows, kPairCols);
  if (most > kMostTiles) return ASGD_EUNSUPPORTED;
  // C by tensor map where its rows (and groups) start at 16-byte boundaries
  CUtensorMap map_c{};
  const long long size = (long long)type_bytes(a.c_type), outer = p.inner ? p.groups : 1;
  p.c_by_map = aligned(a.c, 16) && a.ldc * size % 16 == 0 && (outer == 1 || (a.c_group > 0 && a.c_group * size % 16 == 0));
  if (p.c_by_map) {
    const CUtensorMapDataType type = a.c_type == ASGD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : a.c_type == ASGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    p.c_by_map = encode(&map_c, type, CU_TENSOR_MAP_SWIZZLE_64B, a.c, p.N, p.M, outer, a.ldc * size, a.c_group * size, (unsigned)(64 / size), 32);
  }
  const auto kernel = a.b_square ? product_pair_kernel<false> : product_pair_kernel<true>;
  static std::atomic<unsigned long long> done[2] = {{0}, {0}};
  if (!allow_smem(kernel, kPairSmem, done[a.b_square])) return ASGD_ECUDA;
  const dim3 grid((unsigned)min(most, (long long)(kSMs / 2)) * 2);
  return launch_after(kernel, grid, kPairThreads, kPairSmem, st, p, map_a, map_b, map_c) ? ASGD_OK : ASGD_ECUDA;
}

// Which kernel: the one whose blocks are through first, by the K blocks the busiest of them meets and the time of one.
// Microseconds of a K block, measured where operands come from L2 (4096 x 4096 x 4096; the pair with a scale per column
// from weight gradients of 2048 x 2048): tiles of 16, 32, 64 and 128 rows 0.29, 0.31, 0.43 and 0.66, the pair 0.50, with
// scales per column 0.80; about 1 us a tile for its beginning and end.
enum Kernel { FEW16, FEW32, FEW64, FEW128, PAIR };
Kernel choose(const Params& p) {
  static const int rows_of[5] = {16, 32, 64, 128, kPairRows};
  const double block_us[5] = {0.29, 0.31, 0.43, 0.66, p.sb_shift ? 0.50 : 0.80};
  const int groups = max(p.groups, 1);
  const double kblocks = p.inner ? std::ceil((double)p.kblocks / groups) : p.kblocks;
  Kernel best = FEW16;
  double best_us = 0;
  for (int k = FEW16; k <= PAIR; ++k) {
    const int bm = rows_of[k];
    // tile rows: a group's last one is half full on average, and a group with rows has one at least
    const double tile_rows = p.inner ? (double)ceil_div(p.M, bm) * groups
                             : groups > 1 ? std::max(std::min((double)p.M, (double)groups), (double)p.M / bm + 0.5 * groups) : (double)ceil_div(p.M, bm);
    const double tiles = std::ceil(tile_rows) * (double)ceil_div(p.N, k == PAIR ? kPairCols : kU);
    const int split = k == PAIR ? 1 : split_of(p, bm);
    const double turns = std::ceil(tiles * split / (k == PAIR ? kSMs / 2 : kSMs));
    const double us = turns * (std::ceil(kblocks / split) * block_us[k] + 1.0) + (split > 1 ? 1.0 : 0.0);
    if (k == FEW16 || us < best_us) { best = (Kernel)k; best_us = us; }
  }
  return best;
}

}  // namespace

// For the kernels of other sources that report to the same word and take the same drill (asgd_maps.cuh).
namespace asgd {
namespace experts {
WaitDrill wait_drill() { return {g_wait_limit.load(), g_withhold.load()}; }
int* status_word() {
  static std::atomic<int*> known[64];
  int dev = 0;
  if (!good(cudaGetDevice(&dev))) return nullptr;
  if (dev < 64 && known[dev].load()) return known[dev].load();
  void* at = nullptr;
  if (!good(cudaGetSymbolAddress(&at, g_status))) return nullptr;
  if (dev < 64) known[dev].store(reinterpret_cast<int*>(at));
  return reinterpret_cast<int*>(at);
}
}  // namespace experts
}  // namespace asgd

extern "C" int asgd_product(const asgd_product_args* args, void* stream) {
  if (!args) return ASGD_EINVAL;
  const asgd_product_args& a = *args;
  if (a.M < 0 || a.N < 0 || a.K < 0 || a.groups < 0 || (a.inner != 0 && a.inner != 1) || (a.b_square != 0 && a.b_square != 1)) return ASGD_EINVAL;
  if (!eight_bit_type(a.a_type) || !eight_bit_type(a.b_type) || !float_type(a.c_type)) return ASGD_EINVAL;
  if ((a.groups > 0) != (a.offsets != nullptr) || (a.inner && !a.groups)) return ASGD_EINVAL;
  if (a.lda < a.K || a.ldb < a.K || a.ldc < a.N || (a.K > 0 && (a.lda % 16 || a.ldb % 16))) return ASGD_EINVAL;
  // row, column and inner numbers of whole tiles (256 at most) stay inside 32 bits
  if (std::max({a.M, a.N, a.K}) > ASGD_PRODUCT_MAX || a.groups > ASGD_MAX_EXPERTS) return ASGD_EUNSUPPORTED;
  if (a.M == 0 || a.N == 0) return ASGD_OK;
  if (!a.c || !aligned(a.c, type_bytes(a.c_type)) || !aligned_words(a.offsets)) return ASGD_EINVAL;
  if (a.K > 0 && (!a.a || !a.b || !a.a_scale || !a.b_scale || !aligned(a.a, 16) || !aligned(a.b, 16) || !aligned_words(a.a_scale, a.b_scale))) return ASGD_EINVAL;
  if (a.groups > 1 && !a.inner && (a.b_group % 16 || a.b_group < 0)) return ASGD_EINVAL;
  Params p;
  p.M = (int)a.M; p.N = (int)a.N; p.K = (int)a.K; p.groups = a.groups; p.inner = a.inner;
  p.tiles_n = 0;                                     // and the instruction: by the kernel that takes the call
  p.kblocks = (int)ceil_div(a.K, kKB);
  p.sa = a.a_scale; p.sa_row = a.a_scale_row; p.sa_block = a.a_scale_block;
  p.sb = a.b_scale; p.sb_row = a.b_scale_row; p.sb_block = a.b_scale_block; p.sb_group = a.b_scale_group;
  p.sb_shift = a.b_square ? 7 : 0;
  p.c = a.c; p.ldc = a.ldc; p.c_group = a.c_group; p.c_type = a.c_type; p.c_by_map = 0;
  p.offsets = a.offsets;
  p.idesc = 0;
  p.wait_limit = g_wait_limit.load();
  p.withhold = g_withhold.load();
  cudaStream_t st = (cudaStream_t)stream;
  switch (choose(p)) {
    case FEW16: return launch_few<16>(a, p, st);
    case FEW32: return launch_few<32>(a, p, st);
    case FEW64: return launch_few<64>(a, p, st);
    case FEW128: return launch_few<128>(a, p, st);
    default: return launch_pair(a, p, st);
  }
}

extern "C" int asgd_experts_sync(void* stream) {
  const cudaStream_t st = (cudaStream_t)stream;
  if (!good(cudaStreamSynchronize(st))) return ASGD_ECUDA;
  static std::mutex turn;                              // g_taken holds one answer at a time
  const std::lock_guard<std::mutex> mine(turn);
  int status = 0;
  if (!launch_after(take_status_kernel, dim3(1), 1, 0, st)) return ASGD_ECUDA;
  if (!good(cudaMemcpyFromSymbolAsync(&status, g_taken, sizeof(int), 0, cudaMemcpyDeviceToHost, st))) return ASGD_ECUDA;
  return good(cudaStreamSynchronize(st)) ? status : ASGD_ECUDA;
}

extern "C" int asgd_product_set_wait_drill(uint32_t wait_limit, int32_t withhold) {
  if (wait_limit == 0) return ASGD_EINVAL;
  g_wait_limit.store(wait_limit);
  g_withhold.store(withhold != 0);
  return ASGD_OK;
}
