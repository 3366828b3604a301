// Product of microscaled 4-bit matrices on the tensor cores: dense and grouped over rows.  The contract is in
// include/asgd_fp4.h, the kernels in asgd_product4_few.cuh and asgd_product4_pair.cuh.
#include <algorithm>
#include <cmath>

#include "../../include/asgd_fp4.h"
#include "asgd_maps.cuh"
#include "asgd_product4_few.cuh"
#include "asgd_product4_pair.cuh"

namespace {

constexpr long long kMostTiles = 0x7fffffffll - 2 * kSMs;    // a block's next tile number stays inside 32 bits

// the most tiles of bm x bn there can be: what the offsets say is known on the device alone
long long most_tiles(const Params& p, int bm, int bn) { return (ceil_div(p.M, bm) + p.groups) * ceil_div(p.N, bn); }

// E2M1 operands with scales that are powers of two; columns and rows of the instruction
unsigned instruction4(int cols, int rows) { return 1u << 7 | 1u << 10 | (unsigned)(cols >> 3) << 17 | 1u << 23 | (unsigned)(rows >> 7) << 27; }

// numbers, 128 bytes by `box_rows` rows, and their scales, 16 bytes by `scale_rows` rows
bool encode4(CUtensorMap* numbers, CUtensorMap* scales, const Params4& p, const void* x, long long rows, long long outer, long long ld, long long outer_bytes,
             unsigned box_rows, const void* s, long long s_row, long long s_outer, unsigned scale_rows) {
  return encode(numbers, x, p.K, rows, outer, ld, outer_bytes, box_rows) &&
         encode(scales, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_NONE, s, ceil_div(p.K, ASGD_BLOCK4 / 2), rows, outer, s_row, s_outer, 16, scale_rows);
}

// `split` blocks share a tile (1: a block takes whole tiles in turn)
template <int BN, bool kSplit> int launch_few(const asgd_product4_args& a, Params4 p, int split, cudaStream_t st) {
  CUtensorMap map_u{}, map_v{}, map_su{}, map_sv{};
  if (p.K > 0) {
    if (!encode4(&map_u, &map_su, p, a.b, p.N, std::max(p.groups, 1), a.ldb, a.b_group, kU, a.b_scale, a.b_scale_row, a.b_scale_group, kU)) return ASGD_EINVAL;
    if (!encode4(&map_v, &map_sv, p, a.a, p.M, 1, a.lda, 0, BN, a.a_scale, a.a_scale_row, 0, BN)) return ASGD_EINVAL;
  }
  p.idesc = instruction4(BN, kU);
  p.tiles_n = (int)ceil_div(p.N, kU);
  const long long most = most_tiles(p, BN, kU);
  if (most > kMostTiles) return ASGD_EUNSUPPORTED;
  static std::atomic<unsigned long long> done{0};
  if (!allow_smem(product4_few_kernel<BN, kSplit>, Few4<BN>::kSmem, done)) return ASGD_ECUDA;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;    // see launch_after
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (unsigned)split;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(kSplit ? (unsigned)(most * split) : (unsigned)std::min(most, (long long)kSMs));
  cfg.blockDim = dim3(Few4<BN>::kThreads);
  cfg.dynamicSmemBytes = Few4<BN>::kSmem;
  cfg.stream = st;
  cfg.attrs = attrs;
  cfg.numAttrs = kSplit ? 2 : 1;
  return good(cudaLaunchKernelEx(&cfg, product4_few_kernel<BN, kSplit>, p, map_u, map_v, map_su, map_sv)) ? ASGD_OK : ASGD_ECUDA;
}

// Blocks per tile of the few-rows kernel, as for 8-bit products (split_of in asgd_product.cu): one unit each at least.
int split_of(const Params& p, int bn) {
  const long long most = most_tiles(p, bn, kU);
  for (const int split : {8, 4, 2})
    if (most <= (split == 8 ? 14 : split == 4 ? 32 : kSMs / 2) && p.kblocks >= split) return split;
  return 1;
}
template <int BN> int launch_few(const asgd_product4_args& a, const Params4& p, cudaStream_t st) {
  const int split = split_of(p, BN);
  return split > 1 ? launch_few<BN, true>(a, p, split, st) : launch_few<BN, false>(a, p, 1, st);
}

template <int NT> int launch_pair(const asgd_product4_args& a, Params4 p, cudaStream_t st) {
  CUtensorMap map_a{}, map_b{}, map_sa{}, map_sb{};
  if (p.K > 0) {
    if (!encode4(&map_a, &map_sa, p, a.a, p.M, 1, a.lda, 0, kHalf, a.a_scale, a.a_scale_row, 0, kHalf)) return ASGD_EINVAL;
    if (!encode4(&map_b, &map_sb, p, a.b, p.N, std::max(p.groups, 1), a.ldb, a.b_group, NT / 2, a.b_scale, a.b_scale_row, a.b_scale_group, NT)) return ASGD_EINVAL;
  }
  p.idesc = instruction4(NT, kPairRows);
  p.tiles_n = (int)ceil_div(p.N, NT);
  const long long most = most_tiles(p, kPairRows, NT);
  if (most > kMostTiles) return ASGD_EUNSUPPORTED;
  // C by tensor map where its rows start at 16-byte boundaries
  CUtensorMap map_c{};
  const long long size = (long long)type_bytes(a.c_type);
  p.c_by_map = aligned(a.c, 16) && a.ldc * size % 16 == 0;
  if (p.c_by_map) {
    const CUtensorMapDataType type = a.c_type == ASGD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : a.c_type == ASGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    p.c_by_map = encode(&map_c, type, CU_TENSOR_MAP_SWIZZLE_64B, a.c, p.N, p.M, 1, a.ldc * size, 0, (unsigned)(64 / size), 32);
  }
  static std::atomic<unsigned long long> done{0};
  if (!allow_smem(product4_pair_kernel<NT>, Pair4<NT>::kSmem, done)) return ASGD_ECUDA;
  const dim3 grid((unsigned)std::min(most, (long long)(kSMs / 2)) * 2);
  return launch_after(product4_pair_kernel<NT>, grid, kPairThreads, Pair4<NT>::kSmem, st, p, map_a, map_b, map_sa, map_sb, map_c) ? ASGD_OK : ASGD_ECUDA;
}

// Which kernel: the one whose blocks are through first, by the units and the tiles that the busiest of them meets.  The microseconds of
// each are a fit to a sweep of 64 shapes in which each kernel was forced (dense and grouped, 5 to 16384 rows); there the rule's kernel is the
// best one or within 5 % of it but for two, 6 and 11 % off.
enum Kernel { FEW16, FEW32, FEW64, FEW128, PAIR };
Kernel choose(const Params& p) {
  static const int rows_of[5] = {16, 32, 64, 128, kPairRows};
  static const double unit_us[5] = {0.34, 0.31, 0.34, 1.01, 0.62}, tile_us[5] = {0.3, 0.6, 0.7, 0.6, 0.6};
  const int groups = std::max(p.groups, 1);
  Kernel best = FEW16;
  double best_us = 0;
  for (int k = FEW16; k <= PAIR; ++k) {
    const int bm = rows_of[k];
    // tile rows: a group's last one is half full on average, and a group with rows has one at least
    const double tile_rows = groups > 1 ? std::max(std::min((double)p.M, (double)groups), (double)p.M / bm + 0.5 * groups) : (double)ceil_div(p.M, bm);
    const double tiles = std::ceil(tile_rows) * (double)ceil_div(p.N, k == PAIR ? 256 : kU);
    const int split = k == PAIR ? 1 : split_of(p, bm);
    const double turns = std::ceil(tiles * split / (k == PAIR ? kSMs / 2 : kSMs));
    const double us = turns * (std::ceil((double)p.kblocks / split) * unit_us[k] + tile_us[k]) + (split > 1 ? 0.8 : 0.0) + (k == PAIR ? 1.5 : 0.0);
    if (k == FEW16 || us < best_us) { best = (Kernel)k; best_us = us; }
  }
  return best;
}

}  // namespace

extern "C" int asgd_product4(const asgd_product4_args* args, void* stream) {
  if (!args) return ASGD_EINVAL;
  const asgd_product4_args& a = *args;
  if (a.M < 0 || a.N < 0 || a.K < 0 || a.groups < 0 || !float_type(a.c_type)) return ASGD_EINVAL;
  if ((a.groups > 0) != (a.offsets != nullptr)) return ASGD_EINVAL;
  const long long bytes = ceil_div(a.K, 2), blocks = ceil_div(a.K, ASGD_BLOCK4);
  if (a.lda < bytes || a.ldb < bytes || a.ldc < a.N || a.a_scale_row < blocks || a.b_scale_row < blocks) return ASGD_EINVAL;
  // row, column and inner numbers of whole tiles (256 at most) stay inside 32 bits
  if (std::max({a.M, a.N, a.K}) > ASGD_PRODUCT_MAX || a.groups > ASGD_MAX_EXPERTS) return ASGD_EUNSUPPORTED;
  if (a.M == 0 || a.N == 0) return ASGD_OK;
  if (!a.c || !aligned(a.c, type_bytes(a.c_type)) || !aligned_words(a.offsets)) return ASGD_EINVAL;
  if (a.K > 0) {
    if (!a.a || !a.b || !a.a_scale || !a.b_scale || !aligned(a.a, 16) || !aligned(a.b, 16) || !aligned(a.a_scale, 16) || !aligned(a.b_scale, 16)) return ASGD_EINVAL;
    if (a.lda % 16 || a.ldb % 16 || a.a_scale_row % 16 || a.b_scale_row % 16) return ASGD_EINVAL;
    if (a.groups > 1 && (a.b_group % 16 || a.b_group < 0 || a.b_scale_group % 16 || a.b_scale_group < 0)) return ASGD_EINVAL;
  }
  const WaitDrill drill = wait_drill();
  Params4 p{};
  p.M = (int)a.M; p.N = (int)a.N; p.K = (int)bytes; p.groups = a.groups;
  p.kblocks = (int)ceil_div(bytes, kUnit);
  p.c = a.c; p.ldc = a.ldc; p.c_type = a.c_type;
  p.offsets = a.offsets;
  p.wait_limit = drill.limit;
  p.withhold = drill.withhold;
  p.status = status_word();
  if (!p.status) return ASGD_ECUDA;
  cudaStream_t st = (cudaStream_t)stream;
  switch (choose(p)) {
    case FEW16: return launch_few<16>(a, p, st);
    case FEW32: return launch_few<32>(a, p, st);
    case FEW64: return launch_few<64>(a, p, st);
    case FEW128: return launch_few<128>(a, p, st);
    default: return launch_pair<256>(a, p, st);
  }
}
