// Host side of the kernels that copy by tensor maps: the maps, shared-memory limits, the word that they report to and the
// drill of their waits.
#pragma once

#include <cudaTypedefs.h>

#include <atomic>

#include "asgd_experts_common.cuh"

namespace asgd {
namespace experts {
struct WaitDrill {
  unsigned limit;
  int withhold;
};
WaitDrill wait_drill();                              // what asgd_product_set_wait_drill has set
int* status_word();                                  // the current device's word of asgd_experts_sync (nullptr: a CUDA error)
}  // namespace experts
}  // namespace asgd

namespace {

using namespace asgd::experts;

inline PFN_cuTensorMapEncodeTiled encoder() {
  static std::atomic<PFN_cuTensorMapEncodeTiled> known{nullptr};
  PFN_cuTensorMapEncodeTiled f = known.load();
  if (!f) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (!good(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q)) || !fn) return nullptr;
    f = (PFN_cuTensorMapEncodeTiled)fn;
    known.store(f);
  }
  return f;
}
// a matrix [outer][rows][cols]; strides in bytes; what lies beyond is read as zeros and not written
inline bool encode(CUtensorMap* map, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void* base, long long cols, long long rows, long long outer,
            long long row_bytes, long long outer_bytes, unsigned box_cols, unsigned box_rows) {
  const PFN_cuTensorMapEncodeTiled f = encoder();
  if (!f) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)outer};
  cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)(outer > 1 ? outer_bytes : row_bytes)};
  cuuint32_t box[3] = {box_cols, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return f(map, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 128-byte K blocks of an 8-bit operand
inline bool encode(CUtensorMap* map, const void* base, long long cols, long long rows, long long outer, long long ld, long long outer_stride, unsigned box_rows) {
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_128B, base, cols, rows, outer, ld, outer_stride, 128, box_rows);
}

// Raises a kernel's shared-memory limit, once per device (`done`: a bit per device, of this kernel).
template <typename K> inline bool allow_smem(K kernel, size_t bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  if (!good(cudaGetDevice(&dev))) return false;
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load() & bit)) return true;
  if (!good(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes))) return false;
  done.fetch_or(bit);
  return true;
}

}  // namespace
