// Tensor maps and copies of the paged cache, and the waits and exponentials that
// the attention kernels share.
#pragma once

#include <cuda.h>

#include "attention.cuh"

namespace sls {

// One lane of the warp, the same every time.  The copies and products that one lane
// issues are written as predicated instructions of the whole warp, not as a branch of
// that lane, with operands that are the same in all lanes (prefill of 8192 tokens, the
// products' warp: 556 us with a branch, 525 without, in an early build).
SLS_DEV uint32_t at_elect() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(r));
  return r;
}

SLS_DEV void at_tma3(uint32_t lead, uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                     uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %6, 0;\n"
      " @q cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];\n}\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)), "r"(lead)
      : "memory");
}
SLS_DEV void at_tma4(uint32_t lead, uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                     int w, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %7, 0;\n"
      " @q cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];\n}\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)),
      "r"(lead)
      : "memory");
}

// 2^x by the hardware's approximation (2 units of 2^-23 relative; results below
// 2^-126 are 0).
SLS_DEV float at_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- host: tensor maps ----------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn at_encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// 16-bit elements, 128-byte swizzle, zeros outside the tensor.
inline bool at_map(CUtensorMap* map, int dtype, int rank, const void* base,
                   const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const EncodeTiledFn fn = at_encode_fn();
  if (!fn) return false;
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  return fn(map,
            dtype == SLS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
            (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// K or V of the cache as (element, slot, head, page), boxes of 64 elements and
// `slots` slots of one head: a page number outside the cache reads as zeros.
inline bool at_cache_map(CUtensorMap* map, int dtype, const CacheView& c, const void* base,
                         int slots) {
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)1 << c.page_shift,
                              (cuuint64_t)c.kv_heads, (cuuint64_t)c.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_b, (cuuint64_t)c.head_b, (cuuint64_t)c.page_b};
  const cuuint32_t box[4] = {64, (cuuint32_t)slots, 1, 1};
  return at_map(map, dtype, 4, base, dims, strides, box);
}

// K or V of a cache of codes as (element, slot, head, page), boxes of a head's HD bytes and `slots` slots
// of one head: a page number outside the cache reads as zeros.
template <int HD>
bool at_code_map(CUtensorMap* map, const CacheView& c, const void* base, int slots) {
  const EncodeTiledFn fn = at_encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)1 << c.page_shift,
                              (cuuint64_t)c.kv_heads, (cuuint64_t)c.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.slot_b, (cuuint64_t)c.head_b, (cuuint64_t)c.page_b};
  const cuuint32_t box[4] = {HD, (cuuint32_t)slots, 1, 1}, one[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            HD == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace sls
