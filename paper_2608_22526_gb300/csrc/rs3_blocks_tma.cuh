// rs3_blocks_tma.cuh -- bulk copies of a bank's blocks: tensor maps of its rows, and loads of
// what is read once.
#pragma once

#include "rs3_tc_host.cuh"
#include "rs3_tc_ptx.cuh"

namespace tc {

// A tensor map of `rows` rows of D elements whose copies are `box_rows` rows of `cols` columns, as they lie or in the
// 128-byte swizzle (64 columns of bf16); `promotion`: what L2 fetches around what is asked for.
inline bool make_rows_map(CUtensorMap *m, const void *store, int elem_bytes, int64_t D, int64_t rows, int cols, int box_rows,
                          bool swizzled = false, CUtensorMapL2promotion promotion = CU_TENSOR_MAP_L2_PROMOTION_L2_256B)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)D * (cuuint64_t)elem_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)cols, (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return enc(m, elem_bytes == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void *>(store),
               dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
               promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// tma_load_2d of data that is read once: its lines are the first to leave L2.
__device__ __forceinline__ uint64_t l2_once()
{
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
__device__ __forceinline__ void tma_load_2d_once(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, uint64_t policy)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar), "l"(policy)
        : "memory");
}

}  // namespace tc
