// Tensor maps of bf16 matrices and the tile load through them (the issuing CTA's shared memory only).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace locmoe {

// K-major bf16 matrix [outer...][rows][K] with a box of box_rows x 64 elements, 128-byte swizzle; false on failure.
bool make_map(CUtensorMap* map, const void* ptr, int rank, const uint64_t* dims, uint32_t box_rows);
// Row-major bf16 [outer][rows][cols], cols a multiple of 64, as [outer][cols / 64][rows][64] with a box of chunks x box_rows x 64.
bool make_map_chunks(CUtensorMap* map, const void* ptr, uint64_t cols, uint64_t rows, uint64_t outer, uint32_t box_rows, uint32_t chunks);
// Row-major [outer][rows][cols] for stores, a box of 32 rows x 128 bytes, 128-byte swizzle.
bool make_store_map(CUtensorMap* map, void* ptr, bool f32, uint64_t cols, uint64_t rows, uint64_t outer);

#ifdef __CUDACC__
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {   // by shared-memory address
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1)
                 : "memory");
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int c0, int c1, uint64_t* bar) {
    tma_load_2d(smem_u32(dst), map, c0, c1, smem_u32(bar));
}
#endif

}  // namespace locmoe
