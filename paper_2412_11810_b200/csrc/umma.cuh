// Matrix products on the 5th-generation tensor cores by pairs of SMs (tcgen05, cta_group::2), for 16-bit operands of any
// majorness: the wrappers, and the pipeline that feeds them.
//
// A pair of thread blocks (a cluster of two) computes a 256 x 256 tile: each block keeps 128 rows of A and 128 of B in its
// shared memory and 128 x 256 fp32 accumulators in its tensor memory, and one thread of the even block issues the products
// of both.  Each block thereby loads half of what two single blocks would (32 KB per 64-deep k-block for 128 x 256 of the
// result), which is what the L2 can deliver at the tensor cores' rate.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tma.cuh"

namespace snnk {

constexpr int UM_TILE = 256;            // rows of A and of B per pair of blocks
constexpr int UM_HALF = 128;            // ... per block
constexpr int UM_KB = 64;               // depth of a k-block: 128 bytes of a K-major row
constexpr int UM_STAGES = 6;
constexpr uint32_t UM_OPERAND_BYTES = UM_HALF * UM_KB * 2;      // 16 KB
constexpr uint32_t UM_STAGE_BYTES = 2 * UM_OPERAND_BYTES;
constexpr uint32_t UM_TMEM_COLS = 512;  // two accumulators of 256 columns

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address that `smem_addr` has in the shared memory of another block of the cluster
__device__ __forceinline__ uint32_t peer_address(uint32_t smem_addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr), "r"(rank));
  return a;
}
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Tiled copy into this block's shared memory; the barrier may be the other block's of the pair.
__device__ __forceinline__ void tma_pair_load_3d(void* smem_dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar_addr) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem_u32(smem_dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar_addr) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, const void* smem_src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z),
               "r"(smem_u32(smem_src)) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void bulk_read_done() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ void bulk_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ void pair_tmem_alloc(uint32_t* smem_result, uint32_t n_cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_result)), "r"(n_cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t n_cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(n_cols) : "memory");
}
__device__ __forceinline__ void tcgen05_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Descriptor of an operand tile in shared memory, 128-byte swizzle.  K-major: rows of 64 values (128 bytes), groups of 8
// rows 1024 bytes apart.  MN-major: blocks of 64 (rows of the operand) x 64 (k), a k per 128-byte line; 8 k are 1024 bytes,
// blocks 64 * 128 bytes apart.
template <bool MN_MAJOR> __device__ __forceinline__ uint64_t operand_descriptor(uint32_t smem_addr) {
  uint64_t d = (uint64_t)((smem_addr & 0x3ffffu) >> 4);
  d |= (uint64_t)(MN_MAJOR ? (UM_KB * 128) >> 4 : 1) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// bytes from one k-step of 16 to the next
template <bool MN_MAJOR> __host__ __device__ constexpr uint32_t kstep_bytes() { return MN_MAJOR ? 16 * 128 : 32; }
// kind::f16 with fp32 accumulators, 256 x 256; both operands bf16 or both fp16
__device__ __forceinline__ uint32_t f16_instruction(bool bf16, bool a_mn_major, bool b_mn_major) {
  const uint32_t type = bf16 ? 1u : 0u;
  return (1u << 4) | (type << 7) | (type << 10) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) |
         ((uint32_t)(UM_TILE >> 3) << 17) | ((uint32_t)(UM_TILE >> 4) << 24);
}
__device__ __forceinline__ void pair_mma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc),
      "r"(accumulate ? 1u : 0u) : "memory");
}
// One arrival at the barrier of this offset in both blocks once the products issued so far by this thread are complete.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3) : "memory");
}
// 32 lanes x 32 columns of 32 bits: thread = lane of tensor memory (row), registers = consecutive columns.  The wait is
// part of the statement, so that no use of the registers can move ahead of it.
__device__ __forceinline__ void tmem_load_32(uint32_t taddr, float (&v)[32]) {
  __syncwarp();   // (the whole warp takes part)
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
        "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}

// The same for 16 columns.
__device__ __forceinline__ void tmem_load_16(uint32_t taddr, float (&v)[16]) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr) : "memory");
}

// Host side: a 3-D tensor map [planes][rows][cols] of 16-bit values, rows `pitch` values apart (a multiple of 8), box of
// 64 columns (128 bytes, 128-byte swizzle) x box_rows.
inline bool make_tensor_map_16bit(CUtensorMap* out, const void* base, bool bf16, uint64_t cols, uint64_t rows, uint64_t planes,
                                  uint64_t pitch, uint64_t plane_stride, uint32_t box_rows) {
  tensor_map_encode_fn encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[3] = {cols, rows, planes};
  const cuuint64_t strides[2] = {pitch * 2, plane_stride * 2};
  const cuuint32_t box[3] = {64, box_rows, 1}, elem[3] = {1, 1, 1};
  return encode(out, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides,
                box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace snnk
