// Matrix products on the tensor cores of sm_100a: descriptors, tensor maps and instructions that the kernels of head.cu are put together from.
//
// A pair of CTAs (a cluster of two) multiplies a 256 x BN tile: each CTA brings its 128 rows of A and its half of B's rows into its own shared
// memory by tensor copies, one thread of the first CTA issues the products for both (tcgen05.mma with cta_group::2 reads the two halves where
// they lie), and each CTA finds its 128 rows of the result in its own tensor memory.  Against single CTAs of 128 x BN this halves what B costs in
// shared memory and L2 traffic.  Operands are 16-bit and lie in shared memory in blocks of 64 x 64 elements (128-byte rows, 128-byte swizzle):
// a block's rows may run along the product's inner dimension or across it, so that no matrix is ever transposed in memory.
#pragma once

#include <cuda.h>

#include "stream_pipe.cuh"

namespace solon {
namespace tiles {

constexpr int kBlock = 64;               // elements of a block in either direction
constexpr uint32_t kBlockBytes = kBlock * kBlock * 2;
constexpr int kRows = 128;               // rows of A that a CTA holds

// Descriptor of an operand in shared memory.  Rows along the inner dimension ("K"): groups of eight rows are 1024 bytes apart.  Rows across it
// ("MN"): blocks of 64 result rows are kBlockBytes apart, groups of eight inner indices 1024 bytes.
template <bool ALONG_K>
__device__ __forceinline__ uint64_t operand(uint32_t smem) {
  const uint64_t fixed = (1ull << 46) | (2ull << 61) | ((uint64_t)(1024 >> 4) << 32);      // version, 128-byte swizzle, stride of groups
  return fixed | ((uint64_t)(ALONG_K ? 1 : kBlockBytes >> 4) << 16) | ((smem & 0x3FFFF) >> 4);
}
// 16 inner indices further, in descriptor units of 16 bytes.
template <bool ALONG_K>
constexpr uint32_t kStep16 = ALONG_K ? 32 >> 4 : 2048 >> 4;

// Instruction descriptor: float32 accumulators, both operands bfloat16 or both float16, 256 x n.
__host__ __device__ constexpr uint32_t instruction(bool bf16, bool a_along_k, bool b_along_k, int n) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_along_k ? 0u : 1u) << 15) | ((b_along_k ? 0u : 1u) << 16) |
         ((uint32_t)(n >> 3) << 17) | ((256u >> 4) << 24);
}

__device__ __forceinline__ void multiply(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}

// Arrives at the barrier of this address in both CTAs when all products issued so far are done.
__device__ __forceinline__ void commit_to_both(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(pipe::smem_addr(bar)),
               "h"((uint16_t)3)
               : "memory");
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// pipe::mbar_wait that says whether the phase completed: false once a wait of this CTA has run out.  (The flag is not looked at where there is nothing to wait
// for, which is the case that the loops are made for.)
__device__ __forceinline__ bool waited(uint64_t* bar, uint32_t parity, int* abort_flag, int* status) {
  if (pipe::mbar_try_wait(bar, parity)) return true;
  pipe::mbar_wait(bar, parity, abort_flag, status);
  return !*(volatile int*)abort_flag;
}

template <int COLUMNS>
__device__ __forceinline__ void tmem_alloc(uint32_t* where) {          // one warp of each CTA
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(pipe::smem_addr(where)), "n"(COLUMNS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
template <int COLUMNS>
__device__ __forceinline__ void tmem_free(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLUMNS));
}

// 32 columns of the warp's 32 lanes: register i of lane l is column i of lane l.
__device__ __forceinline__ void tmem_load32(uint32_t tmem, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(tmem));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// One block of a tensor map into this CTA's shared memory; its bytes are counted on the first CTA's barrier of that address.
__device__ __forceinline__ void load_block(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(pipe::smem_addr(bar) & 0xFEFFFFFFu)
      : "memory");
}
// The same of a map by blocks: `block` counts blocks of 64 columns.
__device__ __forceinline__ void load_blocks(uint32_t dst, const CUtensorMap* map, int y, int block, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(0), "r"(y), "r"(block), "r"(z), "r"(pipe::smem_addr(bar) & 0xFEFFFFFFu)
      : "memory");
}
// A block from this CTA's shared memory to where a map says; what lies outside is not written.
__device__ __forceinline__ void store_block(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Arrives at the first CTA's barrier of this address.  (What the arrival orders are reads of tensor memory, by fence_before; a release for the whole
// cluster would wait for this warp's stores to global memory as well: 8 % of the time of short products with much to write.)
__device__ __forceinline__ void arrive_at_first(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .b32 at;\n\tmapa.shared::cluster.u32 at, %0, 0;\n\t"
      "mbarrier.arrive.shared::cluster.b64 _, [at];\n\t}" ::"r"(pipe::smem_addr(bar))
      : "memory");
}

// ------------------------------------------------------------------------------------------------------------ host

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      p = nullptr;
    }
    return (EncodeTiled)p;
  }();
  return fn;
}

inline bool encode_map(CUtensorMap* map, const void* p, CUtensorMapDataType type, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                       const cuuint32_t* box) {
  const EncodeTiled encode = encode_tiled();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return encode && encode(map, type, rank, const_cast<void*>(p), dims, strides, box, ones,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline CUtensorMapDataType type16(bool bf16) { return bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }

// slabs x rows x cols elements of `size` bytes to be written in blocks of 32 rows x 128 bytes.
inline bool output_map(CUtensorMap* map, const void* p, int size, int64_t cols, int64_t rows, int64_t slabs, int64_t pitch, int64_t slab) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)slabs};
  const cuuint64_t strides[2] = {(cuuint64_t)(pitch * size), (cuuint64_t)(slab * size)};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / size), 32, 1};
  return encode_map(map, p, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : size == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_FLOAT64, 3, dims,
                    strides, box);
}

// slabs x rows x cols elements of 16 bits, row pitch and slab distance in elements (multiples of 8); boxes of box_rows x 64.  What lies outside
// reads as zeros and is not written.
inline bool tensor_map(CUtensorMap* map, const void* p, bool bf16, int64_t cols, int64_t rows, int64_t slabs, int64_t pitch, int64_t slab, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)slabs};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)slab * 2};
  const cuuint32_t box[3] = {kBlock, (cuuint32_t)box_rows, 1};
  return encode_map(map, p, type16(bf16), 3, dims, strides, box);
}

// The same by blocks of 64 columns, two of 64 rows a box, one behind the other: one copy where there would be two.  All columns of the last block have to be
// there (a pitch of at least up to its end).
inline bool tensor_map_by_blocks(CUtensorMap* map, const void* p, bool bf16, int64_t cols, int64_t rows, int64_t slabs, int64_t pitch, int64_t slab) {
  const cuuint64_t dims[4] = {kBlock, (cuuint64_t)rows, (cuuint64_t)(cols + kBlock - 1) / kBlock, (cuuint64_t)slabs};
  const cuuint64_t strides[3] = {(cuuint64_t)pitch * 2, kBlock * 2, (cuuint64_t)slab * 2};
  const cuuint32_t box[4] = {kBlock, kBlock, 2, 1};
  return encode_map(map, p, type16(bf16), 4, dims, strides, box);
}

}  // namespace tiles
}  // namespace solon
