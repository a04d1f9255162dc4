// echo_tensor.cuh -- matrix products by pairs of blocks on the tensor cores: barriers, the TMA
// engine, tcgen05 and tensor memory, as the operators' product kernels use them.
//
// A pair of blocks shares a tile (cta_group::2): each holds 128 rows of the first operand and of
// the sums, and half of the second operand's rows.  Stages of 64 columns of the sum are copied
// to both blocks' shared memory (128-byte swizzle), one thread of the pair's first block issues
// the products, and the sums stand in tensor memory, a row a lane.
#pragma once

#include <cuda.h>

#include "echo_ops.cuh"

namespace echo {
namespace {

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// The same place in the pair's first block.
__device__ __forceinline__ uint32_t in_first(uint32_t at) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(r) : "r"(at));
  return r;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
// Sleeps for up to 2 us until the phase of that parity has completed; whether it has.  (Without a time of
// its own, a try comes back soon, and warps that try again and again slow down the threads that copy and
// multiply: 2048 x 2048 by 51200 rows, forward, 278 us instead of 262.)
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok)
               : "r"(bar), "r"(parity), "r"(2000u)
               : "memory");
  return ok;
}
// Bound of every wait of a kernel, and the word in host memory that one sets when it gives up.
struct WaitLimit {
  int32_t *status;
  long long clocks;  // of the SM
};
// Waits until the phase of that parity has completed; false if the block gives up (another
// wait did, or this one's limit has passed).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort, const WaitLimit &w) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > w.clocks) {
      *abort = 1;
      *(volatile int32_t *)w.status = 1;
      __threadfence_system();
      return false;
    }
  }
  return true;
}

// A box of a matrix from (column, row); the column is a multiple of 64.
__device__ __forceinline__ void copy_tile(uint32_t to, const CUtensorMap *map, int col, int row, int z, int plane, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];\n" ::"r"(to),
      "l"(map), "r"(bar), "r"(col), "r"(row), "r"(z), "r"(plane)
      : "memory");
}
// R rows (of P or Q) x 64 columns of the sum from (r, k).  MN: the matrix holds the transpose, so
// boxes of 64 of its rows (the sum) x 64 columns, one behind the other.
template <bool MN, int R>
__device__ __forceinline__ void copy_operand(uint32_t to, const CUtensorMap *map, int r, int k, int z, int plane, uint32_t bar) {
  if constexpr (MN) {
#pragma unroll
    for (int g = 0; g < R / 64; ++g) copy_tile(to + g * 8192, map, r + g * 64, k, z, plane, bar);
  } else {
    copy_tile(to, map, k, r, z, plane, bar);
  }
}

// Descriptor of an operand in shared memory, lines of 128 bytes swizzled in groups of 8 (1024
// bytes).  Lines are rows of the operand, or (MN) of the sum, with 64 rows of the operand on a
// line and the next 64 8192 bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool mn) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(mn ? 8192 >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 16 columns of the sum on: 32 bytes of a line, or 16 lines
constexpr int step16(bool mn) { return (mn ? 2048 : 32) >> 4; }
// 16-bit operands (fp16, or both bf16), fp32 sums, `bn` columns, 256 rows; a_mn, b_mn: MN-major
constexpr uint32_t instruction(int bn, bool a_mn, bool b_mn, bool bf16) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(bn >> 3) << 17 | (256u >> 4) << 24;
}

__device__ __forceinline__ void mma(uint32_t d, uint64_t p, uint64_t q, uint32_t instr, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(p),
               "l"(q), "r"(instr), "r"((uint32_t)add)
               : "memory");
}
// The barriers of both blocks (or of this one) complete once the products issued so far have.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
// 32 columns of this warp's rows of tensor memory; sums_loaded() before the values are used.
struct Sums {
  uint32_t r[32];
};
__device__ __forceinline__ void load_sums(uint32_t at, Sums &s) {
  uint32_t (&r)[32] = s.r;
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void sums_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
// (the wait keeps the compiler from using a register before it: the values pass through it)
__device__ __forceinline__ void pass(Sums &s) {
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(s.r[i]));
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}

// A warp's buffer turns 32 x 32 elements between a row a lane and four lanes to the 64 bytes of
// a row, which is how they meet global memory.  Its halves take turns, so that a half is
// written again only after a synchronisation behind its last reads.  Rows have their 16-byte
// pieces exchanged (64 bytes on, they would meet in the same banks).
__device__ __forceinline__ unsigned char *piece(unsigned char *half, int row, int i) { return half + row * 64 + (i ^ ((row >> 1) & 3)) * 16; }
using Piece = Pack<__half, 8>;

// From a half of the buffer to a matrix of the iteration, by one thread; what is outside the
// matrix is dropped.
__device__ __forceinline__ void store_half(const CUtensorMap *map, const unsigned char *half, int col, int row, int z, int plane) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];\ncp.async.bulk.commit_group;\n" ::"l"(map),
               "r"(smem_u32(half)), "r"(col), "r"(row), "r"(z), "r"(plane)
               : "memory");
}
// Before a half is written: the stores but the last have read theirs, for the whole warp.
__device__ __forceinline__ void half_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;\n" ::: "memory");
  __syncwarp();
}
// What the warp wrote to a half is there for the copy engine.
__device__ __forceinline__ void half_written() {
  asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
  __syncwarp();
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encoder() {
  static const EncodeTiled f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

}  // namespace
}  // namespace echo
