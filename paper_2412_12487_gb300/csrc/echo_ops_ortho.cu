// echo_ops_ortho.cu -- orthogonalised updates by Newton-Schulz products.
//
// With Y the matrix that has n rows and m <= n columns (G, or its transpose), a step is three
// products:
//   A = Y^T Y,  B = b A + c A A,  Y' = a Y + Y B.
// A and B are symmetric, so each product is P Q^T with the sum along the rows of both in memory
// (K-major), but for the first, whose sum runs down Y's columns: the tensor core takes that
// order too (MN-major).  Y is all that a step keeps.  The symmetric products compute the tiles
// that reach the lower triangle and write each block to both places.
//
// Elements are sums of two fp16 numbers times a power of two (the iterate's singular values stay
// near 1, so its elements are at most that): 22 bits of all but small ones (kScaleY), whatever the
// matrices' type, multiplied as high * high + high * low + low * high with sums in fp32.  One
// number an element takes a third of the products, but leaves a bf16 result 2.1e-3 off, 1.7e-3 of
// which is its own rounding.
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace {

// What is stored of Y, A and B: the true value times this.  fp16 holds 2^-24 to 65504, so
// elements up to 16 fit (64 of B), and 22 bits remain of elements down to 2^-14 (2^-12 of B);
// smaller ones keep an error of 2^-37 (2^-35), which the norm of a matrix does not see: 2^32 such
// elements add up to 2^-21.
constexpr int kScaleYLog2 = 12;
constexpr float kScaleY = 1 << kScaleYLog2, kScaleA = 0x1p12f, kScaleB = 0x1p10f;

// -- Frobenius norm ------------------------------------------------------------------------------
// Sums of squares of x, of 2^-90 x and of 2^90 x.  Of up to 2^32 elements between 2^-149 and 2^128
// the second sum stays below 2^108, and the third has no term below 2^-118; the plain one keeps
// its digits for norms from 2^-40 to 2^50.  A block sums a part of one matrix (one without gaps
// comes as a single row).  Bound by the bytes of G: 2048 x 8192 in fp32, 6.7e7 bytes, 15 us, 4.5 TB/s.
template <typename T, int W>
__global__ void __launch_bounds__(256) ortho_norm_kernel(OrthoArgs a, int64_t rows, int64_t cols, float *part, int32_t *arrived, int n_arrived) {
  __shared__ float sh[3][8];
  const float up = 0x1p90f, down = 0x1p-90f;
  kernel_begin();
  next_may_start();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < n_arrived; i += blockDim.x) arrived[i] = 0;
  const int64_t pieces = cols / W, all = rows * pieces;
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    float s[3] = {0.f, 0.f, 0.f};
    const T *g = static_cast<const T *>(a.g) + z * a.g_batch_stride;
    constexpr int kFlight = 4;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 * kFlight + threadIdx.x; i0 < all; i0 += (int64_t)gridDim.x * 256 * kFlight) {
      float v[kFlight][W];
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        const int64_t i = i0 + k * 256;
#pragma unroll
        for (int e = 0; e < W; ++e) v[k][e] = 0.f;
        if (i < all) load_piece<W>(rows == 1 ? g + i * W : g + i / pieces * a.g_stride + i % pieces * W, v[k]);
      }
#pragma unroll
      for (int k = 0; k < kFlight; ++k)
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float x = v[k][e], lo = x * up, hi = x * down;
          s[0] += x * x;
          s[1] += hi * hi;
          s[2] += lo * lo;
        }
    }
    for (int q = 0; q < 3; ++q) {
      s[q] = warp_sum(s[q]);
      if ((threadIdx.x & 31) == 0) sh[q][threadIdx.x >> 5] = s[q];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
      float t = 0.f;
      for (int w = 0; w < 8; ++w) t += sh[threadIdx.x][w];
      part[(z * gridDim.x + blockIdx.x) * 3 + threadIdx.x] = t;
    }
    __syncthreads();
  }
}

// x times a factor that may be outside fp32's range while the product is not: two powers of
// two, each exact, and a number between 1/2 and 1.
struct Factor {
  float p1, p2, f;
  __device__ __forceinline__ float operator()(float x) const { return x * p1 * p2 * f; }
};

// 2^e / (|G| + eps) of matrix z, by a warp, from the parts of its sums of squares.  In fp32: a
// common factor of all elements, and fp64 here took 6 us of every block.
__device__ __forceinline__ Factor inverse_norm(const float *part, int parts, int64_t z, float eps, int e) {
  float s[3] = {0.f, 0.f, 0.f};
  for (int p = threadIdx.x & 31; p < parts; p += 32)
#pragma unroll
    for (int q = 0; q < 3; ++q) s[q] += part[(z * parts + p) * 3 + q];
#pragma unroll
  for (int q = 0; q < 3; ++q) s[q] = warp_sum(s[q]);
  // the plain sum unless it is near the ends of the range; |G| = root * 2^size (a NaN stays one)
  const int size = s[0] > 0x1p100f ? 90 : s[0] < 0x1p-80f ? -90 : 0;
  const float root = sqrtf(size > 0 ? s[1] : size < 0 ? s[2] : s[0]);
  const float inverse = 1.f / (root + ldexpf(eps, -size));
  Factor f{1.f, 1.f, inverse};
  if (inverse > 0.f && isfinite(inverse)) {
    int own = 0;
    f.f = frexpf(inverse, &own);
    const int all = own + e - size, half = all / 2;
    f.p1 = ldexpf(1.f, half);
    f.p2 = ldexpf(1.f, all - half);
  }
  return f;
}

// -- matrices of the iteration --------------------------------------------------------------------
// [plane][batch][rows][ld] fp16; plane 1 is what plane 0 leaves of an element.
constexpr int kPlanes = 2;
struct Planes {
  __half *p;
  int64_t ld, matrix, plane;  // elements of a row, of a matrix, of a plane
};

__device__ __forceinline__ void split(float v, __half (&h)[kPlanes]) {
  h[0] = __float2half_rn(v);
  h[1] = __float2half_rn(v - __half2float(h[0]));
}

// Y = G / (|G| + eps), in pieces of W elements, four of them in flight a thread.  Bound by latency
// while G and Y fit L2, behind the norm: 6 x 2048 x 1024 in bf16, 7.5e7 bytes, 22 us by itself.
template <typename T, int W>
__global__ void __launch_bounds__(256) ortho_start_kernel(OrthoArgs a, int64_t rows, int64_t cols, const float *part, int parts, Planes y) {
  __shared__ Factor factor;
  kernel_begin();
  next_may_start();
  const uint32_t pieces = (uint32_t)(cols / W);
  const int64_t all = rows * pieces, step = (int64_t)gridDim.x * 256 * 4;
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    const T *g = static_cast<const T *>(a.g) + z * a.g_batch_stride;
    __half *to = y.p + z * y.matrix;
    float v[4][W];
    int64_t at[4];
    auto load = [&](int64_t i0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t i = i0 + k * 256;
        if (i >= all) continue;
        // (matrices of up to 2^32 elements: 32 bits hold i where pieces are wide or rows few)
        const uint32_t r = all >> 32 ? (uint32_t)(i / pieces) : (uint32_t)i / pieces, c = (uint32_t)(i - (int64_t)r * pieces);
        load_piece<W>(g + r * a.g_stride + (int64_t)c * W, v[k]);
        at[k] = r * y.ld + (int64_t)c * W;
      }
    };
    int64_t i0 = (int64_t)blockIdx.x * 256 * 4 + threadIdx.x;
    load(i0);
    if (threadIdx.x < 32) {
      const Factor f = inverse_norm(part, parts, z, a.eps, kScaleYLog2);
      if (threadIdx.x == 0) factor = f;
    }
    __syncthreads();
    const Factor f = factor;
    for (; i0 < all; i0 += step) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i0 + k * 256 >= all) continue;
#pragma unroll
        for (int i = 0; i < W; ++i) v[k][i] = f(v[k][i]);
#pragma unroll
        for (int q = 0; q < kPlanes; ++q) {
          Pack<__half, W> h;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            h.v[i] = __float2half_rn(v[k][i]);
            v[k][i] -= __half2float(h.v[i]);  // what the next plane holds
          }
          *reinterpret_cast<Pack<__half, W> *>(to + q * y.plane + at[k]) = h;
        }
      }
      load(i0 + step);
    }
    __syncthreads();
  }
}

// Y = G^T / (|G| + eps).  A block takes 64 x 64 tiles, in bands of 16 rows of tiles, column by
// column, so that the tiles in work at a time make long runs in G and in Y.  Bound by the bytes:
// 2048 x 8192 in fp32, 1.3e8 bytes, 27 us, 4.9 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_turned_kernel(OrthoArgs a, int64_t rows, int64_t cols, const float *part, int parts, Planes y) {
  __shared__ Factor factor;
  __shared__ float tile[64][65];
  kernel_begin();
  next_may_start();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int64_t tiles_r = (rows + 63) / 64, tiles_c = (cols + 63) / 64;
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    if (threadIdx.x < 32) {
      const Factor f = inverse_norm(part, parts, z, a.eps, kScaleYLog2);
      if (threadIdx.x == 0) factor = f;
    }
    __syncthreads();
    const Factor f = factor;
    const T *g = static_cast<const T *>(a.g) + z * a.g_batch_stride;
    for (int64_t t = blockIdx.x; t < tiles_r * tiles_c; t += gridDim.x) {
      const int64_t band = t / (16 * tiles_c), in = t % (16 * tiles_c), high = min((int64_t)16, tiles_r - band * 16);
      const int64_t r0 = (band * 16 + in % high) * 64, c0 = in / high * 64;
      float v[8][2];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int64_t r = r0 + ty + 8 * i, c = c0 + tx + 32 * e;
          v[i][e] = r < rows && c < cols ? to_f(g[r * a.g_stride + c]) : 0.f;
        }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) tile[ty + 8 * i][tx + 32 * e] = f(v[i][e]);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = c0 + ty + 8 * i, r = r0 + 2 * tx;  // two elements of a row of Y: the padding takes an odd end
        if (c >= cols || r >= rows) continue;
        __half h[2][kPlanes];
        split(tile[2 * tx][ty + 8 * i], h[0]);
        split(tile[2 * tx + 1][ty + 8 * i], h[1]);
#pragma unroll
        for (int q = 0; q < kPlanes; ++q)
          *reinterpret_cast<__half2 *>(y.p + q * y.plane + z * y.matrix + c * y.ld + r) = __halves2half2(h[0][q], h[1][q]);
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

// No steps: O = scale G / (|G| + eps).
template <typename T>
__global__ void __launch_bounds__(256) ortho_scale_kernel(OrthoArgs a, int64_t rows, int64_t cols, const float *part, int parts) {
  __shared__ Factor factor;
  kernel_begin();
  next_may_start();
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    if (threadIdx.x < 32) {
      const Factor f = inverse_norm(part, parts, z, a.eps, 0);
      if (threadIdx.x == 0) factor = f;
    }
    __syncthreads();
    const Factor f = factor;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * blockDim.x) {
      const float v = to_f(static_cast<const T *>(a.g)[z * a.g_batch_stride + i / cols * a.g_stride + i % cols]);
      static_cast<T *>(a.o)[z * a.o_batch_stride + i / cols * a.o_stride + i % cols] = from_f<T>(f(v) * a.scale);
    }
    __syncthreads();
  }
}

// -- products --------------------------------------------------------------------------------------
// D = alpha P Q^T + beta C on tiles of 256 x BN, by persistent pairs of blocks that share a
// tile (cta_group::2): each holds 128 rows of P and of the sums, and half of Q's rows, so that
// a pair reads each operand once.  In each block one thread copies 64 columns of its operands
// at a time with the TMA engine (128-byte swizzle) into a ring of stages; a thread of the
// pair's first block issues tcgen05.mma on both blocks' stages; eight warps take the sums out
// of tensor memory, which holds two sets of them.
//
// Tiles that do not fill a round of the pairs are split along the sum, so that the round's other
// pairs have parts of them: each warp writes its part of the sums, and the one that comes last
// adds the parts, in their order, and finishes the tile.  Nobody waits for another block.
//
// The tensor core adds to its fp32 sums with truncation, which is a bias: with one set of sums
// for 12288 columns (2304 additions an element) the result was 8e-5 off.  So a set covers one
// stage, the products of the low parts first, while the sums are small, and the eight warps add
// the sets up in registers, rounding to nearest, while the next set is summed: 7e-7 off there,
// and 6% more clocks than with sets of eight stages.
//
// Large matrices are bound by the tensor cores: 4608 x 12288 in fp32, five steps, 1.3e13
// operations on fp16 numbers, 8.7 to 9.1 ms, 1.5 PFLOP/s.  Small ones are bound by rounds that are
// not full and by what a launch waits for (fill, drain): 6 matrices of 2048 x 1024, 6.8e11 operations,
// 785 to 810 us, 0.8 to 0.9 PFLOP/s, where the symmetric products have 60 tiles for 76 pairs and the
// last one 192 for three rounds; 1003 x 517 14 us a product.
constexpr int kBM = 256, kBK = 64, kRows = 128;  // of a tile, of a stage; rows of P a block holds
constexpr int kThreads = 384;                    // warp 0: copies, 1: products, 4-11: tiles out
// Registers of a thread of warps 0-3 and of 4-11, which hold 128 sums each; together no more
// than the 168 a thread that the block is launched with (65536 / 384, in units of 8).
constexpr int kFewRegs = 56, kManyRegs = 216;
static_assert(128 * kFewRegs + 256 * kManyRegs <= kThreads * 168, "the block's registers");
constexpr int stage_bytes(int bn) { return kPlanes * (kRows + bn / 2) * kBK * 2; }
constexpr int stages(int bn) { return 196608 / stage_bytes(bn); }
constexpr int kOutBytes = 4096;                  // a warp's buffer on the way out: 32 x 32 elements, twice
constexpr size_t smem_bytes(int bn) { return (size_t)stages(bn) * stage_bytes(bn) + 8 * kOutBytes + 256 + 1024; }

struct ProductArgs {
  int64_t batch;
  int M, N, K;
  int tiles_n;          // tiles of a row of tiles (not symmetric)
  int64_t tiles;        // of a matrix
  int64_t whole;        // tiles of the batch that are not split; the others, `split` parts each
  int split;
  float4 *parts;        // sums of the parts: [split tile][part][block of the pair][warp][columns / 4][lane]
  int32_t *arrived;     // [split tile][block of the pair][warp] parts that are there: zeros between launches
  int symmetric;        // D is symmetric: tiles of the lower triangle, each element written twice
  float alpha, beta;
  Planes c;             // C (p may be null)
  void *o;              // the last product: the result instead of D
  int64_t o_stride, o_batch_stride;
  int o_transposed;
  int32_t *status;      // host memory: set when a wait gave up
  long long wait_limit;
  int skip;             // failure injection for tests: this 64-column step is never copied (-1: none)
};

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
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok)
               : "r"(bar), "r"(parity)
               : "memory");
  return ok;
}
// Waits until the phase of that parity has completed; false if the block gives up (another
// wait did, or this one's limit has passed).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort, const ProductArgs &a) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > a.wait_limit) {
      *abort = 1;
      *(volatile int32_t *)a.status = 1;
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
template <bool MN>
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(MN ? 8192 >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 16 columns of the sum on: 32 bytes of a line, or 16 lines
constexpr int step16(bool mn) { return (mn ? 2048 : 32) >> 4; }
// fp16 operands, fp32 sums, `bn` columns, kBM rows
constexpr uint32_t instruction(int bn, bool mn) {
  return 1u << 4 | (mn ? 3u << 15 : 0u) | (uint32_t)(bn >> 3) << 17 | (uint32_t)(kBM >> 4) << 24;
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

// First row and column of a tile.  Symmetric: row i of tiles has (i + 1) kBM / BN of them.
// Otherwise in bands of 8 rows of tiles, column by column, so that the tiles in work share
// operands in L2.
template <int BN>
__device__ __forceinline__ void tile_place(const ProductArgs &a, int64_t t, int &r0, int &c0) {
  constexpr int F = kBM / BN;
  int64_t i, j;
  if (a.symmetric) {
    i = (int64_t)((sqrt(1. + 8. / F * (double)t) - 1.) * 0.5);
    while (i > 0 && F * i * (i + 1) / 2 > t) --i;
    while (F * (i + 1) * (i + 2) / 2 <= t) ++i;
    j = t - F * i * (i + 1) / 2;
  } else {
    const int64_t rows = (a.M + kBM - 1) / kBM, band = t / (8 * a.tiles_n), in = t % (8 * a.tiles_n), high = min((int64_t)8, rows - band * 8);
    i = band * 8 + in % high;
    j = in / high;
  }
  r0 = (int)i * kBM;
  c0 = (int)j * BN;
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

// 32 x 32 elements of a tile out, by a warp: lane r has those of row row0 + r in v, from column
// c.  A symmetric product writes the blocks of the lower triangle and, transposed, those of the
// upper one.  dmap takes rows with exchanged pieces (its 64-byte swizzle), tmap plain ones.
//
// By the copy engine: the tensor core's reads of the stages nearly fill shared memory's
// bandwidth, and every pass through it that the warps do themselves waits for a gap.
__device__ __forceinline__ void block_out(const ProductArgs &a, const CUtensorMap *dmap, const CUtensorMap *tmap, int z, int row0, int c, int lane,
                                          float (&v)[32], unsigned char *buffer, uint32_t &turn) {
  if (a.symmetric && c > row0) return;
#pragma unroll 1
  for (int q = 0; q < kPlanes; ++q) {
    Piece h[4];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      h[i / 8].v[i % 8] = __float2half_rn(v[i]);
      v[i] -= __half2float(h[i / 8].v[i % 8]);  // what the next plane holds
    }
    half_free(lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<Piece *>(piece(buffer + turn, lane, i)) = h[i];
    half_written();
    if (lane == 0) store_half(dmap, buffer + turn, c, row0, z, q);
    turn ^= 2048;
    if (!a.symmetric || c == row0) continue;
    half_free(lane);
    __half *t = reinterpret_cast<__half *>(buffer + turn) + lane;
#pragma unroll
    for (int i = 0; i < 32; ++i) t[i * 32] = h[i / 8].v[i % 8];
    half_written();
    if (lane == 0) store_half(tmap, buffer + turn, row0, c, z, q);
    turn ^= 2048;
  }
}

// The same for the result: through the buffer where its rows are the tile's, so that
// neighbouring lanes write neighbouring elements.
template <typename OUT>
__device__ __forceinline__ void result_out(const ProductArgs &a, int64_t z, int row0, int c, int lane, const float (&v)[32], unsigned char *buffer) {
  OUT *o = static_cast<OUT *>(a.o) + z * a.o_batch_stride;
  if (a.o_transposed) {
    if (row0 + lane < a.M) {
      o += (int64_t)c * a.o_stride + row0 + lane;
#pragma unroll
      for (int i = 0; i < 32; ++i, o += a.o_stride)
        if (c + i < a.N) *o = from_f<OUT>(v[i]);
    }
    return;
  }
  float *f = reinterpret_cast<float *>(buffer);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 32; ++i) f[lane * 32 + (i ^ lane)] = v[i];
  __syncwarp();
  if (c + lane < a.N) {
    o += (int64_t)row0 * a.o_stride + c + lane;
    const int rows = min(32, a.M - row0);
#pragma unroll 4
    for (int r = 0; r < rows; ++r, o += a.o_stride) *o = from_f<OUT>(f[r * 32 + (lane ^ r)]);
  }
}

// OUT: void for a product whose result goes on in planes, else the type of the result.
template <int BN, bool MN, typename OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    ortho_product_kernel(const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap dmap,
                         const __grid_constant__ CUtensorMap tmap, const __grid_constant__ ProductArgs a) {
  constexpr int S = stages(BN), kStage = stage_bytes(BN), kP = kRows * kBK * 2, kQ = BN / 2 * kBK * 2, kCols = BN / 2;
  extern __shared__ unsigned char raw[];
  unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
  unsigned char *buffers = base + S * kStage;
  uint64_t *bars = reinterpret_cast<uint64_t *>(buffers + 8 * kOutBytes);
  __shared__ uint32_t tmem_base;
  __shared__ int give_up;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;  // (clusters of two along x)
  // `full` and `sums_empty` are used in the first block alone, the others in both
  const uint32_t ring = smem_u32(base), full = smem_u32(bars), empty = full + 8 * S, sums_full = empty + 8 * S, sums_empty = sums_full + 16,
                 done = sums_empty + 16;
  volatile int *abort = &give_up;
  if (threadIdx.x == 0) {
    give_up = 0;
    for (int s = 0; s < S; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, 16);
    }
    bar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (threadIdx.x == 32 * 3) {
    asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\n" ::"l"(&pmap), "l"(&qmap) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base)), "r"(2u * BN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = tmem_base;
  // What is above overlaps the end of the kernel before; from here on its results are read.
  kernel_begin();
  next_may_start();
  const int64_t all = a.whole + (a.tiles * a.batch - a.whole) * a.split;
  const int steps = (a.K + kBK - 1) / kBK;  // stages: each has a set of sums

  // Piece of work i: tile t (of the batch), stages k0 to k1 of its sum.
  auto work_at = [&](int64_t i, int64_t &t, int &part, int &k0, int &k1) {
    const int64_t j = i - a.whole;
    const bool whole = j < 0;
    t = whole ? i : a.whole + j / a.split;
    part = whole ? 0 : (int)(j % a.split);
    k0 = whole ? 0 : (int)((int64_t)steps * part / a.split);
    k1 = whole ? steps : (int)((int64_t)steps * (part + 1) / a.split);
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kFewRegs));
    if (warp == 0 && lane == 0) {
      int64_t it = 0;
      bool ok = true;
      for (int64_t i = pair; i < all && ok; i += pairs) {
        int64_t t;
        int r0, c0, part, k0, k1;
        work_at(i, t, part, k0, k1);
        tile_place<BN>(a, t % a.tiles, r0, c0);
        const int z = (int)(t / a.tiles);
        for (int k = k0; k < k1; ++k, ++it) {
          const int s = (int)(it % S);
          ok = k != a.skip && bar_wait(empty + 8 * s, (uint32_t)(it / S + 1) & 1, abort, a);
          if (!ok) break;
          const uint32_t at = ring + s * kStage, bar = in_first(full + 8 * s);
          if (rank == 0) bar_expect(full + 8 * s, 2 * kStage);  // both blocks' copies
#pragma unroll
          for (int q = 0; q < kPlanes; ++q) {
            copy_operand<MN, kRows>(at + q * kP, &pmap, r0 + rank * kRows, k * kBK, z, q, bar);
            copy_operand<MN, kCols>(at + kPlanes * kP + q * kQ, &qmap, c0 + rank * kCols, k * kBK, z, q, bar);
          }
        }
      }
      if (!ok) {  // what is still being copied lands long before this
        const long long t0 = clock64();
        while (clock64() - t0 < 1000000) {
        }
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      int64_t it = 0;
      bool ok = true;
      for (int64_t i = pair; i < all && ok; i += pairs) {
        int64_t t;
        int part, begin, end;
        work_at(i, t, part, begin, end);
        for (int k = begin; k < end; ++k, ++it) {
          const int b = (int)(it & 1), s = (int)(it % S);
          ok = bar_wait(sums_empty + 8 * b, (uint32_t)(it / 2 + 1) & 1, abort, a) && bar_wait(full + 8 * s, (uint32_t)(it / S) & 1, abort, a);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint32_t d = tmem + b * BN;
          const uint64_t p = operand<MN>(ring + s * kStage), q = operand<MN>(ring + s * kStage + kPlanes * kP);
          constexpr uint32_t kInstr = instruction(BN, MN);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk) {
            mma(d, p + step16(MN) * kk, q + step16(MN) * kk + (kQ >> 4), kInstr, kk > 0);
            mma(d, p + step16(MN) * kk + (kP >> 4), q + step16(MN) * kk, kInstr, true);
          }
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk) mma(d, p + step16(MN) * kk, q + step16(MN) * kk, kInstr, true);
          commit_pair(empty + 8 * s);
          commit_pair(sums_full + 8 * b);
        }
      }
      commit(done);  // nothing is in flight when the block ends
      const long long t0 = clock64();
      while (!bar_try(done, 0) && clock64() - t0 <= a.wait_limit) {
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kManyRegs));
    const int quarter = warp & 3, side = (warp - 4) >> 2;  // (a warp reaches the 32 rows of tensor memory of its number modulo 4)
    unsigned char *buffer = buffers + (warp - 4) * kOutBytes;
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + side * kCols;
    int64_t n = 0;
    uint32_t turn = 0;
    bool ok = true;
    for (int64_t i = pair; i < all && ok; i += pairs) {
      int64_t t;
      int r0, c0, part_of, begin, end;
      work_at(i, t, part_of, begin, end);
      tile_place<BN>(a, t % a.tiles, r0, c0);
      const int z = (int)(t / a.tiles), row0 = r0 + rank * kRows + quarter * 32;
      const bool live = row0 < a.M;
      c0 += side * kCols;
      const bool add_c = !MN && a.c.p && part_of == 0;
      const __half *from_c = a.c.p + z * a.c.matrix;
      if (add_c && row0 + lane < a.M) {  // C's part of the tile comes to L2 during the sums
#pragma unroll
        for (int q = 0; q < kPlanes; ++q)
#pragma unroll
          for (int i = 0; i < kCols; i += 64)
            if (c0 + i < a.N) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(from_c + q * a.c.plane + (int64_t)(row0 + lane) * a.c.ld + c0 + i));
      }
      // C is added to the sums a plane of a 32 x 32 block at a time, between the last sets, or
      // before the first one where they are few: then it comes while the first stages do.  Each
      // piece comes one turn ahead, four lanes to the 64 bytes of a row, and changes to a row a lane
      // in the warp's buffer.
      constexpr int kFlight = MN ? 2 : 1;
      constexpr int kParts = kCols / 32, kPieces = MN ? 0 : kPlanes * kParts;
      const int sets = end - begin;
      const bool c_before = add_c && sets <= 2 * kPieces;
      const int set0 = c_before ? kPieces + 1 : 0, first_c = c_before ? 0 : add_c ? sets - kPieces - 1 : sets;  // turns
      Piece ahead[4] = {};
      auto fetch = [&](int u) {
        const int row = row0 + (lane >> 2), col = c0 + u / kPlanes * 32 + (lane & 3) * 8;
        const __half *p = from_c + (int64_t)row * a.c.ld + col + u % kPlanes * a.c.plane;
#pragma unroll
        for (int i = 0; i < 4; ++i)  // (to the end of a piece: within the padding of the row)
          if (row + 8 * i < a.M && col < a.N) ahead[i] = *reinterpret_cast<const Piece *>(p + (int64_t)(8 * i) * a.c.ld);
      };
      float acc[kParts][32] = {};
      for (int turn_c = 0; turn_c < set0 + sets; ++turn_c) {
        if (turn_c >= set0) {
          const int b = (int)(n & 1);
          ok = bar_wait(sums_full + 8 * b, (uint32_t)(n / 2) & 1, abort, a);
          if (!ok) break;
          ++n;
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll
          for (int part = 0; part < kParts; part += kFlight) {
            Sums s[kFlight];
            __syncwarp();
#pragma unroll
            for (int e = 0; e < kFlight; ++e) load_sums(from + b * BN + (part + e) * 32, s[e]);
            sums_loaded();
#pragma unroll
            for (int e = 0; e < kFlight; ++e) {
              pass(s[e]);
#pragma unroll
              for (int i = 0; i < 32; ++i) acc[part + e][i] = fmaf(a.alpha, __uint_as_float(s[e].r[i]), acc[part + e][i]);
            }
          }
          asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive_cluster(in_first(sums_empty + 8 * b));
        }
        if (turn_c < first_c) continue;
        const int u = turn_c - first_c - 1;  // this turn's piece
        if (kPieces && u >= 0 && u < kPieces) {
          half_free(lane);
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<Piece *>(piece(buffer + turn, 8 * i + (lane >> 2), lane & 3)) = ahead[i];
          __syncwarp();
          auto add = [&](auto which) {
            constexpr int part = decltype(which)::value;
            if (part != u / kPlanes) return;
            asm volatile("" ::"n"(part));  // (keeps the blocks apart: as one, they would index the sums in memory)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float f[8];
              unpack<__half, 8>(*reinterpret_cast<const Piece *>(piece(buffer + turn, lane, i)), f);
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[part][8 * i + e] += a.beta * f[e];
            }
          };
          add(Int<0>{});
          add(Int<1>{});
          if constexpr (kParts == 4) {
            add(Int<2>{});
            add(Int<3>{});
          }
          __syncwarp();
        }
        if (u + 1 < kPieces) fetch(u + 1);
      }
      if (!ok) break;
      if (!live) continue;
      if (i >= a.whole && a.split > 1) {
        const int64_t tile = t - a.whole;
        const int64_t place = (int64_t)(rank * 8 + warp - 4) * (kCols / 4 * 32) + lane;
        constexpr int64_t kPart = 16 * (kCols / 4 * 32);
        float4 *mine = a.parts + (tile * a.split + part_of) * kPart + place;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            mine[(part * 8 + e) * 32] = make_float4(acc[part][4 * e], acc[part][4 * e + 1], acc[part][4 * e + 2], acc[part][4 * e + 3]);
        __threadfence();
        __syncwarp();
        int32_t *count = a.arrived + tile * 16 + rank * 8 + warp - 4, before = 0;
        if (lane == 0) before = atomicAdd(count, 1);
        if (__shfl_sync(0xFFFFFFFFu, before, 0) != a.split - 1) continue;  // another part comes later
        if (lane == 0) *count = 0;
        __threadfence();
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[part][e] = 0.f;
#pragma unroll 1
        for (int other = 0; other < a.split; ++other) {
          const float4 *from_part = a.parts + (tile * a.split + other) * kPart + place;
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 f = __ldcg(from_part + (part * 8 + e) * 32);
              acc[part][4 * e] += f.x;
              acc[part][4 * e + 1] += f.y;
              acc[part][4 * e + 2] += f.z;
              acc[part][4 * e + 3] += f.w;
            }
        }
      }
      // One block after the other, in the registers of the first (unrolled, the code is 80 KB and
      // runs once a tile).
      float (&v)[32] = acc[0];
#pragma unroll 1
      for (int c = c0; c < min(a.N, c0 + kCols); c += 32) {
        if constexpr (std::is_void_v<OUT>)
          block_out(a, &dmap, &tmap, z, row0, c, lane, v, buffer, turn);
        else
          result_out<OUT>(a, z, row0, c, lane, v, buffer);
#pragma unroll
        for (int part = 1; part < kParts; ++part)
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[part - 1][i] = acc[part][i];
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  cluster_sync();  // (the other block's products read this one's stages, and signal its barriers)
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2u * BN) : "memory");
  }
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
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

// Boxes of a matrix of the iteration; zeros outside it.
cudaError_t box_map(CUtensorMap *map, const Planes &p, int64_t rows, int64_t cols, int64_t batch, int box_rows, int box_cols,
                    CUtensorMapSwizzle swizzle) {
  if (!encoder()) return cudaErrorNotSupported;
  const cuuint64_t dims[4] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch, (cuuint64_t)kPlanes};
  const cuuint64_t strides[3] = {(cuuint64_t)p.ld * 2, (cuuint64_t)p.matrix * 2, (cuuint64_t)p.plane * 2};
  const cuuint32_t box[4] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, p.p, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}
// 64 columns, for the stages; 32 x 32 for a warp's buffer
cudaError_t tile_map(CUtensorMap *map, const Planes &p, int64_t rows, int64_t cols, int64_t batch, int box_rows) {
  return box_map(map, p, rows, cols, batch, box_rows, 64, CU_TENSOR_MAP_SWIZZLE_128B);
}
cudaError_t out_map(CUtensorMap *map, const Planes &p, int64_t rows, int64_t cols, int64_t batch, bool exchanged) {
  return box_map(map, p, rows, cols, batch, 32, 32, exchanged ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE);
}

int64_t padded(int64_t x) { return (x + 63) / 64 * 64; }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
Planes planes_of(char *&at, int64_t rows, int64_t cols, int64_t batch) {
  Planes p{reinterpret_cast<__half *>(at), padded(cols), rows * padded(cols), batch * rows * padded(cols)};
  at += up256((size_t)kPlanes * p.plane * sizeof(__half));
  return p;
}

}  // namespace

// blocks that sum a matrix for its norm
int norm_parts(const OrthoArgs &a) { return (int)std::clamp<int64_t>(a.m * a.n / 8192, 1, 608); }

// How a product goes: the width of its tiles and the tiles that are split, with the smallest
// estimate of its clocks.  A stage takes 1536 clocks of products at 256 columns, 1080 at 128 (the
// operands' reads from shared memory bound it); joining parts takes about 6000 and, for each part,
// what 256 or 128 KB of a pair's sums take to L2 and back.
struct Plan {
  int bn;
  int64_t tiles, whole;
  int split;
};
Plan plan_product(int64_t M, int64_t N, int64_t K, bool symmetric, int64_t batch, int pairs) {
  Plan best{};
  double least = 0;
  for (const int bn : {256, 128}) {
    const int64_t tm = (M + kBM - 1) / kBM, tiles = symmetric ? kBM / bn * tm * (tm + 1) / 2 : tm * ((N + bn - 1) / bn);
    const int64_t all = tiles * batch, rest = all % pairs, steps = (K + kBK - 1) / kBK;
    const double stage = bn == 256 ? 1536 : 1080, join = bn == 256 ? 3000 : 1500;
    int split = 1;
    double round = rest ? stage * steps : 0;
    for (int64_t p = 2; rest && p <= std::min(pairs / rest, steps); ++p) {
      const double c = stage * ((steps + p - 1) / p) + 6000 + join * p;
      if (c < round) round = c, split = (int)p;
    }
    const double clocks = stage * steps * (all / pairs) + round;
    if (!best.bn || clocks < least) least = clocks, best = {bn, tiles, split > 1 ? all - rest : all, split};
  }
  return best;
}
Plan plan_of(const OrthoArgs &a, int product, int sms) {  // A, B, Y
  return plan_product(product < 2 ? a.m : a.n, a.m, product == 0 ? a.n : a.m, product < 2, a.batch, sms / 2);
}

// parts of the norm; counts and sums of split tiles; Y twice (a product reads one while it
// writes the other), A, B
size_t parts_bytes(const OrthoArgs &a, int sms) {
  size_t most = 0;
  for (int product = 0; product < 3; ++product) {
    const Plan p = plan_of(a, product, sms);
    most = std::max(most, (size_t)(p.tiles * a.batch - p.whole) * p.split * kBM * p.bn * sizeof(float));
  }
  return most;
}
size_t ortho_scratch_bytes(const OrthoArgs &a, int sms) {
  char *at = nullptr;
  for (int i = 0; i < 2; ++i) planes_of(at, a.n, a.m, a.batch);
  for (int i = 0; i < 2; ++i) planes_of(at, a.m, a.m, a.batch);
  return (a.steps ? reinterpret_cast<uintptr_t>(at) + up256((size_t)sms * 8 * sizeof(int32_t)) + parts_bytes(a, sms) : 0) +
         up256((size_t)a.batch * norm_parts(a) * 3 * sizeof(float));
}

cudaError_t launch_orthogonalize(const OrthoArgs &a, int sms, const OpTimer &timed, cudaStream_t st) {
  const int parts = norm_parts(a);
  char *at = static_cast<char *>(a.scratch);
  float *part = reinterpret_cast<float *>(at);
  at += up256((size_t)a.batch * parts * 3 * sizeof(float));
  const int pairs = sms / 2;
  int32_t *arrived = reinterpret_cast<int32_t *>(at);
  const unsigned gz = (unsigned)std::min<int64_t>(a.batch, 65535);
  const int64_t rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
  cudaError_t e = timed("ortho_norm", [&] {
    return with_type(a.type, [&](auto t) {
      using T = decltype(t);
      constexpr int N = 16 / sizeof(T);
      const bool one = a.g_stride == cols || rows == 1;  // without gaps
      const int64_t sum_rows = one ? 1 : rows, sum_cols = one ? rows * cols : cols;
      if (cols % N == 0 && fits_pieces(a.g, a.g_stride, a.type, N) && fits_pieces(a.g, a.g_batch_stride, a.type, N))
        return launch_early(ortho_norm_kernel<T, N>, dim3(parts, gz), 256, 0, st, a, sum_rows, sum_cols, part, arrived, a.steps ? pairs * 16 : 0);
      return launch_early(ortho_norm_kernel<T, 1>, dim3(parts, gz), 256, 0, st, a, sum_rows, sum_cols, part, arrived, a.steps ? pairs * 16 : 0);
    });
  });
  if (e != cudaSuccess) return e;
  if (a.steps == 0)
    return timed("ortho_scale", [&] {
      return with_type(a.type, [&](auto t) {
        return launch_early(ortho_scale_kernel<decltype(t)>, dim3((unsigned)std::min<int64_t>((rows * cols + 255) / 256, sms * 8), gz), 256, 0, st, a, rows,
                            cols, part, parts);
      });
    });
  at += up256((size_t)sms * 8 * sizeof(int32_t));
  float4 *split_parts = reinterpret_cast<float4 *>(at);
  at += parts_bytes(a, sms);
  const Planes Y[2] = {planes_of(at, a.n, a.m, a.batch), planes_of(at, a.n, a.m, a.batch)};
  const Planes A = planes_of(at, a.m, a.m, a.batch), B = planes_of(at, a.m, a.m, a.batch);
  e = timed("ortho_start", [&] {
    return with_type(a.type, [&](auto t) {
      using T = decltype(t);
      constexpr int N = 16 / sizeof(T);
      const int64_t room = std::max<int64_t>(1, sms * 6 / gz);
      auto grid = [&](int64_t want) { return dim3((unsigned)std::min(want, room), gz); };
      if (!a.tall)
        return launch_early(ortho_start_turned_kernel<T>, grid((rows + 63) / 64 * ((cols + 63) / 64)), 256, 0, st, a, rows, cols, part, parts, Y[0]);
      if (cols % N == 0 && fits_pieces(a.g, a.g_stride, a.type, N) && fits_pieces(a.g, a.g_batch_stride, a.type, N))
        return launch_early(ortho_start_kernel<T, N>, grid((rows * cols / N + 1023) / 1024), 256, 0, st, a, rows, cols, part, parts, Y[0]);
      return launch_early(ortho_start_kernel<T, 1>, grid((rows * cols + 1023) / 1024), 256, 0, st, a, rows, cols, part, parts, Y[0]);
    });
  });
  if (e != cudaSuccess) return e;

  struct Matrix {
    const Planes &p;
    int64_t rows, cols;
  };
  const Matrix y[2] = {{Y[0], a.n, a.m}, {Y[1], a.n, a.m}}, sa{A, a.m, a.m}, sb{B, a.m, a.m};
  // D = alpha P Q^T + beta C (mn: P and Q hold the transposes); the result without a D.  D is
  // symmetric where P is Q.
  auto product = [&](int which, const char *name, const Matrix &p, const Matrix &q, bool mn, float alpha, const Planes *c, float beta, const Matrix *d) -> cudaError_t {
    ProductArgs g{};
    const bool symmetric = &p == &q;
    const Plan plan = plan_of(a, which, sms);
    g.batch = a.batch, g.M = (int)(mn ? p.cols : p.rows), g.N = (int)(mn ? q.cols : q.rows), g.K = (int)(mn ? p.rows : p.cols);
    g.symmetric = symmetric;
    g.alpha = alpha, g.beta = beta;
    if (c) g.c = *c;
    g.o = a.o, g.o_stride = a.o_stride, g.o_batch_stride = a.o_batch_stride, g.o_transposed = !a.tall;
    g.status = a.status, g.wait_limit = a.wait_limit, g.skip = a.skip;
    auto go = [&](auto cols_c, auto mn_c, auto out) -> cudaError_t {
      constexpr int BN = decltype(cols_c)::value;
      constexpr bool MN = decltype(mn_c)::value;
      using O = std::remove_pointer_t<decltype(out)>;
      g.tiles_n = (int)((g.N + BN - 1) / BN);
      g.tiles = plan.tiles, g.whole = plan.whole, g.split = plan.split, g.parts = split_parts, g.arrived = arrived;
      CUtensorMap pm, qm, dm{}, tm{};
      cudaError_t r = tile_map(&pm, p.p, p.rows, p.cols, a.batch, MN ? kBK : kRows);
      if (r == cudaSuccess) r = tile_map(&qm, q.p, q.rows, q.cols, a.batch, MN ? kBK : BN / 2);
      if (r == cudaSuccess && d) r = out_map(&dm, d->p, d->rows, d->cols, a.batch, true);
      if (r == cudaSuccess && d && symmetric) r = out_map(&tm, d->p, d->rows, d->cols, a.batch, false);
      auto kernel = ortho_product_kernel<BN, MN, O>;
      if (r == cudaSuccess) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(BN));
      if (r != cudaSuccess) return r;
      return launch_early(kernel, dim3((unsigned)std::min<int64_t>(g.whole + (g.tiles * g.batch - g.whole) * g.split, pairs) * 2), kThreads, smem_bytes(BN), st, pm, qm, dm, tm, g);
    };
    auto with_out = [&](auto cols_c) -> cudaError_t {
      if (mn) return go(cols_c, Int<1>{}, (void *)nullptr);
      if (d) return go(cols_c, Int<0>{}, (void *)nullptr);
      return a.type == ECHO_F32 ? go(cols_c, Int<0>{}, (float *)nullptr)
             : a.type == ECHO_BF16 ? go(cols_c, Int<0>{}, (__nv_bfloat16 *)nullptr)
                                   : go(cols_c, Int<0>{}, (__half *)nullptr);
    };
    return timed(name, [&] { return plan.bn == 128 ? with_out(Int<128>{}) : with_out(Int<256>{}); });
  };
  for (int s = 0; s < a.steps; ++s) {
    const Matrix &now = y[s & 1], &next = y[(s + 1) & 1];
    const bool last = s == a.steps - 1;
    const float out = last ? a.scale / kScaleY : 1.f;
    if ((e = product(0, "ortho_yty", now, now, true, kScaleA / (kScaleY * kScaleY), nullptr, 0.f, &sa)) != cudaSuccess) return e;
    if ((e = product(1, "ortho_aa", sa, sa, false, a.c * (kScaleB / (kScaleA * kScaleA)), &A, a.b * (kScaleB / kScaleA), &sb)) != cudaSuccess) return e;
    // (a Y is added to the sums in fp32: as a on B's diagonal it would cost nothing to add, but the
    // larger sums lose more to truncation, 2.7e-6 instead of 1.0e-6 at 300 x 300)
    if ((e = product(2, "ortho_yb", now, sb, false, out / kScaleB, &now.p, out * a.a, last ? nullptr : &next)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace echo
