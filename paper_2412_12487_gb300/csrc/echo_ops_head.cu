// echo_ops_head.cu -- losses of a language model's head, straight from hidden states and the
// head's weight: softmax cross entropy and distillation from a teacher's top logits, with their
// gradients.
//
// With z[t][v] = <x_t, w_v> scale / tau over the rows of a vocabulary shard, both losses are
//   tau^2 (sum q log q + Q lse - cross),  lse = log sum exp z,  cross = sum of q_k z[id_k],
// for a list of targets (id_k, q_k) a token with Q = sum q_k: one label with q = 1, or a teacher's
// top logits.  The gradient of the products <x_t, w_v> is
//   P[t][v] = coef_t exp(z - lse) - (sum of weight_k where id_k = v),
// and dx = P W, dW = P^T x.
//
// The logits are never kept.  Forward, each tile of the product leaves the largest element and
// the sum of exponentials of each of its rows, and the elements that a target names; a small
// kernel joins them.  Backward, the product is made again for a piece of the vocabulary, whose
// part of P goes to scratch memory for the two products that follow.
//
// Operands are 16-bit numbers on the tensor cores, with sums in fp32:
//   - bf16 and fp16 matrices as they are; fp32 ones as sums of two fp16 numbers times a power of
//     two that the largest element sets (22 bits of elements down to 2^-14 of it, an error of
//     2^-37 of it below), multiplied as high * high + high * low + low * high.  Forward each row
//     has its own power of two, backward x and the weight have one each, as the sums then run over
//     rows;
//   - P, scaled so that its largest element is a power of two, as one number of the matrices' type
//     where the results have 16 bits: an error of up to 2^-8 (bf16) of each element, independent
//     of the others', where the results are rounded to the same (2.4e-3 from 64 bits at the most,
//     1.7e-3 of which is the result's rounding).  For an fp32 dW as the sum of two fp16 numbers,
//     with x as fp16 (scaled in the same way): a gradient added up over micro-batches in fp32
//     would otherwise be 2e-3 off.  That takes dW's products twice.  The two have 22 bits down to
//     2^-18 of P's largest element and an error of 2^-40 of that below: fp16's smallest step is the
//     same for both, so the rows of tokens that hardly any context expects keep fewer bits (2^-30: 10),
//     which no error over the whole of dW shows.
// The tensor core truncates the sums that it adds to, which is a bias, so they are added up in
// registers, rounding to nearest, every few stages (set_of).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "echo_ops.h"
#include "echo_tensor.cuh"

namespace echo {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr int kAmaxParts = 304;  // blocks that look for a largest element, at most

// Where the exponent of a matrix's power of two comes from: the largest elements that blocks
// found (none: the matrix is as it is), or, for one of each row, the largest elements of rows.
struct Scale {
  const float *part;
  int parts;
  const float *rows;
};
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
  return v;
}
__device__ __forceinline__ float largest(Scale s) {
  float m = 0.f;
  for (int i = threadIdx.x & 31; i < s.parts; i += 32) m = fmaxf(m, s.part[i]);
  return warp_max(m);
}
// (-113 to 126: powers of two whose inverses are normal numbers too)
__device__ __forceinline__ int exponent_of(float m) { return m > 0.f ? min(126, 14 - ilogbf(m)) : 0; }
// By a warp, the same in all lanes: the largest element times 2^exponent is 2^14 to 2^15, if it is
// 2^-112 at least (below that it has fewer digits).
__device__ __forceinline__ int exponent(Scale s) { return exponent_of(largest(s)); }
// The same for P, whose largest element becomes 2^15 itself: tokens have the same weight as a rule,
// and 1 is what its targets then round to, not all of them up or down (that left dx 3.0e-3 off in bf16
// where a token's weight is 1 / 1984, and 2.0e-3 so).  What P is multiplied by is 2^exponent times this.
__device__ __forceinline__ float fraction(Scale s) {
  const float m = largest(s), at = ldexpf(m, exponent_of(m));
  return at >= 16384.f && at < 32768.f ? 32768.f / at : 1.f;
}
__device__ __forceinline__ float finite_size(float x) {
  x = fabsf(x);
  return x <= FLT_MAX ? x : 0.f;
}

// -- operands as the tensor cores take them ----------------------------------------------------
// [plane][rows][ld] 16-bit elements; plane 1 is what plane 0 leaves of an element.
struct Operand {
  const void *p;
  int64_t rows, cols, ld, plane;
  int planes;
  bool bf16;
  Scale scale;
};

// Up to two matrices for one launch (grid.y): x and the weight.
struct Source {
  const void *p;
  int64_t rows, cols, stride;
  Scale scale;          // of what it becomes
  const float *live;    // rows that are not live become zeros; null: all are
  void *to;
  int64_t ld, plane;
  float *amax;
  bool down;            // what takes a row back, instead of its largest element
};
struct Sources {
  Source of[2];
};

// The largest finite element of each block's part of a matrix's live rows (without gaps, and all of
// them live, a single row).  Bound by the bytes, or by latency where they are few.
template <typename T, int W>
__global__ void __launch_bounds__(256) head_amax_kernel(Sources s) {
  __shared__ float sh[8];
  kernel_begin();
  next_may_start();
  const Source &m = s.of[blockIdx.y];
  const T *x = static_cast<const T *>(m.p);
  // (a single row: its 16-byte pieces, and what is before and behind them, by the first block)
  int64_t cols = m.cols;
  float most = 0.f;
  if (W > 1 && m.rows == 1) {
    const int64_t before = min(cols, (int64_t)((16 - reinterpret_cast<uintptr_t>(x) % 16) % 16 / sizeof(T))), behind = (cols - before) % W;
    if (blockIdx.x == 0 && threadIdx.x < before + behind)
      most = finite_size(to_f(x[threadIdx.x < before ? (int64_t)threadIdx.x : cols - behind + (threadIdx.x - before)]));
    x += before;
    cols -= before + behind;
  }
  const int64_t pieces = cols / W, all = m.rows * pieces;
  constexpr int kFlight = 8 / (W > 4 ? 2 : 1);
  for (int64_t i0 = (int64_t)blockIdx.x * 256 * kFlight + threadIdx.x; i0 < all; i0 += (int64_t)gridDim.x * 256 * kFlight) {
    float v[kFlight][W];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int64_t i = i0 + k * 256;
#pragma unroll
      for (int e = 0; e < W; ++e) v[k][e] = 0.f;
      if (i < all && m.rows == 1) {
        load_piece<W>(x + i * W, v[k]);
      } else if (i < all) {
        const int64_t r = all >> 32 ? i / pieces : (int64_t)((uint32_t)i / (uint32_t)pieces);
        if (!m.live || m.live[r] != 0.f) load_piece<W>(x + r * m.stride + (i - r * pieces) * W, v[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
#pragma unroll
      for (int e = 0; e < W; ++e) most = fmaxf(most, finite_size(v[k][e]));
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) most = fmaxf(most, sh[w]);
    m.amax[blockIdx.x] = most;
  }
}

// A matrix as PLANES planes of type D (fp16 ones times 2^exponent); rows that are not live become
// zeros, so that whatever they hold (padding) meets nothing in a product.  A thread writes 8 elements
// of a plane at a time (rows of planes are padded for that), and reads them one by one where rows are not
// 16-byte ones.  Bound by the bytes: 5003 x 517 in fp32, 2.1e7 bytes, 9.6 us from cold caches.
template <typename T, typename D, int PLANES, bool WIDE>
__global__ void __launch_bounds__(256) head_pack_kernel(Sources s) {
  __shared__ int sh;
  kernel_begin();
  next_may_start();
  const Source &m = s.of[blockIdx.y];
  if (threadIdx.x < 32) {
    const int e = exponent(m.scale);
    if (threadIdx.x == 0) sh = e;
  }
  __syncthreads();
  constexpr int W = 8, kFlight = 2;
  const float up = ldexpf(1.f, sh);
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  const T *x = static_cast<const T *>(m.p);
  D *to = static_cast<D *>(m.to);
  const float *live = m.live;
  const int64_t stride = m.stride, ld = m.ld, plane = m.plane, cols = m.cols;
  const uint32_t pieces = (uint32_t)((cols + W - 1) / W);
  const int64_t all = m.rows * pieces;
  for (int64_t i0 = first; i0 < all; i0 += step * kFlight) {
    Pack<T, W> raw[kFlight];
    int64_t at[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int64_t i = i0 + k * step;
      if (i >= all) continue;
      const int64_t r = all >> 32 ? i / pieces : (int64_t)((uint32_t)i / pieces), c = (i - r * pieces) * W;
      at[k] = r * ld + c;
#pragma unroll
      for (int e = 0; e < W; ++e) raw[k].v[e] = from_f<T>(0.f);
      if (live && live[r] == 0.f) continue;
      const T *from = x + r * stride + c;
      if (WIDE) {
        raw[k] = *reinterpret_cast<const Pack<T, W> *>(from);
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (c + e < cols) raw[k].v[e] = from[e];
      }
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (i0 + k * step >= all) continue;
      float v[W];
      unpack<T, W>(raw[k], v);
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] *= up;
#pragma unroll
      for (int q = 0; q < PLANES; ++q) {
        const Pack<D, W> h = pack<D, W>(v);
        float back[W];
        unpack<D, W>(h, back);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] -= back[e];  // what the next plane holds
        *reinterpret_cast<Pack<D, W> *>(to + q * plane + at[k]) = h;
      }
    }
  }
}

// fp32 rows as two planes of fp16 each: a row is scaled by its own largest finite element, which is left
// (x), or by the power of two that takes it back (the weight's `down`).  A warp takes a short row, a block a
// longer one: its pieces stay in registers (HELD of a lane; further ones are read again, from L2).  With a warp
// a row of any length the rows on their way are more than L2 holds, and were read twice from memory: 51200 x
// 4096, 1.7e9 bytes, 365 us instead of 280.
template <bool WIDE, int WARPS, int HELD>
__global__ void __launch_bounds__(256) head_pack_rows_kernel(Sources s) {
  __shared__ float of_warps[2][8];
  kernel_begin();
  next_may_start();
  constexpr int W = 8, kLanes = 32 * WARPS, kRows = 8 / WARPS;
  const Source &m = s.of[blockIdx.y];
  const int lane = threadIdx.x % kLanes, warp = threadIdx.x >> 5;
  const int64_t pieces = (m.cols + W - 1) / W;
  __half *to = static_cast<__half *>(m.to);
  int turn = 0;
  for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; r < m.rows; r += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const float *x = static_cast<const float *>(m.p) + r * m.stride;
    float most = 0.f, held[HELD][W];
    auto largest_of = [&](const float (&v)[W]) {
#pragma unroll
      for (int e = 0; e < W; ++e) most = fmaxf(most, finite_size(v[e]));
    };
    if (WIDE) {
#pragma unroll
      for (int k = 0; k < HELD; ++k)
        if (lane + k * kLanes < pieces) load_piece<W>(x + (lane + k * kLanes) * W, held[k]);
#pragma unroll
      for (int k = 0; k < HELD; ++k)
        if (lane + k * kLanes < pieces) largest_of(held[k]);
#pragma unroll 2
      for (int64_t i = lane + HELD * kLanes; i < pieces; i += kLanes) {
        float v[W];
        load_piece<W>(x + i * W, v);
        largest_of(v);
      }
    } else {
#pragma unroll 8
      for (int64_t c = lane; c < m.cols; c += kLanes) most = fmaxf(most, finite_size(x[c]));
    }
    most = warp_max(most);
    if (WARPS > 1) {  // (by turns, so that one wait a row is enough)
      if (threadIdx.x % 32 == 0) of_warps[turn][warp] = most;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, of_warps[turn][k]);
    }
    const int up = exponent_of(most);
    if (lane == 0) m.amax[r] = m.down ? ldexpf(1.f, -up) : most;
    const float by = ldexpf(1.f, up);
    __half *high = to + r * m.ld, *low = high + m.plane;
    auto leave = [&](int64_t i, float (&v)[W]) {
      float back[W];
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] *= by;
      const Pack<__half, W> h = pack<__half, W>(v);
      unpack<__half, W>(h, back);
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] -= back[e];
      *reinterpret_cast<Pack<__half, W> *>(high + i * W) = h;
      store_piece<W>(low + i * W, v);
    };
    if (WIDE) {
#pragma unroll
      for (int k = 0; k < HELD; ++k)
        if (lane + k * kLanes < pieces) leave(lane + k * kLanes, held[k]);
#pragma unroll 2
      for (int64_t i = lane + HELD * kLanes; i < pieces; i += kLanes) {
        float v[W];
        load_piece<W>(x + i * W, v);
        leave(i, v);
      }
    } else {  // (an element a lane: rows at any address are read and written in runs of 32)
#pragma unroll 8
      for (int64_t c = lane; c < m.cols; c += kLanes) {
        const float v = x[c] * by;
        const __half h = __float2half_rn(v);
        high[c] = h;
        low[c] = __float2half_rn(v - __half2float(h));
      }
    }
  }
}

// -- targets -------------------------------------------------------------------------------------
// A token's targets in the order of their rows: [tokens][K] rows of the shard (INT_MAX: none) and
// weights; what the loss needs beside them.
struct Targets {
  int32_t *idx;
  float *weight;
  float *coef;            // backward: of the softmax
  float *live;            // backward: 0 where a token has no gradient
  float *entropy, *mass;  // forward: sum q log q, Q
  float *size_part;       // backward: the largest |coef| + sum |weight| of a block's tokens
  int32_t *arrived;       // of the products: zeros
  int n_arrived;
};

constexpr int kTargetWarps = 8;
constexpr int kMaxTargets = 256;

__device__ __forceinline__ int64_t id_at(const HeadArgs &a, int64_t i) {
  return a.id64 ? static_cast<const int64_t *>(a.ids)[i] : static_cast<const int32_t *>(a.ids)[i];
}
__device__ __forceinline__ int32_t row_of(const HeadArgs &a, int64_t id) {
  return id >= a.v0 && id - a.v0 < a.V ? (int32_t)(id - a.v0) : INT_MAX;
}

// A warp per token: the teacher's distribution, sorted by row by counting the rows before each.
__global__ void __launch_bounds__(kTargetWarps * 32) head_targets_kernel(HeadArgs a, Targets o) {
  __shared__ int32_t rows[kTargetWarps][kMaxTargets];
  __shared__ float sizes[kTargetWarps];
  kernel_begin();
  next_may_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < o.n_arrived; i += blockDim.x) o.arrived[i] = 0;
  const bool grad = a.grad;
  float most_size = 0.f;
  for (int64_t t = (int64_t)blockIdx.x * kTargetWarps + warp; t < a.n; t += (int64_t)gridDim.x * kTargetWarps) {
    float up = 0.f, lse_up = 0.f;  // of the loss (times tau) and of lse (over tau)
    if (grad) {
      up = a.scale * a.tau * a.dloss[t];
      if (a.dlse) lse_up = a.scale / a.tau * a.dlse[t];
    }
    float coef, size;
    if (!a.logits) {
      const int64_t id = id_at(a, t);
      const bool valid = id >= 0;
      const float q = valid ? (grad ? up : 1.f) : 0.f;
      if (lane == 0) {
        o.idx[t] = valid ? row_of(a, id) : INT_MAX;
        o.weight[t] = q;
        if (!grad) o.entropy[t] = 0.f, o.mass[t] = q;
      }
      coef = q + lse_up;
      size = fabsf(coef) + fabsf(q);
    } else {
      float v[kMaxTargets / 32];
      int32_t row[kMaxTargets / 32];
      float most = -INFINITY;
      bool any = false;
      const int own = (a.K - lane + 31) / 32;  // this lane's entries: lane, lane + 32, ...
#pragma unroll
      for (int i = 0; i < kMaxTargets / 32; ++i) {
        v[i] = -INFINITY;
        row[i] = INT_MAX;
        if (i >= own) continue;
        const int64_t at = t * a.K + lane + 32 * i, id = id_at(a, at);
        if (id >= 0) {
          float logit;
          load_param<1>(a.logits, a.logits_type, at, 0.f, &logit);
          v[i] = logit / a.tau;
          row[i] = row_of(a, id);
          any |= !(v[i] == -INFINITY);
        }
        most = fmaxf(most, v[i]);
        rows[warp][lane + 32 * i] = row[i];
      }
      any = __any_sync(0xFFFFFFFFu, any);
      most = warp_max(most);
      float log_sum = a.teacher_lse ? a.teacher_lse[t] : 0.f;
      if (!a.teacher_lse) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kMaxTargets / 32; ++i)
          if (i < own && !(v[i] == -INFINITY)) sum += expf(v[i] - most);
        log_sum = most + logf(warp_sum(sum));
      }
      float mass = 0.f, entropy = 0.f;
#pragma unroll
      for (int i = 0; i < kMaxTargets / 32; ++i) {
        if (i >= own) continue;
        const bool has = !(v[i] == -INFINITY);  // (a missing entry, or one without weight)
        const float log_q = has ? v[i] - log_sum : 0.f, q = has ? expf(log_q) : 0.f;
        mass += q;
        entropy += q * log_q;
        v[i] = grad && has ? q * up : q;
      }
      mass = warp_sum(mass);
      entropy = warp_sum(entropy);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kMaxTargets / 32; ++i) {
        if (i >= own) continue;
        const int k = lane + 32 * i;
        int before = 0;
        for (int j = 0; j < a.K; ++j) before += rows[warp][j] < row[i] || (rows[warp][j] == row[i] && j < k);
        o.idx[t * a.K + before] = row[i];
        o.weight[t * a.K + before] = v[i];
      }
      __syncwarp();
      if (!grad && lane == 0) o.entropy[t] = entropy, o.mass[t] = any ? mass : 0.f;
      coef = (any ? up * mass : 0.f) + lse_up;
      size = fabsf(coef) + (any ? fabsf(up) * mass : 0.f);
    }
    if (grad && lane == 0) {
      o.coef[t] = coef;
      o.live[t] = size;
    }
    most_size = fmaxf(most_size, finite_size(size));
  }
  if (!grad) return;
  if (lane == 0) sizes[warp] = most_size;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kTargetWarps; ++w) most_size = fmaxf(most_size, sizes[w]);
    o.size_part[blockIdx.x] = most_size;
  }
}

// -- products --------------------------------------------------------------------------------------
// D = A B^T on tiles of 256 x 256 by persistent pairs of blocks (echo_tensor.cuh).  The sum may run
// along the rows of an operand in memory (K-major) or down its columns (MN-major), and over several
// pairs of planes.  A launch has up to two products (dx and dW), whose tiles are shared out together.
//
// In each block one thread copies stages into a ring, a thread of the pair's first block issues the
// products, and eight warps take the sums out of tensor memory, which holds two sets of them, add
// them up, and finish the tile while the next one is summed.  What bounds it, at 2048 tokens:
//   - logits, 12288 columns, 6400 rows, bf16: 180 us, 1.79 PFLOP/s, tensor pipe busy 78% of the time.
//     A stage takes 640 to 660 clocks, of which the products are 512: operands come from L2 at 64 bytes
//     a clock and SM, and a copy of half of them (other results wrong) saved 5% only.
//   - logits, 2048 columns, 51200 rows, 64 targets a token: 247 us; 22 rounds where 21.05 would do.
//   - P, 2048 columns, 25600 rows, three planes: 162 us, 10000 clocks a tile to finish beside the 20000
//     of its products, which go slower meanwhile.
//   - dx and dW, 25600 x 2048, fp32 dW (2.15e11 operations on 16-bit numbers for dx, twice that for dW): 357 us; with a
//     16-bit dW 6400 x 12288: 342 us, 1.88 PFLOP/s.
// What counted: 32-bit counters and nothing looked up in a stage's way, which single threads take (a
// stage of 64-bit counters and arguments read from memory: 20% slower); results through the copy engine
// (1236 us for dx and dW with stores by lanes, 451 so); tiles split where rounds are not full, and joined
// through shared memory; longer first sets (lead_of).  Five stages and 64 KB on the way out are as fast
// as six and 32 KB; four are 4% slower.
constexpr int kTile = 256, kHalf = 128, kBK = 64;
constexpr int kThreads = 384;                    // warp 0: copies, 1: products, 4-11: tiles out
constexpr int kFewRegs = 88, kManyRegs = 208;    // a thread of warps 0-3 and of 4-11
static_assert(128 * kFewRegs + 256 * kManyRegs <= kThreads * 168, "the block's registers");
constexpr int kOperandBytes = kHalf * kBK * 2, kStageBytes = 2 * kOperandBytes, kStages = 5;
constexpr int kSlots = 2, kSlotBytes = 4096;     // a warp's buffers on the way out: 32 rows of 128 bytes each
constexpr size_t kSmem = (size_t)kStages * kStageBytes + 8 * kSlots * kSlotBytes + 512 + 1024;

struct Job {
  int M, N, steps;  // rows, columns; stages of a pair of planes
  int pairs, plane_a[3], plane_b[3];
  int lead, lead_part, set;  // stages that the tensor core adds up by itself: of the first two sets of a tile, of a part of one, of the others
  uint32_t instr;
  int tiles_n;
  int64_t tiles;
  Scale scale_a, scale_b;
  int type, add;    // D, times 2^-(both exponents), is written as that type, or added
};
// Who computes what, of two products whose tiles take steps0 and steps1 stages.
//   - Of the first one `whole` tiles, each in `split` parts of (almost) equal length along its sum, a
//     part of every tile and then the next one, go to the pairs of blocks in turn.
//   - Of the tiles of the second one, the pairs that had one part less take `early` each, in turn; the
//     others go to all pairs in turn.
//   - What is left of the first one is the pool: its stages, one tile behind the other, are split evenly
//     over `pool_pairs`, so that a tile has up to three parts as a rule.  It comes first: parts are
//     joined while the next tile is summed.
struct Schedule {
  int64_t whole, tiles1, pool;
  int split, steps0, steps1, early, pool_pairs;
};

struct HeadProduct {
  // Of kOut dx (its first operand K-major, the second MN-major) and dW (both MN-major): either may have no
  // tiles.  Else the logits (both K-major) and nothing.
  Job job[2];
  Schedule schedule;
  float4 *parts;     // sums of parts of tiles: [place][block][warp][columns / 4][lane]
  int32_t *arrived;  // [tile][block][warp] parts that are there: zeros between launches
  WaitLimit wait;
  int skip;          // failure injection for tests: this 64-column step is never copied (-1: none)
  // the logits' product
  int64_t n;         // tokens
  int K, v_begin;    // targets of a token; the piece's first row
  float alpha;       // scale / tau
  const int32_t *idx;
  const float *weight, *coef, *lse;
  const float *w_down;  // forward, fp32: factors of the weight's rows
  float2 *part;      // [columns / 128][n] largest element (times log2 e) and sum of exponentials
  float *picked;     // [n][K] z of the targets
  int p_bf16, p_half;  // planes of P: one of bf16, of fp16
  Scale p_scale;
};
enum { kStats, kGrad, kOut };  // what becomes of the sums

__device__ __forceinline__ void tile_place(const Job &j, int64_t t, int &r0, int &c0) {
  const int64_t rows = (j.M + kTile - 1) / kTile, band = t / (8 * j.tiles_n), in = t % (8 * j.tiles_n), high = min((int64_t)8, rows - band * 8);
  r0 = (int)(band * 8 + in % high) * kTile;
  c0 = (int)(in / high) * kTile;
}

__device__ __forceinline__ void copy_rows(uint32_t to, const CUtensorMap *map, bool mn, int r, int k, int plane, uint32_t bar) {
  if (mn) {
    copy_tile(to, map, r, k, 0, plane, bar);
    copy_tile(to + 8192, map, r + 64, k, 0, plane, bar);
  } else {
    copy_tile(to, map, k, r, 0, plane, bar);
  }
}

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}

// A warp's buffers on the way out take turns: one is written again once the copy engine has read it.
struct Slots {
  unsigned char *base;
  uint32_t turn;
  int lane;
  // The next one, for the whole warp.
  __device__ __forceinline__ unsigned char *next() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(kSlots - 1) : "memory");
    __syncwarp();
    unsigned char *p = base + turn * kSlotBytes;
    turn = (turn + 1) % kSlots;
    return p;
  }
  // All of them.
  __device__ __forceinline__ unsigned char *all() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
    __syncwarp();
    return base;
  }
};
// The 16-byte piece i of a row's 128 bytes, as the copy engine takes them (its 128-byte swizzle): rows
// would meet in the same banks otherwise.
template <typename T>
__device__ __forceinline__ Pack<T, 16 / sizeof(T)> *slot_piece(unsigned char *slot, int row, int i) {
  return reinterpret_cast<Pack<T, 16 / sizeof(T)> *>(slot + row * 128 + (i ^ (row & 7)) * 16);
}
// 32 fp32 columns of a slot added to what a matrix holds; what is outside the matrix is dropped.
__device__ __forceinline__ void add_slot(const CUtensorMap *map, const unsigned char *slot, int col, int row) {
  asm volatile("cp.reduce.async.bulk.tensor.4d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4, %4}], [%1];\ncp.async.bulk.commit_group;\n" ::"l"(map),
               "r"(smem_u32(slot)), "r"(col), "r"(row), "r"(0)
               : "memory");
}

// 32 rows of 64 elements out, by a warp: lane r has those of row row0 + r in v, from column c.
// By the copy engine, which writes it, or adds it to an fp32 matrix (each element by one addition, so
// that the result has one order).
template <typename T>
__device__ __forceinline__ void engine_out(const Job &j, const CUtensorMap *map, int row0, int c, const float *v, Slots &slots) {
  constexpr int kCols = 128 / sizeof(T), kPiece = 16 / sizeof(T);
#pragma unroll
  for (int c1 = 0; c1 < 64; c1 += kCols) {
    if (c + c1 >= j.N) return;
    unsigned char *slot = slots.next();
#pragma unroll
    for (int e = 0; e < 8; ++e) *slot_piece<T>(slot, slots.lane, e) = pack<T, kPiece>(v + c1 + e * kPiece);
    half_written();
    if (slots.lane == 0) {
      if (sizeof(T) == 4 && j.add) add_slot(map, slot, c + c1, row0);
      else store_half(map, slot, c + c1, row0, 0, 0);
    }
  }
}
// What a pair of blocks does, one after the other: stages k0 to k1 of a tile's sum, which is one of
// several parts of it or all.
struct Share {
  int which, k0, k1;
  int64_t tile;
  int64_t count;      // of the tile, among the counts of parts
  int parts;          // 1: all
  int64_t place, first, second, step;  // of this part's sums; of the first and the second; from there on
};
struct Worker {
  const Schedule &s;
  const int pair, pairs;
  int64_t i, j, x, end;
  int early;
  __device__ __forceinline__ Worker(const Schedule &s, int pair, int pairs) : s(s), pair(pair), pairs(pairs), i(pair), x(0), end(0) {
    const int64_t n = s.whole * s.split;
    const int extra = (int)(n % pairs);  // pairs with one part more
    early = extra && pair >= extra ? s.early : 0;
    j = early ? pair - extra : (extra ? (int64_t)s.early * (pairs - extra) : 0) + pair;
    if (pair < s.pool_pairs) x = s.pool * pair / s.pool_pairs, end = s.pool * (pair + 1) / s.pool_pairs;
  }
  __device__ __forceinline__ bool next(Share &w) {
    w.parts = 1;
    if (x < end) {
      const int64_t t = x / s.steps0, base = t * s.steps0;
      w.which = 0, w.tile = s.whole + t, w.count = t;
      w.k0 = (int)(x - base);
      w.k1 = (int)min((int64_t)s.steps0, end - base);
      // pair p begins at floor(pool p / pool_pairs): the last one at or before a stage s is floor(((s + 1) pool_pairs - 1) / pool).
      // A pair has two places: of a tile's beginning, and of its end or a part between.
      const int first = (int)(((base + 1) * s.pool_pairs - 1) / s.pool);
      w.parts = (int)(((base + s.steps0) * s.pool_pairs - 1) / s.pool) - first + 1;
      w.place = 2 * pair + (pair == first), w.first = 2 * first + 1, w.second = 2 * first + 2, w.step = 2;
      x = base + w.k1;
      return true;
    }
    if (i < s.whole * s.split) {
      const int part = s.split > 1 ? (int)(i / s.whole) : 0;
      w.which = 0, w.tile = i - part * s.whole;
      w.k0 = (int)((int64_t)s.steps0 * part / s.split), w.k1 = (int)((int64_t)s.steps0 * (part + 1) / s.split);
      w.parts = s.split, w.count = w.tile;
      w.place = i, w.first = w.tile, w.second = w.tile + s.whole, w.step = s.whole;
      i += pairs;
      return true;
    }
    if (j < s.tiles1) {
      w.which = 1, w.tile = j, w.k0 = 0, w.k1 = s.steps1;
      if (early) {
        const int extra = (int)(s.whole * s.split % pairs);
        j = --early ? j + (pairs - extra) : (int64_t)s.early * (pairs - extra) + pair;
      } else {
        j += pairs;
      }
      return true;
    }
    return false;
  }
};

// A row's targets from a column on, in their order; the one after the next is on its way.
struct Cursor {
  const int32_t *idx;
  const float *weight;
  int K, begin, k, next, after;
  float w, w_after;
  __device__ __forceinline__ void load(int at, int &column, float &x) {
    column = INT_MAX;
    if (at >= K) return;
    const int row = idx[at];
    if (weight) x = weight[at];
    if (row != INT_MAX) column = row - begin;
  }
  // `weights` may be null: w is 0 then
  __device__ __forceinline__ void start(const int32_t *rows, const float *weights, int count, int v_begin, int column) {
    idx = rows, weight = weights, K = count, begin = v_begin, k = 0, w = w_after = 0.f;
    for (int left = K; left;) {  // eight places at a time: their loads do not wait for one another
      const int step = (left + 7) / 8;
      int before = 0;
#pragma unroll
      for (int i = 1; i <= 8; ++i) before += i * step <= left && idx[k + i * step - 1] < v_begin + column;
      k += before * step;
      left = min(step - 1, left - before * step);
    }
    load(k, next, w);
    load(k + 1, after, w_after);
  }
  __device__ __forceinline__ void none() {
    idx = nullptr, weight = nullptr, K = 0, begin = 0, k = 0, next = after = INT_MAX, w = w_after = 0.f;
  }
  __device__ __forceinline__ void step() {
    ++k;
    next = after, w = w_after;
    load(k + 1, after, w_after);
  }
};

// `bytes` contiguous bytes to this block's shared memory.
__device__ __forceinline__ void copy_bytes(uint32_t to, const void *from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
               : "memory");
}

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    head_product_kernel(const __grid_constant__ CUtensorMap amap0, const __grid_constant__ CUtensorMap bmap0, const __grid_constant__ CUtensorMap amap1,
                        const __grid_constant__ CUtensorMap bmap1, const __grid_constant__ CUtensorMap out0, const __grid_constant__ CUtensorMap out1,
                        const __grid_constant__ HeadProduct a) {
  extern __shared__ unsigned char raw[];
  unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) / 1024 * 1024);
  unsigned char *buffers = base + kStages * kStageBytes;
  uint64_t *bars = reinterpret_cast<uint64_t *>(buffers + 8 * kSlots * kSlotBytes);
  __shared__ uint32_t tmem_base;
  __shared__ int give_up;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;  // (clusters of two along x)
  // `full` and `sums_empty` are used in the first block alone, the others in both
  const uint32_t ring = smem_u32(base), full = smem_u32(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages, sums_empty = sums_full + 16,
                 done = sums_empty + 16, joins = done + 8;  // (joins: two of each of the eight warps)
  volatile int *abort = &give_up;
  if (threadIdx.x == 0) {
    give_up = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, 16);
    }
    bar_init(done, 1);
    for (int i = 0; i < 16; ++i) bar_init(joins + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (threadIdx.x == 32 * 3) asm volatile("prefetch.tensormap [%0];\nprefetch.tensormap [%1];\n" ::"l"(&amap0), "l"(&bmap0) : "memory");
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base)), "r"(2u * kTile) : "memory");
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

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kFewRegs));
    if (warp == 0 && lane == 0) {
      // (a stage's way is short: what it takes is in registers, and nothing is divided)
      const uint32_t full_first = in_first(full);
      const WaitLimit wait = a.wait;
      const int skip = a.skip;
      int s = 0;
      uint32_t phase = 1;
      bool ok = true;
      auto copy = [&](auto a_mn, auto b_mn, const CUtensorMap *amap, const CUtensorMap *bmap, const Job &j, const Share &w) {
        // (the pairs of planes of a stage follow one another, so that a plane that two of them read is in L2)
        const int planes = j.pairs;
        int r0, c0, k = w.k0 / planes, p = w.k0 - k * planes;
        tile_place(j, w.tile, r0, c0);
        r0 += rank * kHalf, c0 += rank * kHalf;
        int plane_a = j.plane_a[p], plane_b = j.plane_b[p];
        for (int left = w.k1 - w.k0; left; --left) {
          ok = k != skip && bar_wait(empty + 8 * s, phase, abort, wait);
          if (!ok) break;
          const uint32_t at = ring + s * kStageBytes, bar = full_first + 8 * s;
          if (rank == 0) bar_expect(full + 8 * s, 2 * kStageBytes);  // both blocks' copies
          copy_rows(at, amap, decltype(a_mn)::value, r0, k * kBK, plane_a, bar);
          copy_rows(at + kOperandBytes, bmap, decltype(b_mn)::value, c0, k * kBK, plane_b, bar);
          if (++s == kStages) s = 0, phase ^= 1;
          if (planes == 1) {
            ++k;
          } else {
            if (++p == planes) p = 0, ++k;
            plane_a = j.plane_a[p], plane_b = j.plane_b[p];
          }
        }
      };
      Worker worker(a.schedule, pair, pairs);
      for (Share w; ok && worker.next(w);) {
        if (MODE != kOut) copy(Int<0>{}, Int<0>{}, &amap0, &bmap0, a.job[0], w);
        else if (w.which == 0) copy(Int<0>{}, Int<1>{}, &amap0, &bmap0, a.job[0], w);
        else copy(Int<1>{}, Int<1>{}, &amap1, &bmap1, a.job[1], w);
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      const WaitLimit wait = a.wait;
      int s = 0, b = 0;
      uint32_t phase = 0, sums_phase = 1;  // (of both sets alike: they take turns)
      bool ok = true;
      auto multiply = [&](auto a_mn, auto b_mn, const Job &j, const Share &w) {
        constexpr bool A = decltype(a_mn)::value, B = decltype(b_mn)::value;
        const uint32_t instr = j.instr;
        const int lead = w.parts > 1 ? j.lead_part : j.lead, set = j.set;
        const uint64_t p0 = operand(ring, A), q0 = operand(ring + kOperandBytes, B);
        for (int left = w.k1 - w.k0, in_set = 0, ends = lead, number = 0; left; --left) {
          ok = (in_set || bar_wait(sums_empty + 8 * b, sums_phase, abort, wait)) && bar_wait(full + 8 * s, phase, abort, wait);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint32_t d = tmem + b * kTile;
          const uint64_t p = p0 + (uint32_t)s * (kStageBytes >> 4), q = q0 + (uint32_t)s * (kStageBytes >> 4);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk) mma(d, p + step16(A) * kk, q + step16(B) * kk, instr, kk > 0 || in_set);
          commit_pair(empty + 8 * s);
          if (++s == kStages) s = 0, phase ^= 1;
          if (++in_set == ends || left == 1) {
            commit_pair(sums_full + 8 * b);
            in_set = 0;
            ends = ++number < 2 ? lead : set;
            b ^= 1;
            if (b == 0) sums_phase ^= 1;
          }
        }
      };
      Worker worker(a.schedule, pair, pairs);
      for (Share w; ok && worker.next(w);) {
        if (MODE != kOut) multiply(Int<0>{}, Int<0>{}, a.job[0], w);
        else if (w.which == 0) multiply(Int<0>{}, Int<1>{}, a.job[0], w);
        else multiply(Int<1>{}, Int<1>{}, a.job[1], w);
      }
      commit(done);  // nothing is in flight when the block ends
      const long long t0 = clock64();
      while (!bar_try(done, 0) && clock64() - t0 <= a.wait.clocks) {
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kManyRegs));
    const int quarter = warp & 3, side = (warp - 4) >> 2;  // (a warp reaches the 32 rows of tensor memory of its number modulo 4)
    Slots slots{buffers + (warp - 4) * kSlots * kSlotBytes, 0, lane};
    const uint32_t join = joins + 16 * (warp - 4);
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + side * kHalf;
    constexpr int kParts = kHalf / 32;
    int down[2] = {0, 0};
    for (int w = 0; w < (MODE == kOut ? 2 : 1); ++w) down[w] = -exponent(a.job[w].scale_a) - exponent(a.job[w].scale_b);
    float alpha2 = MODE == kOut ? 1.f : ldexpf(a.alpha, down[0]) * kLog2e;  // (sums become logits over ln 2)
    const float p_up = MODE == kGrad ? ldexpf(fraction(a.p_scale), exponent(a.p_scale)) : 1.f, p_down = MODE == kOut ? 1.f / fraction(a.p_scale) : 1.f;
    int64_t n = 0;
    bool ok = true;
    Worker worker(a.schedule, pair, pairs);
    for (Share w; ok && worker.next(w);) {
      const int which = MODE == kOut ? w.which : 0;
      const Job &j = a.job[which];
      int r0, c0;
      tile_place(j, w.tile, r0, c0);
      const int row0 = r0 + rank * kHalf + quarter * 32;
      c0 += side * kHalf;
      // what the tile's end needs comes during the sums
      const int64_t row = row0 + lane;
      const bool in = row < j.M;
      Cursor at;
      at.none();
      float coef = 0.f, shift = 0.f;
      // (fp32: a power of two of each row, one of each row of the weight.  Half of the row's, the weight's, the other half: the two
      // may be far from one where their product is not, and sums, 2^54 at most, meet neither end of fp32's range on the way)
      const int row_down = MODE == kStats && in && a.w_down ? -exponent_of(a.job[0].scale_a.rows[row]) : 0;
      if (MODE == kStats && a.w_down) alpha2 = ldexpf(a.alpha, row_down / 2) * kLog2e;
      if (MODE != kOut && in) {
        at.start(a.idx + row * a.K, MODE == kGrad ? a.weight + row * a.K : nullptr, a.K, a.v_begin, c0);
        if (MODE == kGrad) {
          // coef exp(z - lse) = coef' exp2(z log2 e - shift): the rounding of shift goes into coef'
          const float lse = a.lse[row];
          coef = a.coef[row] * p_up;
          shift = lse * kLog2e;
          const float rest = fmaf(lse, kLog2e, -shift);
          if (coef != 0.f && fabsf(rest) < 1.f) coef *= exp2f(-rest);
        }
      }
      float acc[kHalf] = {};
      const int lead = w.parts > 1 ? j.lead_part : j.lead, steps = w.k1 - w.k0, after = steps - 2 * lead;  // (stages after the first two sets)
      const int sets = after > 0 ? 2 + (after + j.set - 1) / j.set : steps > lead ? 2 : 1;
      for (int set = 0; set < sets; ++set) {
        const int b = (int)(n & 1);
        ok = __all_sync(0xFFFFFFFFu, bar_wait(sums_full + 8 * b, (uint32_t)(n / 2) & 1, abort, a.wait));  // (a warp gives up as one)
        if (!ok) break;
        ++n;
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          Sums s;
          __syncwarp();
          load_sums(from + b * kTile + part * 32, s);
          sums_loaded();
          pass(s);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const Pair x{__uint_as_float(s.r[e]), __uint_as_float(s.r[e + 1])}, y{acc[part * 32 + e], acc[part * 32 + e + 1]};
            const Pair sum = MODE == kOut ? add2(x, y) : fma2(x, both(alpha2), y);
            acc[part * 32 + e] = sum.a, acc[part * 32 + e + 1] = sum.b;
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_first(sums_empty + 8 * b));
      }
      if (!ok) break;
      if (row0 >= j.M || c0 >= j.N) continue;
      if (w.parts > 1) {
        // this part's sums to memory; who comes last adds the parts, in their order, and goes on with the tile
        constexpr int64_t kPart = 16 * (kHalf / 4 * 32);
        const int64_t place = (int64_t)(rank * 8 + warp - 4) * (kHalf / 4 * 32) + lane;
        float4 *mine = a.parts + w.place * kPart + place;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            mine[(part * 8 + e) * 32] = make_float4(acc[part * 32 + 4 * e], acc[part * 32 + 4 * e + 1], acc[part * 32 + 4 * e + 2], acc[part * 32 + 4 * e + 3]);
        __threadfence();
        __syncwarp();
        int32_t *count = a.arrived + w.count * 16 + rank * 8 + warp - 4, before = 0;
        if (lane == 0) before = atomicAdd(count, 1);
        if (__shfl_sync(0xFFFFFFFFu, before, 0) != w.parts - 1) continue;  // another part comes later
        if (lane == 0) *count = 0;
        __threadfence();
#pragma unroll
        for (int e = 0; e < kHalf; ++e) acc[e] = 0.f;
        // 32 columns of a part at a time come to the warp's buffers, the next ones while these are added
        // (loads to registers, of which the sums leave few, took 10000 clocks a part)
        unsigned char *chunk = slots.all();
        asm volatile("fence.proxy.async;\n" ::: "memory");  // (what other blocks wrote, for the copy engine)
        auto fetch = [&](int q, int c) {
          if (lane != 0 || q >= w.parts) return;
          const float4 *from_part = a.parts + (q ? w.second + (q - 1) * w.step : w.first) * kPart + (place - lane) + c * 256;
          bar_expect(join + 8 * (c & 1), kSlotBytes);
          copy_bytes(smem_u32(chunk) + (c & 1) * kSlotBytes, from_part, kSlotBytes, join + 8 * (c & 1));
        };
        fetch(0, 0);
#pragma unroll 1
        for (int q = 0; q < w.parts && ok; ++q) {
#pragma unroll
          for (int c = 0; c < kParts; ++c) {
            fetch(c == kParts - 1 ? q + 1 : q, (c + 1) % kParts);
            ok = ok && __all_sync(0xFFFFFFFFu, bar_wait(join + 8 * (c & 1), c >> 1, abort, a.wait));  // (each has two phases a part)
            if (ok) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float4 f = *reinterpret_cast<const float4 *>(chunk + (c & 1) * kSlotBytes + (e * 32 + lane) * 16);
                acc[c * 32 + 4 * e] += f.x;
                acc[c * 32 + 4 * e + 1] += f.y;
                acc[c * 32 + 4 * e + 2] += f.z;
                acc[c * 32 + 4 * e + 3] += f.w;
              }
            }
            __syncwarp();
          }
        }
        if (!ok) break;
      }
      if constexpr (MODE == kStats) {
        if (a.w_down) {  // (the array is as long as the tiles)
          const float rest = ldexpf(1.f, row_down - row_down / 2);
#pragma unroll
          for (int e = 0; e < kHalf; e += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(a.w_down + c0 + e);
            acc[e] = acc[e] * f.x * rest, acc[e + 1] = acc[e + 1] * f.y * rest;
            acc[e + 2] = acc[e + 2] * f.z * rest, acc[e + 3] = acc[e + 3] * f.w * rest;
          }
        }
        if (c0 + kHalf > j.N)
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (c0 + part * 32 + e >= j.N) acc[part * 32 + e] = -INFINITY;
        float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int e = 0; e < 32; ++e) m[e & 3] = fmaxf(m[e & 3], acc[part * 32 + e]);
        const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), zero = most == -INFINITY ? 0.f : most;
        Pair sum[2] = {both(0.f), both(0.f)};
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const Pair x = add2({acc[part * 32 + e], acc[part * 32 + e + 1]}, both(-zero));
            sum[e / 2 & 1] = add2(sum[e / 2 & 1], {exp2_fast(x.a), exp2_fast(x.b)});
          }
        sum[0] = add2(sum[0], sum[1]);
        if (in) a.part[(int64_t)(c0 / kHalf) * a.n + row] = make_float2(most, sum[0].a + sum[0].b);
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          const int column0 = c0 + part * 32;
          while (__any_sync(0xFFFFFFFFu, at.next < column0 + 32)) {
            const bool hit = at.next < column0 + 32;
            const int column = hit ? at.next - column0 : 0;
            // the element of that number, a bit of it after the other
            float z[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = column & 16 ? acc[part * 32 + e + 16] : acc[part * 32 + e];
#pragma unroll
            for (int half = 8; half; half >>= 1)
#pragma unroll
              for (int e = 0; e < half; ++e) z[e] = column & half ? z[e + half] : z[e];
            if (hit) {
              a.picked[row * a.K + at.k] = z[0] * kLn2;
              at.step();
            }
          }
        }
        continue;
      }
      // 64 columns and then the others, in the registers of the first (unrolled, the code would be long
      // and runs once a tile).
      float *v = acc;
      const float f1 = ldexpf(p_down, down[which] / 2), f2 = ldexpf(1.f, down[which] - down[which] / 2);
#pragma unroll 1
      for (int c = c0; c < min(j.N, c0 + kHalf); c += 64) {
        if constexpr (MODE == kGrad) {
#pragma unroll
          for (int e = 0; e < 64; ++e) v[e] = coef == 0.f ? 0.f : coef * exp2_fast(v[e] - shift);
#pragma unroll
          for (int e0 = 0; e0 < 64; e0 += 32)
            while (__any_sync(0xFFFFFFFFu, at.next < c + e0 + 32)) {
              const bool hit = at.next < c + e0 + 32;
              const int column = hit ? at.next - c - e0 : -1;
              const float weight = at.w * p_up;
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (column == e) v[e0 + e] -= weight;
              if (hit) at.step();
            }
          int plane = 0;
          if (a.p_bf16) {
            unsigned char *slot = slots.next();
#pragma unroll
            for (int e = 0; e < 8; ++e) *slot_piece<__nv_bfloat16>(slot, lane, e) = pack<__nv_bfloat16, 8>(v + 8 * e);
            half_written();
            if (lane == 0) store_half(&out0, slot, c, row0, 0, plane);
            ++plane;
          }
#pragma unroll 1
          for (; plane < a.p_bf16 + a.p_half; ++plane) {
            unsigned char *slot = slots.next();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const Pack<__half, 8> h = pack<__half, 8>(v + 8 * e);
              float back[8];
              unpack<__half, 8>(h, back);
#pragma unroll
              for (int i = 0; i < 8; ++i) v[8 * e + i] -= back[i];  // what the next plane holds
              *slot_piece<__half>(slot, lane, e) = h;
            }
            half_written();
            if (lane == 0) store_half(&out0, slot, c, row0, 0, plane);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e) v[e] = v[e] * f1 * f2;
          const CUtensorMap *map = which ? &out1 : &out0;
          if (j.type == ECHO_F32) engine_out<float>(j, map, row0, c, v, slots);
          else if (j.type == ECHO_BF16) engine_out<__nv_bfloat16>(j, map, row0, c, v, slots);
          else engine_out<__half>(j, map, row0, c, v, slots);
        }
#pragma unroll
        for (int e = 0; e < 64; ++e) acc[e] = acc[e + 64];
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  if (give_up) {  // stages and parts of tiles that nobody has waited for may be on their way to this block: they land long before this
    const long long t0 = clock64();
    while (clock64() - t0 < 1000000) {
    }
  }
  cluster_sync();  // (the other block's products read this one's stages, and signal its barriers)
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2u * kTile) : "memory");
  }
}

// A result from its fp32 sums, written or added, in pieces of W elements, four of a thread on their way.
// Bound by the bytes.
template <typename T, int W>
__global__ void __launch_bounds__(256) head_round_kernel(const float *from, int64_t ld, int64_t rows, int64_t cols, T *to, int64_t stride, int add) {
  kernel_begin();
  next_may_start();
  const uint32_t pieces = (uint32_t)(cols / W);
  const int64_t all = rows * pieces;
  constexpr int kFlight = 4;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 * kFlight + threadIdx.x; i0 < all; i0 += (int64_t)gridDim.x * 256 * kFlight) {
    float v[kFlight][W];
    Pack<T, W> old[kFlight];
    T *at[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int64_t i = i0 + k * 256;
      at[k] = nullptr;
      if (i >= all) continue;
      const int64_t r = all >> 32 ? i / pieces : (int64_t)((uint32_t)i / pieces), c = (i - r * pieces) * W;
      at[k] = to + r * stride + c;
      load_piece<W>(from + r * ld + c, v[k]);
      if (add) old[k] = *reinterpret_cast<const Pack<T, W> *>(at[k]);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (!at[k]) continue;
      if (add) {
        float x[W];
        unpack<T, W>(old[k], x);
#pragma unroll
        for (int e = 0; e < W; ++e) v[k][e] += x[e];
      }
      store_piece<W>(at[k], v[k]);
    }
  }
}

// -- the end of the forward pass -------------------------------------------------------------------
// A block joins the parts of 32 rows: a warp every 32nd part of all rows, eight of them on their way,
// then a warp a row's targets, in their order.  Bound by latency: 2048 rows of 400 parts, 6.6 MB.
constexpr int kJoinWarps = 32;
__device__ __forceinline__ float2 joined(float2 x, float2 y) {  // (an empty part has -inf and 0)
  const float m = fmaxf(x.x, y.x);
  if (m == -INFINITY) return make_float2(m, x.y + y.y);
  return make_float2(m, x.y * exp2f(x.x - m) + y.y * exp2f(y.x - m));
}
__global__ void __launch_bounds__(kJoinWarps * 32) head_join_kernel(HeadArgs a, Targets t, const float2 *part, int64_t chunks, const float *picked) {
  __shared__ float2 sh[kJoinWarps][33];
  kernel_begin();
  next_may_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int64_t r0 = (int64_t)blockIdx.x * 32; r0 < a.n; r0 += (int64_t)gridDim.x * 32) {
    // a row's targets, while the parts come
    const int64_t row = r0 + warp;
    float cross = 0.f;
    if (row < a.n)
      for (int k = lane; k < a.K; k += 32)
        if (t.idx[row * a.K + k] != INT_MAX) cross += t.weight[row * a.K + k] * picked[row * a.K + k];
    float2 s = make_float2(-INFINITY, 0.f);
    constexpr int kFlight = 8;
    for (int64_t k0 = warp; k0 < chunks; k0 += kFlight * kJoinWarps) {
      float2 v[kFlight];
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        v[k] = make_float2(-INFINITY, 0.f);
        if (k0 + k * kJoinWarps < chunks && r0 + lane < a.n) v[k] = part[(k0 + k * kJoinWarps) * a.n + r0 + lane];
      }
#pragma unroll
      for (int k = 0; k < kFlight; ++k) s = joined(s, v[k]);
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (row < a.n) {
      s = sh[lane][warp];
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        const float2 other = make_float2(__shfl_xor_sync(0xFFFFFFFFu, s.x, d), __shfl_xor_sync(0xFFFFFFFFu, s.y, d));
        s = lane & d ? joined(other, s) : joined(s, other);
      }
      cross = warp_sum(cross);
      if (lane == 0) {
        const float lse = s.x == -INFINITY ? s.y == 0.f ? -INFINITY : NAN : fmaf(s.x, kLn2, logf(s.y)), mass = t.mass[row];
        if (a.loss) a.loss[row] = mass == 0.f ? 0.f : a.tau * a.tau * (t.entropy[row] + fmaf(mass, lse, -cross));
        if (a.lse) a.lse[row] = lse;
        if (a.part) a.part[row] = cross;
      }
    }
    __syncthreads();
  }
}

// -- few tokens of fp32 matrices ---------------------------------------------------------------------
// Planes of the weight are read, written and read again before the tensor cores have them, for tiles of
// 256 tokens: with 51200 x 4096 a call takes 485 us forward and 1060 backward from 17 tokens on, whose
// products alone would be 170.  Up to kFew tokens the products are made in fp32 from the weight as it is,
// read once for the logits (149 us with one token, 206 with eight, 371 with 16; its 839 MB take 124) and
// once for dx, and dW is written once (420, 535 and 880 us, of 371).  Above eight tokens it is neither bytes
// nor arithmetic that bounds them (16: DRAM 28%, the fma pipe 29%): with 128 registers a thread there are 16
// warps an SM, which issue in half of the cycles and wait for the weight in a third of their time.  32 tokens
// would take 957 us forward.
constexpr int kFew = 16, kFewThreads = 256, kFewWarps = kFewThreads / 32;
constexpr int kFewColumns = 512;   // of x in shared memory at a time
constexpr int few_rows(int tokens, bool many) { return tokens > 8 ? 4 : many ? 8 : 2; }  // of the weight, of a warp

// Where x and weight are 16-byte rows, a lane takes four neighbouring columns, else every 32nd.
template <bool WIDE>
__device__ __forceinline__ int few_column(int lane, int e) { return WIDE ? 4 * lane + e : lane + 32 * e; }

// Logits of a block's rows of the weight and all tokens; then the parts and targets of the forward pass, or P.
template <int TOKENS, int R, bool WIDE, bool GRAD>
__global__ void __launch_bounds__(kFewThreads) head_few_kernel(HeadArgs a, Targets t, float2 *part, float *picked, float *P, int64_t ldp) {
  constexpr int kRowsBlock = R * kFewWarps, kAhead = 8 / R;  // (of R rows, 128 columns each are on their way)
  __shared__ alignas(16) float xs[TOKENS][kFewColumns];
  __shared__ float zs[TOKENS][kRowsBlock];
  kernel_begin();
  next_may_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)a.n;
  const float *x = static_cast<const float *>(a.x);
  const int64_t v0 = (int64_t)blockIdx.x * kRowsBlock, first = v0 + warp * R;
  const float *w = static_cast<const float *>(a.w) + first * a.w_stride;
  float acc[R][TOKENS] = {};
  for (int64_t h0 = 0; h0 < a.H; h0 += kFewColumns) {
    for (int i = threadIdx.x; i < TOKENS * kFewColumns; i += kFewThreads) {
      const int row = i / kFewColumns, c = i % kFewColumns;
      xs[row][c] = row < n && h0 + c < a.H ? x[row * a.x_stride + h0 + c] : 0.f;
    }
    __syncthreads();
#pragma unroll 1
    for (int c0 = 0; c0 < kFewColumns && h0 + c0 < a.H; c0 += 128 * kAhead) {
      float f[kAhead][R][4];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int64_t c = h0 + c0 + 128 * u;
          const float *at = w + r * a.w_stride + c;
          const bool row = first + r < a.V;
          if (WIDE) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row && c + 4 * lane < a.H) v = __ldcs(reinterpret_cast<const float4 *>(at + 4 * lane));
            f[u][r][0] = v.x, f[u][r][1] = v.y, f[u][r][2] = v.z, f[u][r][3] = v.w;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[u][r][e] = row && c + few_column<WIDE>(lane, e) < a.H ? __ldcs(at + few_column<WIDE>(lane, e)) : 0.f;
          }
        }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
          const float *at = &xs[k][c0 + 128 * u];
          float g[4];
          if (WIDE) {
            const float4 v = *reinterpret_cast<const float4 *>(at + 4 * lane);
            g[0] = v.x, g[1] = v.y, g[2] = v.z, g[3] = v.w;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = at[few_column<WIDE>(lane, e)];
          }
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][k] = fmaf(f[u][r][e], g[e], acc[r][k]);
        }
    }
    __syncthreads();
  }
  const float alpha = a.scale / a.tau;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int k = 0; k < TOKENS; ++k) {
      const float z = warp_sum(acc[r][k]) * alpha;
      if (lane == 0) zs[k][warp * R + r] = z;
    }
  __syncthreads();
  // a warp a token
  const int rows = (int)min((int64_t)kRowsBlock, a.V - v0);
  for (int k = warp; k < n; k += kFewWarps) {
    const int32_t *idx = t.idx + (int64_t)k * a.K;
    if (!GRAD) {
      float most = -INFINITY, sum = 0.f;
      for (int r = lane; r < rows; r += 32) most = fmaxf(most, zs[k][r] * kLog2e);
      most = warp_max(most);
      const float zero = most == -INFINITY ? 0.f : most;
      for (int r = lane; r < rows; r += 32) sum += exp2f(fmaf(zs[k][r], kLog2e, -zero));
      sum = warp_sum(sum);
      if (lane == 0) part[blockIdx.x * a.n + k] = make_float2(most, sum);
      for (int i = lane; i < a.K; i += 32)
        if (idx[i] >= v0 && idx[i] - v0 < rows) picked[(int64_t)k * a.K + i] = zs[k][idx[i] - v0];
    } else {
      const float coef = t.coef[k], lse = a.lse_in[k];
      for (int r = lane; r < rows; r += 32) {
        float p = coef == 0.f ? 0.f : coef * expf(zs[k][r] - lse);
        for (int i = 0; i < a.K; ++i)
          if (idx[i] - v0 == r) p -= t.weight[(int64_t)k * a.K + i];
        P[k * ldp + v0 + r] = p;
      }
    }
  }
}

// dx's part of a range of the weight's rows, for 1024 columns: [range][token][column].
template <int TOKENS, bool WIDE>
__global__ void __launch_bounds__(kFewThreads) head_few_dx_kernel(HeadArgs a, const float *P, int64_t ldp, float *parts, int64_t rows_range) {
  constexpr int kRowsAt = 64;
  __shared__ alignas(16) float ps[kRowsAt][TOKENS];
  kernel_begin();
  next_may_start();
  const int64_t c0 = (int64_t)blockIdx.x * 4 * kFewThreads, begin = blockIdx.y * rows_range, end = min(a.V, begin + rows_range);
  const float *w = static_cast<const float *>(a.w);
  auto column = [&](int e) { return c0 + (WIDE ? 4 * (int)threadIdx.x + e : (int)threadIdx.x + kFewThreads * e); };
  float acc[TOKENS][4] = {};
  for (int64_t v0 = begin; v0 < end; v0 += kRowsAt) {
    for (int i = threadIdx.x; i < kRowsAt * TOKENS; i += kFewThreads) {
      const int r = i % kRowsAt, k = i / kRowsAt;
      ps[r][k] = k < a.n && v0 + r < end ? P[k * ldp + v0 + r] : 0.f;
    }
    __syncthreads();
    const int rows = (int)min((int64_t)kRowsAt, end - v0);
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
      const float *at = w + (v0 + r) * a.w_stride;
      float f[4] = {};
      if (WIDE) {
        if (column(0) < a.H) load_piece<4>(at + column(0), f);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (column(e) < a.H) f[e] = at[column(e)];
      }
#pragma unroll
      for (int k = 0; k < TOKENS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] = fmaf(ps[r][k], f[e], acc[k][e]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < TOKENS; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k < a.n && column(e) < a.H) parts[(blockIdx.y * a.n + k) * a.H + column(e)] = acc[k][e];
}
// The parts' sum, in their order.
__global__ void __launch_bounds__(256) head_few_dx_join_kernel(HeadArgs a, const float *parts, int ranges) {
  kernel_begin();
  next_may_start();
  const int64_t all = a.n * a.H;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float s = 0.f;
#pragma unroll 8
    for (int q = 0; q < ranges; ++q) s += parts[q * all + i];
    static_cast<float *>(a.dx)[i / a.H * a.dx_stride + i % a.H] = s;
  }
}

// dW: a block has 1024 columns of 64 rows.
template <int TOKENS, typename T, bool WIDE>
__global__ void __launch_bounds__(kFewThreads) head_few_dw_kernel(HeadArgs a, const float *live, const float *P, int64_t ldp) {
  constexpr int kRowsAt = 64;
  __shared__ alignas(16) float ps[kRowsAt][TOKENS];
  kernel_begin();
  next_may_start();
  const int64_t c0 = (int64_t)blockIdx.x * 4 * kFewThreads, v0 = (int64_t)blockIdx.y * kRowsAt;
  auto column = [&](int e) { return c0 + (WIDE ? 4 * (int)threadIdx.x + e : (int)threadIdx.x + kFewThreads * e); };
  float x[TOKENS][4] = {};
#pragma unroll
  for (int k = 0; k < TOKENS; ++k)
    if (k < a.n && live[k] != 0.f)  // (what other tokens hold meets nothing)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (column(e) < a.H) x[k][e] = static_cast<const float *>(a.x)[k * a.x_stride + column(e)];
  for (int i = threadIdx.x; i < kRowsAt * TOKENS; i += kFewThreads) {
    const int r = i % kRowsAt, k = i / kRowsAt;
    ps[r][k] = k < a.n && v0 + r < a.V ? P[k * ldp + v0 + r] : 0.f;
  }
  __syncthreads();
  const int rows = (int)min((int64_t)kRowsAt, a.V - v0);
#pragma unroll 4
  for (int r = 0; r < rows; ++r) {
    T *to = static_cast<T *>(a.dw) + (v0 + r) * a.dw_stride;
    float f[4] = {};
    if (a.accumulate) {
      if (WIDE) {
        if (column(0) < a.H) load_piece<4>(to + column(0), f);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (column(e) < a.H) f[e] = to_f(to[column(e)]);
      }
    }
    float s[4] = {};
#pragma unroll
    for (int k = 0; k < TOKENS; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = fmaf(ps[r][k], x[k][e], s[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] += s[e];
    if (WIDE) {
      if (column(0) < a.H) store_piece<4>(to + column(0), f);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (column(e) < a.H) to[column(e)] = from_f<T>(f[e]);
    }
  }
}

// -- host -------------------------------------------------------------------------------------------
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
int64_t padded(int64_t x) { return (x + 63) / 64 * 64; }

// Scratch memory, from its beginning on; without an address, its size.
struct Carver {
  char *base;
  size_t at = 0;
  template <typename T>
  T *take(int64_t count) {
    T *p = reinterpret_cast<T *>(base + at);
    at += up256((size_t)count * sizeof(T));
    return p;
  }
};

// A matrix that the TMA engine can read where it is: 16-byte rows at 16-byte addresses.
bool readable(const void *p, int64_t rows, int64_t cols, int64_t stride, int type) {
  return type != ECHO_F32 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || (stride % 8 == 0 && stride >= cols && stride < (int64_t)1 << 38));
}
// Whether the copy engine can write a result: rows of 16-byte pieces at 16-byte addresses; sums of 16-bit
// matrices are rounded once, so it does not add to those.  Other results go to fp32 scratch, and from there
// by a kernel of their own.
bool writable(const void *p, int64_t rows, int64_t cols, int64_t stride, int type, bool add) {
  const int size = type_bytes(type);
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || (stride * size % 16 == 0 && stride < (int64_t)1 << 37)) && !(add && type != ECHO_F32);
}
Operand in_place(const void *p, int64_t rows, int64_t cols, int64_t stride, int type) {
  return {p, rows, cols, rows <= 1 ? padded(cols) : stride, 0, 1, type == ECHO_BF16, {}};
}

// Memory of a piece of P at most; a vocabulary whose P is larger is taken in pieces.  Pieces that
// stay in L2 (129 MB) would save no time: the products are bound by the tensor cores, and each
// piece of dx is added up in memory.
constexpr int64_t kPieceBytes = (int64_t)512 << 20;

struct Layout {
  Targets targets;
  float2 *part;
  float *picked;
  int64_t chunks;
  float *amax_x, *amax_w;
  float4 *parts;
  Operand x, w;       // of the logits' product (w: of dx too)
  Operand x_dw;       // of dW
  bool pack_x, pack_w, pack_x_dw;
  int target_blocks;
  // P: planes of a piece
  int p_bf16, p_half;
  int64_t piece, ldp;
  uint16_t *P;
  float *few_p;       // few tokens: P in fp32
  float *dx_sum;      // fp32, where dx is added up over pieces (few tokens: its parts)
  float *dw_sum;      // fp32, of a piece, where dW cannot be written at once
  int64_t sum_ld;
  size_t bytes;
};

bool few_tokens(const HeadArgs &a) { return a.type == ECHO_F32 && a.n <= kFew; }
int few_count(int64_t n) { return n > 8 ? 16 : n > 4 ? 8 : n > 1 ? 4 : 1; }
// Rows of a block: as many as share an x, but four blocks an SM.
int few_block(const HeadArgs &a, int sms) {
  const int n = few_count(a.n), most = few_rows(n, true) * kFewWarps;
  return a.V >= (int64_t)4 * sms * most ? most : few_rows(n, false) * kFewWarps;
}
int64_t few_ranges(const HeadArgs &a, int sms) {  // of the weight's rows, for dx: as many as fill the SMs four times
  const int64_t tiles = (a.H + 4 * kFewThreads - 1) / (4 * kFewThreads);
  return std::clamp<int64_t>(4 * sms / tiles, 1, (a.V + 63) / 64);
}

Layout layout_of(const HeadArgs &a, int sms) {
  Layout l{};
  Carver c{static_cast<char *>(a.scratch)};
  const bool f32 = a.type == ECHO_F32;
  l.target_blocks = (int)std::min<int64_t>((a.n + kTargetWarps - 1) / kTargetWarps, 2 * sms);
  l.targets.idx = c.take<int32_t>(a.n * a.K);
  l.targets.weight = c.take<float>(a.n * a.K);
  if (few_tokens(a)) {
    if (!a.grad) {
      l.chunks = (a.V + few_block(a, sms) - 1) / few_block(a, sms);
      l.targets.entropy = c.take<float>(a.n);
      l.targets.mass = c.take<float>(a.n);
      l.part = c.take<float2>(l.chunks * a.n);
      l.picked = c.take<float>(a.n * a.K);
    } else {
      l.targets.coef = c.take<float>(a.n);
      l.targets.live = c.take<float>(a.n);
      l.targets.size_part = c.take<float>(l.target_blocks);
      l.ldp = padded(a.V);
      l.few_p = c.take<float>(a.n * l.ldp);
      if (a.dx) l.dx_sum = c.take<float>(few_ranges(a, sms) * a.n * a.H);
    }
    l.bytes = c.at;
    return l;
  }
  // (split tiles have two parts for each pair of blocks at most, and are no more than that)
  l.targets.n_arrived = sms * 16;
  l.targets.arrived = c.take<int32_t>(l.targets.n_arrived);
  l.parts = c.take<float4>((int64_t)sms / 2 * 2 * kTile * kTile / 4);
  l.amax_x = c.take<float>(a.grad ? kAmaxParts : f32 ? a.n : 0);  // (of blocks' parts, or of rows)
  l.amax_w = c.take<float>(a.grad ? kAmaxParts : f32 ? (a.V + kTile - 1) / kTile * kTile : 0);  // (or of rows, what takes them back)
  auto planes = [&](int64_t rows, int64_t cols, int count, bool bf16, Scale scale) {
    const int64_t ld = padded(cols);
    return Operand{c.take<uint16_t>(count * rows * ld), rows, cols, ld, rows * ld, count, bf16, scale};
  };
  l.pack_x = !readable(a.x, a.n, a.H, a.x_stride, a.type);
  l.pack_w = !readable(a.w, a.V, a.H, a.w_stride, a.type);
  const Scale none{}, sw = a.grad ? Scale{l.amax_w, kAmaxParts, nullptr} : none, sx = a.grad ? Scale{l.amax_x, kAmaxParts, nullptr} : Scale{nullptr, 0, l.amax_x};
  l.x = l.pack_x ? planes(a.n, a.H, f32 ? 2 : 1, a.type == ECHO_BF16, f32 ? sx : none) : in_place(a.x, a.n, a.H, a.x_stride, a.type);
  l.w = l.pack_w ? planes(a.V, a.H, f32 ? 2 : 1, a.type == ECHO_BF16, f32 ? sw : none) : in_place(a.w, a.V, a.H, a.w_stride, a.type);
  if (!a.grad) {
    l.chunks = (a.V + kHalf - 1) / kHalf;
    l.targets.entropy = c.take<float>(a.n);
    l.targets.mass = c.take<float>(a.n);
    l.part = c.take<float2>(l.chunks * a.n);
    l.picked = c.take<float>(a.n * a.K);
  } else {
    l.targets.coef = c.take<float>(a.n);
    l.targets.live = c.take<float>(a.n);
    l.targets.size_part = c.take<float>(l.target_blocks);
    const bool exact_dw = a.dw && a.dw_type == ECHO_F32;  // (whose P has 22 bits)
    l.p_bf16 = a.type == ECHO_BF16 && (a.dx || !exact_dw);
    l.p_half = f32 || exact_dw ? 2 : a.type == ECHO_F16 ? 1 : 0;
    // dW's x has zeros for tokens without gradients
    l.pack_x_dw = a.dw && !f32;
    if (l.pack_x_dw) {
      const bool as_half = a.type == ECHO_BF16 && exact_dw;
      l.x_dw = planes(a.n, a.H, 1, a.type == ECHO_BF16 && !as_half, as_half ? sx : none);
    } else {
      l.x_dw = l.x;
    }
    const bool dw_sum = a.dw && !writable(a.dw, a.V, a.H, a.dw_stride, a.dw_type, a.accumulate);
    l.sum_ld = padded(a.H);
    const int64_t row_bytes = std::max<int64_t>(1, a.n) * 2 * (l.p_bf16 + l.p_half) + (dw_sum ? 4 * l.sum_ld : 0);
    const int64_t columns = std::max<int64_t>(kTile, a.piece_bytes / row_bytes / kTile * kTile);
    const int64_t pieces = (a.V + columns - 1) / columns;  // of equal size
    l.piece = pieces <= 1 ? a.V : ((a.V + pieces - 1) / pieces + kTile - 1) / kTile * kTile;
    l.ldp = padded(l.piece);
    l.P = c.take<uint16_t>((l.p_bf16 + l.p_half) * a.n * l.ldp);
    if (a.dx && (l.piece < a.V || !writable(a.dx, a.n, a.H, a.dx_stride, a.type, false))) l.dx_sum = c.take<float>(a.n * l.sum_ld);
    if (dw_sum) l.dw_sum = c.take<float>(l.piece * l.sum_ld);
  }
  l.bytes = c.at;
  return l;
}

cudaError_t box_map(CUtensorMap *map, const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t plane, int planes, int box_rows, int box_cols,
                    CUtensorMapSwizzle swizzle, int size = 2, CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_UINT16) {
  if (!encoder()) return cudaErrorNotSupported;
  const cuuint64_t dims[4] = {(cuuint64_t)cols, (cuuint64_t)rows, 1, (cuuint64_t)planes};
  const cuuint64_t far = (cuuint64_t)(planes > 1 ? plane : ld) * size;  // (not used with one plane)
  const cuuint64_t strides[3] = {(cuuint64_t)ld * size, far, far};
  const cuuint32_t box[4] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return encoder()(map, type, 4, const_cast<void *>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}
// Stages of an operand: its rows (and 64 columns of the sum), or (mn) 64 rows of the sum and 64 columns
cudaError_t stage_map(CUtensorMap *map, const Operand &o, bool mn) {
  return box_map(map, o.p, o.rows, o.cols, o.ld, o.plane, o.planes, mn ? kBK : kHalf, kBK, CU_TENSOR_MAP_SWIZZLE_128B);
}

cudaError_t out_to(Job &j, CUtensorMap *map, void *out, int64_t stride, int type, bool add) {
  const int size = type_bytes(type);
  if (j.M <= 1) stride = (j.N + 7) / 8 * 8;
  j.type = type, j.add = add;
  return box_map(map, out, j.M, j.N, stride, 0, 1, 32, 128 / size, CU_TENSOR_MAP_SWIZZLE_128B, size,
                 type == ECHO_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16);
}

// Stages of 64 columns that are summed with truncation: the result is off by about n 2^-25 of its usual size
// for n additions, four a stage.  Taking a set out of tensor memory keeps the tensor core from it for 256
// clocks, half a stage.  So results of 16 bits take 16 stages, those of 32 bits eight (2048 tokens of 12288
// columns: logits 9.1e-7 off with 16, 4.2e-7 with eight; 290 us with four instead of 263 for 51200 rows).
// P for an fp32 dW takes five, as a logit's error is as large a part of it (3% more time).  Short sums, and up
// to 256 tokens, which do not wait for the tensor cores, take three: among few numbers one near zero, off by
// the usual, counts (48 tokens: 1.7e-5 with eight, 5e-6 in fp32).  fp32 matrices, whose stages are summed three
// times over, take three, or two (1003 tokens of 517: 2.5e-6 off with 16, 8.9e-7 with four).
enum { kResult16, kResult32, kExactP };
int set_of(bool f32_matrices, int result, int64_t stages, int64_t tokens) {
  const bool few = tokens <= kTile;
  if (f32_matrices) return few ? 2 : 3;
  return result == kResult16 ? 16 : few || (result == kResult32 && stages <= 12) ? 3 : result == kExactP ? 5 : 8;
}

// The first two sets of a tile, or of each of its parts, are longer: they are summed while the tile before
// is finished, or its parts are joined.  A sum of n stages is off by n as a rule, and so is a tile by the
// mean of its sets' lengths, weighted by them: as long as this leaves it at 11/8 of that of equal sets, and
// no set at more than 32 stages.  (Parts with the lead of a whole sum had means of up to 23 stages where 3 is
// usual, and left fp32 dx of 200 tokens x 256, 51200 rows, 3.1e-6 too small.)
int lead_of(int set, int64_t stages, int64_t parts) {
  return std::min(32, (int)(0.5 * set + std::sqrt(0.25 * set * set + 0.1875 * set * (double)(stages / parts))));
}

// D = A B^T; mn: the operand is held transposed
Job job_of(const Operand &a, bool a_mn, const Operand &b, bool b_mn, bool f32_matrices, int result, int64_t tokens) {
  Job j{};
  j.M = (int)(a_mn ? a.cols : a.rows);
  j.N = (int)(b_mn ? b.cols : b.rows);
  j.steps = (int)(((a_mn ? a.rows : a.cols) + kBK - 1) / kBK);
  for (int p = 0; p < a.planes; ++p)
    for (int q = 0; q < b.planes; ++q)
      if (p + q < 2) j.plane_a[j.pairs] = p, j.plane_b[j.pairs++] = q;
  const int64_t stages = (int64_t)j.steps * j.pairs;
  j.set = set_of(f32_matrices, result, stages, tokens), j.lead = j.lead_part = lead_of(j.set, stages, 1);
  j.instr = instruction(kTile, a_mn, b_mn, a.bf16);
  j.tiles_n = (j.N + kTile - 1) / kTile;
  j.tiles = (int64_t)((j.M + kTile - 1) / kTile) * j.tiles_n;
  j.scale_a = a.scale, j.scale_b = b.scale;
  return j;
}

struct Maps {
  CUtensorMap a[2], b[2], out[2];
};
// The schedule, by an estimate of the pair of blocks that takes longest.  In stages of 560 clocks (512
// of products at 256 columns): joining the parts of a tile takes about 3000 clocks and 3000 for each part.
// Nothing is split where that saves nothing.  Two products have no pool: the first one's operands are
// long, and are in L2 while its tiles are at the same place of their sums.
double joining(int64_t parts) { return (3000. + 3000. * parts) / 560; }
// A tile of few stages takes longer than they do: its results leave in the time of 10 stages in fp32, 6 in 16
// bits, of which only the next tile's lead is hidden (32 tokens, 51200 x 4096, dx and dW: 736 us in fp32 where
// the pairs that take tiles of dW early counted stages only, 368 so; bf16 551 and 200).
double tile_of(const Job &j) {
  const int stages = j.steps * j.pairs;
  return stages + std::max(0., (j.type == ECHO_F32 ? 10. : 6.) - std::min(j.lead, stages));
}
Schedule plan(const Job *j, int pairs) {
  Schedule s{};
  const int64_t tiles = j[0].tiles;
  s.whole = tiles, s.tiles1 = j[1].tiles, s.split = 1;
  s.steps0 = j[0].steps * j[0].pairs, s.steps1 = j[1].steps * j[1].pairs;
  const double tile1 = tile_of(j[1]);
  double least = 0;
  for (int64_t split = 1; split <= std::max<int64_t>(1, s.steps0 / 4) && (split == 1 || tiles * split <= 2 * pairs); ++split) {
    const int64_t n = tiles * split, extra = n % pairs;
    const double length = (double)((s.steps0 + split - 1) / split);
    const int early = extra && s.tiles1 ? (int)std::min<double>(length / tile1 + 0.5, (double)(s.tiles1 / (pairs - extra))) : 0;
    const int64_t late = s.tiles1 - (extra ? early * (pairs - extra) : 0);
    const int64_t most = (late + pairs - 1) / pairs;  // (of a pair; the first ones have it)
    const double clocks = std::max((double)(n / pairs + (extra > 0)) * length, (double)(n / pairs) * length + (double)early * tile1) + (double)most * tile1 +
                          (split > 1 ? joining(split) : 0);
    if (split == 1 || clocks < least) least = clocks, s.split = (int)split, s.early = early;
  }
  const int64_t rest = tiles % pairs, pool = rest * s.steps0;
  if (s.tiles1 || !rest) return s;
  const int pool_pairs = (int)std::clamp<int64_t>(pool / 4, 1, pairs);  // (each has a few stages at least)
  const double clocks = (double)(tiles / pairs * s.steps0) + (double)((pool + pool_pairs - 1) / pool_pairs) + joining(((int64_t)s.steps0 * pool_pairs + pool - 1) / pool + 1);
  if (clocks < least) s.whole = tiles - rest, s.split = 1, s.pool = pool, s.pool_pairs = pool_pairs;
  return s;
}
// The parts of a tile of the first product that has several, at most (Worker's).
int64_t most_parts(const Schedule &s) {
  int64_t most = s.split;
  for (int64_t base = 0; base < s.pool; base += s.steps0)
    most = std::max(most, ((base + s.steps0) * s.pool_pairs - 1) / s.pool - ((base + 1) * s.pool_pairs - 1) / s.pool + 1);
  return most;
}
template <int MODE>
cudaError_t launch_product(const Maps &m, HeadProduct &g, int sms, cudaStream_t st) {
  auto kernel = head_product_kernel<MODE>;
  const int pairs = sms / 2;
  g.schedule = plan(g.job, pairs);
  g.job[0].lead_part = lead_of(g.job[0].set, g.schedule.steps0, most_parts(g.schedule));
  const int64_t busy = std::max<int64_t>(g.schedule.pool_pairs, g.schedule.whole * g.schedule.split + g.schedule.tiles1);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (e != cudaSuccess) return e;
  return launch_early(kernel, dim3((unsigned)std::min<int64_t>(busy, pairs) * 2), kThreads, kSmem, st, m.a[0], m.b[0], m.a[1], m.b[1], m.out[0], m.out[1], g);
}

#define TRY(call)                                \
  do {                                           \
    const cudaError_t _e = (call);               \
    if (_e != cudaSuccess) return _e;            \
  } while (0)

Source source(const void *p, int type, int64_t rows, int64_t cols, int64_t stride) {
  Source m{};
  m.p = p, m.rows = rows, m.cols = cols, m.stride = rows == 1 ? cols : stride;
  return m;
}
// The largest elements of `count` matrices.
cudaError_t launch_amax(Sources s, int count, int type, cudaStream_t st) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    constexpr int N = 16 / sizeof(T);
    bool wide = true;
    for (int i = 0; i < count; ++i) {
      Source &m = s.of[i];
      if (m.stride == m.cols && !m.live) m.cols *= m.rows, m.rows = 1;
      wide &= m.rows == 1 || (m.cols % N == 0 && fits_pieces(m.p, m.stride, type, N));
    }
    return wide ? launch_early(head_amax_kernel<T, N>, dim3(kAmaxParts, count), 256, 0, st, s) : launch_early(head_amax_kernel<T, 1>, dim3(kAmaxParts, count), 256, 0, st, s);
  });
}
// `count` matrices of a type as planes, of bf16 numbers or fp16 ones.
cudaError_t launch_pack(const Sources &s, int count, int type, bool bf16, int sms, cudaStream_t st) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    bool wide = true;
    int64_t most = 1;
    for (int i = 0; i < count; ++i) {
      wide &= s.of[i].cols % 8 == 0 && fits_pieces(s.of[i].p, s.of[i].stride, type, 8);
      most = std::max(most, s.of[i].rows * ((s.of[i].cols + 7) / 8 * 8));
    }
    auto go = [&](auto d, auto planes) {
      auto with = [&](auto w) {
        const dim3 grid((unsigned)std::min<int64_t>((most / 8 + 511) / 512, sms * 8), count);
        return launch_early(head_pack_kernel<T, decltype(d), decltype(planes)::value, decltype(w)::value>, grid, 256, 0, st, s);
      };
      return wide ? with(Int<1>{}) : with(Int<0>{});
    };
    if constexpr (std::is_same_v<T, float>) return go(__half{}, Int<2>{});
    else if constexpr (std::is_same_v<T, __half>) return go(__half{}, Int<1>{});
    else return bf16 ? go(__nv_bfloat16{}, Int<1>{}) : go(__half{}, Int<1>{});
  });
}

// Matrices of rows with a scale each; a lane holds two pieces of 8 columns at least where it can.
cudaError_t launch_pack_rows(const Sources &s, int count, bool wide, int64_t cols, int64_t rows, int sms, cudaStream_t st) {
  auto go = [&](auto kernel, int64_t rows_block) {
    const dim3 grid((unsigned)std::min<int64_t>((rows + rows_block - 1) / rows_block, 8 * sms), count);
    return launch_early(kernel, grid, 256, 0, st, s);
  };
  if (cols <= 1024) return wide ? go(head_pack_rows_kernel<true, 1, 4>, 8) : go(head_pack_rows_kernel<false, 1, 1>, 8);
  if (!wide) return go(head_pack_rows_kernel<false, 8, 1>, 1);
  return cols <= 4096 ? go(head_pack_rows_kernel<true, 8, 2>, 1) : go(head_pack_rows_kernel<true, 8, 6>, 1);
}

cudaError_t launch_round(const float *from, int64_t ld, int64_t rows, int64_t cols, void *to, int64_t stride, int type, bool add, int sms, cudaStream_t st) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      const int64_t blocks = std::min<int64_t>((rows * (cols / W) + 1023) / 1024, sms * 8);
      return launch_early(head_round_kernel<T, W>, dim3((unsigned)blocks), 256, 0, st, from, ld, rows, cols, static_cast<T *>(to), stride, (int)add);
    };
    constexpr int N = 16 / sizeof(T);
    if (cols % N == 0 && fits_pieces(to, stride, type, N)) return go(Int<N>{});
    return cols % 2 == 0 && fits_pieces(to, stride, type, 2) ? go(Int<2>{}) : go(Int<1>{});
  });
}

// f(Int<the number of tokens that the kernels for few of them are made for>, Int<whether rows are 16-byte ones>)
template <typename F>
cudaError_t with_few(int64_t n, bool wide, F &&f) {
  auto with = [&](auto w) {
    switch (few_count(n)) {
      case 1: return f(Int<1>{}, w);
      case 4: return f(Int<4>{}, w);
      case 8: return f(Int<8>{}, w);
      default: return f(Int<16>{}, w);
    }
  };
  return wide ? with(Int<1>{}) : with(Int<0>{});
}
cudaError_t launch_few_dw(const HeadArgs &a, const Layout &l, const OpTimer &timed, cudaStream_t st) {
  const bool wide = a.H % 4 == 0 && fits_pieces(a.dw, a.dw_stride, a.dw_type, 4);
  const dim3 grid((unsigned)((a.H + 4 * kFewThreads - 1) / (4 * kFewThreads)), (unsigned)((a.V + 63) / 64));
  return timed("head_few_dw", [&] {
    return with_type(a.dw_type, [&](auto t) {
      return with_few(a.n, wide, [&](auto tokens, auto w) {
        return launch_early(head_few_dw_kernel<decltype(tokens)::value, decltype(t), decltype(w)::value>, grid, kFewThreads, 0, st, a,
                            (const float *)l.targets.live, (const float *)l.few_p, l.ldp);
      });
    });
  });
}
cudaError_t launch_few(const HeadArgs &a, const Layout &l, int sms, const OpTimer &timed, cudaStream_t st) {
  const bool wide = a.H % 4 == 0 && fits_pieces(a.w, a.w_stride, a.type, 4);
  const unsigned tiles = (unsigned)((a.H + 4 * kFewThreads - 1) / (4 * kFewThreads));
  if (a.V)
    TRY(timed("head_few", [&] {
      return with_few(a.n, wide, [&](auto tokens, auto w) {
        constexpr int N = decltype(tokens)::value;
        constexpr bool W = decltype(w)::value;
        const int block = few_block(a, sms);
        const dim3 grid((unsigned)((a.V + block - 1) / block));
        auto go = [&](auto rows) {
          constexpr int R = decltype(rows)::value;
          if (a.grad) return launch_early(head_few_kernel<N, R, W, true>, grid, kFewThreads, 0, st, a, l.targets, l.part, l.picked, l.few_p, l.ldp);
          return launch_early(head_few_kernel<N, R, W, false>, grid, kFewThreads, 0, st, a, l.targets, l.part, l.picked, l.few_p, l.ldp);
        };
        return block == few_rows(N, true) * kFewWarps ? go(Int<few_rows(N, true)>{}) : go(Int<few_rows(N, false)>{});
      });
    }));
  if (a.dx) {
    const int64_t ranges = few_ranges(a, sms), rows = (a.V + ranges - 1) / ranges;
    TRY(timed("head_few_dx", [&] {
      return with_few(a.n, wide, [&](auto tokens, auto w) {
        return launch_early(head_few_dx_kernel<decltype(tokens)::value, decltype(w)::value>, dim3(tiles, (unsigned)ranges), kFewThreads, 0, st, a,
                            (const float *)l.few_p, l.ldp, l.dx_sum, rows);
      });
    }));
    TRY(timed("head_few_dx", [&] {
      return launch_early(head_few_dx_join_kernel, dim3((unsigned)std::min<int64_t>((a.n * a.H + 255) / 256, 8 * sms)), 256, 0, st, a, (const float *)l.dx_sum,
                          (int)ranges);
    }));
  }
  constexpr int64_t kMost = 65535 * 64;  // rows of a launch (a grid's second dimension)
  for (int64_t v = 0; a.dw && v < a.V; v += kMost) {
    HeadArgs b = a;
    Layout m = l;
    b.V = std::min(kMost, a.V - v);
    b.dw = static_cast<char *>(a.dw) + v * a.dw_stride * type_bytes(a.dw_type);
    m.few_p = l.few_p + v;
    TRY(launch_few_dw(b, m, timed, st));
  }
  return cudaSuccess;
}

}  // namespace

int64_t head_piece_bytes() { return kPieceBytes; }
int head_most_targets() { return kMaxTargets; }
size_t head_scratch_bytes(const HeadArgs &a, int sms) { return layout_of(a, sms).bytes; }

cudaError_t launch_head(const HeadArgs &a, int sms, const OpTimer &timed, cudaStream_t st) {
  const Layout l = layout_of(a, sms);
  const bool f32 = a.type == ECHO_F32;
  TRY(timed("head_targets", [&] { return launch_early(head_targets_kernel, dim3(l.target_blocks), kTargetWarps * 32, 0, st, a, l.targets); }));
  auto join = [&] {
    return timed("head_join", [&] {
      return launch_early(head_join_kernel, dim3((unsigned)std::min<int64_t>((a.n + 31) / 32, 2 * sms)), kJoinWarps * 32, 0, st, a, l.targets, l.part, l.chunks,
                          l.picked);
    });
  };
  if (few_tokens(a)) {
    const cudaError_t e = launch_few(a, l, sms, timed, st);
    return e != cudaSuccess || a.grad ? e : join();
  }
  const bool exact_dw = a.grad && a.dw && a.dw_type == ECHO_F32;
  HeadProduct g{};
  const Source sx = source(a.x, a.type, a.n, a.H, a.x_stride), sw = source(a.w, a.type, a.V, a.H, a.w_stride);
  const bool sized_x = a.grad && (f32 || (l.pack_x_dw && exact_dw && a.type == ECHO_BF16)), sized_w = a.grad && f32;
  Sources s{};
  int count = 0;
  // (rows that are not live do not count: padding may hold any number)
  if (sized_x) s.of[count] = sx, s.of[count].live = l.targets.live, s.of[count++].amax = l.amax_x;
  if (sized_w) s.of[count] = sw, s.of[count++].amax = l.amax_w;
  if (count) TRY(timed("head_amax", [&] { return launch_amax(s, count, a.type, st); }));
  // (backward, the rows of tokens without gradients are zeros in fp32's planes, which both products read)
  auto pack = [&](const Source &m, const Operand &o, const float *live) {
    Source &t = s.of[count++] = m;
    t.scale = o.scale, t.live = live, t.to = const_cast<void *>(o.p), t.ld = o.ld, t.plane = o.plane;
  };
  count = 0;
  if (l.pack_x) pack(sx, l.x, a.grad && f32 ? l.targets.live : nullptr);
  if (l.pack_w && a.V) pack(sw, l.w, nullptr);
  if (count && f32 && !a.grad) {  // (each row has its own scale)
    s.of[0].amax = l.amax_x, s.of[1].amax = l.amax_w, s.of[1].down = true;
    const bool wide = a.H % 8 == 0 && fits_pieces(a.x, s.of[0].stride, a.type, 8) && fits_pieces(a.w, s.of[1].stride, a.type, 8);
    TRY(timed("head_pack", [&] { return launch_pack_rows(s, count, wide, a.H, std::max(a.n, a.V), sms, st); }));
    g.w_down = l.amax_w;
  } else if (count) {
    TRY(timed("head_pack", [&] { return launch_pack(s, count, a.type, l.x.bf16, sms, st); }));
  }
  // (a launch of its own: done by warps of the product that have nothing else to do, it held up the others
  // by more, 60 us instead of 22 for 2048 x 12288 in bf16)
  count = 0;
  if (l.pack_x_dw) pack(sx, l.x_dw, l.targets.live);
  if (count) TRY(timed("head_pack", [&] { return launch_pack(s, count, a.type, l.x_dw.bf16, sms, st); }));
  g.wait = {a.status, a.wait_limit}, g.skip = a.skip;
  g.parts = l.parts, g.arrived = l.targets.arrived;
  g.n = a.n, g.K = a.K, g.alpha = a.scale / a.tau;
  g.idx = l.targets.idx, g.weight = l.targets.weight, g.coef = l.targets.coef, g.lse = a.lse_in;
  Maps m{};
  if (!a.grad) {
    g.part = l.part, g.picked = l.picked;
    if (a.V) {
      g.job[0] = job_of(l.x, false, l.w, false, f32, kResult32, a.n);
      TRY(stage_map(&m.a[0], l.x, false));
      TRY(stage_map(&m.b[0], l.w, false));
      TRY(timed("head_logits", [&] { return launch_product<kStats>(m, g, sms, st); }));
    }
    return join();
  }

  g.p_bf16 = l.p_bf16, g.p_half = l.p_half, g.p_scale = {l.targets.size_part, l.target_blocks, nullptr};
  auto piece_of_dw = [&](int64_t v) -> void * { return static_cast<char *>(a.dw) + v * a.dw_stride * type_bytes(a.dw_type); };
  for (int64_t v = 0; v < a.V; v += l.piece) {
    const int64_t rows = std::min(l.piece, a.V - v);
    Operand w = l.w;
    w.p = static_cast<const uint16_t *>(w.p) + v * w.ld;
    w.rows = rows;
    // the planes of P that dx and dW read
    const int64_t plane = a.n * l.ldp;
    const Operand p{l.P, a.n, rows, l.ldp, plane, l.p_bf16 + l.p_half, false, {}};
    auto planes = [&](bool bf16, int count) {
      Operand o = p;
      o.bf16 = bf16, o.planes = count, o.scale = g.p_scale;
      if (!bf16) o.p = l.P + l.p_bf16 * plane;
      return o;
    };
    HeadProduct h = g;
    h.v_begin = (int)v;
    h.job[0] = job_of(l.x, false, w, false, f32, exact_dw ? kExactP : kResult16, a.n);
    TRY(stage_map(&m.a[0], l.x, false));
    TRY(stage_map(&m.b[0], w, false));
    TRY(box_map(&m.out[0], l.P, a.n, rows, l.ldp, plane, p.planes, 32, 64, CU_TENSOR_MAP_SWIZZLE_128B));
    TRY(timed("head_dlogits", [&] { return launch_product<kGrad>(m, h, sms, st); }));

    HeadProduct d = g;
    if (a.dx) {
      const Operand q = planes(a.type == ECHO_BF16, f32 ? 2 : 1);
      Job &j = d.job[0] = job_of(q, false, w, true, f32, kResult16, a.n);
      TRY(stage_map(&m.a[0], q, false));
      TRY(stage_map(&m.b[0], w, true));
      if (l.dx_sum) TRY(out_to(j, &m.out[0], l.dx_sum, l.sum_ld, ECHO_F32, v > 0));
      else TRY(out_to(j, &m.out[0], a.dx, a.dx_stride, a.type, false));
    }
    if (a.dw) {
      const Operand q = planes(l.x_dw.bf16, f32 || exact_dw ? 2 : 1);
      Job &j = d.job[1] = job_of(q, true, l.x_dw, true, f32, exact_dw ? kResult32 : kResult16, a.n);
      TRY(stage_map(&m.a[1], q, true));
      TRY(stage_map(&m.b[1], l.x_dw, true));
      if (l.dw_sum) TRY(out_to(j, &m.out[1], l.dw_sum, l.sum_ld, ECHO_F32, false));
      else TRY(out_to(j, &m.out[1], piece_of_dw(v), a.dw_stride, a.dw_type, a.accumulate));
    }
    TRY(timed("head_grads", [&] { return launch_product<kOut>(m, d, sms, st); }));
    if (l.dw_sum) TRY(timed("head_round", [&] { return launch_round(l.dw_sum, l.sum_ld, rows, a.H, piece_of_dw(v), a.dw_stride, a.dw_type, a.accumulate, sms, st); }));
  }
  if (!l.dx_sum) return cudaSuccess;
  return timed("head_round", [&] { return launch_round(l.dx_sum, l.sum_ld, a.n, a.H, a.dx, a.dx_stride, a.type, false, sms, st); });
}

}  // namespace echo
