// echo_ops_rotary.cu -- rotary positions of queries and keys, and their gradient.
//
// A pair (a, b) of a head's first `rot` elements becomes scale (a cos - b sin, a sin + b cos) by
// the angle position * frequency of the pair; the gradient is the turn back.  Pairs are
// neighbours, or an element and the one half of `rot` further on.
//
// An angle matters modulo a turn.  Frequencies are held as fractions of a turn times 2^64, so
// the low 64 bits of position * frequency are the angle, for every position, without the digits
// that 32 bits lose far into a context and without 64-bit floating point.
#include <algorithm>
#include <cmath>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace {

constexpr int kThreads = 256, kItems = 4;        // items of a thread in flight
constexpr int kBlocks = 4;                       // of an SM
constexpr int kAngles = 1024, kTokens = 128;     // angles and tokens of a block, at most
static_assert(kRotaryPairs <= kAngles, "a token's angles fit");

struct RotaryPlan {
  int per_head, turned;       // items of a head: two pieces of W elements each; those that are turned
  int heads_block;            // heads of a block (grid.y: groups of them)
  int tokens_block;
  uint32_t by_head, by_token; // ceil(2^32 / divisor)
};

// n / d for n * d < 2^32
__device__ __forceinline__ uint32_t divide(uint32_t n, uint32_t by) { return by ? __umulhi(n, by) : n; }

// A block takes some tokens and heads: their angles once, to shared memory, while the first items
// are on their way.  Bound by the bytes.
template <typename T, int W, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, kBlocks) rotary_kernel(const __grid_constant__ RotaryArgs a, const RotaryPlan p) {
  // cos and sin of pair W j + e, so that neighbouring j are side by side: two e of every j, the next two, ...
  __shared__ alignas(16) float2 angles[kAngles];
  __shared__ int64_t in_at[2][kTokens], out_at[2][kTokens];
  kernel_begin();
  next_may_start();
  const int half = a.rot / 2;
  const uint32_t all = (uint32_t)(a.batch * a.tokens), per_batch = (uint32_t)a.tokens, t0 = blockIdx.x * p.tokens_block;  // (below 2^31)
  const int tokens = (int)min((uint32_t)p.tokens_block, all - t0);
  const int head0 = blockIdx.y * p.heads_block, heads = min(p.heads_block, (int)(a.heads[0] + a.heads[1]) - head0);
  for (int i = threadIdx.x; i < tokens; i += kThreads) {
    const uint32_t b = (t0 + i) / per_batch, t = (t0 + i) - b * per_batch;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      in_at[k][i] = b * a.x_batch[k] + t * a.x_token[k];
      out_at[k][i] = b * a.out_batch[k] + t * a.out_token[k];
    }
  }
  auto position_of = [&](int token) -> int64_t {
    const uint32_t t = t0 + token, b = t / per_batch;
    const int64_t at = b * a.positions_batch + (t - b * per_batch);
    return a.id64 ? static_cast<const int64_t *>(a.positions)[at] : static_cast<const int32_t *>(a.positions)[at];
  };
  int64_t position0 = 0;  // of this thread's first angle: on its way with the items
  if ((int)threadIdx.x < tokens * half) position0 = position_of(threadIdx.x / half);
  __syncthreads();
  const uint32_t per_token = (uint32_t)(heads * p.per_head), items = tokens * per_token;
  const int apart = INTERLEAVED ? W : half;  // the second piece of an item that is turned, from the first
  struct Item {
    Pack<T, W> v[2];
    T *to;
    int pair;  // place of the first pair's angle; or:
  };
  constexpr int kCopied = -1, kCopiedFirst = -2, kNothing = -3;  // both pieces as they are, the first one alone, no item
  auto load = [&](uint32_t i, Item &m) {
    m.pair = kNothing;
    if (i >= items) return;
    uint32_t token = 0;
    if (p.tokens_block > 1) token = heads == p.heads_block ? divide(i, p.by_token) : i / per_token;
    const uint32_t in_token = i - token * per_token, h = divide(in_token, p.by_head), j = in_token - h * p.per_head;
    const int head = head0 + (int)h, k = head >= a.heads[0];
    const int64_t hh = head - (k ? a.heads[0] : 0);
    int first, second = apart;
    if ((int)j < p.turned) {
      first = INTERLEAVED ? 2 * W * (int)j : W * (int)j;
      m.pair = (int)token * half + (W > 1 ? 2 : 1) * (int)j;
    } else {
      first = a.rot + 2 * W * ((int)j - p.turned);
      second = W;
      m.pair = first + W < a.dim ? kCopied : kCopiedFirst;
    }
    const T *from = static_cast<const T *>(a.x[k]) + in_at[k][token] + hh * a.x_head[k] + first;
    m.to = static_cast<T *>(a.out[k]) + out_at[k][token] + hh * a.out_head[k] + first;
    m.v[0] = *reinterpret_cast<const Pack<T, W> *>(from);
    if (m.pair != kCopiedFirst) m.v[1] = *reinterpret_cast<const Pack<T, W> *>(from + second);
  };
  auto finish = [&](const Item &m) {
    if (m.pair == kNothing) return;
    if (m.pair < 0) {
      *reinterpret_cast<Pack<T, W> *>(m.to) = m.v[0];
      if (m.pair == kCopied) *reinterpret_cast<Pack<T, W> *>(m.to + W) = m.v[1];
      return;
    }
    float v[2][W];
    unpack<T, W>(m.v[0], v[0]);
    unpack<T, W>(m.v[1], v[1]);
    float2 angle[W];
    if constexpr (W == 1) {
      angle[0] = angles[m.pair];
    } else {
#pragma unroll
      for (int e = 0; e < W; e += 2) {
        const float4 two = *reinterpret_cast<const float4 *>(angles + m.pair + e * p.turned);
        angle[e] = make_float2(two.x, two.y), angle[e + 1] = make_float2(two.z, two.w);
      }
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const float2 c = angle[e];
      // interleaved: elements 2e and 2e + 1 of the two pieces
      float &x = INTERLEAVED ? v[2 * e / W][2 * e % W] : v[0][e], &y = INTERLEAVED ? v[(2 * e + 1) / W][(2 * e + 1) % W] : v[1][e];
      const float x0 = x;
      x = fmaf(x0, c.x, -__fmul_rn(y, c.y));  // (one order of roundings for every layout)
      y = fmaf(x0, c.y, __fmul_rn(y, c.x));
    }
    store_piece<W>(m.to, v[0]);
    store_piece<W>(m.to + apart, v[1]);
  };
  Item m[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) load(threadIdx.x + k * kThreads, m[k]);
  for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
    const int token = i / half, pair = i - token * half;
    const int64_t position = i == (int)threadIdx.x ? position0 : position_of(token);
    const int64_t turn = (int64_t)((uint64_t)position * a.turns[pair]);  // of a turn, times 2^64: -1/2 to 1/2
    float s, c;
    sincospif(__ll2float_rn(turn) * 0x1p-63f, &s, &c);
    const int at = W == 1 ? pair : (pair % W / 2 * p.turned + pair / W) * 2 + pair % 2;
    angles[token * half + at] = make_float2(c * a.scale, (a.back ? -s : s) * a.scale);
  }
  __syncthreads();
  for (uint32_t i0 = threadIdx.x;;) {
#pragma unroll
    for (int k = 0; k < kItems; ++k) finish(m[k]);
    i0 += kThreads * kItems;
    if (i0 - threadIdx.x >= items) break;
#pragma unroll
    for (int k = 0; k < kItems; ++k) load(i0 + k * kThreads, m[k]);
  }
}

}  // namespace

// A frequency in radians as the fraction of a turn, times 2^64; with 1 / (2 pi) in two doubles, so
// that far positions find all of its bits.
uint64_t rotary_turns(double f) {
  const double high = 0x1.45f306dc9c883p-3, low = -0x1.6b01ec5417056p-57;
  if (f < 0) return -rotary_turns(-f);
  const double p = f * high, rest = std::fma(f, high, -p) + f * low;
  return (uint64_t)((p - std::floor(p)) * 0x1p64) + (uint64_t)std::llrint(rest * 0x1p64);  // (the difference is exact)
}

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t st) {
  return with_type(a.type, [&](auto t) {
    using T = decltype(t);
    auto fits = [&](int W) {
      bool ok = a.rot / 2 % W == 0 && (a.dim - a.rot) % W == 0;
      for (int k = 0; k < 2; ++k)
        if (a.heads[k])
          ok &= fits_pieces(a.x[k], a.x_head[k], a.type, W) && fits_pieces(a.x[k], a.x_token[k], a.type, W) && fits_pieces(a.x[k], a.x_batch[k], a.type, W) &&
                fits_pieces(a.out[k], a.out_head[k], a.type, W) && fits_pieces(a.out[k], a.out_token[k], a.type, W) &&
                fits_pieces(a.out[k], a.out_batch[k], a.type, W);
      return ok;
    };
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      RotaryPlan p{};
      p.turned = a.rot / 2 / W;
      p.per_head = p.turned + (a.dim - a.rot + 2 * W - 1) / (2 * W);
      const int heads = (int)(a.heads[0] + a.heads[1]);
      p.heads_block = std::min(heads, std::max(1, 2048 / p.per_head));
      const int per_token = p.heads_block * p.per_head;
      p.tokens_block = std::max(1, std::min({kThreads * kItems / per_token, kAngles / (a.rot / 2), kTokens}));
      p.by_head = (uint32_t)((((uint64_t)1 << 32) + p.per_head - 1) / p.per_head);
      p.by_token = (uint32_t)((((uint64_t)1 << 32) + per_token - 1) / per_token);
      const dim3 grid((unsigned)((a.batch * a.tokens + p.tokens_block - 1) / p.tokens_block), (unsigned)((heads + p.heads_block - 1) / p.heads_block));
      if (a.interleaved) return launch_early(rotary_kernel<T, W, true>, grid, kThreads, 0, st, a, p);
      return launch_early(rotary_kernel<T, W, false>, grid, kThreads, 0, st, a, p);
    };
    constexpr int N = 16 / sizeof(T);
    return fits(N) ? go(Int<N>{}) : fits(2) ? go(Int<2>{}) : go(Int<1>{});
  });
}

}  // namespace echo
