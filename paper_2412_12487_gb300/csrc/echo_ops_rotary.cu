// echo_ops_rotary.cu -- rotary positions of queries and keys, and their gradient.
//
// A pair (a, b) of a head's first `rot` elements becomes scale (a cos - b sin, a sin + b cos) by
// the angle position * frequency of the pair; the gradient is the turn back.  Pairs are
// neighbours, or an element and the one half of `rot` further on.
//
// An angle matters modulo a turn.  Frequencies are held as fractions of a turn times 2^64, rounded,
// so the low 64 bits of position * frequency are the angle, without the digits that 32 bits lose far
// into a context and without 64-bit floating point.  The half unit that a frequency is off by grows
// with the position: pi 2^-64 |position| radians, fp32's last bits from 2^38 on (1.9e-7 at 2^40).
#include <algorithm>
#include <cmath>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace {

constexpr int kWarps = 4;  // of a block

// An item is two pieces of W elements of a head that are turned together, or copied.  A lane takes the
// same item j of several heads: a warp has `columns` items of `slots` heads at a time.
struct RotaryPlan {
  int items, turned;   // of a head: all, those that are turned
  int columns, slots;
  int column_parts;    // warps for the items of a head
  int head_parts;      // warps for the heads of a token
};

// A warp takes a token and some of its heads.  Its lanes share the work on the angles: the lanes with
// the same item compute some of its pairs each and pass them on.  Nothing waits for another warp (with a
// block's angles in shared memory, and barriers, it took 276 us).  Bound by the bytes where there are many
// tokens: 65536 tokens of 40 heads of 128 in bf16, 1.3e9 bytes, 213 us, 6.3 TB/s; by latency where there
// are few: 2048 tokens of 24 heads, 2.5e7 bytes, 6.9 us.
template <typename T, int W, bool INTERLEAVED>
__global__ void __launch_bounds__(kWarps * 32) rotary_kernel(const __grid_constant__ RotaryArgs a, const RotaryPlan p) {
  kernel_begin();
  next_may_start();
  const int lane = threadIdx.x & 31, half = a.rot / 2;
  const uint32_t tokens = (uint32_t)(a.batch * a.tokens), per_token = p.head_parts * p.column_parts;  // (tokens below 2^31)
  const uint32_t warp = blockIdx.x * kWarps + (threadIdx.x >> 5), n = warp / per_token, in_token = warp - n * per_token;
  if (n >= tokens) return;
  const int head_part = in_token / p.column_parts, column_part = in_token - head_part * p.column_parts;
  const uint32_t b = n / (uint32_t)a.tokens, t = n - b * (uint32_t)a.tokens;
  const int slot = lane / p.columns, j = column_part * p.columns + lane - slot * p.columns;
  const bool mine = slot < p.slots && j < p.items, turned = j < p.turned;
  const int64_t at = b * a.positions_batch + t;
  const int64_t position = a.id64 ? static_cast<const int64_t *>(a.positions)[at] : static_cast<const int32_t *>(a.positions)[at];
  const int first = !turned ? a.rot + 2 * W * (j - p.turned) : INTERLEAVED ? 2 * W * j : W * j;
  const int second = first + (!turned || INTERLEAVED ? W : half);
  const bool both = second < a.dim;  // (or the first piece alone, which is copied)

  const int all = (int)(a.heads[0] + a.heads[1]), heads0 = (int)a.heads[0];
  const int head_end = (int)((int64_t)all * (head_part + 1) / p.head_parts);
  int head = (int)((int64_t)all * head_part / p.head_parts) + slot;
  const T *from[2];
  T *to[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    from[k] = static_cast<const T *>(a.x[k]) + b * a.x_batch[k] + t * a.x_token[k] + first;
    to[k] = static_cast<T *>(a.out[k]) + b * a.out_batch[k] + t * a.out_token[k] + first;
  }
  Pack<T, W> v[2];  // (one item ahead: two or four leave fewer warps, 224 and 265 us instead of 213)
  auto load = [&](int h, Pack<T, W> (&x)[2]) {
    if (!mine || h >= head_end) return;
    const T *f = h < heads0 ? from[0] + h * a.x_head[0] : from[1] + (h - heads0) * a.x_head[1];
    x[0] = *reinterpret_cast<const Pack<T, W> *>(f);
    if (both) x[1] = *reinterpret_cast<const Pack<T, W> *>(f + (second - first));
  };
  load(head, v);

  // cos and sin of the item's pairs: this lane computes those whose number is `slot` modulo `slots`
  float2 angle[W];
  for (int e0 = 0; e0 < W; e0 += p.slots) {
    const int pair = W * j + e0 + slot;
    float2 c = make_float2(1.f, 0.f);
    if (turned && slot < p.slots && e0 + slot < W) {
      const int64_t turn = (int64_t)((uint64_t)position * a.turns[pair]);  // of a turn, times 2^64: -1/2 to 1/2
      float sine, cosine;
      sincospif(__ll2float_rn(turn) * 0x1p-63f, &sine, &cosine);
      c = make_float2(cosine * a.scale, (a.back ? -sine : sine) * a.scale);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const int owner = e - e0;  // (slot that has it)
      const int source = (owner >= 0 && owner < p.slots ? owner : 0) * p.columns + lane - slot * p.columns;
      const float x = __shfl_sync(0xFFFFFFFFu, c.x, source), y = __shfl_sync(0xFFFFFFFFu, c.y, source);
      if (owner >= 0 && owner < p.slots) angle[e] = make_float2(x, y);
    }
  }

  auto finish = [&](int h, const Pack<T, W> (&x)[2]) {
    if (!mine || h >= head_end) return;
    T *o = h < heads0 ? to[0] + h * a.out_head[0] : to[1] + (h - heads0) * a.out_head[1];
    if (!turned) {
      *reinterpret_cast<Pack<T, W> *>(o) = x[0];
      if (both) *reinterpret_cast<Pack<T, W> *>(o + (second - first)) = x[1];
      return;
    }
    float f[2][W];
    unpack<T, W>(x[0], f[0]);
    unpack<T, W>(x[1], f[1]);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const float2 c = angle[e];
      // interleaved: elements 2e and 2e + 1 of the two pieces
      float &x0 = INTERLEAVED ? f[2 * e / W][2 * e % W] : f[0][e], &x1 = INTERLEAVED ? f[(2 * e + 1) / W][(2 * e + 1) % W] : f[1][e];
      const float old = x0;
      x0 = fmaf(old, c.x, -__fmul_rn(x1, c.y));  // (one order of roundings for every layout)
      x1 = fmaf(old, c.y, __fmul_rn(x1, c.x));
    }
    store_piece<W>(o, f[0]);
    store_piece<W>(o + (second - first), f[1]);
  };
  for (; head - slot < head_end; head += p.slots) {
    finish(head, v);
    load(head + p.slots, v);
  }
}

}  // namespace

// A frequency in radians as the fraction of a turn, times 2^64, rounded; with 1 / (2 pi) in two doubles, so
// that far positions find all of its bits.
uint64_t rotary_turns(double f) {
  const double high = 0x1.45f306dc9c883p-3, low = -0x1.6b01ec5417056p-57;
  if (f < 0) return -rotary_turns(-f);
  const double p = f * high, rest = std::fma(f, high, -p) + f * low;
  const double at = (p - std::floor(p)) * 0x1p64, whole = std::floor(at);  // (exact, as is their difference)
  return (uint64_t)whole + (uint64_t)std::llrint(rest * 0x1p64 + (at - whole));
}

cudaError_t launch_rotary(const RotaryArgs &a, int sms, cudaStream_t st) {
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
      p.items = p.turned + (a.dim - a.rot + 2 * W - 1) / (2 * W);
      // as many lanes at work as can be, in runs of eight items at least
      double best = 0;
      for (int c = std::min(p.items, 32); c >= std::min(p.items, 8); --c) {
        const double used = (double)p.items / ((p.items + c - 1) / c * c) * (32 / c * c);
        if (used > best * 1.01) best = used, p.columns = c;
      }
      p.slots = 32 / p.columns;
      p.column_parts = (p.items + p.columns - 1) / p.columns;
      // few tokens are spread over more warps: up to 16 an SM, as far as there are heads
      const int64_t heads = a.heads[0] + a.heads[1], tokens = a.batch * a.tokens;
      p.head_parts = (int)std::clamp<int64_t>(16 * sms / (tokens * p.column_parts), 1, (heads + p.slots - 1) / p.slots);
      const int64_t warps = tokens * p.head_parts * p.column_parts;
      if (warps >= (int64_t)1 << 32) return cudaErrorInvalidConfiguration;
      const unsigned grid = (unsigned)((warps + kWarps - 1) / kWarps);
      if (a.interleaved) return launch_early(rotary_kernel<T, W, true>, dim3(grid), kWarps * 32, 0, st, a, p);
      return launch_early(rotary_kernel<T, W, false>, dim3(grid), kWarps * 32, 0, st, a, p);
    };
    constexpr int N = 16 / sizeof(T);
    return fits(N) ? go(Int<N>{}) : fits(2) ? go(Int<2>{}) : go(Int<1>{});
  });
}

}  // namespace echo
