// echo_ops_norm.cu -- layer norm and its gradients.
#include <algorithm>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace {

// Sum over the threads of a row (blockDim.x, whole warps); `sh`: a slot for each warp of the
// block.  Every row of the block takes part.  The caller alternates two slot arrays, so that
// one barrier a sum is enough.
__device__ __forceinline__ float row_sum(float v, float *sh) {
  v = warp_sum(v);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return v;
  float *row = sh + threadIdx.y * warps;
  if ((threadIdx.x & 31) == 0) row[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < warps; ++w) s += row[w];
  return s;
}

// 1 / sqrt(v), within a rounding: rsqrtf may be 2 units off, and a step of Newton's iteration,
// r + r (1 - v r^2) / 2 with the products' own roundings put back, leaves half a unit.  It takes
// up to 2% of a call, 6% at 65536 x 256 in bf16 (__frsqrt_rn 4% to 10%): every thread does it.
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v), h = v * r;
  const float e = fmaf(-fmaf(v, r, -h), r, fmaf(-h, r, 1.f));
  return fabsf(e) < 1.f ? fmaf(0.5f * r, e, r) : r;  // (not for 0, infinities and NaN)
}

// A thread's E elements of a row lie in E / W pieces blockDim.x apart; in registers they are
// pairs, one piece after the other.
template <typename X, int W, int E>
struct Slice {
  __device__ __forceinline__ static int column(int k) { return (k * (int)blockDim.x + (int)threadIdx.x) * W; }
  // Pieces of the thread that the row has: the first ones.
  __device__ __forceinline__ static int pieces(int H) {
    const int p = H / W - (int)threadIdx.x;
    return p <= 0 ? 0 : min(E / W, (p + (int)blockDim.x - 1) / (int)blockDim.x);
  }
  __device__ __forceinline__ static void store(X *row, const Pair (&v)[E / 2], int pieces) {
    float f[E];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) f[2 * e] = v[e].a, f[2 * e + 1] = v[e].b;
#pragma unroll
    for (int k = 0; k < E / W; ++k)
      if (k < pieces) store_piece<W>(row + column(k), f + k * W);
  }
  // the thread's parameters
  __device__ __forceinline__ static void param(const void *p, int type, float none, Pair (&v)[E / 2], int H) {
    float f[E];
#pragma unroll
    for (int k = 0; k < E / W; ++k) {
#pragma unroll
      for (int i = 0; i < W; ++i) f[k * W + i] = none;
      if (column(k) < H) load_param<W>(p, type, column(k), none, f + k * W);
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) v[e] = {f[2 * e], f[2 * e + 1]};
  }
};

// Rows come through shared memory, copied by the threads of a row while they work on the rows
// before (cp.async, `depth` slots).  In pieces of 16 bytes each thread copies its own; rows in
// narrower pieces (an odd length, stride or address) come in the 16-byte pieces of memory that
// hold them, for which the threads wait for one another.
template <typename X, int W, int E>
struct Rows {
  static constexpr bool kOwn = W * sizeof(X) == 16;
  static size_t slot_bytes(int x, int64_t H) { return kOwn ? (size_t)x * E * sizeof(X) : ((size_t)H * sizeof(X) + 30) / 16 * 16; }

  // `base`: the matrix's first row, before which nothing is read; `mine`: the thread's pieces.
  static __device__ __forceinline__ void copy(unsigned char *slot, const X *base, const X *row, int H, int mine) {
    if constexpr (kOwn) {
#pragma unroll
      for (int k = 0; k < E / W; ++k)
        if (k < mine) copy16(slot + (k * (int)blockDim.x + (int)threadIdx.x) * 16, row + Slice<X, W, E>::column(k), 16);
    } else {
      const uintptr_t begin = reinterpret_cast<uintptr_t>(row), end = begin + (size_t)H * sizeof(X), from = begin / 16 * 16;
      const int pieces = (int)((end - from + 15) / 16);
      for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
        const uintptr_t at = from + (uintptr_t)i * 16;
        if (at >= reinterpret_cast<uintptr_t>(base)) {
          copy16(slot + i * 16, reinterpret_cast<const void *>(at), (int)min((uintptr_t)16, end - at));
        } else {  // (a first row inside such a piece)
          for (uintptr_t b = begin; b < min(end, at + 16); b += sizeof(X)) *reinterpret_cast<X *>(slot + (b - from)) = *reinterpret_cast<const X *>(b);
        }
      }
    }
  }
  // Elements C c .. C c + C - 1 of the thread's (C a multiple of W), zeros where the row has none.
  // (Called apart for threads that have all their pieces, with E / W: the checks fall away.)
  template <int C>
  static __device__ __forceinline__ void read(const unsigned char *slot, const X *row, int mine, int c, Pair (&v)[C / 2]) {
    if constexpr (!kOwn) slot += reinterpret_cast<uintptr_t>(row) % 16;
    float f[C];
#pragma unroll
    for (int i = 0; i < C / W; ++i) {
      const int k = c * (C / W) + i;
      if constexpr (kOwn) {
        Pack<X, W> p{};
        if (k < mine) p = *reinterpret_cast<const Pack<X, W> *>(slot + (k * (int)blockDim.x + (int)threadIdx.x) * 16);
        unpack<X, W>(p, f + i * W);
      } else {
        const int j = k < mine ? Slice<X, W, E>::column(k) : 0;
        unpack<X, W>(*reinterpret_cast<const Pack<X, W> *>(slot + j * (int)sizeof(X)), f + i * W);
#pragma unroll
        for (int u = 0; u < W; ++u) f[i * W + u] = k < mine ? f[i * W + u] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < C / 2; ++e) v[e] = {f[2 * e], f[2 * e + 1]};
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
  // All copies but those of the depth - 2 commits since are there; the slot used last is free.
  static __device__ __forceinline__ void arrived(int depth) {
    if (depth == 2) asm volatile("cp.async.wait_group 0;\n" ::: "memory");
    else if (depth == 3) asm volatile("cp.async.wait_group 1;\n" ::: "memory");
    else asm volatile("cp.async.wait_group 2;\n" ::: "memory");
    if constexpr (!kOwn) __syncthreads();
  }

 private:
  static __device__ __forceinline__ void copy16(void *to, const void *from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
  }
};

// -- forward -----------------------------------------------------------------------------------
// A row stays in the registers of blockDim.x threads, with their parameters, until its output,
// and the block's next rows are on their way meanwhile.  The variance needs one exchange between
// warps: each takes the squared distances from its own mean, and
//   sum (x - mean)^2 = sum over warps of (their sum + n_w (mean_w - mean)^2),
// in which nothing cancels.  The output starts from those distances.  The bytes of x and y would
// bound it; what does is latency.  At 2048 x 12288 in bf16 an SM holds one row's 24 warps (37% of its
// places), which wait for shuffles, shared memory and one another's results; no unit is full (issue
// slots 64%, L1 41%, DRAM 29%).  So arithmetic is in pairs, addresses and bounds are kept from row to
// row, and a row has one barrier (two in pieces of less than 16 bytes).  A call takes 22 to 25 us in
// a row of them, 1.0e8 bytes: up to 4.6 TB/s.  Two rows a block with 32 elements a thread took 16%
// longer.
template <typename X, int W, int E>
__global__ void __launch_bounds__(E > 8 ? 768 : 1024) layer_norm_kernel(NormArgs a, int depth, int slot_bytes) {
  using S = Slice<X, W, E>;
  using R = Rows<X, W, E>;
  extern __shared__ __align__(16) unsigned char ring[];  // [depth][rows of the block]
  kernel_begin();
  next_may_start();
  __shared__ float2 sh[2][32];
  __shared__ float size[32];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, H = (int)a.H;
  const float over_h = 1.f / (float)H;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const X *x = static_cast<const X *>(a.x);
  const int own = S::pieces(H), pitch = (int)blockDim.y * slot_bytes, last = (depth - 1) * pitch;
  unsigned char *slot0 = ring + (int)threadIdx.y * slot_bytes;
  const X *ahead = x + row * a.x_stride;  // next row to copy
  int64_t left = (a.rows - row + step - 1) / step;  // rows from there (of this thread)
  const int64_t jump = step * a.x_stride;
  auto copy_next = [&](int at) {
    if (left > 0) R::copy(slot0 + at, x, ahead, H, own);
    R::commit();
    ahead += jump;
    --left;
  };
  for (int at = 0; at < last; at += pitch) copy_next(at);
  Pair w[E / 2], b[E / 2];
  S::param(a.w, a.p_type, 1.f, w, H);
  S::param(a.b, a.p_type, 0.f, b, H);
  // elements of each warp of a row
  int mine = 0;
#pragma unroll
  for (int k = 0; k < E / W; ++k) mine += max(0, min(32 * W, H - (k * (int)blockDim.x + warp * 32) * W));
  if (threadIdx.y == 0 && lane == 0) size[warp] = (float)mine;
  const float over_mine = mine ? 1.f / (float)mine : 0.f;
  __syncthreads();
  const float n_of = lane < warps ? size[lane] : 0.f;  // of warp `lane`
  int turn = 0, slot = 0;
  const X *from = x + row * a.x_stride;
  X *y = static_cast<X *>(a.y) + row * a.y_stride;
  const int64_t y_jump = step * a.y_stride;
  constexpr int C = W < 2 ? 2 : W;
  for (int64_t row0 = (int64_t)blockIdx.x * blockDim.y; row0 < a.rows; row0 += step, row += step, turn ^= 1, from += jump, y += y_jump) {
    R::arrived(depth);
    Pair v[E / 2];
    auto get = [&](int mine) {
#pragma unroll
      for (int c = 0; c < E / C; ++c) {
        Pair p[C / 2];
        R::template read<C>(slot0 + slot, from, mine, c, p);
#pragma unroll
        for (int e = 0; e < C / 2; ++e) v[c * (C / 2) + e] = p[e];
      }
    };
    if (own == E / W) get(E / W);
    else get(own);
    copy_next(slot == 0 ? last : slot - pitch);
    slot = slot == last ? 0 : slot + pitch;
    Pair s = v[0];
#pragma unroll
    for (int e = 1; e < E / 2; ++e) s = add2(s, v[e]);
    const float mean_w = warp_sum(s.a + s.b) * over_mine;
    Pair m = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      v[e] = add2(v[e], both(-mean_w));
      if (W >= 2) {
        if (2 * e / W < own) m = fma2(v[e], v[e], m);
      } else {  // (the two lie in pieces of their own)
        if (2 * e < own) m.a += v[e].a * v[e].a;
        if (2 * e + 1 < own) m.b += v[e].b * v[e].b;
      }
    }
    float m2 = warp_sum(m.a + m.b), mean = mean_w;
    if (warps > 1) {
      float2 *slots = sh[turn] + threadIdx.y * warps;
      if (lane == 0) slots[warp] = make_float2(mean_w, m2);
      __syncthreads();
      const float2 o = lane < warps ? slots[lane] : make_float2(0.f, 0.f);
      mean = warp_sum(o.x * n_of) * over_h;
      m2 = warp_sum(o.y + n_of * ((o.x - mean) * (o.x - mean)));
    }
    const float rstd = inverse_root(m2 * over_h + a.eps);
    if (row >= a.rows) continue;
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    const Pair scale = both(rstd), shift = both((mean_w - mean) * rstd);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) v[e] = fma2(fma2(v[e], scale, shift), w[e], b[e]);
    S::store(y, v, own);
  }
}

// Rows too long for registers: three passes over the row, a block each, the second and third from
// L2.  The loads' latency bounds it, a pass behind the other: 2048 x 16384 in bf16, 1.3e8 bytes, takes
// 73 us, 2048 x 32768 100 us (1.8 and 2.7 TB/s).
template <typename X, int W>
__global__ void __launch_bounds__(1024) layer_norm_long_kernel(NormArgs a) {
  __shared__ float sh[2][32];
  kernel_begin();
  next_may_start();
  const float over_h = 1.f / (float)a.H;
  const int64_t step = (int64_t)blockDim.x * W;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
    float s = 0.f;
    for (int64_t j = threadIdx.x * W; j < a.H; j += step) {
      float v[W];
      load_piece<W>(x + j, v);
#pragma unroll
      for (int i = 0; i < W; ++i) s += v[i];
    }
    const float mean = row_sum(s, sh[0]) * over_h;
    s = 0.f;
    for (int64_t j = threadIdx.x * W; j < a.H; j += step) {
      float v[W];
      load_piece<W>(x + j, v);
#pragma unroll
      for (int i = 0; i < W; ++i) s += (v[i] - mean) * (v[i] - mean);
    }
    const float rstd = 1.f / sqrtf(row_sum(s, sh[1]) * over_h + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    X *y = static_cast<X *>(a.y) + row * a.y_stride;
    for (int64_t j = threadIdx.x * W; j < a.H; j += step) {
      float v[W], w[W], b[W];
      load_piece<W>(x + j, v);
      load_param<W>(a.w, a.p_type, j, 1.f, w);
      load_param<W>(a.b, a.p_type, j, 0.f, b);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = (v[i] - mean) * rstd * w[i] + b[i];
      store_piece<W>(y + j, v);
    }
  }
}

// -- backward ----------------------------------------------------------------------------------
// With xh = (x - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dweight = sum over rows of dy xh,  dbias = of dy.
// One pass over dy and x: a block goes through its rows, a row among blockDim.x threads that
// keep the sums of dweight and dbias of their columns in registers.  Only those sums stay in
// registers with 16 elements a thread (the weight and the row as well would spill): the row is
// read twice from its slot, and the weight from shared memory (`staged`) or from L2 where the rows
// in flight leave no room.  The bytes of dy, x and dx would bound it; what does is latency, as in the
// forward pass, at twice the reads: at 2048 x 12288 in bf16 L1 is 68% busy (shared memory 51%), the
// issue slots 55%, DRAM 35%, and a call takes 47 to 48 us with the join, 3.2 TB/s.  The blocks'
// partial sums come on top ([blocks][2][H] fp32, written and read once).
template <typename X, int W, int E>
__global__ void __launch_bounds__(E > 8 ? 768 : 1024) layer_norm_grad_kernel(NormGradArgs a, int depth, int slot_bytes, int staged) {
  constexpr int K = E / W;
  using S = Slice<X, W, E>;
  using R = Rows<X, W, E>;
  extern __shared__ __align__(16) unsigned char staging[];  // [depth][x, dy][rows of the block]; the weight
  kernel_begin();
  __shared__ float2 sh[2][32];
  const int T = blockDim.x * blockDim.y, t = threadIdx.y * blockDim.x + threadIdx.x, warps = blockDim.x >> 5, lane = threadIdx.x & 31, H = (int)a.H;
  const float over_h = 1.f / (float)H;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const X *xs = static_cast<const X *>(a.x), *gs = static_cast<const X *>(a.dy);
  const int own = S::pieces(H), pitch = 2 * (int)blockDim.y * slot_bytes, last = (depth - 1) * pitch, g_at = (int)blockDim.y * slot_bytes;
  unsigned char *slot0 = staging + (int)threadIdx.y * slot_bytes;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const X *x_ahead = xs + row * a.x_stride, *g_ahead = gs + row * a.dy_stride;  // next row to copy
  int64_t left = (a.rows - row + step - 1) / step;                               // rows from there (of this thread)
  const int64_t x_jump = step * a.x_stride, g_jump = step * a.dy_stride, d_jump = step * a.dx_stride;
  auto copy_next = [&](int at) {
    if (left > 0) {
      R::copy(slot0 + at, xs, x_ahead, H, own);
      R::copy(slot0 + at + g_at, gs, g_ahead, H, own);
    }
    R::commit();
    x_ahead += x_jump;
    g_ahead += g_jump;
    --left;
  };
  for (int at = 0; at < last; at += pitch) copy_next(at);
  float mean = row < a.rows ? a.mean[row] : 0.f, rstd = row < a.rows ? a.rstd[row] : 0.f;
  Pair dw[E / 2], db[E / 2], kept[E > 8 ? 1 : E / 2];  // (8 elements: the weight's values stay in registers)
  Pair *weights = reinterpret_cast<Pair *>(staging + depth * pitch) + t;  // [E / 2][T], each its own
  if constexpr (E == 8) {
    S::param(a.w, a.p_type, 1.f, kept, H);
  } else if (staged) {
    Pair w[E / 2];
    S::param(a.w, a.p_type, 1.f, w, H);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) weights[e * T] = w[e];
  }
#pragma unroll
  for (int e = 0; e < E / 2; ++e) dw[e] = db[e] = {0.f, 0.f};
  // x, dy and the weight of a thread's elements C c .. C c + C - 1 of a row
  constexpr int C = W < 2 ? 2 : W;
  const X *x_row = xs + row * a.x_stride, *g_row = gs + row * a.dy_stride;
  X *dx = static_cast<X *>(a.dx) + row * a.dx_stride;
  auto read = [&](int mine, int slot, int c, Pair (&x)[C / 2], Pair (&g)[C / 2], Pair (&w)[C / 2]) {
    R::template read<C>(slot0 + slot, x_row, mine, c, x);
    R::template read<C>(slot0 + slot + g_at, g_row, mine, c, g);
    if constexpr (E == 8) {
#pragma unroll
      for (int e = 0; e < C / 2; ++e) w[e] = kept[c * (C / 2) + e];
    } else if (staged) {
#pragma unroll
      for (int e = 0; e < C / 2; ++e) w[e] = weights[(c * (C / 2) + e) * T];
    } else {
      float f[C];
#pragma unroll
      for (int i = 0; i < C / W; ++i) {
        const int k = c * (C / W) + i, j = S::column(k);
#pragma unroll
        for (int u = 0; u < W; ++u) f[i * W + u] = 1.f;
        if (k < own) load_param<W>(a.w, a.p_type, j, 1.f, f + i * W);
      }
#pragma unroll
      for (int e = 0; e < C / 2; ++e) w[e] = {f[2 * e], f[2 * e + 1]};
    }
  };
  int turn = 0, slot = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * blockDim.y; row0 < a.rows; row0 += step, row += step, turn ^= 1) {
    // (16 elements a thread: more than 2048 of a row, which a block then has to itself)
    const bool live = E > 8 || row < a.rows, more = row + step < a.rows;
    const float next_mean = more ? a.mean[row + step] : 0.f, next_rstd = more ? a.rstd[row + step] : 0.f;
    R::arrived(depth);
    copy_next(slot == 0 ? last : slot - pitch);
    const Pair scale = both(rstd), shift = both(-mean);  // (x - mean first: far from zero, x * rstd would lose what they differ by)
    Pair s1 = {0.f, 0.f}, s2 = {0.f, 0.f};
    auto add_up = [&](int mine) {
#pragma unroll
      for (int c = 0; c < E / C; ++c) {
        Pair x[C / 2], g[C / 2], w[C / 2];
        read(mine, slot, c, x, g, w);
#pragma unroll
        for (int e = 0; e < C / 2; ++e) {
          const int at = c * (C / 2) + e;
          const Pair xh = mul2(add2(x[e], shift), scale), gw = mul2(g[e], w[e]);
          dw[at] = fma2(g[e], xh, dw[at]);
          db[at] = add2(db[at], g[e]);
          s1 = add2(s1, gw);
          s2 = fma2(gw, xh, s2);
        }
      }
    };
    if (W > 1 && live && own == E / W) add_up(E / W);
    else if (live) add_up(own);
    if (a.dx) {
      float m1 = warp_sum(s1.a + s1.b), m2 = warp_sum(s2.a + s2.b);
      if (warps > 1) {
        float2 *slots = sh[turn] + threadIdx.y * warps;
        if (lane == 0) slots[threadIdx.x >> 5] = make_float2(m1, m2);
        __syncthreads();
        const float2 o = lane < warps ? slots[lane] : make_float2(0.f, 0.f);
        m1 = warp_sum(o.x);
        m2 = warp_sum(o.y);
      }
      const Pair n1 = both(-m1 * over_h), n2 = both(-m2 * over_h * rstd);
      auto put = [&](int mine) {
#pragma unroll
        for (int c = 0; c < E / C; ++c) {
          Pair x[C / 2], g[C / 2], w[C / 2];
          read(mine, slot, c, x, g, w);
          float f[C];
#pragma unroll
          for (int e = 0; e < C / 2; ++e) {
            const Pair d = mul2(fma2(add2(x[e], shift), n2, fma2(g[e], w[e], n1)), scale);
            f[2 * e] = d.a;
            f[2 * e + 1] = d.b;
          }
#pragma unroll
          for (int i = 0; i < C / W; ++i) {
            const int k = c * (C / W) + i;
            if (k < mine) store_piece<W>(dx + S::column(k), f + i * W);
          }
        }
      };
      if (W > 1 && live && own == E / W) put(E / W);
      else if (live) put(own);
      dx += d_jump;
    }
    x_row += x_jump;
    g_row += g_jump;
    slot = slot == last ? 0 : slot + pitch;
    mean = next_mean;
    rstd = next_rstd;
  }
  next_may_start();
  if (!a.part) return;
  // the block's rows together, in their order, then out
  asm volatile("cp.async.wait_group 0;\n" ::: "memory");
  if (blockDim.y > 1) {
    Pair *sums = reinterpret_cast<Pair *>(staging);  // [blockDim.y - 1][2][E / 2][blockDim.x]
    __syncthreads();
    if (threadIdx.y) {
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        sums[(((threadIdx.y - 1) * 2) * (E / 2) + e) * blockDim.x + threadIdx.x] = dw[e];
        sums[(((threadIdx.y - 1) * 2 + 1) * (E / 2) + e) * blockDim.x + threadIdx.x] = db[e];
      }
    }
    __syncthreads();
    if (threadIdx.y) return;
    for (int y = 0; y < (int)blockDim.y - 1; ++y)
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        dw[e] = add2(dw[e], sums[((y * 2) * (E / 2) + e) * blockDim.x + threadIdx.x]);
        db[e] = add2(db[e], sums[((y * 2 + 1) * (E / 2) + e) * blockDim.x + threadIdx.x]);
      }
  }
  float *part = a.part + (int64_t)blockIdx.x * 2 * a.H;
  float f[2][E];
#pragma unroll
  for (int e = 0; e < E / 2; ++e) f[0][2 * e] = dw[e].a, f[0][2 * e + 1] = dw[e].b, f[1][2 * e] = db[e].a, f[1][2 * e + 1] = db[e].b;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (k >= own) continue;
    store_piece<W>(part + S::column(k), f[0] + k * W);
    store_piece<W>(part + a.H + S::column(k), f[1] + k * W);
  }
}

// Rows too long for that: dx, a block a row, in two passes over it, the second from L2.  Bound by the
// loads' latency: 77 us by itself at 2048 x 16384 in bf16 ...
template <typename X, int W>
__global__ void __launch_bounds__(1024) layer_norm_grad_rows_kernel(NormGradArgs a) {
  __shared__ float sh[4][32];
  kernel_begin();
  next_may_start();
  const float over_h = 1.f / (float)a.H;
  const int64_t step = (int64_t)blockDim.x * W;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 2) {
    const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
    const X *dy = static_cast<const X *>(a.dy) + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int64_t j = threadIdx.x * W; j < a.H; j += step) {
      float v[W], g[W], w[W];
      load_piece<W>(x + j, v);
      load_piece<W>(dy + j, g);
      load_param<W>(a.w, a.p_type, j, 1.f, w);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        s1 += g[i] * w[i];
        s2 += g[i] * w[i] * ((v[i] - mean) * rstd);
      }
    }
    const float m1 = row_sum(s1, sh[turn]) * over_h, m2 = row_sum(s2, sh[turn + 1]) * over_h;
    X *dx = static_cast<X *>(a.dx) + row * a.dx_stride;
    for (int64_t j = threadIdx.x * W; j < a.H; j += step) {
      float v[W], g[W], w[W];
      load_piece<W>(x + j, v);
      load_piece<W>(dy + j, g);
      load_param<W>(a.w, a.p_type, j, 1.f, w);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = rstd * (g[i] * w[i] - m1 - (v[i] - mean) * rstd * m2);
      store_piece<W>(dx + j, v);
    }
  }
}

// ... and partial sums of dweight and dbias, blockDim.x * W columns of one part of the rows a block:
// dy and x once more, 46 us there, 2.9 TB/s.  The whole call takes 129 us, 2.0e8 bytes.
template <typename X, int W>
__global__ void __launch_bounds__(128) layer_norm_grad_columns_kernel(NormGradArgs a) {
  kernel_begin();
  next_may_start();
  const int64_t j = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * W;
  if (j >= a.H) return;
  const int64_t per = (a.rows + a.parts - 1) / a.parts;
  const int64_t begin = min(a.rows, blockIdx.y * per), end = min(a.rows, begin + per);
  float dw[W] = {}, db[W] = {};
#pragma unroll 4
  for (int64_t r = begin; r < end; ++r) {
    float v[W], g[W];
    load_piece<W>(static_cast<const X *>(a.x) + r * a.x_stride + j, v);
    load_piece<W>(static_cast<const X *>(a.dy) + r * a.dy_stride + j, g);
    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      dw[i] += g[i] * ((v[i] - mean) * rstd);
      db[i] += g[i];
    }
  }
  float *part = a.part + (int64_t)blockIdx.y * 2 * a.H + j;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    part[i] = dw[i];
    part[a.H + i] = db[i];
  }
}

__device__ __forceinline__ void put_param(void *p, int type, int64_t j, float v, int accumulate) {
  if (type == ECHO_F32) {
    float *at = static_cast<float *>(p) + j;
    *at = accumulate ? *at + v : v;
  } else if (type == ECHO_BF16) {
    __nv_bfloat16 *at = static_cast<__nv_bfloat16 *>(p) + j;
    *at = __float2bfloat16_rn(accumulate ? __bfloat162float(*at) + v : v);
  } else {
    __half *at = static_cast<__half *>(p) + j;
    *at = __float2half_rn(accumulate ? __half2float(*at) + v : v);
  }
}

// dweight and dbias from their parts: 32 columns of one of the two a block, its warps taking
// the parts in turn, then the warps' sums in order, so that calls repeat to the bit.  152 parts of
// 12288 columns, 1.5e7 bytes, take 8.7 us by themselves.
constexpr int kJoinWarps = 16;

__global__ void __launch_bounds__(kJoinWarps * 32) layer_norm_grad_join_kernel(NormGradArgs a) {
  __shared__ float sh[kJoinWarps][33];
  kernel_begin();
  next_may_start();
  const int64_t j = (int64_t)blockIdx.x * 32 + threadIdx.x;  // of [dweight, dbias]: 2 H columns
  float s = 0.f;
  if (j < 2 * a.H) {
#pragma unroll 8
    for (int p = threadIdx.y; p < a.parts; p += kJoinWarps) s += a.part[(int64_t)p * 2 * a.H + j];
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y || j >= 2 * a.H) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) s += sh[w][threadIdx.x];
  void *to = j < a.H ? a.dw : a.db;
  if (to) put_param(to, a.p_type, j < a.H ? j : j - a.H, s, a.accumulate);
}

// Widest pieces (16 bytes of X, two elements, or one) that all rows and parameters of a call
// allow, as f's argument.
template <typename X, typename F>
cudaError_t with_pieces(int64_t H, std::initializer_list<std::pair<const void *, int64_t>> rows, int x_type,
                        std::initializer_list<const void *> params, int p_type, F &&f) {
  auto fits = [&](int W) {
    if (H % W) return false;
    for (const auto &r : rows)
      if (r.first && !fits_pieces(r.first, r.second, x_type, W)) return false;
    for (const void *p : params)
      if (p && !fits_pieces(p, 0, p_type, W)) return false;
    return true;
  };
  constexpr int N = 16 / sizeof(X);
  return fits(N) ? f(Int<N>{}) : fits(2) ? f(Int<2>{}) : f(Int<1>{});
}

int row_threads(int64_t H, int E) { return (int)std::min<int64_t>(1024, (H + 32 * E - 1) / (32 * E) * 32); }

constexpr int64_t kCached = 768 * 16;  // longest rows of the one-pass kernels
// Elements of a row that a thread takes.  With 16 a row's sums and addresses take fewer
// instructions (forward, 16384 x 2048 in bf16: 27 us, 31 with 8); backward, more warps are worth
// more up to 256 threads a row (8192 x 1024 in fp32: 22 us with 8, 28 with 16).
int row_elements(int64_t H, int arrays) { return H <= (arrays == 2 ? 2048 : 256) ? 8 : 16; }

// Shape of a one-pass kernel for rows of H elements, `arrays` of them read: threads of a row,
// rows at a time, slots (up to 4, as two blocks' shared memory allows), bytes of a slot.
struct Shape {
  int E, x, y, depth, slot, staged;
  size_t smem;
};
template <typename X, int W>
Shape row_shape(int64_t H, int arrays) {
  Shape s{};
  s.E = row_elements(H, arrays);
  s.x = row_threads(H, s.E);
  s.y = std::max(1, 256 / s.x);
  s.slot = (int)(s.E == 8 ? Rows<X, W, 8>::slot_bytes(s.x, H) : Rows<X, W, 16>::slot_bytes(s.x, H));
  const size_t row = (size_t)s.y * arrays * s.slot, room = s.E > 8 ? 200 << 10 : 100 << 10;
  const size_t weights = arrays == 2 && s.E > 8 ? (size_t)s.x * s.y * s.E * sizeof(float) : 0;
  s.staged = weights && row * 2 + weights <= room;
  s.depth = (int)std::clamp<size_t>((room - (s.staged ? weights : 0)) / row, 2, 4);
  s.smem = row * s.depth + (s.staged ? weights : 0);
  if (arrays == 2) s.smem = std::max(s.smem, (size_t)(s.y - 1) * 2 * s.E * s.x * sizeof(float));
  return s;
}
// Blocks of it that an SM takes: 80 registers a thread with 16 elements, 64 with 8.
int blocks_of(const Shape &s) {
  return (int)std::max<size_t>(1, std::min<size_t>((s.E > 8 ? 768 : 1024) / (s.x * s.y), (220 << 10) / (s.smem + 2048)));
}
// A grid that goes through its rows in turns has to lie evenly on the SMs, which blocks that come
// while another kernel ends do not by themselves: where it fills them, a block asks for so much
// shared memory that no more than its share fit an SM (4999 x 1537 in fp32, backward: 40 us a
// call in a row of them, 63 without).  Backward, up to as many blocks as SMs get an SM each in the
// same way (64 x 2048 in bf16, in a graph: 4.8 us, 5.2 to 6.2 where they come several to an SM; 100 x
// 1537 in fp32 6.0 and 6.6).  Forward, and for less than a quarter of the SMs, it changes nothing but
// the call, which sets the kernel's limit (0.6 us).
size_t even_smem(const Shape &s, int64_t grid, int sms, int arrays) {
  if (arrays == 2 && grid <= sms && grid > sms / 4) return std::max<size_t>(s.smem, (228 << 10) / 2);
  return grid > sms && grid % sms == 0 ? std::max<size_t>(s.smem, (228 << 10) / (grid / sms + 1)) : s.smem;
}

constexpr int kMostSmem = 224 << 10;  // a block's, beside what the kernels hold for their sums

template <typename K, typename... A>
cudaError_t launch_rows(K kernel, const Shape &s, int arrays, int64_t grid, int sms, cudaStream_t st, const A &...args) {
  const size_t smem = even_smem(s, grid, sms, arrays);
  if (smem > 40 << 10) {  // (one limit for all lengths: calls of other threads, or a graph's, may lie between)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e != cudaSuccess) return e;
  }
  return launch_early(kernel, dim3((unsigned)grid), dim3(s.x, s.y), smem, st, args...);
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs &a, int sms, cudaStream_t st) {
  return with_type(a.x_type, [&](auto t) {
    using X = decltype(t);
    return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.y, a.y_stride}}, a.x_type, {a.w, a.b}, a.p_type, [&](auto wide) {
      constexpr int W = decltype(wide)::value;
      if (a.H > kCached) {
        return launch_early(layer_norm_long_kernel<X, W>, dim3((unsigned)std::min<int64_t>(a.rows, sms * 2)), 1024, 0, st, a);
      }
      const Shape s = row_shape<X, W>(a.H, 1);
      auto go = [&](auto each) {
        constexpr int E = decltype(each)::value;
        const int64_t grid = std::min<int64_t>((a.rows + s.y - 1) / s.y, (int64_t)sms * blocks_of(s));
        return launch_rows(layer_norm_kernel<X, W, E>, s, 1, grid, sms, st, a, s.depth, s.slot);
      };
      return s.E == 8 ? go(Int<8>{}) : go(Int<16>{});
    });
  });
}

namespace {
// Blocks of the backward kernel, each with a partial sum of the parameters' gradients.
int grad_blocks(const Shape &s, int64_t rows, int sms) { return (int)std::min<int64_t>((rows + s.y - 1) / s.y, (int64_t)std::min(2, blocks_of(s)) * sms); }
}  // namespace

int layer_norm_grad_parts(const NormGradArgs &a, int sms) {
  if (a.H > kCached) return (int)std::max<int64_t>(1, std::min<int64_t>({a.rows / 8, (int64_t)sms, 65535}));
  int parts = 0;
  (void)with_type(a.x_type, [&](auto t) {
    using X = decltype(t);
    return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dx, a.dx_stride}}, a.x_type, {a.w}, a.p_type, [&](auto wide) {
      parts = grad_blocks(row_shape<X, decltype(wide)::value>(a.H, 2), a.rows, sms);
      return cudaSuccess;
    });
  });
  return parts;
}

cudaError_t launch_layer_norm_grad(const NormGradArgs &a, int sms, const OpTimer &timed, cudaStream_t st) {
  const bool params = a.dw || a.db;
  cudaError_t e = cudaSuccess;
  if (a.rows && (a.dx || params))
    e = with_type(a.x_type, [&](auto t) {
      using X = decltype(t);
      return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dx, a.dx_stride}}, a.x_type, {a.w}, a.p_type, [&](auto wide) {
        constexpr int W = decltype(wide)::value;
        if (a.H > kCached) {
          cudaError_t r = cudaSuccess;
          const int64_t cols = 128 * W;
          if (params)  // (before dx: it may overwrite dy or x)
            r = timed("layer_norm_grad_columns", [&] {
              return launch_early(layer_norm_grad_columns_kernel<X, W>, dim3((unsigned)((a.H + cols - 1) / cols), a.parts), 128, 0, st, a);
            });
          if (r == cudaSuccess && a.dx)
            r = timed("layer_norm_grad_rows", [&] {
              return launch_early(layer_norm_grad_rows_kernel<X, W>, dim3((unsigned)std::min<int64_t>(a.rows, INT32_MAX)), row_threads(a.H, 8), 0, st, a);
            });
          return r;
        }
        const Shape s = row_shape<X, W>(a.H, 2);
        auto go = [&](auto each) {
          constexpr int E = decltype(each)::value;
          return timed("layer_norm_grad", [&] {
            return launch_rows(layer_norm_grad_kernel<X, W, E>, s, 2, grad_blocks(s, a.rows, sms), sms, st, a, s.depth, s.slot, s.staged);
          });
        };
        return s.E == 8 ? go(Int<8>{}) : go(Int<16>{});
      });
    });
  if (e != cudaSuccess || !params) return e;
  return timed("layer_norm_grad_join", [&] {
    return launch_early(layer_norm_grad_join_kernel, dim3((unsigned)((2 * a.H + 31) / 32)), dim3(32, kJoinWarps), 0, st, a);
  });
}

}  // namespace echo
