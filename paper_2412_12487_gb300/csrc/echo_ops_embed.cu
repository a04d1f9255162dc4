// echo_ops_embed.cu -- embedding lookup in a vocabulary shard, and its gradient.
#include <cooperative_groups.h>

#include <algorithm>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace cg = cooperative_groups;

namespace {

// Row of the shard that token t reads, or -1: the id's distance from the first id, taken
// without overflow for any id.
__device__ __forceinline__ int64_t shard_row(const void *ids, int id64, int64_t t, int64_t v0, int64_t V) {
  const int64_t id = id64 ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
  const uint64_t row = (uint64_t)id - (uint64_t)v0;  // (v0 >= 0: an id below it wraps to beyond V)
  return row < (uint64_t)V ? (int64_t)row : -1;
}

// -- lookup ----------------------------------------------------------------------------------
// out[t] = scale * table[row of t], zeros without one.  Bound by the bytes read and written.  A
// warp takes 32 * kLookup pieces of one token, then those of another: the next token's id is
// read while this one's row is on its way, so that a token costs one latency and not two.  2048
// tokens of 12288, fp32 to bf16, 8.4e7 bytes: 15.6 us in a row of calls, 5.35 TB/s; half the
// pieces, in registers for six blocks an SM, took 6.5 us more.
constexpr int kLookup = 4;

template <typename T, typename O, int W>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, int64_t pieces, int64_t chunks, int64_t units) {
  kernel_begin();
  next_may_start();
  const T *table = static_cast<const T *>(a.table);
  O *out = static_cast<O *>(a.out);
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
  int64_t unit = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  if (unit >= units) return;
  // units go token by token; a step of `warps` units is this many tokens and chunks
  const int64_t t_step = warps / chunks, c_step = warps % chunks;
  int64_t t = unit / chunks, c = unit % chunks;
  int64_t row = shard_row(a.ids, a.id64, t, a.v0, a.V);
  for (;;) {
    const int64_t p0 = c * (32 * kLookup) + lane;
    Pack<T, W> in[kLookup];
    if (row >= 0) {
      const T *from = table + row * a.table_stride;
#pragma unroll
      for (int k = 0; k < kLookup; ++k)
        if (p0 + k * 32 < pieces) in[k] = *reinterpret_cast<const Pack<T, W> *>(from + (p0 + k * 32) * W);
    }
    O *to = out + t * a.out_stride;
    const bool mine = row >= 0;
    unit += warps;
    t += t_step;
    c += c_step;
    if (c >= chunks) c -= chunks, ++t;
    if (unit < units) row = shard_row(a.ids, a.id64, t, a.v0, a.V);
#pragma unroll
    for (int k = 0; k < kLookup; ++k) {
      float f[W];
      if (mine) unpack<T, W>(in[k], f);
#pragma unroll
      for (int i = 0; i < W; ++i) f[i] = mine ? f[i] * a.scale : 0.f;
      if (p0 + k * 32 < pieces) store_piece<W>(to + (p0 + k * 32) * W, f);
    }
    if (unit >= units) break;
  }
}

// -- gradient: tokens sorted by row ------------------------------------------------------------
// A stable radix sort, 8 bits a pass, by one cluster of 8 blocks: 256 warps each own a
// contiguous range of the tokens.  A pass counts each warp's digits, takes the running sum over
// (digit, block, warp) with the blocks' totals exchanged through distributed shared memory, and
// places each token behind those before it.  The order of equal rows is the tokens', so the
// sums' order is fixed.  Bound by the latency of its steps, not by the tokens, so the first
// kHeld tokens of each thread (all of them up to 32768 tokens) stay in registers from their
// count to their place.  16384 tokens of 51200 rows, two passes, take 21 us.
constexpr int kSortBlocks = 8, kSortWarps = 32, kHeld = 4;

__global__ void __cluster_dims__(kSortBlocks) __launch_bounds__(kSortWarps * 32) embed_sort_kernel(EmbedGradArgs a, int passes) {
  __shared__ int32_t cnt[kSortWarps][256];
  __shared__ int32_t tot[256], start[256];
  __shared__ int32_t sums[8];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned below = (1u << lane) - 1;
  kernel_begin();
  next_may_start();
  int64_t n = a.n;
  for (int pass = 0; pass < passes; ++pass) {
    const uint32_t *key_in = a.key[(pass + 1) & 1], *tok_in = a.tok[(pass + 1) & 1];
    uint32_t *key_out = a.key[pass & 1], *tok_out = a.tok[pass & 1];
    const int64_t per_warp = ((n + kSortBlocks * kSortWarps - 1) / (kSortBlocks * kSortWarps) + 31) / 32 * 32;
    const int64_t begin = min(n, (rank * kSortWarps + warp) * per_warp), end = min(n, begin + per_warp);
    auto key_at = [&](int64_t i) -> int64_t {  // -1: no token, or one of another shard
      if (i >= end) return -1;
      return pass == 0 ? shard_row(a.ids, a.id64, i, a.v0, a.V) : (int64_t)__ldcg(key_in + i);
    };
    auto token_at = [&](int64_t i) { return pass == 0 || i >= end ? (uint32_t)i : __ldcg(tok_in + i); };
    auto digit_of = [&](int64_t key) { return key < 0 ? 256 : (int)(key >> (8 * pass)) & 255; };
    // place of a token among its warp's with the same digit, which is counted on the way
    auto count = [&](int64_t key) {
      const int digit = digit_of(key);
      const unsigned same = __match_any_sync(0xFFFFFFFFu, digit);
      const int32_t before = key < 0 ? 0 : cnt[warp][digit];
      __syncwarp();
      if (key >= 0 && !(same & below)) cnt[warp][digit] = before + __popc(same);
      __syncwarp();
      return before + __popc(same & below);
    };
    int64_t key[kHeld];
    uint32_t tok[kHeld];
    int32_t place[kHeld];
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
      key[h] = key_at(begin + h * 32 + lane);
      tok[h] = token_at(begin + h * 32 + lane);
    }
    for (int i = tid; i < kSortWarps * 64; i += blockDim.x) reinterpret_cast<int4 *>(cnt)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (begin + h * 32 < end) place[h] = count(key[h]);
    for (int64_t i = begin + kHeld * 32; i < end; i += 32) (void)count(key_at(i + lane));
    __syncthreads();
    {  // running sums over the warps: four threads a digit, eight warps each
      const int digit = tid >> 2, w0 = (tid & 3) * 8;
      int32_t c[8], run = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        c[w] = cnt[w0 + w][digit];
        run += c[w];
      }
      int32_t upto = run;
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        const int32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, d, 4);
        if ((tid & 3) >= d) upto += v;
      }
      int32_t base = upto - run;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        cnt[w0 + w][digit] = base;
        base += c[w];
      }
      if ((tid & 3) == 3) tot[digit] = upto;
    }
    cluster.sync();
    int32_t all = 0, before = 0, upto = 0;
    if (tid < 256) {
#pragma unroll
      for (int b = 0; b < kSortBlocks; ++b) {
        const int32_t c = cluster.map_shared_rank(tot, b)[tid];
        before += b < rank ? c : 0;
        all += c;
      }
      upto = all;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += v;
      }
      if (lane == 31) sums[warp] = upto;
    }
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      upto += w < warp ? sums[w] : 0;
      total += sums[w];
    }
    if (tid < 256) start[tid] = upto - all + before;  // where the block's tokens of a digit begin
    __syncthreads();
    auto put = [&](int64_t k, uint32_t t, int64_t at) {
      key_out[at] = (uint32_t)k;
      tok_out[at] = t;
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
      if (key[h] >= 0) put(key[h], tok[h], (int64_t)start[digit_of(key[h])] + cnt[warp][digit_of(key[h])] + place[h]);
    if (begin + kHeld * 32 < end) {  // the others are counted again, behind those
      __syncwarp();
#pragma unroll
      for (int h = 0; h < kHeld; ++h) (void)count(key[h]);
      for (int64_t i = begin + kHeld * 32; i < end; i += 32) {
        const int64_t k = key_at(i + lane);
        const int32_t at = count(k);  // (from the warp's base on)
        if (k >= 0) put(k, token_at(i + lane), (int64_t)start[digit_of(k)] + at);
      }
    }
    __threadfence();
    cluster.sync();  // (the other blocks' tokens, and their reads of `tot`)
    n = total;
  }
  if (rank == 0 && tid == 0) *a.count = (int32_t)n;
}

// The same order for few tokens, on all SMs at once: a token's place is the number of tokens
// before it, counted against every other token (a warp takes four, 32 others at a time).  The
// counts grow with the square of the tokens, but nothing waits for another block: with the
// events around them, 2048 tokens take 10 us (16 by the passes above), 4096 13 us (22), 8192
// 27 us (22).
constexpr int kRankTokens = 5120, kRankWarps = 8, kRankEach = 4;

__global__ void __launch_bounds__(kRankWarps * 32) embed_rank_kernel(EmbedGradArgs a, uint32_t *key_out, uint32_t *tok_out) {
  extern __shared__ __align__(16) uint32_t rows[];  // of every token, padded to 128; ~0: none of the shard
  kernel_begin();
  next_may_start();
  const int n = (int)a.n, padded = (n + 127) / 128 * 128, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < padded; i += blockDim.x) rows[i] = i < n ? (uint32_t)shard_row(a.ids, a.id64, i, a.v0, a.V) : ~0u;
  __syncthreads();
  const int t0 = (blockIdx.x * kRankWarps + (threadIdx.x >> 5)) * kRankEach;
  uint32_t mine[kRankEach];
  int before[kRankEach] = {}, all = 0;
#pragma unroll
  for (int k = 0; k < kRankEach; ++k) mine[k] = t0 + k < n ? rows[t0 + k] : ~0u;
  for (int i = lane * 4; i < padded; i += 128) {
    const uint4 o = *reinterpret_cast<const uint4 *>(rows + i);
    const uint32_t other[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      all += other[e] != ~0u;
#pragma unroll
      for (int k = 0; k < kRankEach; ++k) before[k] += other[e] < mine[k] || (other[e] == mine[k] && i + e < t0 + k);
    }
  }
#pragma unroll
  for (int k = 0; k < kRankEach; ++k) {
    const int at = __reduce_add_sync(0xFFFFFFFFu, before[k]);
    if (lane == k && mine[k] != ~0u) {
      key_out[at] = mine[k];
      tok_out[at] = (uint32_t)(t0 + k);
    }
  }
  all = __reduce_add_sync(0xFFFFFFFFu, all);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = all;
}

// -- gradient: sums ----------------------------------------------------------------------------
// The sorted tokens are cut into windows of a.window; a warp sums one window over 32 * kWide
// columns, so that every warp has the same work however the tokens fall on the rows.  A row
// that lies inside a window is written at once; the part of a row that a window's edge cuts
// goes to `part` ([window][0: began before it, 1: began in it][H]) and embed_join_kernel adds
// the parts in order.  Bound by the bytes of dy and of the rows: 16384 tokens of 2048 in bf16 into 51200
// rows, 2.8e8 bytes of which zeros are most, take 57 us, 4.9 TB/s.
//
// Unless the call accumulates, other blocks of the grid, between those of the sums, write zeros
// to the rows that no token has: each marks which of kClear rows have any among the sorted ones.
constexpr int kClear = 32;

template <typename T>
__device__ void clear_rows(const EmbedGradArgs &a, const uint32_t *key, int64_t count, int64_t v0) {
  __shared__ uint32_t has;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t v1 = min(a.V, v0 + kClear);
  if (threadIdx.x == 0) has = 0;
  __syncthreads();
  int64_t lo = 0, hi = count;  // the first token of these rows: a 33-fold search by each warp
  while (lo < hi) {
    const int64_t step = (hi - lo + 32) / 33, at = lo + (lane + 1) * step - 1;
    const unsigned less = __ballot_sync(0xFFFFFFFFu, at < hi && key[at] < v0);
    const int below = __popc(less);
    const int64_t next = lo + below * step;
    hi = min(hi, below < 32 ? next + step - 1 : hi);
    lo = next;
  }
  for (int64_t i = lo + threadIdx.x; i < count; i += blockDim.x) {
    const uint32_t k = key[i];
    if (k >= v1) break;
    atomicOr(&has, 1u << (k - v0));
  }
  __syncthreads();
  const int64_t bytes = a.H * (int64_t)sizeof(T), pitch = a.dtable_stride * (int64_t)sizeof(T);
  unsigned char *table = static_cast<unsigned char *>(a.dtable);
  const bool wide = bytes % 16 == 0 && pitch % 16 == 0 && reinterpret_cast<uintptr_t>(table) % 16 == 0;
  for (int64_t v = v0 + warp; v < v1; v += blockDim.x >> 5) {
    if (has >> (v - v0) & 1) continue;
    unsigned char *at = table + v * pitch;
    if (wide) {
      for (int64_t i = lane; i < bytes / 16; i += 32) reinterpret_cast<uint4 *>(at)[i] = make_uint4(0, 0, 0, 0);
    } else {
      for (int64_t i = lane; i < a.H; i += 32) reinterpret_cast<T *>(at)[i] = T{};
    }
  }
}
template <typename D, typename T, int W>
__global__ void __launch_bounds__(256, 3) embed_sum_kernel(EmbedGradArgs a, const uint32_t *key, const uint32_t *tok, int64_t chunks, int64_t clears) {
  kernel_begin();
  next_may_start();
  constexpr int N = 16 / sizeof(D), K = N / W;              // columns of a lane, in K pieces
  constexpr int kBatch = W * sizeof(D) >= 4 ? 8 : 4;        // rows of dy in flight (a 16-bit piece takes a register)
  const int lane = threadIdx.x & 31;
  const int64_t count = *a.count;
  // `clears` of the blocks clear rows, spread evenly over the grid
  const int64_t cleared = (int64_t)blockIdx.x * clears / gridDim.x;
  if (((int64_t)blockIdx.x + 1) * clears / gridDim.x != cleared) {
    clear_rows<T>(a, key, count, cleared * kClear);
    return;
  }
  const int64_t unit = ((blockIdx.x - cleared) * blockDim.x + threadIdx.x) >> 5;
  const int64_t w0 = unit / chunks * a.window, col0 = unit % chunks * (32 * N) + lane * W;
  if (w0 >= count) return;
  const int m = (int)min((int64_t)a.window, count - w0);
  const uint32_t my_key = lane < m ? key[w0 + lane] : 0, my_tok = lane < m ? tok[w0 + lane] : 0;
  const uint32_t first = __shfl_sync(0xFFFFFFFFu, my_key, 0), last = __shfl_sync(0xFFFFFFFFu, my_key, m - 1);
  const bool cut_before = w0 > 0 && key[w0 - 1] == first, cut_after = w0 + m < count && key[w0 + m] == last;
  const D *dy = static_cast<const D *>(a.dy);
  T *dtable = static_cast<T *>(a.dtable);
  float acc[K][W];
  auto flush = [&](uint32_t row, bool head, bool tail) {
    const bool from_before = head && cut_before, to_after = tail && cut_after;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t j = col0 + k * 32 * W;
      if (j >= a.H) continue;
      if (from_before || to_after) {
        store_piece<W>(a.part + ((w0 / a.window) * 2 + (from_before ? 0 : 1)) * a.H + j, acc[k]);
      } else {
        T *at = dtable + row * a.dtable_stride + j;
        float old[W];
        if (a.accumulate) load_piece<W>(at, old);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[k][i] = acc[k][i] * a.scale + (a.accumulate ? old[i] : 0.f);
        store_piece<W>(at, acc[k]);
      }
    }
  };
  uint32_t row = first;
  bool head = true;
#pragma unroll
  for (int k = 0; k < K; ++k)
    for (int i = 0; i < W; ++i) acc[k][i] = 0.f;
  for (int t0 = 0; t0 < m; t0 += kBatch) {
    Pack<D, W> in[kBatch][K];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t t = __shfl_sync(0xFFFFFFFFu, my_tok, (t0 + u) & 31);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (t0 + u < m && col0 + k * 32 * W < a.H)
          in[u][k] = *reinterpret_cast<const Pack<D, W> *>(dy + t * a.dy_stride + col0 + k * 32 * W);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const uint32_t r = __shfl_sync(0xFFFFFFFFu, my_key, (t0 + u) & 31);
      if (t0 + u >= m) continue;
      const bool next = r != row;
      if (next) {
        flush(row, head, false);
        row = r;
        head = false;
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float f[W];
        unpack<D, W>(in[u][k], f);
        if (col0 + k * 32 * W < a.H) {
#pragma unroll
          for (int i = 0; i < W; ++i) acc[k][i] = next ? f[i] : acc[k][i] + f[i];
        }
      }
    }
  }
  flush(row, head, true);
}

// Rows that windows cut: the warp of the window in which the row begins adds its parts, in
// order.  Latency bounds it: most windows have nothing to add, and a frequent row's parts are read
// 16 at a time (13 us by itself there; its start lies behind the sums').
template <typename T, int W>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedGradArgs a, const uint32_t *key, int64_t chunks) {
  kernel_begin();
  next_may_start();
  const int lane = threadIdx.x & 31;
  const int64_t unit = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int64_t w = unit / chunks, j = unit % chunks * (32 * W) + lane * W;
  const int64_t count = *a.count, P = a.window, end = (w + 1) * P;
  if (end >= count) return;
  // three keys at once, and the first keys of the windows behind, 32 at a time
  const int64_t at = lane == 0 ? end - 1 : lane == 1 ? max((int64_t)0, w * P - 1) : end;
  const uint32_t k = lane < 3 ? key[at] : 0, row = __shfl_sync(0xFFFFFFFFu, k, 0);
  if (__shfl_sync(0xFFFFFFFFu, k, 2) != row || (w > 0 && __shfl_sync(0xFFFFFFFFu, k, 1) == row)) return;  // no row begins here and is cut
  const int64_t windows = (count + P - 1) / P;
  int64_t last = w + 1;  // the last window that begins with this row
  for (;;) {
    const int64_t u = last + 1 + lane;
    const unsigned differs = __ballot_sync(0xFFFFFFFFu, u >= windows || key[u * P] != row);
    last += differs ? __ffs(differs) - 1 : 32;
    if (differs) break;
  }
  if (j >= a.H) return;
  float acc[W];
  load_piece<W>(a.part + (w * 2 + 1) * a.H + j, acc);
#pragma unroll 16
  for (int64_t u = w + 1; u <= last; ++u) {
    float f[W];
    load_piece<W>(a.part + u * 2 * a.H + j, f);
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] += f[i];
  }
  T *to = static_cast<T *>(a.dtable) + row * a.dtable_stride + j;
  float old[W];
  if (a.accumulate) load_piece<W>(to, old);
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = acc[i] * a.scale + (a.accumulate ? old[i] : 0.f);
  store_piece<W>(to, acc);
}

int sort_passes(int64_t V) {
  int bits = 1;
  while (bits < 31 && ((int64_t)1 << bits) < V) ++bits;
  return (bits + 7) / 8;
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs &a, int sms, cudaStream_t st) {
  return with_type(a.table_type, [&](auto t) {
    return with_type(a.out_type, [&](auto o) {
      using T = decltype(t);
      using O = decltype(o);
      constexpr int N = 16 / sizeof(O);
      auto go = [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int64_t pieces = a.H / W, chunks = (pieces + 32 * kLookup - 1) / (32 * kLookup);
        if (a.n > INT64_MAX / chunks) return cudaErrorInvalidValue;
        const int64_t units = a.n * chunks;
        return launch_early(embed_kernel<T, O, W>, dim3((unsigned)std::min<int64_t>((units + 7) / 8, (int64_t)sms * 6)), 256, 0, st, a, pieces, chunks, units);
      };
      auto fits = [&](int W) {
        return a.H % W == 0 && fits_pieces(a.table, a.table_stride, a.table_type, W) && fits_pieces(a.out, a.out_stride, a.out_type, W);
      };
      return fits(N) ? go(Int<N>{}) : fits(2) ? go(Int<2>{}) : go(Int<1>{});
    });
  });
}

// Windows small enough that the sums occupy the SMs, 24 warps each.
int embed_grad_window(int64_t n, int64_t H, int sms) {
  int P = 8;
  while (P < 32 && n / (2 * P) * ((H + 255) / 256) >= (int64_t)sms * 24) P *= 2;
  return P;
}

cudaError_t launch_embed_sort(const EmbedGradArgs &a, cudaStream_t st) {
  if (a.n <= kRankTokens) {
    const int last = (sort_passes(a.V) + 1) & 1, each = kRankWarps * kRankEach;
    return launch_early(embed_rank_kernel, dim3((unsigned)std::max<int64_t>(1, (a.n + each - 1) / each)), kRankWarps * 32,
                        (size_t)((a.n + 127) / 128 * 128) * 4, st, a, a.key[last], a.tok[last]);
  }
  return launch_early(embed_sort_kernel, kSortBlocks, kSortWarps * 32, 0, st, a, sort_passes(a.V));
}

cudaError_t launch_embed_sum(const EmbedGradArgs &a, cudaStream_t st) {
  const int last = (sort_passes(a.V) + 1) & 1;
  return with_type(a.dy_type, [&](auto d) {
    return with_type(a.dtable_type, [&](auto t) {
      using D = decltype(d);
      using T = decltype(t);
      constexpr int N = 16 / sizeof(D);
      auto go = [&](auto w) {
        constexpr int W = decltype(w)::value;
        const int64_t chunks = (a.H + 32 * N - 1) / (32 * N), units = (a.n + a.window - 1) / a.window * chunks;
        const int64_t clears = a.accumulate ? 0 : (a.V + kClear - 1) / kClear;
        return launch_early(embed_sum_kernel<D, T, W>, dim3((unsigned)((units + 7) / 8 + clears)), 256, 0, st, a, a.key[last], a.tok[last], chunks, clears);
      };
      auto fits = [&](int W) {
        return a.H % W == 0 && fits_pieces(a.dy, a.dy_stride, a.dy_type, W) && fits_pieces(a.dtable, a.dtable_stride, a.dtable_type, W);
      };
      return fits(N) ? go(Int<N>{}) : fits(2) ? go(Int<2>{}) : go(Int<1>{});
    });
  });
}

cudaError_t launch_embed_join(const EmbedGradArgs &a, cudaStream_t st) {
  const int last = (sort_passes(a.V) + 1) & 1;
  return with_type(a.dtable_type, [&](auto t) {
    using T = decltype(t);
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      const int64_t chunks = (a.H + 32 * W - 1) / (32 * W), units = (a.n + a.window - 1) / a.window * chunks;
      return launch_early(embed_join_kernel<T, W>, dim3((unsigned)((units + 7) / 8)), 256, 0, st, a, a.key[last], chunks);
    };
    return a.H % 4 == 0 && fits_pieces(a.dtable, a.dtable_stride, a.dtable_type, 4) ? go(Int<4>{}) : go(Int<1>{});
  });
}

}  // namespace echo
