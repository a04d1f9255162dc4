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
// out[t] = scale * table[row of t], zeros without one.  Bound by the bytes read and written.
// A thread takes kLookup pieces of one row; their loads are in flight together.
constexpr int kLookup = 4;

template <typename T, typename O, int W>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, int64_t pieces, int64_t steps) {
  const T *table = static_cast<const T *>(a.table);
  O *out = static_cast<O *>(a.out);
  for (int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; t < a.n; t += (int64_t)gridDim.x * blockDim.y) {
    const int64_t row = shard_row(a.ids, a.id64, t, a.v0, a.V);
    for (int64_t s = blockIdx.y; s < steps; s += gridDim.y) {
      const int64_t p0 = s * kLookup * blockDim.x + threadIdx.x;
      float f[kLookup][W];
#pragma unroll
      for (int k = 0; k < kLookup; ++k) {
        const int64_t p = p0 + k * (int)blockDim.x;
#pragma unroll
        for (int i = 0; i < W; ++i) f[k][i] = 0.f;
        if (row >= 0 && p < pieces) load_piece<W>(table + row * a.table_stride + p * W, f[k]);
      }
#pragma unroll
      for (int k = 0; k < kLookup; ++k) {
        const int64_t p = p0 + k * (int)blockDim.x;
#pragma unroll
        for (int i = 0; i < W; ++i) f[k][i] = row >= 0 ? f[k][i] * a.scale : 0.f;
        if (p < pieces) store_piece<W>(out + t * a.out_stride + p * W, f[k]);
      }
    }
  }
}

// -- gradient: tokens sorted by row ------------------------------------------------------------
// A stable radix sort, 8 bits a pass, by one cluster of 8 blocks: 256 warps each own a
// contiguous range of the tokens.  A pass counts each warp's digits, takes the running sum
// over (digit, block, warp) with the blocks' totals exchanged through distributed shared
// memory, and places each token behind those before it.  The order of equal rows is the
// tokens', so the sums' order is fixed.  Bound by the latency of its steps: one token a
// thread up to 8192 tokens.
constexpr int kSortBlocks = 8, kSortWarps = 32;

__global__ void __cluster_dims__(kSortBlocks) __launch_bounds__(kSortWarps * 32) embed_sort_kernel(EmbedGradArgs a, int passes) {
  __shared__ int32_t cnt[kSortWarps][256];
  __shared__ int32_t tot[256];
  __shared__ int32_t sums[8];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned below = (1u << lane) - 1;
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
    for (int i = tid; i < kSortWarps * 256; i += blockDim.x) cnt[0][i] = 0;
    __syncthreads();
    for (int64_t i = begin; i < end; i += 32) {
      const int64_t key = key_at(i + lane);
      const int digit = key < 0 ? 256 : (int)(key >> (8 * pass)) & 255;
      const unsigned same = __match_any_sync(0xFFFFFFFFu, digit);
      if (key >= 0 && !(same & below)) cnt[warp][digit] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (tid < 256) {
      int32_t run = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const int32_t c = cnt[w][tid];
        cnt[w][tid] = run;
        run += c;
      }
      tot[tid] = run;
    }
    cluster.sync();
    int32_t all = 0, before = 0, upto = 0;
    if (tid < 256) {
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
    if (tid < 256) {
      for (int w = 0; w < warp; ++w) upto += sums[w];
      for (int w = 0; w < kSortWarps; ++w) cnt[w][tid] += upto - all + before;
    }
    int64_t total = 0;
    for (int w = 0; w < 8; ++w) total += sums[w];
    __syncthreads();
    for (int64_t i = begin; i < end; i += 32) {
      const int64_t key = key_at(i + lane);
      const int digit = key < 0 ? 256 : (int)(key >> (8 * pass)) & 255;
      const unsigned same = __match_any_sync(0xFFFFFFFFu, digit);
      if (key >= 0) {
        const int64_t at = cnt[warp][digit] + __popc(same & below);
        key_out[at] = (uint32_t)key;
        tok_out[at] = pass == 0 ? (uint32_t)(i + lane) : __ldcg(tok_in + i + lane);
      }
      __syncwarp();
      if (key >= 0 && !(same & below)) cnt[warp][digit] += __popc(same);
      __syncwarp();
    }
    __threadfence();
    cluster.sync();  // (the other blocks' tokens, and their reads of `tot`)
    n = total;
  }
  if (rank == 0 && tid == 0) *a.count = (int32_t)n;
}

// -- gradient: sums ----------------------------------------------------------------------------
// The sorted tokens are cut into windows of a.window; a warp sums one window over 32 * kWide
// columns, so that every warp has the same work however the tokens fall on the rows.  A row
// that lies inside a window is written at once; the part of a row that a window's edge cuts
// goes to `part` ([window][0: began before it, 1: began in it][H]) and embed_join_kernel adds
// the parts in order.  Bound by the bytes of dy and of the rows.
constexpr int kBatch = 8;  // rows of dy in flight

template <typename D, typename T, int W>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedGradArgs a, const uint32_t *key, const uint32_t *tok, int64_t chunks) {
  constexpr int N = 16 / sizeof(D), K = N / W;  // columns of a lane, in K pieces
  const int lane = threadIdx.x & 31;
  const int64_t unit = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int64_t w0 = unit / chunks * a.window, col0 = unit % chunks * (32 * N) + lane * W;
  const int64_t count = *a.count;
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

// Rows that windows cut: the warp of the window in which the row begins adds its parts.
template <typename T, int W>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedGradArgs a, const uint32_t *key, int64_t chunks) {
  const int lane = threadIdx.x & 31;
  const int64_t unit = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int64_t w = unit / chunks, j = unit % chunks * (32 * W) + lane * W;
  const int64_t count = *a.count, P = a.window;
  if ((w + 1) * P >= count) return;
  const uint32_t row = key[(w + 1) * P - 1];
  if (key[(w + 1) * P] != row || (w > 0 && key[w * P - 1] == row)) return;  // no row begins here and is cut
  int64_t lo = w + 1, hi = (count - 1) / P;  // the last window that begins with this row
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) / 2;
    if (key[mid * P] == row) lo = mid;
    else hi = mid - 1;
  }
  if (j >= a.H) return;
  float acc[W];
  load_piece<W>(a.part + (w * 2 + 1) * a.H + j, acc);
#pragma unroll 4
  for (int64_t u = w + 1; u <= lo; ++u) {
    float f[W];
    load_piece<W>(a.part + u * 2 * a.H + j, f);
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] += f[i];
  }
  T *at = static_cast<T *>(a.dtable) + row * a.dtable_stride + j;
  float old[W];
  if (a.accumulate) load_piece<W>(at, old);
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = acc[i] * a.scale + (a.accumulate ? old[i] : 0.f);
  store_piece<W>(at, acc);
}

// Zeros to every row, before the rows of tokens are written.
template <typename T, int W>
__global__ void __launch_bounds__(256) embed_clear_kernel(EmbedGradArgs a, int64_t pieces) {
  const float zero[W] = {};
  T *dtable = static_cast<T *>(a.dtable);
  for (int64_t v = blockIdx.x; v < a.V; v += gridDim.x)
    for (int64_t p = threadIdx.x; p < pieces; p += blockDim.x) store_piece<W>(dtable + v * a.dtable_stride + p * W, zero);
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
        const int64_t pieces = a.H / W;
        int x = 32;
        while (x < 256 && x * kLookup < pieces) x *= 2;
        const int64_t steps = (pieces + (int64_t)x * kLookup - 1) / ((int64_t)x * kLookup);
        const dim3 block(x, 256 / x);
        const int64_t gx = std::min<int64_t>((a.n + block.y - 1) / block.y, INT32_MAX);
        embed_kernel<T, O, W><<<dim3((unsigned)gx, (unsigned)std::min<int64_t>(steps, 65535)), block, 0, st>>>(a, pieces, steps);
        return cudaGetLastError();
      };
      auto fits = [&](int W) {
        return a.H % W == 0 && fits_pieces(a.table, a.table_stride, a.table_type, W) && fits_pieces(a.out, a.out_stride, a.out_type, W);
      };
      return fits(N) ? go(Int<N>{}) : fits(2) ? go(Int<2>{}) : go(Int<1>{});
    });
  });
}

int embed_grad_window(int64_t n, int64_t H, int sms) {
  int P = 8;
  while (P < 32 && n / P * ((H + 255) / 256) > (int64_t)sms * 32) P *= 2;
  return P;
}

cudaError_t launch_embed_sort(const EmbedGradArgs &a, cudaStream_t st) {
  embed_sort_kernel<<<kSortBlocks, kSortWarps * 32, 0, st>>>(a, sort_passes(a.V));
  return cudaGetLastError();
}

cudaError_t launch_embed_clear(const EmbedGradArgs &a, int sms, cudaStream_t st) {
  return with_type(a.dtable_type, [&](auto t) {
    using T = decltype(t);
    constexpr int N = 16 / sizeof(T);
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      embed_clear_kernel<T, W><<<(unsigned)std::min<int64_t>(a.V, sms * 8), 256, 0, st>>>(a, a.H / W);
      return cudaGetLastError();
    };
    return a.H % N == 0 && fits_pieces(a.dtable, a.dtable_stride, a.dtable_type, N) ? go(Int<N>{}) : go(Int<1>{});
  });
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
        embed_sum_kernel<D, T, W><<<(unsigned)((units + 7) / 8), 256, 0, st>>>(a, a.key[last], a.tok[last], chunks);
        return cudaGetLastError();
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
      embed_join_kernel<T, W><<<(unsigned)((units + 7) / 8), 256, 0, st>>>(a, a.key[last], chunks);
      return cudaGetLastError();
    };
    return a.H % 4 == 0 && fits_pieces(a.dtable, a.dtable_stride, a.dtable_type, 4) ? go(Int<4>{}) : go(Int<1>{});
  });
}

}  // namespace echo
