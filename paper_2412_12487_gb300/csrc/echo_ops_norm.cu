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

// -- forward -----------------------------------------------------------------------------------
// A row stays in the registers of blockDim.x threads, E elements each, between its mean, the
// sum of its squared distances from it, and its output: x is read once.  Bound by the bytes.
template <typename X, int W, int E>
__global__ void __launch_bounds__(1024) layer_norm_kernel(NormArgs a) {
  constexpr int K = E / W;
  __shared__ float sh[2][32];
  const float over_h = 1.f / (float)a.H;
  for (int64_t row0 = (int64_t)blockIdx.x * blockDim.y; row0 < a.rows; row0 += (int64_t)gridDim.x * blockDim.y) {
    const int64_t row = row0 + threadIdx.y;
    const bool live = row < a.rows;
    const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
    float v[K][W];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t j = ((int64_t)k * blockDim.x + threadIdx.x) * W;
#pragma unroll
      for (int i = 0; i < W; ++i) v[k][i] = 0.f;
      if (live && j < a.H) load_piece<W>(x + j, v[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < W; ++i) s += v[k][i];
    const float mean = row_sum(s, sh[0]) * over_h;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool in = ((int64_t)k * blockDim.x + threadIdx.x) * W < a.H;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        v[k][i] -= mean;
        s += in ? v[k][i] * v[k][i] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(row_sum(s, sh[1]) * over_h + a.eps);
    if (!live) continue;
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    X *y = static_cast<X *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t j = ((int64_t)k * blockDim.x + threadIdx.x) * W;
      if (j >= a.H) continue;
      float w[W], b[W];
      load_param<W>(a.w, a.p_type, j, 1.f, w);
      load_param<W>(a.b, a.p_type, j, 0.f, b);
#pragma unroll
      for (int i = 0; i < W; ++i) v[k][i] = v[k][i] * rstd * w[i] + b[i];
      store_piece<W>(y + j, v[k]);
    }
  }
}

// Rows too long for registers: three passes over the row, a block each.
template <typename X, int W>
__global__ void __launch_bounds__(1024) layer_norm_long_kernel(NormArgs a) {
  __shared__ float sh[2][32];
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
// dx, a block a row: the row's two sums, then its elements.
template <typename X, int W>
__global__ void __launch_bounds__(1024) layer_norm_grad_rows_kernel(NormGradArgs a) {
  __shared__ float sh[4][32];
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

// Partial sums of dweight and dbias: a block takes blockDim.x * W columns of one part of the rows.
template <typename X, int W>
__global__ void __launch_bounds__(128) layer_norm_grad_columns_kernel(NormGradArgs a) {
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
// the parts in turn, then the warps' sums in order.
constexpr int kJoinWarps = 16;

__global__ void __launch_bounds__(kJoinWarps * 32) layer_norm_grad_join_kernel(NormGradArgs a) {
  __shared__ float sh[kJoinWarps][33];
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

}  // namespace

cudaError_t launch_layer_norm(const NormArgs &a, int sms, cudaStream_t st) {
  return with_type(a.x_type, [&](auto t) {
    using X = decltype(t);
    return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.y, a.y_stride}}, a.x_type, {a.w, a.b}, a.p_type, [&](auto wide) {
      constexpr int W = decltype(wide)::value;
      if (a.H > 1024 * 32) {
        layer_norm_long_kernel<X, W><<<(unsigned)std::min<int64_t>(a.rows, sms * 2), 1024, 0, st>>>(a);
        return cudaGetLastError();
      }
      auto go = [&](auto each) {
        constexpr int E = decltype(each)::value;
        const int x = row_threads(a.H, E);
        const dim3 block(x, std::max(1, 128 / x));
        const int64_t grid = std::min<int64_t>((a.rows + block.y - 1) / block.y, INT32_MAX);
        layer_norm_kernel<X, W, E><<<(unsigned)grid, block, 0, st>>>(a);
        return cudaGetLastError();
      };
      return a.H <= 2048 ? go(Int<8>{}) : a.H <= 8192 ? go(Int<16>{}) : go(Int<32>{});
    });
  });
}

int layer_norm_grad_parts(int64_t rows, int64_t H, int x_type, int sms) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({rows / 8, (int64_t)sms, 65535}));
}

cudaError_t launch_layer_norm_grad_rows(const NormGradArgs &a, int sms, cudaStream_t st) {
  return with_type(a.x_type, [&](auto t) {
    using X = decltype(t);
    return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dx, a.dx_stride}}, a.x_type, {a.w}, a.p_type, [&](auto wide) {
      constexpr int W = decltype(wide)::value;
      layer_norm_grad_rows_kernel<X, W><<<(unsigned)std::min<int64_t>(a.rows, INT32_MAX), row_threads(a.H, 8), 0, st>>>(a);
      return cudaGetLastError();
    });
  });
}

cudaError_t launch_layer_norm_grad_columns(const NormGradArgs &a, cudaStream_t st) {
  return with_type(a.x_type, [&](auto t) {
    using X = decltype(t);
    return with_pieces<X>(a.H, {{a.x, a.x_stride}, {a.dy, a.dy_stride}}, a.x_type, {}, a.p_type, [&](auto wide) {
      constexpr int W = decltype(wide)::value;
      const int64_t cols = 128 * W;
      layer_norm_grad_columns_kernel<X, W><<<dim3((unsigned)((a.H + cols - 1) / cols), a.parts), 128, 0, st>>>(a);
      return cudaGetLastError();
    });
  });
}

cudaError_t launch_layer_norm_grad_join(const NormGradArgs &a, cudaStream_t st) {
  layer_norm_grad_join_kernel<<<(unsigned)((2 * a.H + 31) / 32), dim3(32, kJoinWarps), 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace echo
