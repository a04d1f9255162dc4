// echo_ops_ortho.cu -- orthogonalised updates by Newton-Schulz products.
#include <algorithm>

#include "echo_ops.cuh"
#include "echo_ops.h"

namespace echo {

namespace {

// -- Frobenius norm ------------------------------------------------------------------------------
// Sums of squares of x, of 2^-60 x and of 2^60 x: one of them neither overflows nor underflows,
// whatever the size of the elements.  A block sums a part of one matrix.
constexpr int kNormParts = 64;

template <typename T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(OrthoArgs a, int64_t rows, int64_t cols, float *part) {
  __shared__ float sh[3][8];
  const float up = 0x1p60f, down = 0x1p-60f;
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    float s[3] = {0.f, 0.f, 0.f};
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
      const T *g = static_cast<const T *>(a.g) + z * a.g_batch_stride + r * a.g_stride;
      for (int64_t j = threadIdx.x; j < cols; j += blockDim.x) {
        const float v = to_f(g[j]), lo = v * up, hi = v * down;
        s[0] += v * v;
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
      part[(z * kNormParts + blockIdx.x) * 3 + threadIdx.x] = t;
    }
    __syncthreads();
  }
}

// 1 / (|G| + eps) of a matrix, from the parts of its sums of squares.
__device__ double inverse_norm(const float *part, int64_t z, float eps) {
  double s[3] = {0., 0., 0.};
  for (int p = 0; p < kNormParts; ++p)
    for (int q = 0; q < 3; ++q) s[q] += part[(z * kNormParts + p) * 3 + q];
  // (the plain sum unless it is near the ends of the fp32 range; a NaN stays one)
  const double norm = s[0] > 1e30 ? sqrt(s[1]) * 0x1p60 : s[0] < 1e-24 ? sqrt(s[2]) * 0x1p-60 : sqrt(s[0]);
  return 1. / (norm + (double)eps);
}

// X = G / (|G| + eps) in fp32, [m][n]
template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(OrthoArgs a, const float *part, float *X) {
  __shared__ double inv;
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    __syncthreads();
    if (threadIdx.x == 0) inv = inverse_norm(part, z, a.eps);
    __syncthreads();
    const T *g = static_cast<const T *>(a.g) + z * a.g_batch_stride;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < a.m * a.n; i += (int64_t)gridDim.x * blockDim.x) {
      const int64_t r = i / a.n, c = i % a.n;
      X[z * a.m * a.n + i] = (float)((double)to_f(a.tall ? g[c * a.g_stride + r] : g[r * a.g_stride + c]) * inv);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) ortho_finish_kernel(OrthoArgs a, const float *X) {
  for (int64_t z = blockIdx.y; z < a.batch; z += gridDim.y) {
    T *o = static_cast<T *>(a.o) + z * a.o_batch_stride;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < a.m * a.n; i += (int64_t)gridDim.x * blockDim.x) {
      const int64_t r = i / a.n, c = i % a.n;
      o[a.tall ? c * a.o_stride + r : r * a.o_stride + c] = from_f<T>(a.scale * X[z * a.m * a.n + i]);
    }
  }
}

// D = alpha P Q + beta C of [M][K] and [K][N] (or Q transposed) matrices without gaps, 64 x 64 a block.
__global__ void __launch_bounds__(256) ortho_product_kernel(int64_t batch, int M, int N, int K, const float *P, const float *Q, bool q_transposed,
                                                            const float *C, float alpha, float beta, float *D) {
  __shared__ float sp[16][65], sq[16][65];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  for (int64_t z = blockIdx.z; z < batch; z += gridDim.z) {
    const float *p = P + z * M * K, *q = Q + z * N * K;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
      for (int i = threadIdx.x; i < 1024; i += 256) {
        const int r = i >> 4, k = i & 15;
        sp[k][r] = r0 + r < M && k0 + k < K ? p[(int64_t)(r0 + r) * K + k0 + k] : 0.f;
        if (q_transposed) {
          sq[k][r] = c0 + r < N && k0 + k < K ? q[(int64_t)(c0 + r) * K + k0 + k] : 0.f;
        } else {
          const int kk = i >> 6, c = i & 63;
          sq[kk][c] = c0 + c < N && k0 + kk < K ? q[(int64_t)(k0 + kk) * N + c0 + c] : 0.f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] += sp[k][ty + 16 * i] * sq[k][tx + 16 * j];
      __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int r = r0 + ty + 16 * i, c = c0 + tx + 16 * j;
        if (r >= M || c >= N) continue;
        const int64_t at = z * M * N + (int64_t)r * N + c;
        D[at] = alpha * acc[i][j] + (C ? beta * C[at] : 0.f);
      }
  }
}

}  // namespace

// norm parts; X, the next X, A, B in fp32
size_t ortho_scratch_bytes(const OrthoArgs &a, int) {
  return (size_t)a.batch * (kNormParts * 3 + 2 * a.m * a.n + 2 * a.m * a.m) * sizeof(float);
}

cudaError_t launch_orthogonalize(const OrthoArgs &a, int sms, const OpTimer &timed, cudaStream_t st) {
  float *X = static_cast<float *>(a.scratch), *X2 = X + a.batch * a.m * a.n, *A = X2 + a.batch * a.m * a.n, *B = A + a.batch * a.m * a.m;
  float *part = B + a.batch * a.m * a.m;
  const unsigned gz = (unsigned)std::min<int64_t>(a.batch, 65535);
  const int64_t rows = a.tall ? a.n : a.m, cols = a.tall ? a.m : a.n;
  cudaError_t e = timed("ortho_norm", [&] {
    return with_type(a.type, [&](auto t) {
      ortho_norm_kernel<decltype(t)><<<dim3(kNormParts, gz), 256, 0, st>>>(a, rows, cols, part);
      return cudaGetLastError();
    });
  });
  if (e != cudaSuccess) return e;
  const dim3 flat((unsigned)std::min<int64_t>((a.m * a.n + 255) / 256, sms * 8), gz);
  e = timed("ortho_start", [&] {
    return with_type(a.type, [&](auto t) {
      ortho_start_kernel<decltype(t)><<<flat, 256, 0, st>>>(a, part, X);
      return cudaGetLastError();
    });
  });
  const int m = (int)a.m, n = (int)a.n;
  auto product = [&](int N, int K, const float *P, const float *Q, bool qt, const float *C, float alpha, float beta, float *D) {
    return timed("ortho_product", [&] {
      ortho_product_kernel<<<dim3((N + 63) / 64, (m + 63) / 64, gz), 256, 0, st>>>(a.batch, m, N, K, P, Q, qt, C, alpha, beta, D);
      return cudaGetLastError();
    });
  };
  for (int s = 0; s < a.steps && e == cudaSuccess; ++s) {
    e = product(m, n, X, X, true, nullptr, 1.f, 0.f, A);
    if (e == cudaSuccess) e = product(m, m, A, A, true, A, a.c, a.b, B);
    if (e == cudaSuccess) e = product(n, m, B, X, false, X, 1.f, a.a, X2);
    std::swap(X, X2);
  }
  if (e != cudaSuccess) return e;
  return timed("ortho_finish", [&] {
    return with_type(a.type, [&](auto t) {
      ortho_finish_kernel<decltype(t)><<<flat, 256, 0, st>>>(a, X);
      return cudaGetLastError();
    });
  });
}

}  // namespace echo
