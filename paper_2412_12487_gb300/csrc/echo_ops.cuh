// echo_ops.cuh -- element types, pieces of rows and sums over threads, for the operators'
// kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>
#include <cstring>
#include <type_traits>

#include "echo.h"

namespace echo {

// Every kernel of the operators is launched early: its blocks may take their places while the
// kernel before ends, and wait there until all of that one's results are to be read.  Each calls
// kernel_begin() before it touches memory, so the order of a stream holds whatever lies between
// (embedding 2048 tokens of 12288: 15.6 us a call in a row of them, 18.3 with plain launches).
// A kernel that says next_may_start() lets the next one's blocks come before its own have ended.
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const A &...args) {
  cudaLaunchConfig_t how{};
  how.gridDim = grid;
  how.blockDim = block;
  how.dynamicSmemBytes = smem;
  how.stream = st;
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  how.attrs = &early;
  how.numAttrs = 1;
  return cudaLaunchKernelEx(&how, kernel, P(args)...);
}
__device__ __forceinline__ void kernel_begin() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

// A piece: W consecutive elements of a row, at a multiple of the piece's size (16 bytes at
// most: a larger one is several loads).  Rows that cannot be cut into wide pieces (an odd
// length, stride or address) are cut into narrower ones; neighbouring threads always take
// neighbouring pieces.
template <typename T, int W>
struct alignas(sizeof(T) * W <= 16 ? sizeof(T) * W : 16) Pack {
  T v[W];
};
template <typename T, int W>
__device__ __forceinline__ void unpack(const Pack<T, W> p, float *f) {
  if constexpr (W % 2 == 0 && std::is_same_v<T, __nv_bfloat16>) {  // a bf16 is the upper half of its fp32
    uint32_t r[W / 2];
    memcpy(r, &p, sizeof r);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      f[2 * i] = __uint_as_float(r[i] << 16);
      f[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = to_f(p.v[i]);
  }
}
template <typename T, int W>
__device__ __forceinline__ Pack<T, W> pack(const float *f) {
  Pack<T, W> p;
  if constexpr (W % 2 == 0 && std::is_same_v<T, __nv_bfloat16>) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) reinterpret_cast<__nv_bfloat162 *>(p.v)[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  } else if constexpr (W % 2 == 0 && std::is_same_v<T, __half>) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) reinterpret_cast<__half2 *>(p.v)[i] = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) p.v[i] = from_f<T>(f[i]);
  }
  return p;
}
template <int W, typename T>
__device__ __forceinline__ void load_piece(const T *at, float *f) {
  const Pack<T, W> p = *reinterpret_cast<const Pack<T, W> *>(at);  // (as one piece)
  unpack<T, W>(p, f);
}
template <int W, typename T>
__device__ __forceinline__ void store_piece(T *at, const float *f) {
  *reinterpret_cast<Pack<T, W> *>(at) = pack<T, W>(f);
}

// Piece of a vector of parameters whose type is known at run time; `none` without one.
template <int W>
__device__ __forceinline__ void load_param(const void *p, int type, int64_t j, float none, float *f) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = none;
  } else if (type == ECHO_F32) {
    load_piece<W>(static_cast<const float *>(p) + j, f);
  } else if (type == ECHO_BF16) {
    load_piece<W>(static_cast<const __nv_bfloat16 *>(p) + j, f);
  } else {
    load_piece<W>(static_cast<const __half *>(p) + j, f);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Pairs of fp32 numbers: one instruction for both.
struct Pair {
  float a, b;
};
__device__ __forceinline__ uint64_t bits(Pair p) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(p.a), "f"(p.b));
  return r;
}
__device__ __forceinline__ Pair pair(uint64_t r) {
  Pair p;
  asm("mov.b64 {%0, %1}, %2;\n" : "=f"(p.a), "=f"(p.b) : "l"(r));
  return p;
}
__device__ __forceinline__ Pair both(float x) { return {x, x}; }
__device__ __forceinline__ Pair fma2(Pair x, Pair y, Pair z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(bits(x)), "l"(bits(y)), "l"(bits(z)));
  return pair(r);
}
__device__ __forceinline__ Pair add2(Pair x, Pair y) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(bits(x)), "l"(bits(y)));
  return pair(r);
}
__device__ __forceinline__ Pair mul2(Pair x, Pair y) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(bits(x)), "l"(bits(y)));
  return pair(r);
}

constexpr int type_bytes(int type) { return type == ECHO_F32 ? 4 : 2; }

// Whether rows `stride` elements apart can be read in pieces of W elements.
inline bool fits_pieces(const void *p, int64_t stride, int type, int W) {
  const int64_t a = std::min<int64_t>(16, (int64_t)type_bytes(type) * W);
  return reinterpret_cast<uintptr_t>(p) % a == 0 && stride * type_bytes(type) % a == 0;
}

// f(an element of the type)
template <typename F>
auto with_type(int type, F &&f) {
  if (type == ECHO_F32) return f(float{});
  if (type == ECHO_BF16) return f(__nv_bfloat16{});
  return f(__half{});
}
template <int I>
struct Int {
  static constexpr int value = I;
};

}  // namespace echo
