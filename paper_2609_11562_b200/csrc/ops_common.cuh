// What the operators beside the fused call share: element types, 16-byte pieces of a row, launch checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "entwine_ops.h"

namespace entwine {

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};
template <>
struct Elem<float> {
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};

// V consecutive elements moved as one access: 16 bytes, or a single element where a row does not start on a
// 16-byte boundary.
template <typename T, int V>
struct alignas(sizeof(T) * V) Piece {
  T e[V];
};

inline bool aligned_rows(const void* p, int64_t ld, int64_t elem_bytes, int64_t bytes = 16) {
  return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0 && (ld * elem_bytes) % bytes == 0;
}

// an element pointer that may be null only where there is nothing behind it
inline bool bad_pointer(const void* p, int64_t elem_bytes) {
  return p == nullptr || reinterpret_cast<uintptr_t>(p) % uintptr_t(elem_bytes) != 0;
}

inline int launched(cudaError_t e) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e == cudaSuccess) return ENTWINE_OK;
  cudaGetLastError();
  return ENTWINE_ERR_CUDA;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace entwine
