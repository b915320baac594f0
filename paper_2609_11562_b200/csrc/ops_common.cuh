// What the operators beside the fused call share: element types, 16-byte pieces of a row, launch checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstring>
#include <type_traits>

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

// V consecutive elements moved as one access.
template <typename T, int V>
struct alignas(sizeof(T) * V) Piece {
  T e[V];
};

// The elements of a piece in fp32.  16-bit ones are taken from the 32-bit words that hold two of them: element by
// element the compiler spends three instructions on each.
template <typename T, int V>
__device__ __forceinline__ void unpack(const Piece<T, V>& v, float (&f)[V]) {
  if constexpr (sizeof(T) == 2 && V >= 2) {
    uint32_t w[V / 2];
    memcpy(w, &v, sizeof(v));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        __half2 h;
        memcpy(&h, &w[i], 4);
        const float2 d = __half22float2(h);
        f[2 * i] = d.x;
        f[2 * i + 1] = d.y;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = Elem<T>::up(v.e[e]);
  }
}

// fp32 values rounded to a piece, two at a time.
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> pack(const float (&f)[V]) {
  Piece<T, V> o;
  if constexpr (sizeof(T) == 2 && V >= 2) {
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        memcpy(&w[i], &h, 4);
      } else {
        const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        memcpy(&w[i], &h, 4);
      }
    }
    memcpy(&o, w, sizeof(o));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = Elem<T>::down(f[e]);
  }
  return o;
}

// A piece that is read once, zeros where `there` is false.  As an instruction of its own, in order with its
// neighbours, so that a batch of them is in flight together whatever the compiler makes of the code around it.
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_if(const T* p, bool there) {
  static_assert(sizeof(T) * V == 16, "sixteen bytes");
  uint4 w;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=&r"(w.x), "=&r"(w.y), "=&r"(w.z), "=&r"(w.w)
      : "l"(p), "r"(int(there)));
  Piece<T, V> v;
  memcpy(&v, &w, 16);
  return v;
}

// Memory that may be read: a matrix from its first element to its last.
struct Span {
  uintptr_t lo, hi;
};
template <typename T>
__host__ __device__ __forceinline__ Span span_of(const T* p, int64_t rows, int64_t cols, int64_t ld) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, rows > 0 ? lo + uintptr_t(((rows - 1) * ld + cols) * int64_t(sizeof(T))) : lo};
}

// Sixteen bytes of elements that start anywhere in a matrix: the two aligned words around them, put together by byte
// shifts.  What lies around the elements is read only inside the matrix (another row, or the space between rows);
// at its very ends, where alone() is true, the elements are read one by one.
template <typename T>
struct Anywhere {
  static constexpr int V = 16 / sizeof(T);
  uint4 a, b;
  uint32_t shift;

  static __device__ __forceinline__ bool alone(const T* p, const Span& inside) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~uintptr_t(15);
    return base < inside.lo || base + (at == base ? 16 : 32) > inside.hi;
  }
  // Both words, zeros where `there` is false; instructions of their own, so that those of a batch are in flight together.
  __device__ __forceinline__ void fetch(const T* p, bool there) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~uintptr_t(15);
    shift = uint32_t(at & 15);
    a = word(base, there);
    b = word(base + 16, there && shift != 0);
  }
  __device__ __forceinline__ Piece<T, V> get() const {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = shift & 4 ? w[i + 1] : w[i];
    const uint32_t bits = (shift & 3) * 8;
    const uint4 o = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                               __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
    Piece<T, V> v;
    memcpy(&v, &o, 16);
    return v;
  }
  static __device__ __forceinline__ Piece<T, V> one_by_one(const T* p) {
    Piece<T, V> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = p[e];
    return v;
  }
  // One piece by itself.
  static __device__ __forceinline__ Piece<T, V> load(const T* p, const Span& inside) {
    if (alone(p, inside)) return one_by_one(p);
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~uintptr_t(15);
    Anywhere<T> v;
    v.shift = uint32_t(at & 15);
    v.a = *reinterpret_cast<const uint4*>(base);
    v.b = v.shift ? *reinterpret_cast<const uint4*>(base + 16) : v.a;
    return v.get();
  }

 private:
  static __device__ __forceinline__ uint4 word(uintptr_t at, bool there) {
    uint4 w;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(w.x), "=&r"(w.y), "=&r"(w.z), "=&r"(w.w)
        : "l"(at), "r"(int(there)));
    return w;
  }
};

// How a row that starts anywhere falls into aligned 16-byte pieces: `head` elements before the first of them, `pieces`
// of them, and the rest of H elements behind.
template <typename T>
struct Cut {
  int64_t head, pieces, ends;  // ends: elements outside the pieces
  __device__ __forceinline__ Cut(const T* row, int64_t H) {
    constexpr int V = 16 / sizeof(T);
    head = min(int64_t((16 - reinterpret_cast<uintptr_t>(row) % 16) % 16 / sizeof(T)), H);
    pieces = (H - head) / V;
    ends = H - pieces * V;
  }
  // element number of the i-th one outside the pieces
  __device__ __forceinline__ int64_t end(int64_t i) const { return i < head ? i : i + pieces * (16 / sizeof(T)); }
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

// SMs of the current device (148 where that cannot be told).
inline int sm_count() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace entwine
