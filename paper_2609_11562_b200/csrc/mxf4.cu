// Rows to 4-bit floats with a power-of-two scale per 32 elements, and back (entwine_quant_mxf4, entwine_dequant_mxf4).
#include <cuda_fp4.h>

#include <algorithm>
#include <cstring>

#include "ops_common.cuh"

namespace entwine {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;  // elements that share a scale
constexpr int64_t kMaxRows = 2147483647;
constexpr int64_t kMaxCols = 2147483647 - 65536;  // column numbers of a CTA's last, idle threads fit 32 bits

struct Params {
  void* x;         // values, read or written
  uint8_t* q;      // codes, two a byte
  uint8_t* scale;  // scale bytes
  int64_t rows, ldx, ldq, lds;
  int cols, row_threads;
};

// Eight elements of a row of `cols`, zeros behind its end.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int left, float (&f)[8]) {
  if (VEC && left >= 8) {
    constexpr int V = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
      float g[V];
      unpack<T, V>(reinterpret_cast<const Piece<T, V>*>(p)[i], g);
#pragma unroll
      for (int e = 0; e < V; ++e) f[i * V + e] = g[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = e < left ? Elem<T>::up(p[e]) : 0.0f;
  }
}

// Two values as codes, the first in the low half: to the nearest, ties to the even code, the largest where above it.
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  return uint32_t(__nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest));
}

// Four lanes have a block: its largest magnitude's exponent, two less, is the scale's (6 = 1.5 * 2^2 is the largest
// code).  The product with the inverse power of two is exact as far as the rounding to a code can see.
template <typename T, int P, bool VEC>
__global__ void __launch_bounds__(kThreads) quant_mxf4_kernel(const Params a) {
  const int slot = int(threadIdx.x) / a.row_threads, lane = int(threadIdx.x) - slot * a.row_threads;
  const int64_t row = int64_t(blockIdx.x) * (blockDim.x / a.row_threads) + slot;
  const bool there = row < a.rows;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  uint8_t* const q = a.q + row * a.ldq;
  uint8_t* const scale = a.scale + row * a.lds;
  const int step = 8 * P * a.row_threads, cols = there ? a.cols : 0;
  // (whole warps go through the loop together: they vote on the blocks' scales)
  for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
    const int c0 = int(base);
    float f[P][8];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * a.row_threads + lane);
      load8<T, VEC>(x + at, max(cols - at, 0), f[i]);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * a.row_threads + lane);
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[i][e]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2)) >> 23;
      if (at >= cols) continue;
      const bool fine = top < 255;
      const uint32_t byte = fine ? (top > 2 ? top - 2 : 0) : 255;
      const float up = __uint_as_float((254 - byte) << 23);
      uint32_t w = 0;
      if (fine) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) w |= codes2(f[i][e] * up, f[i][e + 1] * up) << (4 * e);
      }
      if (at % kBlock == 0) scale[at / kBlock] = uint8_t(byte);
      if (VEC && at + 8 <= a.cols) {
        *reinterpret_cast<uint32_t*>(q + at / 2) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          if (at + e < a.cols) q[(at + e) / 2] = uint8_t(w >> (4 * e));
      }
    }
  }
}

template <typename T, int P, bool VEC>
__global__ void __launch_bounds__(kThreads) dequant_mxf4_kernel(const Params a) {
  const int slot = int(threadIdx.x) / a.row_threads, lane = int(threadIdx.x) - slot * a.row_threads;
  const int64_t row = int64_t(blockIdx.x) * (blockDim.x / a.row_threads) + slot;
  if (row >= a.rows) return;
  T* const x = static_cast<T*>(a.x) + row * a.ldx;
  const uint8_t* const q = a.q + row * a.ldq;
  const uint8_t* const scale = a.scale + row * a.lds;
  const int step = 8 * P * a.row_threads;
  for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
    const int c0 = int(base);
    uint32_t w[P], byte[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * a.row_threads + lane);
      w[i] = byte[i] = 0;
      if (at < a.cols) {
        byte[i] = scale[at / kBlock];
        if (VEC && at + 8 <= a.cols) {
          w[i] = *reinterpret_cast<const uint32_t*>(q + at / 2);
        } else {
#pragma unroll
          for (int e = 0; e < 8; e += 2)
            if (at + e < a.cols) w[i] |= uint32_t(q[(at + e) / 2]) << (4 * e);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * a.row_threads + lane);
      if (at >= a.cols) continue;
      // 2^(byte-127); 2^-127 is half of the least normal number, 255 stands for NaN
      const float s = __uint_as_float(byte[i] == 255 ? 0x7fffffffu : byte[i] ? byte[i] << 23 : 0x00400000u);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2(__nv_fp4x2_storage_t((w[i] >> (4 * e)) & 0xff), __NV_E2M1);
        const float2 d = __half22float2(__half2(h));
        f[e] = d.x * s;
        f[e + 1] = d.y * s;
      }
      if (VEC && at + 8 <= a.cols) {
        constexpr int V = 16 / sizeof(T);
#pragma unroll
        for (int j = 0; j < 8 / V; ++j) {
          float g[V];
#pragma unroll
          for (int e = 0; e < V; ++e) g[e] = f[j * V + e];
          reinterpret_cast<Piece<T, V>*>(x + at)[j] = pack<T, V>(g);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < a.cols) x[at + e] = Elem<T>::down(f[e]);
      }
    }
  }
}

template <typename T, int P>
int run_by(Params a, bool back, bool vec, cudaStream_t stream) {
  const int64_t groups = (int64_t(a.cols) + 7) / 8;
  // whole warps of a row's threads where a row has that much
  a.row_threads = int(std::min<int64_t>(kThreads, (groups + P * 32 - 1) / (P * 32) * 32));
  while (a.row_threads > 4 && a.row_threads / 2 * P >= groups) a.row_threads /= 2;
  const int per_cta = kThreads / a.row_threads;
  const int64_t chunks = (groups + P * a.row_threads - 1) / (P * a.row_threads);
  const dim3 grid(unsigned((a.rows + per_cta - 1) / per_cta), unsigned(std::min<int64_t>(chunks, 65535)));
  auto kernel = back ? (vec ? dequant_mxf4_kernel<T, P, true> : dequant_mxf4_kernel<T, P, false>)
                     : (vec ? quant_mxf4_kernel<T, P, true> : quant_mxf4_kernel<T, P, false>);
  kernel<<<grid, per_cta * a.row_threads, 0, stream>>>(a);
  return launched(cudaSuccess);
}

template <typename T>
int run(const Params& a, bool back, cudaStream_t stream) {
  const bool vec = aligned_rows(a.x, a.ldx, sizeof(T)) && aligned_rows(a.q, a.ldq, 1, 4);
  // little work: one group a thread, for the latency
  return a.rows * int64_t(a.cols) < (1 << 20) ? run_by<T, 1>(a, back, vec, stream) : run_by<T, 4>(a, back, vec, stream);
}

int convert(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* q, int64_t ldq,
            const void* scale, int64_t lds, bool back, void* stream) {
  if (dtype != ENTWINE_BF16 && dtype != ENTWINE_FP16 && dtype != ENTWINE_FP32) return ENTWINE_ERR_INVALID;
  if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols || ldx < cols || ldq < (cols + 1) / 2 ||
      lds < (cols + kBlock - 1) / kBlock)
    return ENTWINE_ERR_INVALID;
  if (rows == 0) return ENTWINE_OK;
  if (bad_pointer(x, dtype == ENTWINE_FP32 ? 4 : 2) || bad_pointer(q, 1) || bad_pointer(scale, 1)) return ENTWINE_ERR_INVALID;
  Params a;
  std::memset(&a, 0, sizeof(a));
  a.x = const_cast<void*>(x);
  a.q = static_cast<uint8_t*>(const_cast<void*>(q));
  a.scale = static_cast<uint8_t*>(const_cast<void*>(scale));
  a.rows = rows;
  a.ldx = ldx;
  a.ldq = ldq;
  a.lds = lds;
  a.cols = int(cols);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return run<__nv_bfloat16>(a, back, s);
    case ENTWINE_FP16: return run<__half>(a, back, s);
    default: return run<float>(a, back, s);
  }
}

}  // namespace
}  // namespace entwine

using namespace entwine;

extern "C" {

int entwine_quant_mxf4(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq, void* scale,
                       int64_t lds, void* stream) {
  return convert(x, dtype, rows, cols, ldx, q, ldq, scale, lds, false, stream);
}

int entwine_dequant_mxf4(const void* q, int64_t ldq, const void* scale, int64_t lds, int64_t rows, int64_t cols, void* x,
                         int dtype, int64_t ldx, void* stream) {
  return convert(x, dtype, rows, cols, ldx, q, ldq, scale, lds, true, stream);
}

}  // extern "C"
