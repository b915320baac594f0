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
  int cols;
  int q_wide;      // rows of codes start on 8-byte boundaries (4, on the way back)
};

// Two values as codes, the first in the low half: to the nearest, ties to the even code, the largest where above it.
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  return uint32_t(__nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest));
}

// Sixteen elements of a row, zeros behind the row's end: as they lie in memory where they are whole and aligned, else put
// together from the aligned words around them, which are read inside the matrix only.
template <typename T, bool WHOLE>
struct Half {
  static constexpr int V = 16 / sizeof(T), N = 16 / V;
  Piece<T, V> v[N];
  __device__ __forceinline__ void load(const T* p, int left, const Span& inside) {
    if constexpr (WHOLE) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = left > i * V ? reinterpret_cast<const Piece<T, V>*>(p)[i] : Piece<T, V>{};
    } else if (left >= 16 && !Anywhere<T>::alone(p, inside) && !Anywhere<T>::alone(p + (N - 1) * V, inside)) {
      Anywhere<T> w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i].fetch(p + i * V, true);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = w[i].get();
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) v[i].e[e] = i * V + e < left ? p[i * V + e] : Elem<T>::down(0.0f);
    }
  }
  __device__ __forceinline__ uint32_t top() const {  // fp32 bits of the largest magnitude (infinity or above: not finite)
    if constexpr (sizeof(T) == 2) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint32_t w[4];
        memcpy(w, &v[i], 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __vmaxu2(m, w[j] & 0x7fff7fffu);
      }
      const uint16_t h = uint16_t(max(m & 0xffffu, m >> 16));
      T t;
      memcpy(&t, &h, 2);
      return __float_as_uint(Elem<T>::up(t));
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) m = max(m, __float_as_uint(v[i].e[e]) & 0x7fffffffu);
      return m;
    }
  }
  __device__ __forceinline__ uint2 codes(float up) const {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float f[V];
      unpack<T, V>(v[i], f);
#pragma unroll
      for (int e = 0; e < V; e += 2) w[(i * V + e) / 8] |= codes2(f[e] * up, f[e + 1] * up) << (4 * ((i * V + e) % 8));
    }
    return make_uint2(w[0], w[1]);
  }
};

// Two lanes have a block: its largest magnitude's exponent, two less, is the scale's (6 = 1.5 * 2^2 is the largest code).
// The product with the inverse power of two is exact as far as the rounding to a code can see.  Bound by its instructions,
// 92 for eight elements, beside the read of x: 4096 x 5120 bf16 take 14.4 us cold, 53 MB, 63 % of the issue slots (four lanes
// a block, of which each worked the scale out: 27 us).
template <typename T, int P, bool WHOLE>
__global__ void __launch_bounds__(kThreads) quant_mxf4_kernel(const Params a) {
  const int lane = int(threadIdx.x), width = int(blockDim.x);
  const int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
  const bool there = row < a.rows;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  uint8_t* const q = a.q + row * a.ldq;
  uint8_t* const scale = a.scale + row * a.lds;
  const int step = 16 * P * width, cols = there ? a.cols : 0;
  const Span inside = span_of(static_cast<const T*>(a.x), a.rows, a.cols, a.ldx);
  // (whole warps go through the loop together: they vote on the blocks' scales)
  for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
    const int c0 = int(base);
    Half<T, WHOLE> h[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 16 * (i * width + lane);
      h[i].load(x + at, cols - at, inside);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 16 * (i * width + lane);
      uint32_t top = h[i].top();
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1)) >> 23;
      if (at >= cols) continue;
      const bool fine = top < 255;
      const uint32_t byte = fine ? (top > 2 ? top - 2 : 0) : 255;
      uint2 w = h[i].codes(__uint_as_float((254 - byte) << 23));
      if (!fine) w = make_uint2(0, 0);
      if (at % kBlock == 0) scale[at / kBlock] = uint8_t(byte);
      if ((WHOLE || a.q_wide) && at + 16 <= cols) {
        *reinterpret_cast<uint2*>(q + at / 2) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 16; e += 2)
          if (at + e < cols) q[(at + e) / 2] = uint8_t((e < 8 ? w.x : w.y) >> (4 * (e % 8)));
      }
    }
  }
}

// 2^(byte-127); 2^-127 is half of the least normal number, 255 stands for NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 255 ? 0x7fffffffu : byte ? byte << 23 : 0x00400000u);
}
__device__ __forceinline__ float2 values2(uint32_t codes) {
  const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2(__nv_fp4x2_storage_t(codes), __NV_E2M1);
  return __half22float2(__half2(h));
}

// Groups of eight values, all of them whole and aligned: 16-byte stores side by side.  4096 x 5120 bf16 take 11.4 us cold, 77 %
// of the issue slots.
template <typename T, int P>
__global__ void __launch_bounds__(kThreads) dequant_mxf4_kernel(const Params a) {
  const int lane = int(threadIdx.x), width = int(blockDim.x);
  const int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= a.rows) return;
  T* const x = static_cast<T*>(a.x) + row * a.ldx;
  const uint8_t* const q = a.q + row * a.ldq;
  const uint8_t* const scale = a.scale + row * a.lds;
  const int step = 8 * P * width;
  for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
    const int c0 = int(base);
    uint32_t w[P], byte[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * width + lane);
      w[i] = byte[i] = 0;
      if (at < a.cols) {
        byte[i] = scale[at / kBlock];
        w[i] = *reinterpret_cast<const uint32_t*>(q + at / 2);
      }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * width + lane);
      if (at >= a.cols) continue;
      const float s = scale_of(byte[i]);
      constexpr int V = 16 / sizeof(T);
#pragma unroll
      for (int j = 0; j < 8 / V; ++j) {
        float g[V];
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float2 d = values2((w[i] >> (4 * (j * V + e))) & 0xff);
          g[e] = d.x * s;
          g[e + 1] = d.y * s;
        }
        reinterpret_cast<Piece<T, V>*>(x + at)[j] = pack<T, V>(g);
      }
    }
  }
}

// Rows that start anywhere: a warp has 256 columns at a time, and a lane stores eight of them 32 apart, so that its stores
// lie beside its neighbours'.  Codes and scale of a column come from the lane that has read those of its group of eight.
template <typename T, int P>
__global__ void __launch_bounds__(kThreads) dequant_mxf4_anywhere_kernel(const Params a) {
  const int lane = int(threadIdx.x), width = int(blockDim.x);
  const int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= a.rows) return;
  T* const x = static_cast<T*>(a.x) + row * a.ldx;
  const uint8_t* const q = a.q + row * a.ldq;
  const uint8_t* const scale = a.scale + row * a.lds;
  const int step = 8 * P * width;
  for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
    const int c0 = int(base);
    uint32_t w[P], byte[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = c0 + 8 * (i * width + lane);
      w[i] = byte[i] = 0;
      if (at < a.cols) {
        byte[i] = scale[at / kBlock];
        if (a.q_wide && at + 8 <= a.cols) {
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
      const int first = c0 + 8 * (i * width + (lane & ~31)) + (lane & 31);
      const float s = scale_of(byte[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int from = 4 * e + (lane & 31) / 8;
        const uint32_t code = __shfl_sync(0xffffffffu, w[i], from) >> (4 * (lane & 7)) & 15;
        const float v = values2(code).x * __shfl_sync(0xffffffffu, s, from);
        if (first + 32 * e < a.cols) x[first + 32 * e] = Elem<T>::down(v);
      }
    }
  }
}

// Threads of a row and rows of a CTA: whole warps of a row's threads where a row has that many pieces.
template <int P>
dim3 shape(int64_t pieces, int least) {
  int width = int(std::min<int64_t>(kThreads, (pieces + P * 32 - 1) / (P * 32) * 32));
  while (width > least && width / 2 * P >= pieces) width /= 2;
  return dim3(unsigned(width), unsigned(kThreads / width));
}
dim3 grid_of(const Params& a, const dim3& block, int64_t per_chunk) {
  const int64_t chunks = (a.cols + per_chunk - 1) / per_chunk;
  return dim3(unsigned((a.rows + block.y - 1) / block.y), unsigned(std::min<int64_t>(chunks, 65535)));
}

template <typename T>
int run(Params a, bool back, cudaStream_t stream) {
  // little work: one piece a thread, for the latency
  const bool little = a.rows * int64_t(a.cols) < (1 << 20), aligned = aligned_rows(a.x, a.ldx, sizeof(T));
  if (back) {
    // groups of eight elements, all whole and on 16 bytes' (codes: 4 bytes') boundaries
    const bool whole = a.cols % 8 == 0 && aligned && aligned_rows(a.q, a.ldq, 1, 4);
    const int64_t groups = (int64_t(a.cols) + 7) / 8;
    const int least = whole ? 4 : 32;  // (else by whole warps)
    const dim3 block = little ? shape<1>(groups, least) : shape<4>(groups, least);
    a.q_wide = aligned_rows(a.q, a.ldq, 1, 4);
    auto kernel = little ? (whole ? dequant_mxf4_kernel<T, 1> : dequant_mxf4_anywhere_kernel<T, 1>)
                         : (whole ? dequant_mxf4_kernel<T, 4> : dequant_mxf4_anywhere_kernel<T, 4>);
    kernel<<<grid_of(a, block, int64_t(little ? 8 : 32) * block.x), block, 0, stream>>>(a);
  } else {
    // pieces of sixteen elements, made of whole words of 16 bytes; codes on 8 bytes' boundaries
    a.q_wide = aligned_rows(a.q, a.ldq, 1, 8);
    const bool whole = a.cols % (16 / int(sizeof(T))) == 0 && aligned && a.q_wide;
    const int64_t halves = (int64_t(a.cols) + 15) / 16;
    const dim3 block = little ? shape<1>(halves, 2) : shape<2>(halves, 2);
    auto kernel = little ? (whole ? quant_mxf4_kernel<T, 1, true> : quant_mxf4_kernel<T, 1, false>)
                         : (whole ? quant_mxf4_kernel<T, 2, true> : quant_mxf4_kernel<T, 2, false>);
    kernel<<<grid_of(a, block, int64_t(little ? 16 : 32) * block.x), block, 0, stream>>>(a);
  }
  return launched(cudaSuccess);
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
