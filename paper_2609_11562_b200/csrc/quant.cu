// Rows to 8-bit integers with a scale each (entwine_quant_i8).
#include "ops_common.cuh"

namespace entwine {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxRows = 2147483647;  // grid limit

// One row's quantiser.  q = rint(127 x / amax) of the exact quotient: the product with the rounded factor 127/amax
// is within 2^-16 of it, so only values within 2^-14 of a half need a second look, which compares 127|x| with
// (k + 1/2) amax in fp64, where both products are exact (24 + 8 bits).
struct RowQuant {
  float pre;     // a power of two that keeps 127/amax finite and normal (1 but for extreme rows)
  float factor;  // 127 / (amax pre)
  float amax;    // amax pre
  bool zero;     // the row is all zeros or not finite

  __device__ __forceinline__ explicit RowQuant(uint32_t amax_bits) {
    amax = __uint_as_float(amax_bits);
    zero = amax_bits == 0 || amax_bits >= 0x7f800000u;
    pre = amax < 0x1p-60f ? 0x1p64f : (amax > 0x1p60f ? 0x1p-64f : 1.0f);
    amax *= pre;
    factor = __fdiv_rn(127.0f, amax);
  }
  __device__ __forceinline__ int operator()(float x) const {
    if (zero) return 0;
    const float xs = x * pre;
    const float t = xs * factor;
    float q = rintf(t);
    if (fabsf(t - q) > 0.5f - 0x1p-14f) {
      const float a = fabsf(t), k = floorf(a);
      const double l = 127.0 * double(fabsf(xs)), h = (double(k) + 0.5) * double(amax);
      const float up = l > h || (l == h && (int(k) & 1)) ? 1.0f : 0.0f;
      q = copysignf(k + up, t);
    }
    return int(q);
  }
  static __device__ __forceinline__ float scale(uint32_t amax_bits) {
    return amax_bits >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : __fdiv_rn(__uint_as_float(amax_bits), 127.0f);
  }
};

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// One CTA per row, the row read twice.  |x| as unsigned bits: their maximum is the maximum of the magnitudes, and
// infinities and NaN lie above every finite value.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) quant_rows_kernel(const T* x, int64_t cols, int64_t ldx, int8_t* q,
                                                              int64_t ldq, float* scale) {
  using In = Piece<T, V>;
  using Out = Piece<int8_t, V>;
  __shared__ uint32_t part[kThreads / 32];
  const int64_t row = blockIdx.x;
  const T* xr = x + row * ldx;
  int8_t* qr = q + row * ldq;
  const int64_t pieces = cols / V;
  uint32_t m = 0;
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
    const In v = reinterpret_cast<const In*>(xr)[i];
#pragma unroll
    for (int e = 0; e < V; ++e) m = max(m, abs_bits(Elem<T>::up(v.e[e])));
  }
  for (int64_t i = pieces * V + threadIdx.x; i < cols; i += kThreads) m = max(m, abs_bits(Elem<T>::up(xr[i])));
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = m;
  __syncthreads();
  m = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) m = max(m, part[w]);
  if (threadIdx.x == 0) scale[row] = RowQuant::scale(m);
  const RowQuant quant(m);
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
    const In v = reinterpret_cast<const In*>(xr)[i];
    Out o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = int8_t(quant(Elem<T>::up(v.e[e])));
    reinterpret_cast<Out*>(qr)[i] = o;
  }
  for (int64_t i = pieces * V + threadIdx.x; i < cols; i += kThreads) qr[i] = int8_t(quant(Elem<T>::up(xr[i])));
}

template <typename T>
int quant_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq, float* scale,
               cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(x, ldx, sizeof(T)) && aligned_rows(q, ldq, 1, V);
  auto kernel = vec ? quant_rows_kernel<T, V> : quant_rows_kernel<T, 1>;
  kernel<<<unsigned(rows), kThreads, 0, stream>>>(static_cast<const T*>(x), cols, ldx, static_cast<int8_t*>(q), ldq,
                                                  scale);
  return launched(cudaSuccess);
}

}  // namespace
}  // namespace entwine

using namespace entwine;

extern "C" int entwine_quant_i8(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, void* q,
                                int64_t ldq, float* scale, void* stream) {
  if (dtype != ENTWINE_BF16 && dtype != ENTWINE_FP16 && dtype != ENTWINE_FP32) return ENTWINE_ERR_INVALID;
  if (rows < 0 || rows > kMaxRows || cols < 1 || ldx < cols || ldq < cols) return ENTWINE_ERR_INVALID;
  if (rows == 0) return ENTWINE_OK;
  if (bad_pointer(x, dtype == ENTWINE_FP32 ? 4 : 2) || bad_pointer(q, 1) || bad_pointer(scale, 4))
    return ENTWINE_ERR_INVALID;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return quant_rows<__nv_bfloat16>(x, rows, cols, ldx, q, ldq, scale, s);
    case ENTWINE_FP16: return quant_rows<__half>(x, rows, cols, ldx, q, ldq, scale, s);
    default: return quant_rows<float>(x, rows, cols, ldx, q, ldq, scale, s);
  }
}
