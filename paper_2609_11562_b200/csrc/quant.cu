// Rows to 8-bit integers with a scale each (entwine_quant_i8).
#include <algorithm>
#include <cstring>

#include "ops_common.cuh"

namespace entwine {
namespace {

constexpr int kThreads = 256;       // of the kernel that reads a row twice, and of several short rows together
constexpr int kMaxRowThreads = 512;
constexpr int kMaxPieces = 8;       // of 16 bytes, of a row held by one thread
constexpr int64_t kFewRows = 1024;
constexpr int64_t kMaxRows = 2147483647;  // grid limit

// What decides on which side of a half a quotient u = 127 x / amax lies, by type.  With x = a 2^i and amax = d 2^j, both
// a and d of p bits, u is a tie or at least u / (254 a) > u 2^-(p+8) away from every half.  The product x * factor, which
// is not rounded before it is rounded to a level, is within u 2^-23 of u; so for p = 8 and 11 (bf16, fp16) it lies on
// the right side but for ties: 254 a 2^i = (2k+1) d 2^j, where the prime 127 divides 2k+1 or d.  2k+1 = 127 is
// |x| = amax/2: the tie goes up, to 64, and a factor rounded up puts the product at 63.5 or above.  127 | d makes a
// bf16 factor a power of two (d = 254) and its ties exact; fp16 rows with such a d take the exact way.  In fp32 every
// product is tested.
template <typename T>
struct Border;
template <>
struct Border<__nv_bfloat16> {
  static constexpr bool kTest = false;
  static __device__ __forceinline__ bool careful(uint32_t) { return false; }
};
template <>
struct Border<__half> {
  static constexpr bool kTest = false;
  static __device__ __forceinline__ bool careful(uint32_t amax_bits) {
    return (((amax_bits >> 13) & 0x3ff) | 0x400) % 127 == 0;
  }
};
template <>
struct Border<float> {
  static constexpr bool kTest = true;
  static __device__ __forceinline__ bool careful(uint32_t) { return false; }
};

// One row's quantiser: q = rint(127 x / amax) of the exact quotient.
template <typename T>
struct RowQuant {
  float factor;  // 127 / amax, rounded up
  float amax;
  float pre;     // rows of extreme magnitude: a power of two, applied to x and amax, that keeps all this in range
  bool zero;     // the row is all zeros or not finite
  bool careful;  // every element takes the exact way

  __device__ __forceinline__ explicit RowQuant(uint32_t amax_bits) {
    amax = __uint_as_float(amax_bits);
    zero = amax_bits == 0 || amax_bits >= 0x7f800000u;
    pre = amax < 0x1p-60f ? 0x1p64f : (amax > 0x1p60f ? 0x1p-64f : 1.0f);
    careful = zero || pre != 1.0f || Border<T>::careful(amax_bits);
    amax *= pre;
    factor = __fdiv_ru(127.0f, amax);
  }
  // Near a half 127|x| is compared with (k + 1/2) amax.  Both products are kept as an fp32 value and its exact rest
  // (24 + 8 bits); their difference is exact because they agree to 2^-16.
  __device__ __forceinline__ uint32_t exact(float x) const {
    if (zero) return 0;
    x *= pre;
    const float t = x * factor, a = fabsf(t), k = floorf(a), h = k + 0.5f;
    float level = rintf(a);
    if (fabsf(a - h) < 0x1p-14f) {
      x = fabsf(x);
      const float l = 127.0f * x, m = h * amax;
      const float over = (l - m) + (__fmaf_rn(127.0f, x, -l) - __fmaf_rn(h, amax, -m));
      level = over > 0.0f || (over == 0.0f && (int(k) & 1)) ? k + 1.0f : k;
    }
    return uint32_t(int(copysignf(level, t)));
  }
  // V elements at once: adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves it in the low bits.
  template <int V>
  __device__ __forceinline__ Piece<int8_t, V> operator()(const Piece<T, V>& v) const {
    uint32_t q[V];
    float f[V], off = 0.0f;
    unpack<T, V>(v, f);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float r = __fmaf_rn(f[e], factor, 0x1.8p23f);
      if constexpr (Border<T>::kTest) off = fmaxf(off, fabsf(__fmaf_rn(f[e], factor, -(r - 0x1.8p23f))));
      q[e] = __float_as_uint(r);
    }
    if (careful || off > 0.5f - 0x1p-14f) {
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = exact(f[e]);
    }
    Piece<int8_t, V> o;
    if constexpr (V >= 4) {
      uint32_t w[V / 4];
#pragma unroll
      for (int e = 0; e < V; e += 4)
        w[e / 4] = __byte_perm(__byte_perm(q[e], q[e + 1], 0x0040), __byte_perm(q[e + 2], q[e + 3], 0x0040), 0x5410);
      memcpy(&o, w, sizeof(o));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) o.e[e] = int8_t(q[e]);
    }
    return o;
  }
  __device__ __forceinline__ int8_t operator()(T x) const { return int8_t(exact(Elem<T>::up(x))); }
  static __device__ __forceinline__ float scale(uint32_t amax_bits) {
    return amax_bits >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : __fdiv_rn(__uint_as_float(amax_bits), 127.0f);
  }
};

// |x| as unsigned bits: their maximum is the maximum of the magnitudes, and infinities and NaN lie above every
// finite value.  Two 16-bit elements are compared by one instruction; the bits of the largest become fp32 at the end.
template <typename T>
__device__ __forceinline__ uint32_t abs_bits(T v) {
  return __float_as_uint(Elem<T>::up(v)) & 0x7fffffffu;
}
template <typename T, int V>
struct RunningMax {
  static constexpr bool kPairs = sizeof(T) == 2 && V >= 2;
  uint32_t m = 0;
  __device__ __forceinline__ void take(const Piece<T, V>& v) {
    if constexpr (kPairs) {
      uint32_t w[V / 2];
      memcpy(w, &v, sizeof(v));
#pragma unroll
      for (int i = 0; i < V / 2; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) m = max(m, abs_bits(v.e[e]));
    }
  }
  __device__ __forceinline__ uint32_t bits() const {
    if constexpr (kPairs) {
      const uint16_t h = uint16_t(max(m & 0xffffu, m >> 16));
      T v;
      memcpy(&v, &h, 2);
      return abs_bits(v);
    }
    return m;
  }
};

// The maximum over the warps of a row.
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* part, int first_warp, int warps) {
  m = __reduce_max_sync(0xffffffffu, m);
  if (warps == 1) return m;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = m;
  __syncthreads();
  for (int w = 0; w < warps; ++w) m = max(m, part[first_warp + w]);
  return m;
}

// A row in registers: 2^log_threads threads (whole warps) hold up to P pieces of 16 bytes each, a CTA as many rows as
// fit.  One read of x, one write of q: 8192 rows of 3584 bf16 take 18.7 us, 4.7 TB/s, 4096 of 8192 fp32 28 us, 6.0 TB/s.
// Bound by the latency of a row's chain (load, maximum, factor, store) against the registers that hold rows: two or four
// pieces a thread 23.7 and 19.8 us, loads of the next row kept in flight by persistent CTAs 30 us (fewer rows fit).
template <typename T, int P>
__global__ void __launch_bounds__(kMaxRowThreads) quant_rows_kernel(const T* x, int64_t rows, int cols, int64_t ldx,
                                                                    int8_t* q, int64_t ldq, float* scale,
                                                                    int log_threads) {
  constexpr int V = 16 / sizeof(T);
  using In = Piece<T, V>;
  using Out = Piece<int8_t, V>;
  __shared__ uint32_t part[kMaxRowThreads / 32];
  const int slot = int(threadIdx.x) >> log_threads, row_threads = 1 << log_threads;
  const int lane = int(threadIdx.x) & (row_threads - 1);
  const int64_t row = int64_t(blockIdx.x) * (blockDim.x >> log_threads) + slot;
  const int pieces = cols / V, tail = cols % V;
  const T* xr = x + row * ldx;
  In v[P];
  T last{};
  RunningMax<T, V> top;
  if (row < rows) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      v[p] = p * row_threads + lane < pieces ? reinterpret_cast<const In*>(xr)[p * row_threads + lane] : In{};
    if (lane < tail) last = xr[pieces * V + lane];
#pragma unroll
    for (int p = 0; p < P; ++p) top.take(v[p]);
  }
  const uint32_t m = row_max(max(top.bits(), abs_bits(last)), part, slot << (log_threads - 5), 1 << (log_threads - 5));
  if (row >= rows) return;
  const RowQuant<T> quant(m);
  int8_t* qr = q + row * ldq;
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (p * row_threads + lane < pieces) reinterpret_cast<Out*>(qr)[p * row_threads + lane] = quant(v[p]);
  if (lane < tail) qr[pieces * V + lane] = quant(last);
  if (lane == 0) scale[row] = RowQuant<T>::scale(m);
}

// One CTA per row, the row read twice: rows too long for the registers, and rows that do not start on 16-byte
// boundaries, element by element (V = 1).  8192 contiguous rows of 3583 bf16 take 37 us (padded to 3584: 20), of 1021 18 us;
// four rows of 65536 fp32 23 us.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) quant_long_rows_kernel(const T* x, int64_t cols, int64_t ldx, int8_t* q,
                                                                   int64_t ldq, float* scale) {
  using In = Piece<T, V>;
  using Out = Piece<int8_t, V>;
  __shared__ uint32_t part[kThreads / 32];
  const int64_t row = blockIdx.x;
  const T* xr = x + row * ldx;
  int8_t* qr = q + row * ldq;
  const int64_t pieces = cols / V;
  RunningMax<T, V> top;
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads) top.take(reinterpret_cast<const In*>(xr)[i]);
  uint32_t m = top.bits();
  for (int64_t i = pieces * V + threadIdx.x; i < cols; i += kThreads) m = max(m, abs_bits(xr[i]));
  m = row_max(m, part, 0, kThreads / 32);
  if (threadIdx.x == 0) scale[row] = RowQuant<T>::scale(m);
  const RowQuant<T> quant(m);
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads)
    reinterpret_cast<Out*>(qr)[i] = quant(reinterpret_cast<const In*>(xr)[i]);
  for (int64_t i = pieces * V + threadIdx.x; i < cols; i += kThreads) qr[i] = quant(xr[i]);
}

template <typename T>
int quant_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, void* q, int64_t ldq, float* scale,
               cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(x, ldx, sizeof(T)) && aligned_rows(q, ldq, 1, V);
  const T* xt = static_cast<const T*>(x);
  int8_t* qt = static_cast<int8_t*>(q);
  const int64_t pieces = (cols + V - 1) / V;
  if (!vec || pieces > kMaxPieces * int64_t(kMaxRowThreads)) {
    auto kernel = vec ? quant_long_rows_kernel<T, V> : quant_long_rows_kernel<T, 1>;
    kernel<<<unsigned(rows), kThreads, 0, stream>>>(xt, cols, ldx, qt, ldq, scale);
    return launched(cudaSuccess);
  }
  // few rows: many threads with little each, for the latency; many rows: many pieces per thread
  const int most = rows < kFewRows ? 2 : kMaxPieces;
  int log_threads = 5;
  while ((2 << log_threads) <= kMaxRowThreads && (int64_t(most) << log_threads) < pieces) ++log_threads;
  const int64_t each = (pieces + (1 << log_threads) - 1) >> log_threads;
  auto kernel = each <= 2 ? quant_rows_kernel<T, 2> : each <= 4 ? quant_rows_kernel<T, 4> : quant_rows_kernel<T, kMaxPieces>;
  const int threads = std::max(64, 1 << log_threads), per_cta = threads >> log_threads;
  kernel<<<unsigned((rows + per_cta - 1) / per_cta), threads, 0, stream>>>(xt, rows, int(cols), ldx, qt, ldq, scale,
                                                                           log_threads);
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
