// Tokens sorted by expert and back with weights applied, and the gradients (entwine_moe_*).
#include <algorithm>

#include "ops_common.cuh"

namespace entwine {
namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxExperts = 1024;
constexpr int64_t kMaxGrid = 2147483647;

// Expert of assignment i, or E where it is dropped.
template <typename Id>
__device__ __forceinline__ int expert_of(const Id* ids, int64_t i, int E) {
  const Id e = ids[i];
  return e >= 0 && e < Id(E) ? int(e) : E;
}

// Stable counting sort of n assignments by expert, one CTA.  Every warp owns a run of consecutive assignments and a
// row of counts; the counts become start positions by a scan over warps and experts; then each warp walks its run
// again, 32 assignments at a time, ranking equal experts among its lanes by a vote.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads) moe_sort_kernel(const Id* ids, int64_t n, int E, int32_t* offsets,
                                                                int32_t* row_of) {
  extern __shared__ int32_t counts[];  // [kSortWarps][E]
  __shared__ int32_t warp_total[kSortWarps];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t run = (n + kSortThreads - 1) / kSortThreads * 32;
  const int64_t first = min(int64_t(warp) * run, n), last = min(first + run, n);
  int32_t* mine = counts + warp * E;
  for (int i = threadIdx.x; i < kSortWarps * E; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  for (int64_t i0 = first; i0 < last; i0 += 32) {
    const int64_t i = i0 + lane;
    const int e = i < last ? expert_of(ids, i, E) : E;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    if (e < E && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // thread e: the counts of expert e become the starts of the warps' runs inside its rows
  const int e = threadIdx.x;
  int32_t total = 0;
  if (e < E)
    for (int w = 0; w < kSortWarps; ++w) {
      const int32_t c = counts[w * E + e];
      counts[w * E + e] = total;
      total += c;
    }
  int32_t sum = total;  // inclusive scan over the experts
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) warp_total[warp] = sum;
  __syncthreads();
  int32_t before = 0;
  for (int w = 0; w < warp; ++w) before += warp_total[w];
  const int32_t start = before + sum - total;
  if (e < E) {
    offsets[e] = start;
    if (e == E - 1) offsets[E] = start + total;
    for (int w = 0; w < kSortWarps; ++w) counts[w * E + e] += start;
  }
  __syncthreads();
  for (int64_t i0 = first; i0 < last; i0 += 32) {
    const int64_t i = i0 + lane;
    const int x = i < last ? expert_of(ids, i, E) : E;
    const unsigned same = __match_any_sync(0xffffffffu, x);
    const int32_t base = x < E ? mine[x] : 0;
    __syncwarp();
    if (x < E && lane == __ffs(same) - 1) mine[x] = base + __popc(same);
    __syncwarp();
    if (i < last) row_of[i] = x < E ? base + __popc(same & ((1u << lane) - 1)) : -1;
  }
}

// One CTA per token: its row is read once and written to each of its places.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) moe_move_kernel(const T* x, int64_t H, int64_t ldx, const float* x_scale,
                                                            const int32_t* row_of, int64_t k, T* rows, int64_t ldr,
                                                            float* row_scale) {
  using P = Piece<T, V>;
  const int64_t t = blockIdx.x, pieces = H / V;
  const T* src = x + t * ldx;
  const int32_t* to = row_of + t * k;
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
    const P v = reinterpret_cast<const P*>(src)[i];
    for (int64_t j = 0; j < k; ++j)
      if (to[j] >= 0) reinterpret_cast<P*>(rows + to[j] * ldr)[i] = v;
  }
  for (int64_t i = pieces * V + threadIdx.x; i < H; i += kThreads) {
    const T v = src[i];
    for (int64_t j = 0; j < k; ++j)
      if (to[j] >= 0) rows[to[j] * ldr + i] = v;
  }
  if (x_scale)
    for (int64_t j = threadIdx.x; j < k; j += kThreads)
      if (to[j] >= 0) row_scale[to[j]] = x_scale[t];
}

// One CTA per token: the weighted sum of its rows (w null: weights of one).
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) moe_combine_kernel(const T* y, int64_t n_rows, int64_t H, int64_t ldy,
                                                               const float* w, const int32_t* row_of, int64_t k,
                                                               T* out, int64_t ldo) {
  using P = Piece<T, V>;
  const int64_t t = blockIdx.x, pieces = H / V;
  const int32_t* at = row_of + t * k;
  const float* wt = w ? w + t * k : nullptr;
  T* dst = out + t * ldo;
  for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
    for (int64_t j = 0; j < k; ++j) {
      const int64_t r = at[j];
      if (r < 0 || r >= n_rows) continue;
      const P v = reinterpret_cast<const P*>(y + r * ldy)[i];
      const float f = wt ? wt[j] : 1.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fmaf(f, Elem<T>::up(v.e[e]), acc[e]);
    }
    P o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = Elem<T>::down(acc[e]);
    reinterpret_cast<P*>(dst)[i] = o;
  }
  for (int64_t i = pieces * V + threadIdx.x; i < H; i += kThreads) {
    float acc = 0.0f;
    for (int64_t j = 0; j < k; ++j) {
      const int64_t r = at[j];
      if (r >= 0 && r < n_rows) acc = fmaf(wt ? wt[j] : 1.0f, Elem<T>::up(y[r * ldy + i]), acc);
    }
    dst[i] = Elem<T>::down(acc);
  }
}

// One CTA per token: dy of its rows, and the dot products that are the gradients of its weights.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) moe_combine_bwd_kernel(const T* dout, int64_t H, int64_t ldo, const T* y,
                                                                   int64_t n_rows, int64_t ldy, const float* w,
                                                                   const int32_t* row_of, int64_t k, T* dy,
                                                                   int64_t lddy, float* dw) {
  using P = Piece<T, V>;
  __shared__ float part[kThreads / 32];
  const int64_t t = blockIdx.x, pieces = H / V;
  const T* g = dout + t * ldo;
  for (int64_t j = 0; j < k; ++j) {
    const int64_t r = row_of[t * k + j];
    if (r < 0 || r >= n_rows) {
      if (threadIdx.x == 0) dw[t * k + j] = 0.0f;
      continue;
    }
    const float f = w[t * k + j];
    const T* yr = y + r * ldy;
    T* dr = dy + r * lddy;
    float dot = 0.0f;
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
      const P a = reinterpret_cast<const P*>(g)[i], b = reinterpret_cast<const P*>(yr)[i];
      P o;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float ge = Elem<T>::up(a.e[e]);
        dot = fmaf(ge, Elem<T>::up(b.e[e]), dot);
        o.e[e] = Elem<T>::down(f * ge);
      }
      reinterpret_cast<P*>(dr)[i] = o;
    }
    for (int64_t i = pieces * V + threadIdx.x; i < H; i += kThreads) {
      const float ge = Elem<T>::up(g[i]);
      dot = fmaf(ge, Elem<T>::up(yr[i]), dot);
      dr[i] = Elem<T>::down(f * ge);
    }
    dot = warp_sum(dot);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      float s = part[0];
      for (int i = 1; i < kThreads / 32; ++i) s += part[i];
      dw[t * k + j] = s;
    }
    __syncthreads();
  }
}

template <typename Id>
int sort(const void* ids, int64_t n, int E, int32_t* offsets, int32_t* row_of, cudaStream_t stream) {
  const int smem = kSortWarps * E * 4;
  cudaError_t e = cudaFuncSetAttribute(moe_sort_kernel<Id>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kSortWarps * kMaxExperts * 4);
  if (e == cudaSuccess)
    moe_sort_kernel<Id><<<1, kSortThreads, smem, stream>>>(static_cast<const Id*>(ids), n, E, offsets, row_of);
  return launched(e);
}

template <typename T>
int move(const void* x, int64_t T_, int64_t H, int64_t ldx, const float* x_scale, const int32_t* row_of, int64_t k,
         void* rows, int64_t ldr, float* row_scale, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  auto kernel = aligned_rows(x, ldx, sizeof(T)) && aligned_rows(rows, ldr, sizeof(T)) ? moe_move_kernel<T, V>
                                                                                       : moe_move_kernel<T, 1>;
  kernel<<<unsigned(T_), kThreads, 0, stream>>>(static_cast<const T*>(x), H, ldx, x_scale, row_of, k,
                                                static_cast<T*>(rows), ldr, row_scale);
  return launched(cudaSuccess);
}

template <typename T>
int combine(const void* y, int64_t n_rows, int64_t H, int64_t ldy, const float* w, const int32_t* row_of, int64_t T_,
            int64_t k, void* out, int64_t ldo, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  auto kernel = aligned_rows(y, ldy, sizeof(T)) && aligned_rows(out, ldo, sizeof(T)) ? moe_combine_kernel<T, V>
                                                                                      : moe_combine_kernel<T, 1>;
  kernel<<<unsigned(T_), kThreads, 0, stream>>>(static_cast<const T*>(y), n_rows, H, ldy, w, row_of, k,
                                                static_cast<T*>(out), ldo);
  return launched(cudaSuccess);
}

template <typename T>
int combine_bwd(const void* dout, int64_t T_, int64_t H, int64_t ldo, const void* y, int64_t n_rows, int64_t ldy,
                const float* w, const int32_t* row_of, int64_t k, void* dy, int64_t lddy, float* dw,
                cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(dout, ldo, sizeof(T)) && aligned_rows(y, ldy, sizeof(T)) &&
                   aligned_rows(dy, lddy, sizeof(T));
  auto kernel = vec ? moe_combine_bwd_kernel<T, V> : moe_combine_bwd_kernel<T, 1>;
  kernel<<<unsigned(T_), kThreads, 0, stream>>>(static_cast<const T*>(dout), H, ldo, static_cast<const T*>(y), n_rows,
                                                ldy, w, row_of, k, static_cast<T*>(dy), lddy, dw);
  return launched(cudaSuccess);
}

int elem_bytes(int dtype) { return dtype == ENTWINE_FP32 ? 4 : (dtype == ENTWINE_I8 ? 1 : 2); }
bool floating(int dtype) { return dtype == ENTWINE_BF16 || dtype == ENTWINE_FP16 || dtype == ENTWINE_FP32; }

// T*k assignments, each with a 32-bit row number
bool bad_routing(int64_t T, int64_t k) { return T < 0 || T > kMaxGrid || k < 1 || k > kMaxGrid || T * k > kMaxGrid; }

int weighted_sum(const void* y, int dtype, int64_t n_rows, int64_t H, int64_t ldy, const float* w,
                 const int32_t* row_of, int64_t T, int64_t k, void* out, int64_t ldo, cudaStream_t s) {
  if (!floating(dtype) || bad_routing(T, k) || n_rows < 0 || n_rows > kMaxGrid || H < 1 || ldy < H || ldo < H)
    return ENTWINE_ERR_INVALID;
  if (T == 0) return ENTWINE_OK;
  const int size = elem_bytes(dtype);
  if ((n_rows > 0 && bad_pointer(y, size)) || bad_pointer(row_of, 4) || bad_pointer(out, size))
    return ENTWINE_ERR_INVALID;
  switch (dtype) {
    case ENTWINE_BF16: return combine<__nv_bfloat16>(y, n_rows, H, ldy, w, row_of, T, k, out, ldo, s);
    case ENTWINE_FP16: return combine<__half>(y, n_rows, H, ldy, w, row_of, T, k, out, ldo, s);
    default: return combine<float>(y, n_rows, H, ldy, w, row_of, T, k, out, ldo, s);
  }
}

}  // namespace
}  // namespace entwine

using namespace entwine;

extern "C" {

int entwine_moe_dispatch(const void* x, int dtype, int64_t T, int64_t H, int64_t ldx, const float* x_scale,
                         const void* ids, int ids64, int64_t k, int64_t E, void* rows, int64_t ldr,
                         float* row_scale, int32_t* offsets, int32_t* row_of, void* stream) {
  if ((!floating(dtype) && dtype != ENTWINE_I8) || bad_routing(T, k) || H < 1 || ldx < H || ldr < H || E < 1 ||
      E > kMaxExperts || bad_pointer(offsets, 4) || (x_scale == nullptr) != (row_scale == nullptr))
    return ENTWINE_ERR_INVALID;
  const int size = elem_bytes(dtype);
  if (T > 0 && (bad_pointer(x, size) || bad_pointer(ids, ids64 ? 8 : 4) || bad_pointer(rows, size) ||
                bad_pointer(row_of, 4) || (x_scale && (bad_pointer(x_scale, 4) || bad_pointer(row_scale, 4)))))
    return ENTWINE_ERR_INVALID;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  int rc = ids64 ? sort<int64_t>(ids, T * k, int(E), offsets, row_of, s)
                 : sort<int32_t>(ids, T * k, int(E), offsets, row_of, s);
  if (rc != ENTWINE_OK || T == 0) return rc;
  switch (size) {  // rows are moved as they are: only the size of an element counts
    case 1: return move<uint8_t>(x, T, H, ldx, x_scale, row_of, k, rows, ldr, row_scale, s);
    case 2: return move<uint16_t>(x, T, H, ldx, x_scale, row_of, k, rows, ldr, row_scale, s);
    default: return move<uint32_t>(x, T, H, ldx, x_scale, row_of, k, rows, ldr, row_scale, s);
  }
}

int entwine_moe_dispatch_bwd(const void* d_rows, int dtype, int64_t n_rows, int64_t H, int64_t ldr,
                             const int32_t* row_of, int64_t T, int64_t k, void* dx, int64_t ldx, void* stream) {
  return weighted_sum(d_rows, dtype, n_rows, H, ldr, nullptr, row_of, T, k, dx, ldx,
                      static_cast<cudaStream_t>(stream));
}

int entwine_moe_combine(const void* y, int dtype, int64_t n_rows, int64_t H, int64_t ldy, const float* w,
                        const int32_t* row_of, int64_t T, int64_t k, void* out, int64_t ldo, void* stream) {
  if (T > 0 && bad_pointer(w, 4)) return ENTWINE_ERR_INVALID;
  return weighted_sum(y, dtype, n_rows, H, ldy, w, row_of, T, k, out, ldo, static_cast<cudaStream_t>(stream));
}

int entwine_moe_combine_bwd(const void* dout, int dtype, int64_t T, int64_t H, int64_t ldo, const void* y,
                            int64_t n_rows, int64_t ldy, const float* w, const int32_t* row_of, int64_t k, void* dy,
                            int64_t lddy, float* dw, void* stream) {
  if (!floating(dtype) || bad_routing(T, k) || n_rows < 0 || n_rows > kMaxGrid || H < 1 || ldo < H || ldy < H ||
      lddy < H)
    return ENTWINE_ERR_INVALID;
  if (T == 0) return ENTWINE_OK;
  const int size = elem_bytes(dtype);
  if (bad_pointer(dout, size) || (n_rows > 0 && (bad_pointer(y, size) || bad_pointer(dy, size))) || bad_pointer(w, 4) ||
      bad_pointer(row_of, 4) || bad_pointer(dw, 4))
    return ENTWINE_ERR_INVALID;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return combine_bwd<__nv_bfloat16>(dout, T, H, ldo, y, n_rows, ldy, w, row_of, k, dy, lddy, dw, s);
    case ENTWINE_FP16: return combine_bwd<__half>(dout, T, H, ldo, y, n_rows, ldy, w, row_of, k, dy, lddy, dw, s);
    default: return combine_bwd<float>(dout, T, H, ldo, y, n_rows, ldy, w, row_of, k, dy, lddy, dw, s);
  }
}

}  // extern "C"
