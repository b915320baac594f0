// Tokens sorted by expert and back with weights applied, and the gradients (entwine_moe_*).
#include <algorithm>
#include <type_traits>

#include "ops_common.cuh"
#include "sm100.cuh"

namespace entwine {
namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCtas = 8;      // CTAs of the sort: one cluster
constexpr int kIdsAhead = 8;      // loads of assignments in flight per lane
constexpr int kMaxExperts = 1024;
constexpr int kChunk = 8;         // assignments of a token placed and written together
// Assignments of a token read together by the sums.  Four loads of 16 bytes per thread at four or five CTAs per SM
// reach 94-100 % of the copy rate; eight cost the registers of half of the CTAs (8192 tokens of 4096 bf16, eight
// experts each: forward 94 us with four, 116 with eight; backward 175, 344).
constexpr int kReads = 4;
constexpr int64_t kMaxGrid = 2147483647;
// up to this many assignments of this many tokens every token's CTA ranks its own ones against all others: 256 tokens to
// eight experts each take 7.8 us that way, 11.8 by the sort; 2048 tokens to one 16.5 and 11.6
constexpr int64_t kSmallRouting = 2048, kSmallTokens = 512;
constexpr int64_t kFewTokens = 1024;  // below this a token's row is spread over several CTAs

// Expert of an assignment, or E where it is dropped.
template <typename Id>
__device__ __forceinline__ int expert_of(Id e, int E) {
  return e >= 0 && e < Id(E) ? int(e) : E;
}

// Inclusive scan over the lanes of a warp.
__device__ __forceinline__ int32_t warp_scan(int32_t v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Stable counting sort of n assignments by expert, one cluster of eight CTAs.  Every warp owns a run of consecutive
// assignments and a row of counts in shared memory; the counts become start positions by a scan over a CTA's warps,
// over the CTAs (whose totals are read through distributed shared memory) and over the experts; then each warp walks
// its run again, 32 assignments at a time, ranking equal experts among its lanes by votes on the bits of the
// expert's number (a match instruction takes 64 cycles of its SM: 36 us for the 131072 assignments of 16384 tokens).
template <typename Id>
__global__ void __launch_bounds__(kSortThreads) moe_sort_kernel(const Id* ids, int64_t n, int E, int32_t* offsets,
                                                                int32_t* row_of) {
  extern __shared__ int32_t counts[];  // [kSortWarps][E], then the CTA's totals [E]
  __shared__ int32_t warp_total[kSortWarps];
  const int cta = int(cluster_ctarank()), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t walkers = kSortCtas * kSortWarps;
  const int64_t run = (n + walkers * 32 - 1) / (walkers * 32) * 32;
  const int64_t first = min((int64_t(cta) * kSortWarps + warp) * run, n), last = min(first + run, n);
  int32_t* mine = counts + warp * E;
  int32_t* totals = counts + kSortWarps * E;
  const int bits = 32 - __clz(E);  // of an expert's number, E (dropped) among them
  for (int i = threadIdx.x; i < kSortWarps * E; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  for (int64_t i0 = first; i0 < last; i0 += 32 * kIdsAhead) {
    Id id[kIdsAhead];
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) id[u] = i0 + 32 * u + lane < last ? ids[i0 + 32 * u + lane] : Id(-1);
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) {
      if (i0 + 32 * u >= last) break;
      const int e = expert_of(id[u], E);
      if (e < E) atomicAdd(&mine[e], 1);  // counts: no order to depend on
    }
  }
  __syncthreads();
  // thread e: the counts of expert e become the starts of the warps' runs inside its rows
  const int e = threadIdx.x;
  int32_t total = 0;
  if (e < E) {
    for (int w = 0; w < kSortWarps; ++w) {
      const int32_t c = counts[w * E + e];
      counts[w * E + e] = total;
      total += c;
    }
    totals[e] = total;
  }
  __syncwarp();
  cluster_sync_all();
  int32_t before = 0;  // of this expert, in the CTAs before this one
  total = 0;
  if (e < E) {
    int32_t t[kSortCtas];
#pragma unroll
    for (int c = 0; c < kSortCtas; ++c) t[c] = ld_cluster(map_to_cta(smem_u32(totals + e), c));
#pragma unroll
    for (int c = 0; c < kSortCtas; ++c) {
      if (c < cta) before += t[c];
      total += t[c];
    }
  }
  const int32_t sum = warp_scan(total, lane);
  if (lane == 31) warp_total[warp] = sum;
  __syncthreads();
  int32_t start = sum - total;
  for (int w = 0; w < warp; ++w) start += warp_total[w];
  if (e < E) {
    if (cta == 0) {
      offsets[e] = start;
      if (e == E - 1) offsets[E] = start + total;
    }
    for (int w = 0; w < kSortWarps; ++w) counts[w * E + e] += start + before;
  }
  __syncwarp();
  cluster_sync_all();  // (also: no CTA leaves while its totals are read)
  for (int64_t i0 = first; i0 < last; i0 += 32 * kIdsAhead) {
    Id id[kIdsAhead];
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) id[u] = i0 + 32 * u + lane < last ? ids[i0 + 32 * u + lane] : Id(-1);
#pragma unroll
    for (int u = 0; u < kIdsAhead; ++u) {
      const int64_t i = i0 + 32 * u + lane;
      if (i0 + 32 * u >= last) break;
      const int x = expert_of(id[u], E);
      unsigned same = 0xffffffffu;
      for (int b = 0; b < bits; ++b) {
        const bool one = (x >> b) & 1;
        const unsigned ones = __ballot_sync(0xffffffffu, one);
        same &= one ? ones : ~ones;
      }
      const int32_t base = x < E ? mine[x] : 0;
      __syncwarp();
      if (x < E && lane == __ffs(same) - 1) mine[x] = base + __popc(same);
      __syncwarp();
      if (i < last) row_of[i] = x < E ? base + __popc(same & ((1u << lane) - 1)) : -1;
    }
  }
}

// A token's row written to its places, `to` in shared or global memory: read once for each kChunk of them where all rows
// start on 16-byte boundaries (V > 1), else put together anew for each place, whose pieces lie differently.
template <typename T, int V>
__device__ __forceinline__ void move_row(const T* src, int64_t H, const int32_t* to, int64_t k, T* rows, int64_t ldr,
                                         const Span& inside) {
  if constexpr (V > 1) {
    const int64_t pieces = H / V;
    for (int64_t j0 = 0; j0 < k; j0 += kChunk) {
      int32_t r[kChunk];
#pragma unroll
      for (int j = 0; j < kChunk; ++j) r[j] = j0 + j < k ? to[j0 + j] : -1;
      for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
        const uint4 v = reinterpret_cast<const uint4*>(src)[i];  // (moved as one thing, whatever the elements)
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
          if (r[j] >= 0) reinterpret_cast<uint4*>(rows + r[j] * ldr)[i] = v;
      }
      for (int64_t i = pieces * V + threadIdx.x; i < H; i += kThreads)
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
          if (r[j] >= 0) rows[r[j] * ldr + i] = src[i];
    }
  } else {
    for (int64_t j = 0; j < k; ++j) {
      if (to[j] < 0) continue;
      T* const dst = rows + to[j] * ldr;
      const Cut<T> cut(dst, H);
      for (int64_t i = threadIdx.x; i < cut.pieces; i += kThreads) {
        const int64_t e = cut.head + i * (16 / int64_t(sizeof(T)));
        const Piece<T, 16 / sizeof(T)> v = Anywhere<T>::load(src + e, inside);
        uint4 bits;
        memcpy(&bits, &v, 16);
        *reinterpret_cast<uint4*>(dst + e) = bits;
      }
      for (int64_t i = threadIdx.x; i < cut.ends; i += kThreads) dst[cut.end(i)] = src[cut.end(i)];
    }
  }
}

// One CTA per token, behind the sort.  16384 tokens of 4096 bytes to eight places each: 95 us, 6.2 TB/s.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) moe_move_kernel(const T* x, int64_t H, int64_t ldx, const float* x_scale,
                                                            const int32_t* row_of, int64_t k, T* rows, int64_t ldr,
                                                            float* row_scale) {
  const int64_t t = blockIdx.x;
  const int32_t* to = row_of + t * k;
  move_row<T, V>(x + t * ldx, H, to, k, rows, ldr, span_of(x, gridDim.x, H, ldx));
  if (x_scale)
    for (int64_t j = threadIdx.x; j < k; j += kThreads)
      if (to[j] >= 0) row_scale[to[j]] = x_scale[t];
}

// Few assignments: sort and move in one launch, a CTA per token.  The row of an assignment is the number of
// assignments to lower experts plus that of earlier ones to its own, counted over all n by the token's CTA; the last
// CTA of the grid counts the experts' rows for the offsets.
template <typename T, int V, typename Id>
__global__ void __launch_bounds__(kThreads) moe_dispatch_small_kernel(const T* x, int64_t T_, int64_t H, int64_t ldx,
                                                                      const float* x_scale, const Id* ids, int k, int E,
                                                                      T* rows, int64_t ldr, float* row_scale,
                                                                      int32_t* offsets, int32_t* row_of) {
  __shared__ int32_t all[kSmallRouting];
  __shared__ int32_t table[kMaxExperts];  // the last CTA: rows of each expert; the others: rows of the assignments
  const int n = int(T_) * k, lane = threadIdx.x % 32, t = blockIdx.x;
  for (int i = threadIdx.x; i < n; i += kThreads) all[i] = expert_of(ids[i], E);
  if (t == T_) {
    __shared__ int32_t warp_total[kThreads / 32];
    constexpr int kEach = kMaxExperts / kThreads;
    for (int e = threadIdx.x; e < kMaxExperts; e += kThreads) table[e] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (all[i] < E) atomicAdd(&table[all[i]], 1);  // counts: no order to depend on
    __syncthreads();
    int32_t c[kEach], total = 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) total += c[u] = table[threadIdx.x * kEach + u];
    const int32_t sum = warp_scan(total, lane);
    if (lane == 31) warp_total[threadIdx.x / 32] = sum;
    __syncthreads();
    int32_t start = sum - total;
    for (int w = 0; w < int(threadIdx.x) / 32; ++w) start += warp_total[w];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int e = threadIdx.x * kEach + u;
      if (e <= E) offsets[e] = start;
      start += c[u];
    }
    if (E == kMaxExperts && threadIdx.x == kThreads - 1) offsets[E] = start;
    return;
  }
  __shared__ int32_t part[kThreads / 32][kChunk];
  __syncthreads();
  for (int j0 = 0; j0 < k; j0 += kChunk) {
    int32_t e[kChunk], count[kChunk];
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
      e[j] = j0 + j < k ? all[t * k + j0 + j] : E;
      count[j] = 0;
    }
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int32_t o = all[i];
#pragma unroll
      for (int j = 0; j < kChunk; ++j) count[j] += o < e[j] + (i < t * k + j0 + j ? 1 : 0) ? 1 : 0;
    }
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
      const int32_t c = __reduce_add_sync(0xffffffffu, count[j]);
      if (lane == j) part[threadIdx.x / 32][j] = c;
    }
    __syncthreads();
    if (threadIdx.x < kChunk && j0 + int(threadIdx.x) < k) {
      const int j = j0 + threadIdx.x;
      int32_t r = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) r += part[w][threadIdx.x];
      if (all[t * k + j] >= E) r = -1;
      row_of[int64_t(t) * k + j] = r;
      part[0][threadIdx.x] = r;
      if (r >= 0 && x_scale) row_scale[r] = x_scale[t];
    }
    __syncthreads();
    move_row<T, V>(x + t * ldx, H, part[0], min(k - j0, kChunk), rows, ldr, span_of(x, T_, H, ldx));
    __syncthreads();
  }
}

// The weighted sum of a token's rows (w null: weights of one).  Bound by reading the rows: J assignments of U pieces
// of the token are in flight together, and a row is spread over several CTAs where there are few tokens.
template <typename T, int V, int J, int U>
__global__ void __launch_bounds__(kThreads, 5) moe_combine_kernel(const T* y, int64_t n_rows, int64_t H, int64_t ldy,
                                                                   const float* w, const int32_t* row_of, int64_t k,
                                                                   T* out, int64_t ldo) {
  using P = Piece<T, V>;
  const int64_t t = blockIdx.x, pieces = H / V, step = int64_t(gridDim.y) * blockDim.x;
  const int32_t* at = row_of + t * k;
  const float* wt = w ? w + t * k : nullptr;
  T* dst = out + t * ldo;
  const int64_t first = int64_t(blockIdx.y) * blockDim.x + threadIdx.x;
  for (int64_t i0 = first; i0 < pieces; i0 += U * step) {
    float acc[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[u][e] = 0.0f;
    for (int64_t j0 = 0; j0 < k; j0 += J) {
      P v[J][U];
      float f[J];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int64_t r = j0 + j < k ? at[j0 + j] : -1;
        const bool there = r >= 0 && r < n_rows;
        f[j] = !there ? 0.0f : wt ? wt[j0 + j] : 1.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t i = i0 + u * step;
          v[j][u] = load_if<T, V>(y + r * ldy + i * V, there && i < pieces);
        }
      }
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float ye[V];
          unpack<T, V>(v[j][u], ye);
#pragma unroll
          for (int e = 0; e < V; ++e) acc[u][e] = fmaf(f[j], ye[e], acc[u][e]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * step < pieces) reinterpret_cast<P*>(dst)[i0 + u * step] = pack<T, V>(acc[u]);
  }
  for (int64_t i = pieces * V + first; i < H; i += step) {
    float acc = 0.0f;
    for (int64_t j = 0; j < k; ++j) {
      const int64_t r = at[j];
      if (r >= 0 && r < n_rows) acc = fmaf(wt ? wt[j] : 1.0f, Elem<T>::up(y[r * ldy + i]), acc);
    }
    dst[i] = Elem<T>::down(acc);
  }
}

// The same for rows that start anywhere: a thread takes an aligned piece of the token and puts the pieces of its rows
// together from the words around them.  8192 tokens of 4095 bf16, eight experts each: 209 to 219 us (94 to 99 of 4096,
// where rows start on 16-byte boundaries); fp32 134.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) moe_combine_anywhere_kernel(const T* y, int64_t n_rows, int64_t H,
                                                                           int64_t ldy, const float* w,
                                                                           const int32_t* row_of, int64_t k, T* out,
                                                                           int64_t ldo) {
  constexpr int V = 16 / sizeof(T);
  using P = Piece<T, V>;
  const int64_t t = blockIdx.x, step = int64_t(gridDim.y) * blockDim.x;
  const int32_t* at = row_of + t * k;
  const float* wt = w ? w + t * k : nullptr;
  T* dst = out + t * ldo;
  const Cut<T> cut(dst, H);
  const Span inside = span_of(y, n_rows, H, ldy);
  const int64_t first = int64_t(blockIdx.y) * blockDim.x + threadIdx.x;
  for (int64_t i = first; i < cut.pieces; i += step) {
    const int64_t x = cut.head + i * V;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
    for (int64_t j0 = 0; j0 < k; j0 += kReads) {
      Anywhere<T> v[kReads];
      const T* from[kReads];
      float f[kReads];
      bool there[kReads], alone = false;
#pragma unroll
      for (int j = 0; j < kReads; ++j) {
        const int64_t r = j0 + j < k ? at[j0 + j] : -1;
        there[j] = r >= 0 && r < n_rows;
        from[j] = y + r * ldy + x;
        f[j] = !there[j] ? 0.0f : wt ? wt[j0 + j] : 1.0f;
        alone = alone || (there[j] && Anywhere<T>::alone(from[j], inside));
      }
#pragma unroll
      for (int j = 0; j < kReads; ++j) v[j].fetch(from[j], there[j] && !alone);
#pragma unroll
      for (int j = 0; j < kReads; ++j) {
        const P piece = alone && there[j] ? Anywhere<T>::one_by_one(from[j]) : v[j].get();
        float ye[V];
        unpack<T, V>(piece, ye);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = fmaf(f[j], ye[e], acc[e]);
      }
    }
    *reinterpret_cast<P*>(dst + x) = pack<T, V>(acc);
  }
  for (int64_t i = first; i < cut.ends; i += step) {
    const int64_t x = cut.end(i);
    float acc = 0.0f;
    for (int64_t j = 0; j < k; ++j) {
      const int64_t r = at[j];
      if (r >= 0 && r < n_rows) acc = fmaf(wt ? wt[j] : 1.0f, Elem<T>::up(y[r * ldy + x]), acc);
    }
    dst[x] = Elem<T>::down(acc);
  }
}

// One CTA per token: dy of its rows, and the dot products that are the gradients of its weights.  Bound by reading
// y and writing dy; up to four assignments are handled in one walk over the token's gradient.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 4) moe_combine_bwd_kernel(const T* dout, int64_t H, int64_t ldo, const T* y,
                                                                   int64_t n_rows, int64_t ldy, const float* w,
                                                                   const int32_t* row_of, int64_t k, T* dy,
                                                                   int64_t lddy, float* dw) {
  using P = Piece<T, V>;
  __shared__ float part[kThreads / 32][kReads];
  const int64_t t = blockIdx.x, pieces = H / V;
  const T* g = dout + t * ldo;
  for (int64_t j0 = 0; j0 < k; j0 += kReads) {
    int32_t r[kReads];
    float f[kReads], dot[kReads];
#pragma unroll
    for (int j = 0; j < kReads; ++j) {
      r[j] = j0 + j < k ? row_of[t * k + j0 + j] : -1;
      if (r[j] >= n_rows) r[j] = -1;
      f[j] = r[j] >= 0 ? w[t * k + j0 + j] : 0.0f;
      dot[j] = 0.0f;
    }
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
      const P a = reinterpret_cast<const P*>(g)[i];
      P b[kReads];
#pragma unroll
      for (int j = 0; j < kReads; ++j) b[j] = r[j] >= 0 ? reinterpret_cast<const P*>(y + r[j] * ldy)[i] : P{};
      float ge[V];
      unpack<T, V>(a, ge);
#pragma unroll
      for (int j = 0; j < kReads; ++j) {
        if (r[j] < 0) continue;
        float ye[V], d[V];
        unpack<T, V>(b[j], ye);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dot[j] = fmaf(ge[e], ye[e], dot[j]);
          d[e] = f[j] * ge[e];
        }
        reinterpret_cast<P*>(dy + r[j] * lddy)[i] = pack<T, V>(d);
      }
    }
    for (int64_t i = pieces * V + threadIdx.x; i < H; i += kThreads) {
      const float ge = Elem<T>::up(g[i]);
#pragma unroll
      for (int j = 0; j < kReads; ++j) {
        if (r[j] < 0) continue;
        dot[j] = fmaf(ge, Elem<T>::up(y[r[j] * ldy + i]), dot[j]);
        dy[r[j] * lddy + i] = Elem<T>::down(f[j] * ge);
      }
    }
#pragma unroll
    for (int j = 0; j < kReads; ++j) {
      const float d = warp_sum(dot[j]);
      if (threadIdx.x % 32 == j) part[threadIdx.x / 32][j] = d;
    }
    __syncthreads();
    if (threadIdx.x < kReads && j0 + threadIdx.x < k) {
      float s = part[0][threadIdx.x];
#pragma unroll
      for (int i = 1; i < kThreads / 32; ++i) s += part[i][threadIdx.x];
      dw[t * k + j0 + threadIdx.x] = s;
    }
    __syncthreads();
  }
}

// The same for rows that start anywhere, one row of dy after another in its own aligned pieces (8192 tokens of 4095
// bf16, eight experts each: 317 to 396 us, aligned 174 to 181).
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) moe_combine_bwd_anywhere_kernel(const T* dout, int64_t H, int64_t ldo,
                                                                               const T* y, int64_t n_rows, int64_t ldy,
                                                                               const float* w, const int32_t* row_of,
                                                                               int64_t k, T* dy, int64_t lddy,
                                                                               float* dw) {
  constexpr int V = 16 / sizeof(T);
  using P = Piece<T, V>;
  __shared__ float part[2][kThreads / 32];
  const int64_t t = blockIdx.x;
  const T* g = dout + t * ldo;
  const Span in_g = span_of(dout, gridDim.x, H, ldo), in_y = span_of(y, n_rows, H, ldy);
  int turn = 0;
  for (int64_t j = 0; j < k; ++j) {
    const int64_t r = row_of[t * k + j];
    if (r < 0 || r >= n_rows) {
      if (threadIdx.x == 0) dw[t * k + j] = 0.0f;
      continue;
    }
    const float f = w[t * k + j];
    const T* yr = y + r * ldy;
    T* dr = dy + r * lddy;
    const Cut<T> cut(dr, H);
    float dot = 0.0f;
    for (int64_t i = threadIdx.x; i < cut.pieces; i += kThreads) {
      const int64_t x = cut.head + i * V;
      const P a = Anywhere<T>::load(g + x, in_g), b = Anywhere<T>::load(yr + x, in_y);
      float ge[V], ye[V], d[V];
      unpack<T, V>(a, ge);
      unpack<T, V>(b, ye);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dot = fmaf(ge[e], ye[e], dot);
        d[e] = f * ge[e];
      }
      *reinterpret_cast<P*>(dr + x) = pack<T, V>(d);
    }
    for (int64_t i = threadIdx.x; i < cut.ends; i += kThreads) {
      const int64_t x = cut.end(i);
      const float ge = Elem<T>::up(g[x]);
      dot = fmaf(ge, Elem<T>::up(yr[x]), dot);
      dr[x] = Elem<T>::down(f * ge);
    }
    dot = warp_sum(dot);
    if (threadIdx.x % 32 == 0) part[turn][threadIdx.x / 32] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      float s = part[turn][0];
#pragma unroll
      for (int i = 1; i < kThreads / 32; ++i) s += part[turn][i];
      dw[t * k + j] = s;
    }
    turn ^= 1;
  }
}

template <typename Id>
int sort(const void* ids, int64_t n, int E, int32_t* offsets, int32_t* row_of, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(moe_sort_kernel<Id>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (kSortWarps + 1) * kMaxExperts * 4);
  if (e != cudaSuccess) return launched(e);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kSortCtas);
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = size_t(kSortWarps + 1) * E * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {kSortCtas, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return launched(cudaLaunchKernelEx(&cfg, moe_sort_kernel<Id>, static_cast<const Id*>(ids), n, E, offsets, row_of));
}

template <typename T, typename Id>
int dispatch(const void* x, int64_t T_, int64_t H, int64_t ldx, const float* x_scale, const void* ids, int64_t k, int E,
             void* rows, int64_t ldr, float* row_scale, int32_t* offsets, int32_t* row_of, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(x, ldx, sizeof(T)) && aligned_rows(rows, ldr, sizeof(T));
  const T* xt = static_cast<const T*>(x);
  T* rt = static_cast<T*>(rows);
  if (T_ <= kSmallTokens && T_ * k <= kSmallRouting) {
    auto kernel = vec ? moe_dispatch_small_kernel<T, V, Id> : moe_dispatch_small_kernel<T, 1, Id>;
    kernel<<<unsigned(T_ + 1), kThreads, 0, stream>>>(xt, T_, H, ldx, x_scale, static_cast<const Id*>(ids), int(k), E,
                                                      rt, ldr, row_scale, offsets, row_of);
    return launched(cudaSuccess);
  }
  const int rc = sort<Id>(ids, T_ * k, E, offsets, row_of, stream);
  if (rc != ENTWINE_OK) return rc;
  auto kernel = vec ? moe_move_kernel<T, V> : moe_move_kernel<T, 1>;
  kernel<<<unsigned(T_), kThreads, 0, stream>>>(xt, H, ldx, x_scale, row_of, k, rt, ldr, row_scale);
  return launched(cudaSuccess);
}

template <typename T>
int dispatch_ids(const void* x, int64_t T_, int64_t H, int64_t ldx, const float* x_scale, const void* ids, int ids64,
                 int64_t k, int E, void* rows, int64_t ldr, float* row_scale, int32_t* offsets, int32_t* row_of,
                 cudaStream_t s) {
  return ids64 ? dispatch<T, int64_t>(x, T_, H, ldx, x_scale, ids, k, E, rows, ldr, row_scale, offsets, row_of, s)
               : dispatch<T, int32_t>(x, T_, H, ldx, x_scale, ids, k, E, rows, ldr, row_scale, offsets, row_of, s);
}

template <typename T>
int combine(const void* y, int64_t n_rows, int64_t H, int64_t ldy, const float* w, const int32_t* row_of, int64_t T_,
            int64_t k, void* out, int64_t ldo, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(y, ldy, sizeof(T)) && aligned_rows(out, ldo, sizeof(T));
  auto kernel = !vec ? moe_combine_anywhere_kernel<T>
                : k <= kReads / 2 ? moe_combine_kernel<T, V, kReads / 2, 2> : moe_combine_kernel<T, V, kReads, 1>;
  // one piece per thread until the tokens alone fill the GPU
  const int64_t pieces = (H + V - 1) / V;
  const int threads = pieces <= 128 || T_ < kFewTokens ? 128 : kThreads;
  const int64_t parts = T_ < kFewTokens ? std::min<int64_t>((pieces + threads - 1) / threads, 64) : 1;
  kernel<<<dim3(unsigned(T_), unsigned(parts)), threads, 0, stream>>>(static_cast<const T*>(y), n_rows, H, ldy, w,
                                                                      row_of, k, static_cast<T*>(out), ldo);
  return launched(cudaSuccess);
}

template <typename T>
int combine_bwd(const void* dout, int64_t T_, int64_t H, int64_t ldo, const void* y, int64_t n_rows, int64_t ldy,
                const float* w, const int32_t* row_of, int64_t k, void* dy, int64_t lddy, float* dw,
                cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned_rows(dout, ldo, sizeof(T)) && aligned_rows(y, ldy, sizeof(T)) &&
                   aligned_rows(dy, lddy, sizeof(T));
  auto kernel = vec ? moe_combine_bwd_kernel<T, V> : moe_combine_bwd_anywhere_kernel<T>;
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
  switch (size) {  // rows are moved as they are: only the size of an element counts
    case 1:
      return dispatch_ids<uint8_t>(x, T, H, ldx, x_scale, ids, ids64, k, int(E), rows, ldr, row_scale, offsets, row_of, s);
    case 2:
      return dispatch_ids<uint16_t>(x, T, H, ldx, x_scale, ids, ids64, k, int(E), rows, ldr, row_scale, offsets, row_of, s);
    default:
      return dispatch_ids<uint32_t>(x, T, H, ldx, x_scale, ids, ids64, k, int(E), rows, ldr, row_scale, offsets, row_of, s);
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
