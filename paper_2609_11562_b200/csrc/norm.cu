// Dropout from a counter-based generator (entwine_dropout), layer norm of residual + dropout(x) and its gradients
// (entwine_layer_norm, entwine_layer_norm_bwd).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "ops_common.cuh"
#include "sm100.cuh"

namespace entwine {
namespace {

constexpr int kGroup = 8;  // columns that one call of the generator decides on
constexpr int64_t kMaxCols = 2147483647 - 65536;  // column numbers of a CTA's last, idle threads fit 32 bits
constexpr int64_t kMaxRows = 2147483647;

// ------------------------------------------------------------------------------------------
// the generator
// ------------------------------------------------------------------------------------------
// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): a
// bijection of a 128-bit counter under a 64-bit key.  The counter is (column / 8, row, offset), the key the seed; its
// four words are eight 16-bit numbers, one for each column.  16 bits decide whether an element is kept with probability
// 1 - t / 65536 exactly, and what is kept is multiplied with 65536 / (65536 - t): the expectation is exact, p itself is
// taken to the nearest 2^-16.  With 32 bits an element the generator, 40 instructions a call, would be the bound instead
// of the memory.
struct Dropout {
  const int64_t* rng;  // {seed, offset}
  uint32_t t16;        // t * 65536: elements whose number is below t are dropped
  float scale;
  uint32_t row0;       // number of the first row
};

struct Stream {
  uint32_t k0, k1, o0, o1;
  __device__ __forceinline__ explicit Stream(const int64_t* rng) {
    const uint64_t seed = rng ? uint64_t(rng[0]) : 0, offset = rng ? uint64_t(rng[1]) : 0;
    k0 = uint32_t(seed);
    k1 = uint32_t(seed >> 32);
    o0 = uint32_t(offset);
    o1 = uint32_t(offset >> 32);
  }
  // The words of P groups of a row, `step` groups apart, round by round together: they share the keys.
  template <int P>
  __device__ __forceinline__ void words(uint32_t group, uint32_t step, uint32_t row, uint32_t (&c)[P][4]) const {
    uint32_t a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      c[i][0] = group + i * step;
      c[i][1] = row;
      c[i][2] = o0;
      c[i][3] = o1;
    }
#pragma unroll
    for (int r = 0; r < 10; ++r) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const uint64_t m = uint64_t(c[i][0]) * 0xD2511F53u, n = uint64_t(c[i][2]) * 0xCD9E8D57u;
        c[i][0] = uint32_t(n >> 32) ^ c[i][1] ^ a;
        c[i][1] = uint32_t(n);
        c[i][2] = uint32_t(m >> 32) ^ c[i][3] ^ b;
        c[i][3] = uint32_t(m);
      }
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
  }
};
// Two fp32 values in one register pair, and arithmetic on both at once.
struct Two {
  unsigned long long v;
  Two() = default;
  __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit Two(float a) : Two(a, a) {}
  __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Two add(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two mul(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// Number e of a group's eight is at least t: its word, the number shifted to the top, is at least t * 65536.
__device__ __forceinline__ bool kept(const uint32_t (&c)[4], int e, uint32_t t16) {
  return (e & 1 ? c[e / 2] : c[e / 2] << 16) >= t16;
}
// A dropped element is 0 whatever it held.
__device__ __forceinline__ void drop8(const uint32_t (&c)[4], const Dropout& d, float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = kept(c, 2 * j, d.t16) ? f[2 * j] : 0.0f, b = kept(c, 2 * j + 1, d.t16) ? f[2 * j + 1] : 0.0f;
    mul(Two(a, b), Two(d.scale)).get(f[2 * j], f[2 * j + 1]);
  }
}
__device__ __forceinline__ float drop1(const Stream& s, const Dropout& d, uint32_t row, uint32_t col, float f) {
  uint32_t c[1][4];
  s.words<1>(col / kGroup, 0, row, c);
  uint32_t w = c[0][0];
#pragma unroll
  for (int i = 1; i < 4; ++i) w = int(col % kGroup) / 2 == i ? c[0][i] : w;
  return (col & 1 ? w : w << 16) >= d.t16 ? f * d.scale : 0.0f;
}

// ------------------------------------------------------------------------------------------
// groups of eight elements
// ------------------------------------------------------------------------------------------
// Eight elements as they lie in memory: four words of a 16-bit type, eight of fp32.
template <typename T>
struct Raw {
  static constexpr int V = 16 / sizeof(T), N = 8 / V;
  Piece<T, V> v[N];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = reinterpret_cast<const Piece<T, V>*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<Piece<T, V>*>(p)[i] = v[i];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float g[V];
      unpack<T, V>(v[i], g);
#pragma unroll
      for (int e = 0; e < V; ++e) f[i * V + e] = g[e];
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float g[V];
#pragma unroll
      for (int e = 0; e < V; ++e) g[e] = f[i * V + e];
      v[i] = pack<T, V>(g);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = Piece<T, V>{};
  }
};
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
  Raw<T> r;
  r.load(p);
  r.get(f);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  Raw<T> r;
  r.set(f);
  r.store(p);
}

// Rows that start anywhere go element by element, and so that a warp's accesses lie side by side: it has 256 columns at a
// time, a lane eight of them 32 apart.  (Eight neighbouring ones a lane touch as many lines with each access as all eight
// accesses need together.)  `left` columns of the row lie at and behind the lane's first.
template <typename T>
__device__ __forceinline__ void load_apart(const T* p, int left, float (&f)[8]) {
  T v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 32 * e < left ? p[32 * e] : Elem<T>::down(0.0f);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = Elem<T>::up(v[e]);
}
template <typename T>
__device__ __forceinline__ void store_apart(T* p, int left, const float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (32 * e < left) p[32 * e] = Elem<T>::down(f[e]);
}
// The first column of a row's thread in its i-th turn.
__device__ __forceinline__ int first_apart(int i, int width, int lane) {
  return (i * width + (lane & ~31)) * kGroup + (lane & 31);
}
// Its eight columns lie in eight groups of the warp's 32, of which every lane has called the generator for one.
__device__ __forceinline__ void drop_apart(const uint32_t (&c)[4], const Dropout& d, int lane, float (&f)[8]) {
  uint32_t mine = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) mine |= uint32_t(kept(c, e, d.t16)) << e;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t group = __shfl_sync(0xffffffffu, mine, 4 * e + (lane & 31) / 8);
    f[e] = group >> (lane & 7) & 1 ? f[e] * d.scale : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ float rounded(float f) {
  return Elem<T>::up(Elem<T>::down(f));
}

__device__ __forceinline__ void twos(const float (&f)[8], Two (&t)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = Two(f[2 * j], f[2 * j + 1]);
}
__device__ __forceinline__ void ones(const Two (&t)[4], float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j].get(f[2 * j], f[2 * j + 1]);
}

// Weights: of the rows' type, or fp32.
template <typename T>
struct Weights {
  const void* at;
  bool wide;
  __device__ __forceinline__ void load(int col, float (&f)[8]) const {
    if (wide) load8(static_cast<const float*>(at) + col, f);
    else load8(static_cast<const T*>(at) + col, f);
  }
  __device__ __forceinline__ void apart(int col, int left, float (&f)[8]) const {
    if (wide) load_apart(static_cast<const float*>(at) + col, left, f);
    else load_apart(static_cast<const T*>(at) + col, left, f);
  }
  __device__ __forceinline__ float one(int col) const {
    return wide ? static_cast<const float*>(at)[col] : Elem<T>::up(static_cast<const T*>(at)[col]);
  }
};

// ------------------------------------------------------------------------------------------
// dropout
// ------------------------------------------------------------------------------------------
struct DropParams {
  const void* x;
  const void* residual;
  void* out;
  int64_t rows, ldx, ldr, ldo;
  int cols;
  Dropout d;
};

constexpr int kDropThreads = 256;

// P groups of eight elements a thread; a CTA (threads of a row x rows) goes from rows to rows.  16384 x 4096 bf16: 55 us.
// The generator takes 18 us of that (its wide multiplications issue at a quarter of the rate), so everything else has to be
// short: set-up is paid once a thread, and whole groups have no element-wise alternative beside them.
template <typename T, int P>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropParams a) {
  const int lane = int(threadIdx.x), width = int(blockDim.x);
  const Stream rng(a.d.rng);
  const int full = a.cols / kGroup, step = P * width;
  const int64_t stride = int64_t(gridDim.x) * blockDim.y;
  for (int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y; row < a.rows; row += stride) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const r = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
    T* const out = static_cast<T*>(a.out) + row * a.ldo;
    const uint32_t number = a.d.row0 + uint32_t(row);
    for (int g0 = int(blockIdx.y) * step + lane; g0 < full; g0 += int(gridDim.y) * step) {
      Raw<T> v[P], res[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int g = g0 + i * width;
        if (g < full) {
          v[i].load(x + int64_t(g) * kGroup);
          if (r) res[i].load(r + int64_t(g) * kGroup);
        }
      }
      uint32_t c[P][4];
      rng.words<P>(uint32_t(g0), uint32_t(width), number, c);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int g = g0 + i * width;
        if (g < full) {
          float f[8];
          v[i].get(f);
          drop8(c[i], a.d, f);
          if (r) {
            float h[8];
            res[i].get(h);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += h[e];
          }
          store8(out + int64_t(g) * kGroup, f);
        }
      }
    }
    const int col = full * kGroup + lane;
    if (blockIdx.y == 0 && lane < kGroup && col < a.cols) {
      float f = drop1(rng, a.d, number, uint32_t(col), Elem<T>::up(x[col]));
      if (r) f += Elem<T>::up(r[col]);
      out[col] = Elem<T>::down(f);
    }
  }
}

// The same for rows that start anywhere.
template <typename T, int P>
__global__ void __launch_bounds__(kDropThreads) dropout_anywhere_kernel(const DropParams a) {
  const int lane = int(threadIdx.x), width = int(blockDim.x), step = P * width * kGroup;
  const Stream rng(a.d.rng);
  const int64_t stride = int64_t(gridDim.x) * blockDim.y;
  for (int64_t row = int64_t(blockIdx.x) * blockDim.y + threadIdx.y; row < a.rows; row += stride) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const r = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
    T* const out = static_cast<T*>(a.out) + row * a.ldo;
    for (int64_t base = int64_t(blockIdx.y) * step; base < a.cols; base += int64_t(gridDim.y) * step) {
      float f[P][8], res[P][8];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int64_t c = base + first_apart(i, width, lane);
        const int left = int(a.cols - c);
        load_apart(x + c, left, f[i]);
        if (r) load_apart(r + c, left, res[i]);
      }
      uint32_t w[P][4];
      rng.words<P>(uint32_t(base / kGroup) + uint32_t(lane), uint32_t(width), a.d.row0 + uint32_t(row), w);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int64_t c = base + first_apart(i, width, lane);
        drop_apart(w[i], a.d, lane, f[i]);
        if (r) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[i][e] += res[i][e];
        }
        store_apart(out + c, int(a.cols - c), f[i]);
      }
    }
  }
}

template <typename T, int P>
int run_dropout_by(const DropParams& a, bool vec, cudaStream_t stream) {
  const int64_t groups = (int64_t(a.cols) + kGroup - 1) / kGroup, chunks = (groups + P * kDropThreads - 1) / (P * kDropThreads);
  // whole warps of a row's threads, as many as share its groups evenly; fewer where a short row has fewer groups
  int width = int((groups + P * chunks * 32 - 1) / (P * chunks * 32) * 32);
  while (vec && width > 8 && width / 2 * P >= groups) width /= 2;
  const int high = std::max(1, kDropThreads / width);
  // a few rows for every thread where there are many
  const int64_t bands = (a.rows + high - 1) / high, y = std::min<int64_t>(chunks, 1024);
  const dim3 grid(unsigned(std::min(bands, std::max<int64_t>(1, int64_t(sm_count()) * 32 / y))), unsigned(y));
  auto kernel = vec ? dropout_kernel<T, P> : dropout_anywhere_kernel<T, P>;
  kernel<<<grid, dim3(width, high), 0, stream>>>(a);
  return launched(cudaSuccess);
}

template <typename T>
int run_dropout(const DropParams& a, cudaStream_t stream) {
  const bool vec = aligned_rows(a.x, a.ldx, sizeof(T)) && aligned_rows(a.out, a.ldo, sizeof(T)) &&
                   (!a.residual || aligned_rows(a.residual, a.ldr, sizeof(T)));
  // little work: one group a thread, for the latency
  return a.rows * int64_t(a.cols) < (1 << 20) ? run_dropout_by<T, 1>(a, vec, stream) : run_dropout_by<T, 4>(a, vec, stream);
}

// ------------------------------------------------------------------------------------------
// layer norm
// ------------------------------------------------------------------------------------------
struct NormParams {
  const void* x;
  const void* residual;
  const void* weight;
  const void* bias;
  void* hidden;
  void* out;
  float* mean;
  float* rstd;
  int64_t rows, ldx, ldr, ldh, ldo;
  int cols, wide;
  float eps;
  Dropout d;
};

// Sum over the threads of a row: whole warps, threadIdx.x of them, from the CTA's warp first_warp on.
template <typename F>
__device__ __forceinline__ F row_sum(F v, F* part, int first_warp, int warps) {
  v = warp_sum(v);
  if (warps == 1) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) part[first_warp + threadIdx.x / 32] = v;
  __syncthreads();
  return warp_sum(lane < warps ? part[first_warp + lane] : F(0));
}

// A row in registers: P groups a thread, all of them whole and there (FULL), or up to P and one element of the last,
// incomplete group.  The mean first, then the mean of the squared distances from it: no difference of large sums.  A CTA is
// threads of a row x rows.  8192 x 5120 bf16 with dropout and residual take 74 us, 4.5 TB/s, 55 % of the issue slots with 25
// warps an SM: bound by the latency of a row's chain (loads, two sums) against the registers that hold rows, and by its
// instructions, 282 for eight columns.  More groups a thread are better (two: 83 us, one: 106): fewer threads meet at a row's
// sums; two fp32 operations an instruction, 75 us before.
template <typename T, int P, bool FULL, bool DROP>
__global__ void __launch_bounds__(P == 4 ? 512 : 1024) norm_rows_kernel(const NormParams a) {
  __shared__ float part[2][32];
  const int slot = int(threadIdx.y), lane = int(threadIdx.x), width = int(blockDim.x);
  const int64_t row = int64_t(blockIdx.x) * blockDim.y + slot;
  const bool there = row < a.rows;
  const int full = !there ? 0 : FULL ? P * width : a.cols / kGroup, tail = full * kGroup + lane;
  const bool has_tail = !FULL && there && lane < kGroup && tail < a.cols;
  auto whole = [&](int i) { return FULL ? there : i * width + lane < full; };
  const uint32_t number = a.d.row0 + uint32_t(row);
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  T* const hidden = a.hidden ? static_cast<T*>(a.hidden) + row * a.ldh : nullptr;
  Raw<T> v[P];
  float last = 0.0f, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int g = i * width + lane;
    if (whole(i)) v[i].load(x + g * kGroup);
    else v[i].zero();
  }
  if (has_tail) last = Elem<T>::up(x[tail]);
  if (DROP || res) {
    Raw<T> r[P];
    if (res) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int g = i * width + lane;
        if (whole(i)) r[i].load(res + g * kGroup);
      }
    }
    uint32_t c[P][4];
    const Stream rng(DROP ? a.d.rng : nullptr);
    if constexpr (DROP) rng.words<P>(uint32_t(lane), uint32_t(width), number, c);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (whole(i)) {
        float f[8];
        v[i].get(f);
        if constexpr (DROP) drop8(c[i], a.d, f);
        if (res) {
          float h[8];
          Two t[4], u[4];
          r[i].get(h);
          twos(f, t);
          twos(h, u);
#pragma unroll
          for (int j = 0; j < 4; ++j) t[j] = add(t[j], u[j]);
          ones(t, f);
        }
        v[i].set(f);  // rounded, as it is written
      }
    }
    if (has_tail) {
      if (DROP) last = drop1(rng, a.d, number, uint32_t(tail), last);
      last = rounded<T>(res ? last + Elem<T>::up(res[tail]) : last);
    }
  }
  Two h[P][4], all(0.0f);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (hidden && whole(i)) v[i].store(hidden + (i * width + lane) * kGroup);
    float f[8];
    v[i].get(f);
    twos(f, h[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) all = add(all, h[i][j]);
  }
  if (hidden && has_tail) hidden[tail] = Elem<T>::down(last);
  float even, odd;
  all.get(even, odd);
  sum = even + odd + last;
  const int warps = width / 32, first_warp = slot * warps;
  const float mean = row_sum(sum, part[0], first_warp, warps) / float(a.cols);
  const Two minus_mean(-mean);
  all = Two(0.0f);
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (whole(i)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[i][j] = add(h[i][j], minus_mean);
        all = fma(h[i][j], h[i][j], all);
      }
    }
  all.get(even, odd);
  float square = even + odd;
  if (has_tail) {
    last -= mean;
    square = fmaf(last, last, square);
  }
  const float rstd = 1.0f / sqrtf(row_sum(square, part[1], first_warp, warps) / float(a.cols) + a.eps);
  if (!there) return;
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const Weights<T> weight{a.weight, a.wide != 0}, bias{a.bias, a.wide != 0};
  T* const out = static_cast<T*>(a.out) + row * a.ldo;
  const Two by_rstd(rstd);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int g = i * width + lane;
    if (whole(i)) {
      float w[8], b[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      weight.load(g * kGroup, w);
      if (a.bias) bias.load(g * kGroup, b);
      Two t[4], u[4];
      twos(w, t);
      twos(b, u);
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = fma(mul(h[i][j], by_rstd), t[j], u[j]);
      ones(t, w);
      store8(out + g * kGroup, w);
    }
  }
  if (has_tail) out[tail] = Elem<T>::down(fmaf(last * rstd, weight.one(tail), a.bias ? bias.one(tail) : 0.0f));
}

constexpr int kLongThreads = 512;

// Rows too long for registers: a CTA goes through one three times.  What it normalises it reads again from hidden, or
// computes again where that is not kept.  A thread adds up the eight values of a turn in fp32, the turns in 64 bits: in
// fp32, which rounds equal values to the same side again and again, the mean of 2^24 of them was off by 2.6e-4 of it.
template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_long_rows_kernel(const NormParams a) {
  __shared__ double part[2][32];
  const int lane = int(threadIdx.x);
  const int64_t row = blockIdx.x;
  const Stream rng(a.d.rng);
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  T* const hidden = a.hidden ? static_cast<T*>(a.hidden) + row * a.ldh : nullptr;
  T* const out = static_cast<T*>(a.out) + row * a.ldo;
  constexpr int64_t kStep = int64_t(kLongThreads) * kGroup;
  auto values = [&](int64_t base, int64_t c, int left, float (&f)[8]) {
    load_apart(x + c, left, f);
    if (a.d.rng) {
      uint32_t w[1][4];
      rng.words<1>(uint32_t(base / kGroup) + uint32_t(lane), 0, a.d.row0 + uint32_t(row), w);
      drop_apart(w[0], a.d, lane, f);
    }
    float r[8] = {};
    if (res) load_apart(res + c, left, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = rounded<T>(res ? f[e] + r[e] : f[e]);
  };
  float f[8];
  double sum = 0.0;
  for (int64_t base = 0; base < a.cols; base += kStep) {
    const int64_t c = base + first_apart(0, kLongThreads, lane);
    const int left = int(a.cols - c);
    values(base, c, left, f);
    if (hidden) store_apart(hidden + c, left, f);
    float turn = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) turn += f[e];  // (0 behind the row's end)
    sum += turn;
  }
  const float mean = float(row_sum(sum, part[0], 0, kLongThreads / 32) / a.cols);
  sum = 0.0;
  for (int64_t base = 0; base < a.cols; base += kStep) {
    const int64_t c = base + first_apart(0, kLongThreads, lane);
    const int left = int(a.cols - c);
    if (hidden) load_apart(hidden + c, left, f);
    else values(base, c, left, f);
    float turn = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (32 * e < left) turn = fmaf(f[e] - mean, f[e] - mean, turn);
    sum += turn;
  }
  const float rstd = 1.0f / sqrtf(float(row_sum(sum, part[1], 0, kLongThreads / 32) / a.cols) + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const Weights<T> weight{a.weight, a.wide != 0}, bias{a.bias, a.wide != 0};
  for (int64_t base = 0; base < a.cols; base += kStep) {
    const int64_t c = base + first_apart(0, kLongThreads, lane);
    const int left = int(a.cols - c);
    if (hidden) load_apart(hidden + c, left, f);
    else values(base, c, left, f);
    float w[8], b[8] = {};
    weight.apart(int(c), left, w);
    if (a.bias) bias.apart(int(c), left, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = fmaf((f[e] - mean) * rstd, w[e], b[e]);
    store_apart(out + c, left, f);
  }
}

// The same for rows that start anywhere.
template <typename T, int P>
__global__ void __launch_bounds__(1024) norm_rows_anywhere_kernel(const NormParams a) {
  __shared__ float part[2][32];
  const int slot = int(threadIdx.y), lane = int(threadIdx.x), width = int(blockDim.x);
  const int64_t row = int64_t(blockIdx.x) * blockDim.y + slot;
  const int cols = row < a.rows ? a.cols : 0;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  T* const hidden = a.hidden ? static_cast<T*>(a.hidden) + row * a.ldh : nullptr;
  float h[P][8], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) load_apart(x + first_apart(i, width, lane), cols - first_apart(i, width, lane), h[i]);
  if (a.d.rng || res) {
    const Stream rng(a.d.rng);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = first_apart(i, width, lane);
      float r[8] = {};
      if (res) load_apart(res + c, cols - c, r);
      if (a.d.rng) {
        uint32_t w[1][4];
        rng.words<1>(uint32_t(i * width + lane), 0, a.d.row0 + uint32_t(row), w);
        drop_apart(w[0], a.d, lane, h[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = rounded<T>(res ? h[i][e] + r[e] : h[i][e]);
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = first_apart(i, width, lane);
    if (hidden) store_apart(hidden + c, cols - c, h[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += h[i][e];  // (0 behind the row's end)
  }
  const int warps = width / 32, first_warp = slot * warps;
  const float mean = row_sum(sum, part[0], first_warp, warps) / float(a.cols);
  float square = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int left = cols - first_apart(i, width, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[i][e] -= mean;
      if (32 * e < left) square = fmaf(h[i][e], h[i][e], square);
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum(square, part[1], first_warp, warps) / float(a.cols) + a.eps);
  if (cols == 0) return;
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const Weights<T> weight{a.weight, a.wide != 0}, bias{a.bias, a.wide != 0};
  T* const out = static_cast<T*>(a.out) + row * a.ldo;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = first_apart(i, width, lane), left = cols - c;
    float w[8], b[8] = {};
    weight.apart(c, left, w);
    if (a.bias) bias.apart(c, left, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = fmaf(h[i][e] * rstd, w[e], b[e]);
    store_apart(out + c, left, h[i]);
  }
}

template <typename T, bool DROP>
auto pick_norm(int each, bool full) {
  if (!full)
    return each == 4   ? norm_rows_kernel<T, 4, false, DROP>
           : each == 2 ? norm_rows_kernel<T, 2, false, DROP>
                       : norm_rows_kernel<T, 1, false, DROP>;
  return each == 4   ? norm_rows_kernel<T, 4, true, DROP>
         : each == 2 ? norm_rows_kernel<T, 2, true, DROP>
                     : norm_rows_kernel<T, 1, true, DROP>;
}

template <typename T>
int run_norm(const NormParams& a, cudaStream_t stream) {
  auto aligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool vec = aligned_rows(a.x, a.ldx, sizeof(T)) && aligned_rows(a.out, a.ldo, sizeof(T)) &&
                   (!a.residual || aligned_rows(a.residual, a.ldr, sizeof(T))) &&
                   (!a.hidden || aligned_rows(a.hidden, a.ldh, sizeof(T))) && aligned(a.weight) &&
                   (!a.bias || aligned(a.bias));
  const int groups = (a.cols + kGroup - 1) / kGroup;
  if (groups > 2048) {
    norm_long_rows_kernel<T><<<unsigned(a.rows), kLongThreads, 0, stream>>>(a);
    return launched(cudaSuccess);
  }
  // Groups a thread: few rows, many threads with little each, for the latency; else four, or what divides a row evenly.
  auto fits = [&](int p) { return vec && a.cols % kGroup == 0 && groups % (32 * p) == 0 && groups / p <= (p == 4 ? 512 : 1024); };
  const int most = a.rows < 512 ? 1 : a.rows < 2048 ? 2 : 4;
  int each = most;
  while (each > 1 && !fits(each)) each /= 2;
  const bool full = fits(each);
  if (!full) {
    // little that is not there (20000 rows of 300 with four groups a thread: 63 us, of 128 groups' places for 38); at most two
    // groups where rows start anywhere (four: 233 us instead of 165 for 8192 rows of 5121 bf16)
    auto idle = [&](int p) { return (groups + 32 * p - 1) / (32 * p) * 32 * p * 4 > groups * 5; };
    each = std::min(most, vec ? 4 : 2);
    while (each > 1 && idle(each)) each /= 2;
    if (groups > each * 1024) each = 2;  // (2048 groups at most)
  }
  const int width = (groups + each * 32 - 1) / (each * 32) * 32, high = std::max(1, 128 / width);
  const unsigned grid = unsigned((a.rows + high - 1) / high);
  auto kernel = !vec ? (each == 1 ? norm_rows_anywhere_kernel<T, 1> : norm_rows_anywhere_kernel<T, 2>)
                : a.d.rng ? pick_norm<T, true>(each, full) : pick_norm<T, false>(each, full);
  kernel<<<grid, dim3(width, high), 0, stream>>>(a);
  return launched(cudaSuccess);
}

// ------------------------------------------------------------------------------------------
// layer norm, gradients
// ------------------------------------------------------------------------------------------
struct GradParams {
  const void* dout;
  const void* hidden;
  const void* weight;
  const float* mean;
  const float* rstd;
  const void* dhidden;
  void* dx;
  void* dresidual;
  float* work;  // [parts][2][cols]: each part's sums over its rows, of the weight's gradient and the bias's
  int64_t rows, ldo, ldh, lddh, lddx, lddr;
  int cols, wide;
  Dropout d;
};

// How the rows are spread: every CTA gives a part of the sums.  `ctas` is the most of them that any type and alignment of
// these extents launches; the workspace has room for so many.
struct GradPlan {
  int each, width, high, ctas;  // groups of eight columns a thread, threads of a row, rows of a CTA at a time
  bool in_registers;
};

constexpr int kGradThreads = 512;        // at most
constexpr int kGradHalf = 320;           // at most, where two CTAs and their rows of 16-bit elements share an SM
constexpr int kGradHalfWide = 256;       // at most, where two and their rows of fp32 do
constexpr int kGradWide = 352;           // at most, where two CTAs without rows in shared memory do
constexpr int kGradSms = 148;             // (the extents alone say how large the workspace is)
constexpr int kStripRows = 64;           // rows of a part where the columns are summed by themselves
// Two CTAs of the kernel that copies rows ahead share an SM (registers, and shared memory: 88 and 110 KB of 16-bit elements, 112
// KB of fp32).
template <typename T>
constexpr bool two_copy(int threads) {
  return threads <= (sizeof(T) == 2 ? kGradHalf : kGradHalfWide);
}
// Rows that it has under way or in work with `each` groups a thread: as many as the SM's shared memory holds.
template <typename T>
__host__ __device__ constexpr int copy_depth(int each) {
  return sizeof(T) == 2 && each == 2 ? 3 : 2;
}
// Its shared memory for `places` threads: those rows' dout, hidden and dhidden; the weights, in fp32, with two groups.
template <typename T>
constexpr int copy_bytes(int each, int places) {
  return places * each * kGroup * (3 * copy_depth<T>(each) * int(sizeof(T)) + (each == 2 ? 4 : 0));
}

GradPlan grad_plan(int64_t rows, int64_t cols) {
  GradPlan g;
  const int64_t groups = (cols + kGroup - 1) / kGroup;
  g.in_registers = groups <= 4 * kGradThreads;
  if (!g.in_registers) {
    g.each = g.high = 1;
    g.width = kLongThreads;
    g.ctas = int(std::min<int64_t>(256, std::max<int64_t>(1, (rows + kStripRows - 1) / kStripRows)));
    return g;
  }
  g.each = groups <= 2 * kGradThreads ? 2 : 4;
  g.width = int((groups + g.each * 32 - 1) / (g.each * 32)) * 32;
  g.high = std::max(1, 256 / g.width);
  const int resident = g.each == 2 && g.width <= kGradWide ? 2 : 1;
  g.ctas = int(std::min<int64_t>((rows + g.high - 1) / g.high, int64_t(resident) * kGradSms));
  g.ctas = std::max(1, g.ctas);
  return g;
}

// Two sums over the threads of a row, of 16 warps at most: the halves of a warp take one each.  `part` is one of two buffers
// in turn: one barrier a row.
__device__ __forceinline__ float2 row_sum2(float2 v, float2* part, int first_warp, int warps) {
  const int lane = threadIdx.x & 31;
  const bool upper = lane & 16;
  float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xffffffffu, upper ? v.x : v.y, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (warps > 1) {
    if ((lane & 15) == 0) reinterpret_cast<float*>(part)[2 * (first_warp + threadIdx.x / 32) + (lane >> 4)] = s;
    __syncthreads();
    s = (lane & 15) < warps ? reinterpret_cast<const float*>(part)[2 * (first_warp + (lane & 15)) + (lane >> 4)] : 0.0f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  const float other = __shfl_xor_sync(0xffffffffu, s, 16);
  return upper ? make_float2(other, s) : make_float2(s, other);
}

// A CTA's part of the sums: put(to) writes a thread's own to a [2][cols].  Those of several
// rows at a time meet in shared memory first.
template <typename F>
__device__ __forceinline__ void put_sums(const GradParams& a, float* pool, int slot, int high, const F& put) {
  float* const part = a.work + int64_t(blockIdx.x) * 2 * a.cols;
  grid_let_next_start();  // (the launch that adds the parts; it waits for them)
  if (high == 1) {
    put(part);
    return;
  }
  __syncthreads();  // (what else the pool was for is over)
  put(pool + slot * 2 * a.cols);
  __syncthreads();
  for (int i = int(threadIdx.y * blockDim.x + threadIdx.x); i < 2 * a.cols; i += int(blockDim.x * blockDim.y)) {
    float v = pool[i];
    for (int s = 1; s < high; ++s) v += pool[s * 2 * a.cols + i];
    part[i] = v;
  }
}

// With g = dout weight and n = (hidden - mean) rstd: dh = rstd (g - mean(g) - n mean(g n)) + dhidden.  A thread keeps its
// columns from row to row, and with them their sums of dout n and dout.  This form is for rows that start anywhere.  With four
// groups a thread the second half of a row reads it again.
template <typename T, int P, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS <= kGradWide ? 2 : 1) norm_grad_anywhere_kernel(const GradParams a) {
  extern __shared__ float pool[];
  __shared__ float2 part[2][32];
  const int slot = int(threadIdx.y), lane = int(threadIdx.x), width = int(blockDim.x), high = int(blockDim.y);
  const int warps = width / 32, first_warp = slot * warps;
  const Weights<T> weight{a.weight, a.wide != 0};
  const Stream rng(a.d.rng);
  const float per_col = 1.0f / float(a.cols);
  float dw[P][8] = {}, db[P][8] = {};
  int turn = 0;
  for (int64_t row0 = int64_t(blockIdx.x) * high; row0 < a.rows; row0 += int64_t(gridDim.x) * high, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool there = row < a.rows;
    const int cols = there ? a.cols : 0;
    const T* const dout = static_cast<const T*>(a.dout) + row * a.ldo;
    const T* const hidden = static_cast<const T*>(a.hidden) + row * a.ldh;
    constexpr int KEEP = P <= 2 ? P : 1;
    float g[KEEP][8], n[KEEP][8];
    float2 s = make_float2(0.0f, 0.0f);
    const float mean = there ? a.mean[row] : 0.0f, rstd = there ? a.rstd[row] : 0.0f;
    auto load = [&](int i) {
      const int c = first_apart(i, width, lane);
      load_apart(dout + c, cols - c, g[i % KEEP]);  // (0 behind the row's end, and so is what is made of it)
      load_apart(hidden + c, cols - c, n[i % KEEP]);
    };
    if constexpr (KEEP == P) {
#pragma unroll
      for (int i = 0; i < P; ++i) load(i);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = first_apart(i, width, lane), k = i % KEEP;
      if constexpr (KEEP < P) load(i);
      float w[8];
      weight.apart(c, cols - c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[k][e] = (n[k][e] - mean) * rstd;
        dw[i][e] = 32 * e < cols - c ? fmaf(g[k][e], n[k][e], dw[i][e]) : dw[i][e];
        db[i][e] += g[k][e];
        g[k][e] *= w[e];
        s.x += g[k][e];
        s.y = 32 * e < cols - c ? fmaf(g[k][e], n[k][e], s.y) : s.y;
      }
    }
    s = row_sum2(s, part[turn], first_warp, warps);
    s.x *= per_col;
    s.y *= per_col;
    if (!there) continue;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = first_apart(i, width, lane), k = i % KEEP;
      if constexpr (KEEP < P) {
        float w[8];
        load(i);
        weight.apart(c, cols - c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          n[k][e] = (n[k][e] - mean) * rstd;
          g[k][e] *= w[e];
        }
      }
      float f[8] = {};
      if (a.dhidden) load_apart(static_cast<const T*>(a.dhidden) + row * a.lddh + c, cols - c, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = fmaf(rstd, g[k][e] - s.x - n[k][e] * s.y, f[e]);
      if (a.dresidual) store_apart(static_cast<T*>(a.dresidual) + row * a.lddr + c, cols - c, f);
      if (a.d.rng) {
        uint32_t w[1][4];
        rng.words<1>(uint32_t(i * width + lane), 0, a.d.row0 + uint32_t(row), w);
        drop_apart(w[0], a.d, lane, f);
      }
      store_apart(static_cast<T*>(a.dx) + row * a.lddx + c, cols - c, f);
    }
  }
  put_sums(a, pool, slot, high, [&](float* sums) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = first_apart(i, width, lane);
      store_apart(sums + c, a.cols - c, dw[i]);
      store_apart(sums + a.cols + c, a.cols - c, db[i]);
    }
  });
}

// The same for rows on 16-byte boundaries (FULL: whose groups are all whole and there).  Every thread copies its own pieces
// of dout, hidden and dhidden ahead, into places of shared memory that no other thread looks at: D rows are under way or in
// work, and the only barrier of a row is that of its two sums.  What the second half of a row needs is read again instead of
// held in registers, the weights (in fp32) too: 96 registers have to do where two CTAs share an SM.  8192 x 5120 bf16 with
// dropout and the residual stream's gradient take 102 us with the sums' launch (5), 4.1 TB/s, half of the issue slots; loads in
// order instead of copies ahead 236 us, one fp32 operation an instruction and weights from global memory 120.
template <typename T, int P, int THREADS, bool FULL>
__global__ void __launch_bounds__(THREADS, two_copy<T>(THREADS) ? 2 : 1) norm_grad_kernel(const GradParams a) {
  constexpr int D = copy_depth<T>(P), N = Raw<T>::N, V = Raw<T>::V, kRow = 3 * P * N * THREADS;  // 16-byte places of a row
  constexpr bool KEPT = P == 2;  // weights kept in shared memory, fp32, behind the rows
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float2 part[2][32];
  const int slot = int(threadIdx.y), lane = int(threadIdx.x), width = int(blockDim.x), high = int(blockDim.y);
  const int full = FULL ? P * width : a.cols / kGroup, tail = full * kGroup + lane;
  const bool has_tail = !FULL && lane < kGroup && tail < a.cols;
  const int warps = width / 32, first_warp = slot * warps;
  const Weights<T> weight{a.weight, a.wide != 0};
  const Stream rng(a.d.rng);
  const float per_col = 1.0f / float(a.cols);
  const int64_t stride = int64_t(gridDim.x) * high;
  int64_t row = int64_t(blockIdx.x) * high + slot, ahead = row;
  const T *dout = static_cast<const T*>(a.dout) + row * a.ldo + lane * kGroup,
          *hidden = static_cast<const T*>(a.hidden) + row * a.ldh + lane * kGroup,
          *dhidden = a.dhidden ? static_cast<const T*>(a.dhidden) + row * a.lddh + lane * kGroup : nullptr;
  uint4* const mine = reinterpret_cast<uint4*>(ring) + slot * width + lane;
  auto whole = [&](int i) { return FULL || i * width + lane < full; };
  // the next row of this thread's to place d
  auto fetch = [&](int d) {
    if (ahead < a.rows) {
      const uint32_t to = smem_u32(mine + d * kRow);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (whole(i)) {
#pragma unroll
          for (int piece = 0; piece < N; ++piece) {
            const int at = i * width * kGroup + piece * V;
            cp_async16(to + ((0 * P + i) * N + piece) * THREADS * 16, dout + at);
            cp_async16(to + ((1 * P + i) * N + piece) * THREADS * 16, hidden + at);
            if (a.dhidden) cp_async16(to + ((2 * P + i) * N + piece) * THREADS * 16, dhidden + at);
          }
        }
    }
    cp_async_commit();
    ahead += stride;
    dout += stride * a.ldo;
    hidden += stride * a.ldh;
    if (a.dhidden) dhidden += stride * a.lddh;
  };
  auto get = [&](const uint4* from, int what, int i, Two (&t)[4]) {
    Raw<T> r;
#pragma unroll
    for (int piece = 0; piece < N; ++piece) {
      const uint4 w = from[((what * P + i) * N + piece) * THREADS];
      memcpy(&r.v[piece], &w, 16);
    }
    float f[8];
    r.get(f);
    twos(f, t);
  };
  uint4* const kept_weights = mine + D * kRow;
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (whole(i)) {
        float w[8];
        weight.load((i * width + lane) * kGroup, w);
        uint4 v[2];
        memcpy(v, w, sizeof(v));
        kept_weights[2 * i * THREADS] = v[0];
        kept_weights[(2 * i + 1) * THREADS] = v[1];
      }
  }
  auto get_weight = [&](int i, Two (&t)[4]) {
    float w[8];
    if constexpr (KEPT) {
      const uint4 v[2] = {kept_weights[2 * i * THREADS], kept_weights[(2 * i + 1) * THREADS]};
      memcpy(w, v, sizeof(v));
    } else {
      weight.load((i * width + lane) * kGroup, w);
    }
    twos(w, t);
  };
  Two dw[P][4], db[P][4];
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[i][j] = db[i][j] = Two(0.0f);
  float dw_tail = 0.0f, db_tail = 0.0f;
  int turn = 0, d = 0;
#pragma unroll
  for (int i = 0; i < D - 1; ++i) fetch(i);
  float mean = 0.0f, rstd = 0.0f, next_mean = row < a.rows ? a.mean[row] : 0.0f, next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
  for (int64_t row0 = int64_t(blockIdx.x) * high; row0 < a.rows; row0 += stride, row += stride, turn ^= 1) {
    const bool there = row < a.rows;
    fetch(d + D - 1 < D ? d + D - 1 : d - 1);
    mean = next_mean;
    rstd = next_rstd;
    if (row + stride < a.rows) {
      next_mean = a.mean[row + stride];
      next_rstd = a.rstd[row + stride];
    }
    cp_async_wait<D - 1>();
    const uint4* const from = mine + d * kRow;
    const Two minus_mean(-mean), by_rstd(rstd);
    Two sum(0.0f), dot(0.0f);
    float2 s = make_float2(0.0f, 0.0f);
    float g_tail = 0.0f, n_tail = 0.0f;
    if (there) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (whole(i)) {
          Two g[4], h[4], w[4];
          get(from, 0, i, g);
          get(from, 1, i, h);
          get_weight(i, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const Two n = mul(add(h[j], minus_mean), by_rstd);
            dw[i][j] = fma(g[j], n, dw[i][j]);
            db[i][j] = add(db[i][j], g[j]);
            const Two gw = mul(g[j], w[j]);
            sum = add(sum, gw);
            dot = fma(gw, n, dot);
          }
        }
      }
      if (has_tail) {
        g_tail = Elem<T>::up(static_cast<const T*>(a.dout)[row * a.ldo + tail]);
        n_tail = (Elem<T>::up(static_cast<const T*>(a.hidden)[row * a.ldh + tail]) - mean) * rstd;
        dw_tail = fmaf(g_tail, n_tail, dw_tail);
        db_tail += g_tail;
        g_tail *= weight.one(tail);
        s.x += g_tail;
        s.y = fmaf(g_tail, n_tail, s.y);
      }
    }
    float even, odd;
    sum.get(even, odd);
    s.x += even + odd;
    dot.get(even, odd);
    s.y += even + odd;
    s = row_sum2(s, part[turn], first_warp, warps);
    s.x *= per_col;
    s.y *= per_col;
    const Two minus_sum(-s.x), minus_dot(-s.y);
    if (there) {
      T* const dresidual = a.dresidual ? static_cast<T*>(a.dresidual) + row * a.lddr : nullptr;
      T* const dx = static_cast<T*>(a.dx) + row * a.lddx;
      const uint32_t number = a.d.row0 + uint32_t(row);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (whole(i)) {
          const int g0 = i * width + lane;
          Two g[4], h[4], w[4], t[4];
          get(from, 0, i, g);
          get(from, 1, i, h);
          get_weight(i, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) t[j] = Two(0.0f);
          if (a.dhidden) get(from, 2, i, t);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const Two n = mul(add(h[j], minus_mean), by_rstd);
            t[j] = fma(by_rstd, fma(n, minus_dot, fma(g[j], w[j], minus_sum)), t[j]);
          }
          float f[8];
          ones(t, f);
          if (dresidual) store8(dresidual + g0 * kGroup, f);
          if (a.d.rng) {
            uint32_t c[1][4];
            rng.words<1>(uint32_t(g0), 0, number, c);
            drop8(c[0], a.d, f);
          }
          store8(dx + g0 * kGroup, f);
        }
      }
      if (has_tail) {
        float f = fmaf(rstd, g_tail - s.x - n_tail * s.y,
                       a.dhidden ? Elem<T>::up(static_cast<const T*>(a.dhidden)[row * a.lddh + tail]) : 0.0f);
        if (dresidual) dresidual[tail] = Elem<T>::down(f);
        if (a.d.rng) f = drop1(rng, a.d, number, uint32_t(tail), f);
        dx[tail] = Elem<T>::down(f);
      }
    }
    if (++d == D) d = 0;
  }
  cp_async_wait<0>();
  put_sums(a, reinterpret_cast<float*>(ring), slot, high, [&](float* sums) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (whole(i)) {
        float f[8];
        ones(dw[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[(i * width + lane) * kGroup + e] = f[e];
        ones(db[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[a.cols + (i * width + lane) * kGroup + e] = f[e];
      }
    }
    if (has_tail) {
      sums[tail] = dw_tail;
      sums[a.cols + tail] = db_tail;
    }
  });
}

// By threads (256, 320 or 512); four groups a thread only where two rows of 512 such threads fit (16-bit types).
template <typename T, bool FULL>
auto pick_grad(int each, int threads) {
  if constexpr (sizeof(T) == 2)
    if (each == 4) return norm_grad_kernel<T, 4, kGradThreads, FULL>;
  return threads == 256         ? norm_grad_kernel<T, 2, 256, FULL>
         : threads == kGradHalf ? norm_grad_kernel<T, 2, kGradHalf, FULL>
                                : norm_grad_kernel<T, 2, kGradThreads, FULL>;
}

// Rows too long for that: dx by a CTA that reads a row twice (its two sums as in norm_long_rows_kernel), ...
template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_grad_long_rows_kernel(const GradParams a) {
  __shared__ double part[2][32];
  const int lane = int(threadIdx.x);
  const int64_t row = blockIdx.x;
  const T* const dout = static_cast<const T*>(a.dout) + row * a.ldo;
  const T* const hidden = static_cast<const T*>(a.hidden) + row * a.ldh;
  const Weights<T> weight{a.weight, a.wide != 0};
  const Stream rng(a.d.rng);
  const float mean = a.mean[row], rstd = a.rstd[row];
  constexpr int64_t kStep = int64_t(kLongThreads) * kGroup;
  // g = dout weight and n of a turn's columns; behind the row's end g is 0
  auto load = [&](int64_t c, int left, float (&g)[8], float (&n)[8]) {
    float w[8];
    load_apart(dout + c, left, g);
    load_apart(hidden + c, left, n);
    weight.apart(int(c), left, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      g[e] *= w[e];
      n[e] = (n[e] - mean) * rstd;
    }
  };
  float g[8], n[8];
  double sum = 0.0, dot = 0.0;
  for (int64_t base = 0; base < a.cols; base += kStep) {
    const int64_t c = base + first_apart(0, kLongThreads, lane);
    const int left = int(a.cols - c);
    load(c, left, g, n);
    float2 turn = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (32 * e < left) {
        turn.x += g[e];
        turn.y = fmaf(g[e], n[e], turn.y);
      }
    sum += turn.x;
    dot += turn.y;
  }
  const float2 s = make_float2(float(row_sum(sum, part[0], 0, kLongThreads / 32) / a.cols),
                               float(row_sum(dot, part[1], 0, kLongThreads / 32) / a.cols));
  for (int64_t base = 0; base < a.cols; base += kStep) {
    const int64_t c = base + first_apart(0, kLongThreads, lane);
    const int left = int(a.cols - c);
    float f[8] = {};
    load(c, left, g, n);
    if (a.dhidden) load_apart(static_cast<const T*>(a.dhidden) + row * a.lddh + c, left, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = fmaf(rstd, g[e] - s.x - n[e] * s.y, f[e]);
    if (a.dresidual) store_apart(static_cast<T*>(a.dresidual) + row * a.lddr + c, left, f);
    if (a.d.rng) {
      uint32_t w[1][4];
      rng.words<1>(uint32_t(base / kGroup) + uint32_t(lane), 0, a.d.row0 + uint32_t(row), w);
      drop_apart(w[0], a.d, lane, f);
    }
    store_apart(static_cast<T*>(a.dx) + row * a.lddx + c, left, f);
  }
}

// ... and the sums of a column over a part of the rows by a thread.
template <typename T>
__global__ void __launch_bounds__(128) norm_grad_columns_kernel(const GradParams a, int parts) {
  const int64_t c = int64_t(blockIdx.x) * 128 + threadIdx.x;
  if (c >= a.cols) return;
  const int part = int(blockIdx.y);
  const int64_t first = a.rows * part / parts, end = a.rows * (part + 1) / parts;
  float dw = 0.0f, db = 0.0f;
  for (int64_t row = first; row < end; ++row) {
    const float dy = Elem<T>::up(static_cast<const T*>(a.dout)[row * a.ldo + c]);
    const float n = (Elem<T>::up(static_cast<const T*>(a.hidden)[row * a.ldh + c]) - a.mean[row]) * a.rstd[row];
    dw = fmaf(dy, n, dw);
    db += dy;
  }
  a.work[int64_t(part) * 2 * a.cols + c] = dw;
  a.work[int64_t(part) * 2 * a.cols + a.cols + c] = db;
}

constexpr int kSumThreads = 512;

// The parts' sums added up, in a fixed order: X columns a CTA.
template <int X>
__global__ void __launch_bounds__(kSumThreads) norm_sum_kernel(const float* work, int parts, int cols, float* dweight,
                                                               float* dbias) {
  constexpr int Y = kSumThreads / X;
  __shared__ float sums[Y][X + 1];
  const int x = int(threadIdx.x) % X, y = int(threadIdx.x) / X;
  const int64_t c = int64_t(blockIdx.x) * X + x;
  const float* const in = work + int64_t(blockIdx.y) * cols + c;
  float v = 0.0f;
  grid_wait();
  if (c < cols) {
#pragma unroll 8
    for (int i = y; i < parts; i += Y) v += in[int64_t(i) * 2 * cols];
  }
  sums[y][x] = v;
#pragma unroll
  for (int half = Y / 2; half > 0; half /= 2) {
    __syncthreads();
    if (y < half) sums[y][x] += sums[y + half][x];
  }
  if (y == 0 && c < cols) (blockIdx.y == 0 ? dweight : dbias)[c] = sums[0][x];
}

template <typename T>
int run_grad(const GradParams& a, float* dweight, float* dbias, cudaStream_t stream) {
  const GradPlan plan = grad_plan(a.rows, a.cols);
  int parts = a.rows > 0 ? plan.ctas : 0;  // (of no rows the sums are 0)
  auto aligned = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  if (a.rows == 0) {
  } else if (plan.in_registers) {
    const bool vec = aligned_rows(a.dout, a.ldo, sizeof(T)) && aligned_rows(a.hidden, a.ldh, sizeof(T)) &&
                     aligned_rows(a.dx, a.lddx, sizeof(T)) && (!a.dhidden || aligned_rows(a.dhidden, a.lddh, sizeof(T))) &&
                     (!a.dresidual || aligned_rows(a.dresidual, a.lddr, sizeof(T))) && aligned(a.weight);
    const dim3 threads(plan.width, plan.high);
    if (vec && (plan.each == 2 || sizeof(T) == 2)) {
      const int count = plan.width * plan.high;
      const int places = plan.each == 4 || count > kGradHalf ? kGradThreads : count > 256 ? kGradHalf : 256;
      // no more CTAs than the GPU holds at once: others would begin when these end (8192 x 5632 bf16 114 us instead of 124,
      // 4096 x 5120 fp32 116 instead of 120)
      if (!two_copy<T>(places)) parts = std::min(parts, kGradSms);
      const bool full = a.cols == plan.width * plan.each * kGroup;
      const int bytes = copy_bytes<T>(plan.each, places);
      auto kernel = full ? pick_grad<T, true>(plan.each, places) : pick_grad<T, false>(plan.each, places);
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
      if (e != cudaSuccess) return launched(e);
      kernel<<<unsigned(parts), threads, bytes, stream>>>(a);
    } else {
      // (the registers of 256 threads hold what spills with 352, 45 and 54 us for 8192 rows of 1021 bf16; but two CTAs of up to
      // 352 are worth it, 217 us instead of 267 for 8192 rows of 5121)
      const int count = plan.width * plan.high;
      auto kernel = plan.each == 4       ? norm_grad_anywhere_kernel<T, 4, kGradThreads>
                    : count <= 256       ? norm_grad_anywhere_kernel<T, 2, 256>
                    : count <= kGradWide ? norm_grad_anywhere_kernel<T, 2, kGradWide>
                                         : norm_grad_anywhere_kernel<T, 2, kGradThreads>;
      const int pool = plan.high > 1 ? plan.high * 2 * a.cols * 4 : 0;  // (32 KB at most: 256 threads' 16 columns)
      kernel<<<unsigned(parts), threads, pool, stream>>>(a);
    }
  } else {
    norm_grad_long_rows_kernel<T><<<unsigned(a.rows), kLongThreads, 0, stream>>>(a);
    const dim3 grid(unsigned((int64_t(a.cols) + 127) / 128), unsigned(parts));
    norm_grad_columns_kernel<T><<<grid, 128, 0, stream>>>(a, parts);
  }
  const int rc = launched(cudaSuccess);
  if (rc != ENTWINE_OK) return rc;
  // (narrow strips where there are few columns: more CTAs, fewer parts for each thread)
  const int x = a.cols >= 4096 ? 32 : 8;
  const dim3 grid(unsigned((int64_t(a.cols) + x - 1) / x), dbias ? 2 : 1);
  auto kernel = x == 32 ? norm_sum_kernel<32> : norm_sum_kernel<8>;
  // It may start while the parts' launch ends, and waits for it: 777 x 1021 fp32 in 12.1 us instead of 12.9.
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kSumThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = a.rows > 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, static_cast<const float*>(a.work), parts, a.cols, dweight, dbias));
}

bool floating(int dtype) { return dtype == ENTWINE_BF16 || dtype == ENTWINE_FP16 || dtype == ENTWINE_FP32; }
int64_t bytes_of(int dtype) { return dtype == ENTWINE_FP32 ? 4 : 2; }

// p, the generator's state and the first row's number; false where they cannot be.
bool make_dropout(double p, const int64_t* rng, int64_t row0, int64_t rows, Dropout* d) {
  if (!(p >= 0.0 && p < 1.0) || row0 < 0 || row0 > (int64_t(1) << 32) - rows) return false;
  const double t = std::nearbyint(p * 65536.0);
  if (t > 65535.0 || (p > 0.0 && bad_pointer(rng, 8))) return false;
  d->rng = t > 0.0 ? rng : nullptr;
  d->t16 = uint32_t(t) << 16;
  d->scale = float(65536.0 / (65536.0 - t));
  d->row0 = uint32_t(row0);
  return true;
}

}  // namespace
}  // namespace entwine

using namespace entwine;

extern "C" {

int entwine_dropout(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* residual, int64_t ldr,
                    double p, const int64_t* rng, int64_t row0, void* out, int64_t ldo, void* stream) {
  if (!floating(dtype) || rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols || ldx < cols || ldo < cols ||
      (residual && ldr < cols))
    return ENTWINE_ERR_INVALID;
  DropParams a;
  std::memset(&a, 0, sizeof(a));
  if (!make_dropout(p, rng, row0, rows, &a.d)) return ENTWINE_ERR_INVALID;
  if (rows == 0) return ENTWINE_OK;
  const int64_t elem = bytes_of(dtype);
  if (bad_pointer(x, elem) || bad_pointer(out, elem) || (residual && bad_pointer(residual, elem))) return ENTWINE_ERR_INVALID;
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.rows = rows;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldo = ldo;
  a.cols = int(cols);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return run_dropout<__nv_bfloat16>(a, s);
    case ENTWINE_FP16: return run_dropout<__half>(a, s);
    default: return run_dropout<float>(a, s);
  }
}

int entwine_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* residual,
                       int64_t ldr, double p, const int64_t* rng, int64_t row0, const void* weight, const void* bias,
                       int w_dtype, float eps, void* hidden, int64_t ldh, void* out, int64_t ldo, float* mean, float* rstd,
                       void* stream) {
  if (!floating(dtype) || (w_dtype != dtype && w_dtype != ENTWINE_FP32) || rows < 0 || rows > kMaxRows || cols < 1 ||
      cols > kMaxCols || ldx < cols || ldo < cols || (residual && ldr < cols) || (hidden && ldh < cols) || !(eps >= 0.0f))
    return ENTWINE_ERR_INVALID;
  NormParams a;
  std::memset(&a, 0, sizeof(a));
  if (!make_dropout(p, rng, row0, rows, &a.d)) return ENTWINE_ERR_INVALID;
  if (rows == 0) return ENTWINE_OK;
  const int64_t elem = bytes_of(dtype), w_elem = bytes_of(w_dtype);
  if (bad_pointer(x, elem) || bad_pointer(out, elem) || (residual && bad_pointer(residual, elem)) ||
      (hidden && bad_pointer(hidden, elem)) || bad_pointer(weight, w_elem) || (bias && bad_pointer(bias, w_elem)) ||
      (mean && bad_pointer(mean, 4)) || (rstd && bad_pointer(rstd, 4)))
    return ENTWINE_ERR_INVALID;
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.bias = bias;
  a.hidden = hidden;
  a.out = out;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = rows;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldh = ldh;
  a.ldo = ldo;
  a.cols = int(cols);
  a.wide = w_dtype == ENTWINE_FP32;
  a.eps = eps;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return run_norm<__nv_bfloat16>(a, s);
    case ENTWINE_FP16: return run_norm<__half>(a, s);
    default: return run_norm<float>(a, s);
  }
}

int entwine_layer_norm_bwd_work(int64_t rows, int64_t cols, int64_t* floats) {
  if (!floats || rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return ENTWINE_ERR_INVALID;
  *floats = int64_t(grad_plan(rows, cols).ctas) * 2 * cols;
  return ENTWINE_OK;
}

int entwine_layer_norm_bwd(const void* dout, int dtype, int64_t rows, int64_t cols, int64_t ldo, const void* hidden,
                           int64_t ldh, const void* weight, int w_dtype, const float* mean, const float* rstd,
                           const void* dhidden, int64_t lddh, double p, const int64_t* rng, int64_t row0, void* dx,
                           int64_t lddx, void* dresidual, int64_t lddr, float* dweight, float* dbias, float* work,
                           int64_t work_floats, void* stream) {
  if (!floating(dtype) || (w_dtype != dtype && w_dtype != ENTWINE_FP32) || rows < 0 || rows > kMaxRows || cols < 1 ||
      cols > kMaxCols || ldo < cols || ldh < cols || lddx < cols || (dhidden && lddh < cols) || (dresidual && lddr < cols))
    return ENTWINE_ERR_INVALID;
  GradParams a;
  std::memset(&a, 0, sizeof(a));
  if (!make_dropout(p, rng, row0, rows, &a.d)) return ENTWINE_ERR_INVALID;
  const int64_t elem = bytes_of(dtype), w_elem = bytes_of(w_dtype);
  if (bad_pointer(dweight, 4) || (dbias && bad_pointer(dbias, 4)) || bad_pointer(work, 4) ||
      work_floats < int64_t(grad_plan(rows, cols).ctas) * 2 * cols)
    return ENTWINE_ERR_INVALID;
  // (without rows the sums are still written)
  if (rows > 0 && (bad_pointer(dout, elem) || bad_pointer(hidden, elem) || bad_pointer(weight, w_elem) ||
                   bad_pointer(mean, 4) || bad_pointer(rstd, 4) || (dhidden && bad_pointer(dhidden, elem)) ||
                   bad_pointer(dx, elem) || (dresidual && bad_pointer(dresidual, elem))))
    return ENTWINE_ERR_INVALID;
  a.dout = dout;
  a.hidden = hidden;
  a.weight = weight;
  a.mean = mean;
  a.rstd = rstd;
  a.dhidden = dhidden;
  a.dx = dx;
  a.dresidual = dresidual;
  a.work = work;
  a.rows = rows;
  a.ldo = ldo;
  a.ldh = ldh;
  a.lddh = lddh;
  a.lddx = lddx;
  a.lddr = lddr;
  a.cols = int(cols);
  a.wide = w_dtype == ENTWINE_FP32;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case ENTWINE_BF16: return run_grad<__nv_bfloat16>(a, dweight, dbias, s);
    case ENTWINE_FP16: return run_grad<__half>(a, dweight, dbias, s);
    default: return run_grad<float>(a, dweight, dbias, s);
  }
}

}  // extern "C"
