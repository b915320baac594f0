// Product in 4-bit floats with a power-of-two scale per 32 elements, for one weight matrix or one per expert
// (entwine_gemm_mxf4, entwine_gemm_mxf4_grouped).
//
// As in the int8 product the tensor core computes a tile of C transposed: the 128 lanes of an accumulator are output
// channels (rows of B), its columns tokens (rows of A), the instruction as narrow as the number of tokens.  The scales
// lie in memory as rows beside the codes' rows, so that rows sorted by expert may start anywhere; the tensor core wants
// them by 128 rows and four blocks of K, rows r, r + 32, r + 64 and r + 96 side by side.  Warps with nothing else to do
// bring them four bytes at a time to those places.
#include <algorithm>
#include <cstring>

#include "ops_common.cuh"
#include "sm100.cuh"

namespace entwine {
namespace {

constexpr int kChannels = 128;       // channels of a tile
constexpr int kKBytes = 128;         // bytes of codes per row and pipeline stage (one swizzled row): 256 elements
constexpr int kScaleBytes = 8;       // their scales
constexpr int kThreads = 128;
constexpr int kMaxSplit = 8;
constexpr int kMaxGroups = 1024;
constexpr int64_t kMaxK = int64_t(1) << 24;
constexpr int64_t kMaxExtent = 2147483647;
constexpr int64_t kMaxRows = kMaxExtent - 65536;                  // row and channel numbers of the last tiles, which reach
constexpr int64_t kMaxChannels = kMaxExtent - 255;                // behind the matrix, fit 32 bits

// Bounded waits that ran out on this device; it only grows.
__device__ unsigned long long g_waits_failed;

struct Maps {
  CUtensorMap a;  // tokens [M][K/2]
  CUtensorMap b;  // channels [G][N][K/2]
};

struct Params {
  const uint8_t* scale_a;
  const uint8_t* scale_b;
  const float* bias;
  const int32_t* offsets;  // NULL: one expert that owns every row
  void* c;
  int64_t ldc, ldsa, ldsb, scale_stride;
  int c_step;              // bytes on whose multiples every row of C starts, 16 at most
  int M, N, G;
  int kbytes, kscales;     // bytes of a row's codes and scales
  int token_tiles;         // an upper bound with experts
  int split;               // CTAs that share the length K of a tile
  int withhold;            // block of K that the first tile's first CTA or pair does not load; -1: none
  unsigned long long wait_ns;  // budget of every wait
};

__device__ __noinline__ void wait_failed() { atomicAdd(&g_waits_failed, 1ull); }

// Bounded wait for a phase of a barrier.
__device__ __forceinline__ bool wait_bar(const Params& P, uint32_t bar, uint32_t parity) {
  unsigned long long t0 = 0;
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long now = globaltimer_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > P.wait_ns) break;
  }
  wait_failed();
  return false;
}

template <int TOKENS>
struct Tile {
  static constexpr int kCodes = (kChannels + TOKENS) * kKBytes;   // of a stage, then the scales of both
  static constexpr int kScales = 1024;                            // of 128 rows
  static constexpr int kStageBytes = kCodes + 2 * kScales;
  // two CTAs per SM
  static constexpr int kStages = TOKENS >= 128 ? 3 : TOKENS >= 64 ? 4 : 5;
  static constexpr int kSmem = kStages * kStageBytes + 1024;
  // accumulator, then two buffers of scales: eight columns of each operand's
  static constexpr int kScaleCol = TOKENS;
  static constexpr int kTmemCols = TOKENS <= 32 ? 64 : 2 * TOKENS;
};

// Expert and token rows of token tile `tile`, found by one warp: experts have ceil(rows / TOKENS) tiles each.
template <int TOKENS>
__device__ __forceinline__ void find_tile(const Params& P, int tile, int lane, int* group, int* m0, int* m_end) {
  *group = -1;
  int before = 0;
  for (int g0 = 0; g0 < P.G; g0 += 32) {
    const int g = g0 + lane;
    int lo = 0, hi = 0;
    if (g < P.G) {
      lo = min(max(P.offsets[g], 0), P.M);
      hi = min(max(P.offsets[g + 1], lo), P.M);
    }
    const int tiles = (hi - lo + TOKENS - 1) / TOKENS;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    const int first = before + sum - tiles;
    const unsigned here = __ballot_sync(0xffffffffu, tile >= first && tile < first + tiles);
    if (here) {
      const int src = __ffs(here) - 1;
      *group = g0 + src;
      *m0 = __shfl_sync(0xffffffffu, lo + (tile - first) * TOKENS, src);
      *m_end = __shfl_sync(0xffffffffu, hi, src);
      return;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
}

// Scales of one stage of ROWS rows, by THREADS threads: two words a row, zeros (a scale that nothing is multiplied with)
// for rows and blocks that are not there.  Word w of row r goes to place w * 512 + r % 32 * 16 + r / 32 * 4 of its 128 rows.
template <int ROWS, int THREADS>
__device__ __forceinline__ void fetch_scales(const uint8_t* scales, int64_t ld, int rows, int at, int row_bytes,
                                             uint32_t smem, int thread) {
#pragma unroll
  for (int i0 = 0; i0 < 2 * ROWS; i0 += THREADS) {
    const int i = i0 + thread, r = i / 2, w = i % 2;
    if (2 * ROWS % THREADS == 0 || i < 2 * ROWS) {
      const int left = row_bytes - at - 4 * w;
      const bool there = r < rows && left > 0;
      cp_async4(smem + r / 128 * 1024 + w * 512 + r % 32 * 16 + r % 128 / 32 * 4,
                there ? scales + r * ld + at + 4 * w : scales, there ? uint32_t(min(left, 4)) : 0u);
    }
  }
}

// One tile of 128 channels x TOKENS tokens per cluster of one to eight CTAs, which share the length K: each sums its
// blocks of K, then the partial sums meet through distributed shared memory, added in the order of the CTAs, each CTA
// finishing its share of the tokens.  So a decoding step reads the weights with all SMs.
template <int TOKENS, typename Out>
__global__ void __launch_bounds__(kThreads) gemm_mxf4_kernel(const __grid_constant__ Maps maps,
                                                             const __grid_constant__ Params P) {
  using T = Tile<TOKENS>;
  constexpr int S = T::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * S + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ int job[3];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = int(cluster_ctarank()), index = int(blockIdx.x) / P.split;
  const int n0 = index / P.token_tiles * kChannels, tile = index % P.token_tiles;
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, done = full + 16 * S;
  const int all = (P.kbytes + kKBytes - 1) / kKBytes;  // blocks of K; this CTA's:
  const int first = int(int64_t(all) * rank / P.split), blocks = int(int64_t(all) * (rank + 1) / P.split) - first;

  int issued = 0;
  bool ok = true;
  int g = 0, m0 = tile * TOKENS, m_end = P.M;
  const int withhold = blockIdx.x == 0 ? P.withhold : -1;
  auto load = [&]() {
    const int s = issued % S;
    const uint32_t at = ring + s * T::kStageBytes;
    if (issued != withhold && elect_one()) {
      mbar_arrive_expect_tx(full + 8 * s, T::kCodes);
      tma_load_3d(at, &maps.b, (first + issued) * kKBytes, n0, g, full + 8 * s);
      tma_load_2d(at + kChannels * kKBytes, &maps.a, (first + issued) * kKBytes, m0, full + 8 * s);
    }
    __syncwarp();
    ++issued;
  };
  if (warp == 0) {
    if (lane == 0) {
      tma_prefetch_map(&maps.a);
      tma_prefetch_map(&maps.b);
    }
    if (P.offsets) {
      g = -1;
      find_tile<TOKENS>(P, tile, lane, &g, &m0, &m_end);
    }
    if (lane == 0) {
      job[0] = g;
      job[1] = m0;
      job[2] = m_end;
      for (int s = 0; s < S; ++s) {
        mbar_init(full + 8 * s, 3);  // the codes, two warps' scales
        mbar_init(empty + 8 * s, 1);
      }
      mbar_init(done, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (g >= 0)  // the first loads need nothing that the rest of the CTA prepares
      while (issued < min(S, blocks)) load();
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  g = job[0];
  m0 = job[1];
  m_end = job[2];
  if (g < 0) {  // fewer tiles than the bound
    if (warp == 1) tmem_dealloc(tmem, T::kTmemCols);
    return;
  }
  // this lane's four channels in the last step
  const int n = n0 + 4 * lane;
  float add[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) add[i] = n + i < P.N && P.bias ? P.bias[int64_t(g) * P.N + n + i] : 0.0f;

  if (warp == 0) {
    while (issued < blocks) {
      if (!(ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * (issued % S), (issued / S - 1) & 1)))) break;
      load();
    }
  } else if (warp == 1) {
    for (int i = 0; i < blocks; ++i) {
      const int s = i % S;
      if (!(ok = __all_sync(0xffffffffu, wait_bar(P, full + 8 * s, (i / S) & 1)))) break;
      // the products that read this buffer of scales are done
      if (i >= 2 && !(ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * ((i - 2) % S), ((i - 2) / S) & 1)))) break;
      tc_fence_after();
      const uint32_t at = ring + s * T::kStageBytes, scales = tmem + T::kScaleCol + i % 2 * 16;
      const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
      const uint64_t ds = smem_desc_scales(at + T::kCodes);
      if (elect_one()) {
#pragma unroll
        for (int w = 0; w < 4; ++w) tmem_copy_scales(scales + 4 * w, ds + w * (512 >> 4));
#pragma unroll
        for (int k = 0; k < kKBytes / 32; ++k)
          umma_mxf4(tmem, da + 2 * k, db + 2 * k, instr_desc_mxf4(TOKENS, kChannels, k % 2), scales + k / 2 * 4,
                    scales + 8 + k / 2 * 4, i > 0 || k > 0);
        tc_commit(empty + 8 * s);
      }
      __syncwarp();
    }
    if (elect_one()) tc_commit(done);
  } else {
    // scales, two stages under way
    constexpr int kLag = 2;
    const uint8_t* const sa = P.scale_a + int64_t(m0) * P.ldsa;
    const uint8_t* const sb = P.scale_b + int64_t(g) * P.scale_stride + int64_t(n0) * P.ldsb;
    const int thread = threadIdx.x - 64;
    auto hand_over = [&](int i) {  // stage i's words have arrived
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8 * (i % S));
    };
    int i = 0;
    for (; i < blocks; ++i) {
      if (i >= S && !(ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * (i % S), (i / S - 1) & 1)))) break;
      const uint32_t at = ring + i % S * T::kStageBytes + T::kCodes;
      fetch_scales<kChannels, 64>(sb, P.ldsb, P.N - n0, (first + i) * kScaleBytes, P.kscales, at, thread);
      fetch_scales<TOKENS, 64>(sa, P.ldsa, P.M - m0, (first + i) * kScaleBytes, P.kscales, at + T::kScales, thread);
      cp_async_commit();
      cp_async_wait<kLag>();
      if (i >= kLag) hand_over(i - kLag);
    }
    cp_async_wait<0>();
    for (int j = max(0, i - kLag); j < i; ++j) hand_over(j);
  }
  __syncwarp();
  ok = wait_bar(P, done, 0) && ok;
  tc_fence_after();
  ok = !__syncthreads_or(!ok);
  if (!ok && warp == 0) {
    // copies still under way end before the CTA does; the one whose wait ran out is not the last of them
    for (int i = issued > S ? issued - S : 0; i < issued; ++i) wait_bar(P, full + 8 * (i % S), (i / S) & 1);
    __syncwarp();
  }
  // The partial sums go to shared memory, over the operands: [TOKENS][channels].
  const int used = min(TOKENS, m_end - m0);
  {
    constexpr int kCols = TOKENS < 32 ? TOKENS : 32;
    const uint32_t mine = ring + threadIdx.x * 4;
#pragma unroll 1
    for (int j0 = 0; j0 < used; j0 += kCols) {
      uint32_t v[kCols];
      if constexpr (kCols == 16) tmem_ld16(tmem + (uint32_t(warp) << 21) + j0, v);
      else tmem_ld32(tmem + (uint32_t(warp) << 21) + j0, v);
      tmem_ld_wait(v);
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(mine + (j0 + j) * kChannels * 4), "r"(v[j]) : "memory");
    }
  }
  if (P.split > 1) cluster_sync_all();
  else __syncthreads();
  // Every warp finishes tokens, four channels per lane.
  if (ok) {
    const bool vec = P.c_step >= int(4 * sizeof(Out)) && n + 4 <= P.N;
    for (int j = rank + warp * P.split; j < used; j += P.split * (kThreads / 32)) {
      const uint32_t at = ring + (j * kChannels + 4 * lane) * 4;
      float o[4] = {add[0], add[1], add[2], add[3]};
      int4 part[kMaxSplit];
#pragma unroll
      for (int r = 0; r < kMaxSplit; ++r) part[r] = r < P.split ? ld_cluster_v4(map_to_cta(at, r)) : make_int4(0, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < kMaxSplit; ++r) {
        o[0] += __int_as_float(part[r].x);
        o[1] += __int_as_float(part[r].y);
        o[2] += __int_as_float(part[r].z);
        o[3] += __int_as_float(part[r].w);
      }
      Out* const c = static_cast<Out*>(P.c) + int64_t(m0 + j) * P.ldc + n;
      if (vec) {
        *reinterpret_cast<Piece<Out, 4>*>(c) = pack<Out, 4>(o);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < P.N) c[i] = Elem<Out>::down(o[i]);
      }
    }
  }
  __syncwarp();
  if (P.split > 1) cluster_sync_all();  // no CTA leaves while its sums are read
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, T::kTmemCols);
}

template <int TOKENS, typename Out>
int run(const Maps& maps, Params P, cudaStream_t stream) {
  using T = Tile<TOKENS>;
  const int64_t token_tiles = P.offsets ? P.M / TOKENS + P.G : (P.M + TOKENS - 1) / TOKENS;
  const int64_t tiles = token_tiles * ((P.N + kChannels - 1) / kChannels);
  const int blocks = (P.kbytes + kKBytes - 1) / kKBytes;
  P.split = 1;
  while (P.split * TOKENS < 512 && P.split < kMaxSplit && tiles * P.split * 2 <= 2 * int64_t(sm_count()) &&
         blocks >= P.split * 4)
    P.split *= 2;
  if (tiles * P.split > kMaxExtent) return ENTWINE_ERR_INVALID;
  P.token_tiles = int(token_tiles);
  auto kernel = gemm_mxf4_kernel<TOKENS, Out>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
  if (e != cudaSuccess) return launched(e);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * P.split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = T::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {unsigned(P.split), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, maps, P));
}

bool make_maps(Maps* maps, const void* A, int64_t lda, const void* B, int64_t ldb, int64_t expert_stride,
               const Params& P, int tokens) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  const cuuint32_t one[3] = {1, 1, 1};
  cuuint64_t dims[3] = {cuuint64_t(P.kbytes), cuuint64_t(P.M), 1};
  cuuint64_t strides[2] = {cuuint64_t(lda), 0};
  cuuint32_t box[3] = {kKBytes, cuuint32_t(tokens), 1};
  if (fn(&maps->a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(A), dims, strides, box, one,
         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return false;
  dims[1] = cuuint64_t(P.N);
  dims[2] = cuuint64_t(P.G);
  strides[0] = cuuint64_t(ldb);
  strides[1] = cuuint64_t(expert_stride);
  box[1] = kChannels;
  return fn(&maps->b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(B), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Out>
int run_as(const void* A, int64_t lda, const void* B, int64_t ldb, int64_t expert_stride, const Params& P,
           cudaStream_t stream) {
  const int rows = (P.M + P.G - 1) / P.G;  // of an average expert
  Maps maps;
  // the narrowest tile that holds them
  const int tokens = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  if (!make_maps(&maps, A, lda, B, ldb, expert_stride, P, tokens)) return ENTWINE_ERR_CUDA;
  switch (tokens) {
    case 16: return run<16, Out>(maps, P, stream);
    case 32: return run<32, Out>(maps, P, stream);
    case 64: return run<64, Out>(maps, P, stream);
    default: return run<128, Out>(maps, P, stream);
  }
}

int gemm(const void* A, int64_t lda, const void* scale_a, int64_t ldsa, const void* B, int64_t ldb, int64_t expert_stride,
         const void* scale_b, int64_t ldsb, int64_t scale_stride, const float* bias, const int32_t* offsets, void* C,
         int c_dtype, int64_t ldc, int64_t M, int64_t N, int64_t K, int64_t G, void* stream) {
  if (c_dtype != ENTWINE_BF16 && c_dtype != ENTWINE_FP16 && c_dtype != ENTWINE_FP32) return ENTWINE_ERR_INVALID;
  if (M < 0 || M > kMaxRows || N < 1 || N > kMaxChannels || K < 1 || K > kMaxK || G < 1 || G > kMaxGroups || G * N > kMaxExtent)
    return ENTWINE_ERR_INVALID;
  const int64_t kbytes = (K + 1) / 2, kscales = (K + 31) / 32;
  if (ldc < N || lda < kbytes || ldb < kbytes || ldsa < kscales || ldsb < kscales) return ENTWINE_ERR_INVALID;
  // a matrix of one row has no row distance, a single expert no distance to the next
  const int64_t row = (kbytes + 15) / 16 * 16, scale_row = (kscales + 3) / 4 * 4;
  if (M == 1) lda = row, ldsa = scale_row;
  if (N == 1) ldb = row, ldsb = scale_row;
  if (G == 1) expert_stride = ldb, scale_stride = ldsb;
  if (lda % 16 || ldb % 16 || expert_stride % 16 || expert_stride < kbytes || ldsa % 4 || ldsb % 4 || scale_stride % 4 ||
      scale_stride < kscales)
    return ENTWINE_ERR_INVALID;
  if (G > 1 && (expert_stride < (N - 1) * ldb + kbytes || scale_stride < (N - 1) * ldsb + kscales)) return ENTWINE_ERR_INVALID;
  if (M == 0) return ENTWINE_OK;
  if (bad_pointer(A, 16) || bad_pointer(B, 16) || bad_pointer(scale_a, 4) || bad_pointer(scale_b, 4) ||
      (bias && bad_pointer(bias, 4)) || bad_pointer(C, c_dtype == ENTWINE_FP32 ? 4 : 2))
    return ENTWINE_ERR_INVALID;
  Params P;
  std::memset(&P, 0, sizeof(P));
  P.scale_a = static_cast<const uint8_t*>(scale_a);
  P.scale_b = static_cast<const uint8_t*>(scale_b);
  P.bias = bias;
  P.offsets = offsets;
  P.c = C;
  P.ldc = ldc;
  P.ldsa = ldsa;
  P.ldsb = ldsb;
  P.scale_stride = scale_stride;
  const uint64_t starts = reinterpret_cast<uintptr_t>(C) | uint64_t(ldc) * (c_dtype == ENTWINE_FP32 ? 4 : 2);
  P.c_step = int(std::min<uint64_t>(starts & (~starts + 1), 16));
  P.M = int(M);
  P.N = int(N);
  P.G = int(G);
  P.kbytes = int(kbytes);
  P.kscales = int(kscales);
  const WaitSettings w = wait_settings();
  P.withhold = w.withhold;
  P.wait_ns = w.budget_ns;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (c_dtype) {
    case ENTWINE_BF16: return run_as<__nv_bfloat16>(A, lda, B, ldb, expert_stride, P, s);
    case ENTWINE_FP16: return run_as<__half>(A, lda, B, ldb, expert_stride, P, s);
    default: return run_as<float>(A, lda, B, ldb, expert_stride, P, s);
  }
}

}  // namespace

cudaError_t mxf4_failed_waits(unsigned long long* n, cudaStream_t stream) {
  return cudaMemcpyFromSymbolAsync(n, g_waits_failed, sizeof(*n), 0, cudaMemcpyDeviceToHost, stream);
}

}  // namespace entwine

using namespace entwine;

extern "C" {

int entwine_gemm_mxf4(const void* A, int64_t lda, const void* scale_a, int64_t ldsa, const void* B, int64_t ldb,
                      const void* scale_b, int64_t ldsb, const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M,
                      int64_t N, int64_t K, void* stream) {
  return gemm(A, lda, scale_a, ldsa, B, ldb, 0, scale_b, ldsb, 0, bias, nullptr, C, c_dtype, ldc, M, N, K, 1, stream);
}

int entwine_gemm_mxf4_grouped(const void* A, int64_t lda, const void* scale_a, int64_t ldsa, const void* B, int64_t ldb,
                              int64_t expert_stride, const void* scale_b, int64_t ldsb, int64_t scale_stride,
                              const float* bias, const int32_t* offsets, void* C, int c_dtype, int64_t ldc, int64_t M,
                              int64_t N, int64_t K, int64_t G, void* stream) {
  if (M > 0 && bad_pointer(offsets, 4)) return ENTWINE_ERR_INVALID;
  return gemm(A, lda, scale_a, ldsa, B, ldb, expert_stride, scale_b, ldsb, scale_stride, bias, offsets, C, c_dtype, ldc, M, N,
              K, G, stream);
}

}  // extern "C"
