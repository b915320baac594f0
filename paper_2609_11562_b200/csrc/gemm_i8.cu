// Product in 8-bit integers with token and channel scales, for one weight matrix or one per expert
// (entwine_gemm_i8, entwine_gemm_i8_grouped).
//
// The tensor core computes a tile of C transposed: the 128 lanes of an accumulator are output channels (rows of B),
// its columns tokens (rows of A).  With few tokens the instruction is as narrow as their number (16 at least), so
// that a decoding step pays for reading B and nothing else; and a warp's lanes, consecutive channels, store
// consecutive elements of a row of C.
#include <algorithm>
#include <cstring>

#ifndef PAIRMIN
#define PAIRMIN 256
#endif

#include "ops_common.cuh"
#include "sm100.cuh"

namespace entwine {
namespace {

constexpr int kChannels = 128;       // channels of a tile
constexpr int kKBytes = 128;         // elements of K per pipeline stage (one swizzled row)
constexpr int kThreads = 128;
constexpr int kMaxGroups = 1024;
constexpr int64_t kMaxK = 131071;    // 128 * 128 * K < 2^31
constexpr int64_t kMaxExtent = 2147483647;
constexpr unsigned long long kWaitBudgetNs = 2000000000ull;

__device__ int g_wait_failed;        // set when a bounded wait ran out, read by entwine_ops_status

struct Maps {
  CUtensorMap a;  // tokens [M][K]
  CUtensorMap b;  // channels [G][N][K]
};

// (a pair tile: 256 channels, up to 256 tokens)
constexpr int kPairThreads = 320;    // TMA warp, MMA warp, eight epilogue warps
constexpr int kPairChannels = 256;
constexpr int kPairTokens = 256;
constexpr int kPairStageBytes = 32768;
constexpr int kBand = 16;            // token tiles that share a walk over the channels: their rows stay in L2

struct Params {
  const float* scale_a;
  const float* scale_b;
  const float* bias;
  const int32_t* offsets;  // null: one matrix for all rows
  void* c;
  int64_t ldc;
  int M, N, K, G;
  int token_tiles;         // an upper bound with experts
  int tile_rows;           // most tokens of a pair tile, a multiple of 32
};

// Bounded wait for a phase of a barrier.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = globaltimer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (globaltimer_ns() - t0 > kWaitBudgetNs) {
      g_wait_failed = 1;
      return false;
    }
  }
}

template <int TOKENS>
struct Tile {
  static constexpr int kStageBytes = (kChannels + TOKENS) * kKBytes;
  // all of the shared memory for one CTA per SM with wide tiles, two CTAs per SM with narrow ones
  static constexpr int kStages = TOKENS >= 256 ? 4 : TOKENS >= 128 ? 6 : TOKENS >= 64 ? 4 : TOKENS >= 32 ? 5 : 6;
  static constexpr int kSmem = kStages * kStageBytes + 1024;
  static constexpr int kTmemCols = TOKENS < 32 ? 32 : TOKENS;
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

template <int TOKENS, typename Out>
__global__ void __launch_bounds__(kThreads) gemm_i8_kernel(const __grid_constant__ Maps maps,
                                                           const __grid_constant__ Params P) {
  using T = Tile<TOKENS>;
  constexpr int S = T::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * S + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ int job[3];
  __shared__ float token_scale[TOKENS];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int n0 = int(blockIdx.x / P.token_tiles) * kChannels, tile = int(blockIdx.x % P.token_tiles);
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, done = full + 16 * S;

  if (warp == 0) {
    int g = 0, m0 = tile * TOKENS, m_end = P.M;
    if (P.offsets) find_tile<TOKENS>(P, tile, lane, &g, &m0, &m_end);
    if (lane == 0) {
      job[0] = g;
      job[1] = m0;
      job[2] = m_end;
      for (int s = 0; s < S; ++s) {
        mbar_init(full + 8 * s, 1);
        mbar_init(empty + 8 * s, 1);
      }
      mbar_init(done, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  __syncthreads();
  const int g = job[0], m0 = job[1], m_end = job[2];
  if (g < 0) return;  // fewer tiles than the bound
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), T::kTmemCols);
  for (int i = threadIdx.x; i < TOKENS; i += kThreads) token_scale[i] = m0 + i < m_end ? P.scale_a[m0 + i] : 0.0f;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int blocks = (P.K + kKBytes - 1) / kKBytes;

  int issued = 0;
  bool ok = true;
  if (threadIdx.x == 0) {
    for (; issued < blocks; ++issued) {
      const int s = issued % S;
      if (issued >= S && !(ok = wait_bar(empty + 8 * s, (issued / S - 1) & 1))) break;
      const uint32_t at = ring + s * T::kStageBytes;
      mbar_arrive_expect_tx(full + 8 * s, T::kStageBytes);
      tma_load_3d(at, &maps.b, issued * kKBytes, n0, g, full + 8 * s);
      tma_load_2d(at + kChannels * kKBytes, &maps.a, issued * kKBytes, m0, full + 8 * s);
    }
  } else if (threadIdx.x == 32) {
    // int32 accumulator, signed 8-bit operands, both K-major
    constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (uint32_t(TOKENS >> 3) << 17) |
                               (uint32_t(kChannels >> 4) << 24);
    for (int i = 0; i < blocks; ++i) {
      const int s = i % S;
      if (!(ok = wait_bar(full + 8 * s, (i / S) & 1))) break;
      tc_fence_after();
      const uint32_t at = ring + s * T::kStageBytes;
      const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
#pragma unroll
      for (int k = 0; k < kKBytes / 32; ++k) umma_i8(tmem, da + 2 * k, db + 2 * k, idesc, i > 0 || k > 0);
      tc_commit(empty + 8 * s);
    }
    tc_commit(done);
  }
  __syncwarp();
  ok = wait_bar(done, 0) && ok;
  tc_fence_after();
  ok = !__syncthreads_or(!ok);
  if (ok) {
    const int n = n0 + threadIdx.x;
    const float sb = n < P.N ? P.scale_b[int64_t(g) * P.N + n] : 0.0f;
    const float add = n < P.N && P.bias ? P.bias[int64_t(g) * P.N + n] : 0.0f;
    Out* c = static_cast<Out*>(P.c) + int64_t(m0) * P.ldc + n;
    constexpr int kCols = 16;
#pragma unroll 1
    for (int j0 = 0; j0 < TOKENS && m0 + j0 < m_end; j0 += kCols) {
      uint32_t v[kCols];
      tmem_ld16(tmem + (uint32_t(warp) << 21) + j0, v);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < kCols; ++j) {
        // the sum is exact; its conversion, the two products and the last rounding are the only inexact steps
        const float f = fmaf(__int2float_rn(int(v[j])) * token_scale[j0 + j], sb, add);
        if (n < P.N && m0 + j0 + j < m_end) c[int64_t(j0 + j) * P.ldc] = Elem<Out>::down(f);
      }
    }
  } else if (threadIdx.x == 0) {
    // copies still under way end before the CTA does
    for (int i = issued > S ? issued - S : 0; i < issued; ++i) wait_bar(full + 8 * (i % S), (i / S) & 1);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, T::kTmemCols);
}

// ------------------------------------------------------------------------------------------
// many tokens: CTA pairs, persistent
// ------------------------------------------------------------------------------------------
// Two CTAs of a cluster compute 256 channels x up to 256 tokens (tcgen05 cta_group::2: 128 channels each, each loading
// half of the tokens), so that an SM takes in 64 bytes per cycle at the full MMA rate instead of 96.  A tile is as
// wide as its tokens, in steps of 32: an expert's last rows cost what they are.  Two accumulators in TMEM: the
// epilogue of a tile runs beside the products of the next.
struct PairTile {
  int g, m0, rows, n0;
};

template <typename Out>
struct PairCfg {
  static constexpr int kStages = sizeof(Out) == 4 ? 5 : 6;
  static constexpr int kStagingBytes = 32 * 32 * sizeof(Out);  // of a warp: 32 tokens x 32 channels
  static constexpr int kSmem = kStages * kPairStageBytes + 8 * kStagingBytes + 1024;
};

// Tile t of the walk.  first[g]: token tiles of the experts before g.  An expert's tiles are as equal as steps of 32
// rows allow; bands of kBand of them walk over the channels together.
__device__ __forceinline__ PairTile pair_tile(const Params& P, const int* first, const int* start, int channel_tiles,
                                              int t) {
  const int u = t / channel_tiles;
  int g = 0;
  for (int step = 512; step > 0; step >>= 1)  // the last expert whose tiles start at or before u
    if (g + step < P.G && first[g + step] <= u) g += step;
  const int tiles = first[g + 1] - first[g];
  int local = t - first[g] * channel_tiles;
  const int band = local / (kBand * channel_tiles);
  local -= band * kBand * channel_tiles;
  const int in_band = min(kBand, tiles - band * kBand);
  const int m = band * kBand + local % in_band;
  const int total = start[2 * g + 1] - start[2 * g];
  const int height = ((total + tiles - 1) / tiles + 31) / 32 * 32;
  PairTile r;
  r.g = g;
  r.m0 = start[2 * g] + m * height;
  r.rows = min(height, start[2 * g + 1] - r.m0);
  r.n0 = local / in_band * kPairChannels;
  return r;
}

template <typename Out>
__global__ void __launch_bounds__(kPairThreads, 1) gemm_i8_pair_kernel(const __grid_constant__ Maps maps,
                                                                       const __grid_constant__ Params P) {
  using C = PairCfg<Out>;
  constexpr int S = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * S + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ int first[kMaxGroups + 1], start[2 * kMaxGroups];
  __shared__ __align__(16) float token_scale[8][32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = int(cluster_ctarank());
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, tfull = full + 16 * S, tempty = tfull + 16,
                 drain = tempty + 16;

  // token tiles of each expert, then their running sum
  for (int g = threadIdx.x; g < P.G; g += kPairThreads) {
    int lo = 0, hi = P.M;
    if (P.offsets) {
      lo = min(max(P.offsets[g], 0), P.M);
      hi = min(max(P.offsets[g + 1], lo), P.M);
    }
    start[2 * g] = lo;
    start[2 * g + 1] = hi;
    first[g + 1] = (hi - lo + P.tile_rows - 1) / P.tile_rows;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull + 8 * a, 1);
      mbar_init(tempty + 8 * a, 16);
    }
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    first[0] = 0;
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    int before = 0;
    for (int g0 = 0; g0 < P.G; g0 += 32) {
      int sum = g0 + lane < P.G ? first[g0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      sum += before;
      if (g0 + lane < P.G) first[g0 + lane + 1] = sum;
      before = __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  __syncthreads();
  cluster_sync_all();  // both CTAs' barriers exist before either signals
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int channel_tiles = (P.N + kPairChannels - 1) / kPairChannels;
  const int total = first[P.G] * channel_tiles, pair = int(blockIdx.x) / 2, pairs = int(gridDim.x) / 2;
  const int blocks = (P.K + kKBytes - 1) / kKBytes;

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t bytes = kChannels * kKBytes + P.tile_rows / 2 * kKBytes;  // that each CTA brings
      int stage = 0;
      uint32_t phase = 0;
      long long issued = 0;
      bool ok = true;
      for (int t = pair; ok && t < total; t += pairs) {
        const PairTile w = pair_tile(P, first, start, channel_tiles, t);
        const int half = (w.rows + 31) / 32 * 16;
        for (int b = 0; b < blocks; ++b) {
          if (!(ok = wait_bar(empty + 8 * stage, phase ^ 1))) break;
          const uint32_t at = ring + stage * kPairStageBytes, bar = map_to_cta(full + 8 * stage, 0);
          if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, 2 * bytes);
          tma_load_3d_pair(at, &maps.b, b * kKBytes, w.n0 + rank * kChannels, w.g, bar);
          tma_load_2d_pair(at + kChannels * kKBytes, &maps.a, b * kKBytes, w.m0 + rank * half, bar);
          ++issued;
          if (++stage == S) stage = 0, phase ^= 1;
        }
      }
      // after a wait that ran out: copies still under way end before the CTA does
      for (int i = 0; !ok && rank == 0 && i < S && i < issued; ++i) {
        if (--stage < 0) stage = S - 1, phase ^= 1;
        if (!wait_bar(full + 8 * stage, phase)) break;
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int t = pair; ok && t < total; t += pairs) {
        const PairTile w = pair_tile(P, first, start, channel_tiles, t);
        const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (uint32_t((w.rows + 31) / 32 * 4) << 17) |
                               (uint32_t(kPairChannels >> 4) << 24);
        if (!(ok = wait_bar(tempty + 8 * acc, acc_phase ^ 1))) break;
        tc_fence_after();
        const uint32_t d = tmem + acc * kPairTokens;
        for (int b = 0; b < blocks; ++b) {
          if (!(ok = wait_bar(full + 8 * stage, phase))) break;
          tc_fence_after();
          const uint32_t at = ring + stage * kPairStageBytes;
          const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
#pragma unroll
          for (int k = 0; k < kKBytes / 32; ++k) umma_i8_pair(d, da + 2 * k, db + 2 * k, idesc, b > 0 || k > 0);
          tc_commit_pair(empty + 8 * stage);
          if (++stage == S) stage = 0, phase ^= 1;
        }
        if (ok) tc_commit_pair(tfull + 8 * acc);
        if ((acc ^= 1) == 0) acc_phase ^= 1;
      }
      if (!ok) {  // products under way end before the TMEM is given back
        tc_commit_pair(drain);
        wait_bar(drain, 0);
      }
    }
  } else {
    // Epilogue: a warp owns 32 channels (its lane quarter of the accumulator), a lane one of them; groups of four
    // warps take turns at the 32-token chunks of a tile.  Values go through the warp's own staging, so that 16-byte
    // stores carry 32 channels of eight (fp32: four) tokens at a time.
    const int q = warp & 3, group = (warp - 2) / 4;
    Out* const staging = reinterpret_cast<Out*>(smem_raw + (ring - smem_u32(smem_raw)) + S * kPairStageBytes +
                                                (warp - 2) * C::kStagingBytes);
    float* const sa = token_scale[warp - 2];
    constexpr int kVec = 16 / sizeof(Out), kLanesPerRow = 32 / kVec, kRowsPerStore = 32 / kLanesPerRow;
    const bool vec = reinterpret_cast<uintptr_t>(P.c) % 16 == 0 && P.ldc * sizeof(Out) % 16 == 0;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int t = pair; t < total; t += pairs) {
      const PairTile w = pair_tile(P, first, start, channel_tiles, t);
      const int n0 = w.n0 + rank * kChannels + q * 32, n = n0 + lane;
      const float sb = n < P.N ? P.scale_b[int64_t(w.g) * P.N + n] : 0.0f;
      const float add = n < P.N && P.bias ? P.bias[int64_t(w.g) * P.N + n] : 0.0f;
      const bool ok = __all_sync(0xffffffffu, wait_bar(tfull + 8 * acc, acc_phase));
      if (!ok) break;
      tc_fence_after();
      const int chunks = (w.rows + 31) / 32;
      for (int c = group; c < chunks; c += 2) {
        uint32_t v[32];
        tmem_ld32(tmem + (uint32_t(q) << 21) + acc * kPairTokens + c * 32, v);
        sa[lane] = c * 32 + lane < w.rows ? P.scale_a[w.m0 + c * 32 + lane] : 0.0f;
        tmem_ld_wait();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 s4 = *reinterpret_cast<const float4*>(sa + j);
          staging[(j + 0) * 32 + lane] = Elem<Out>::down(fmaf(__int2float_rn(int(v[j + 0])) * s4.x, sb, add));
          staging[(j + 1) * 32 + lane] = Elem<Out>::down(fmaf(__int2float_rn(int(v[j + 1])) * s4.y, sb, add));
          staging[(j + 2) * 32 + lane] = Elem<Out>::down(fmaf(__int2float_rn(int(v[j + 2])) * s4.z, sb, add));
          staging[(j + 3) * 32 + lane] = Elem<Out>::down(fmaf(__int2float_rn(int(v[j + 3])) * s4.w, sb, add));
        }
        __syncwarp();
        const int rows = min(32, w.rows - c * 32);
        Out* const out = static_cast<Out*>(P.c) + int64_t(w.m0 + c * 32) * P.ldc + n0;
        if (vec && n0 + 32 <= P.N) {
          const int r0 = lane / kLanesPerRow, x = lane % kLanesPerRow * kVec;
#pragma unroll
          for (int i = 0; i < 32 / kRowsPerStore; ++i) {
            const int r = i * kRowsPerStore + r0;
            if (r < rows) *reinterpret_cast<uint4*>(out + r * P.ldc + x) = *reinterpret_cast<const uint4*>(staging + r * 32 + x);
          }
        } else if (n < P.N) {
          for (int r = 0; r < rows; ++r) out[r * P.ldc + lane] = staging[r * 32 + lane];
        }
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty + 8 * acc, 0));
      if ((acc ^= 1) == 0) acc_phase ^= 1;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA signals the other's barriers any more
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

template <typename Out>
int run_pairs(const Maps& maps, Params P, cudaStream_t stream) {
  using C = PairCfg<Out>;
  const int64_t token_tiles = P.offsets ? P.M / P.tile_rows + P.G : (P.M + P.tile_rows - 1) / P.tile_rows;
  const int64_t tiles = token_tiles * ((P.N + kPairChannels - 1) / kPairChannels);
  if (tiles > kMaxExtent) return ENTWINE_ERR_INVALID;
  auto kernel = gemm_i8_pair_kernel<Out>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (e != cudaSuccess) return launched(e);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(std::min<int64_t>(2 * tiles, sm_count() / 2 * 2)));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {2, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return launched(cudaLaunchKernelEx(&cfg, kernel, maps, P));
}

// The height of the pair tiles: as many waves of the pairs as there are, each as long as its tiles are high (and a
// part that does not depend on it).
int pair_rows(const Params& P) {
  if (P.G > 1) return kPairTokens;
  const int64_t channel_tiles = (P.N + kPairChannels - 1) / kPairChannels, pairs = sm_count() / 2;
  int best = kPairTokens;
  int64_t least = 0;
  for (int rows = kPairTokens; rows >= 96; rows -= 32) {
    const int64_t token_tiles = (P.M + rows - 1) / rows, waves = (token_tiles * channel_tiles + pairs - 1) / pairs;
    const int64_t cost = waves * (rows + 32);
    if (least == 0 || cost < least) least = cost, best = rows;
  }
  return best;
}

template <int TOKENS, typename Out>
int run(const Maps& maps, Params P, cudaStream_t stream) {
  using T = Tile<TOKENS>;
  const int64_t token_tiles = P.offsets ? P.M / TOKENS + P.G : (P.M + TOKENS - 1) / TOKENS;
  const int64_t grid = token_tiles * ((P.N + kChannels - 1) / kChannels);
  if (grid > kMaxExtent) return ENTWINE_ERR_INVALID;
  P.token_tiles = int(token_tiles);
  auto kernel = gemm_i8_kernel<TOKENS, Out>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
  if (e == cudaSuccess) kernel<<<unsigned(grid), kThreads, T::kSmem, stream>>>(maps, P);
  return launched(e);
}

bool make_maps(Maps* maps, const void* A, int64_t lda, const void* B, int64_t ldb, int64_t expert_stride,
               const Params& P, int tokens) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  const cuuint32_t one[3] = {1, 1, 1};
  cuuint64_t dims[3] = {cuuint64_t(P.K), cuuint64_t(P.M), 1};
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
  if (rows > PAIRMIN) {
    Params Q = P;
    Q.tile_rows = pair_rows(P);
    Maps maps;
    if (!make_maps(&maps, A, lda, B, ldb, expert_stride, Q, Q.tile_rows / 2)) return ENTWINE_ERR_CUDA;
    return run_pairs<Out>(maps, Q, stream);
  }
  // the narrowest tile that holds them
  const int tokens = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
  Maps maps;
  if (!make_maps(&maps, A, lda, B, ldb, expert_stride, P, tokens)) return ENTWINE_ERR_CUDA;
  switch (tokens) {
    case 16: return run<16, Out>(maps, P, stream);
    case 32: return run<32, Out>(maps, P, stream);
    case 64: return run<64, Out>(maps, P, stream);
    case 128: return run<128, Out>(maps, P, stream);
    default: return run<256, Out>(maps, P, stream);
  }
}

int gemm(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb, int64_t expert_stride,
         const float* scale_b, const float* bias, const int32_t* offsets, void* C, int c_dtype, int64_t ldc, int64_t M,
         int64_t N, int64_t K, int64_t G, void* stream) {
  if (c_dtype != ENTWINE_BF16 && c_dtype != ENTWINE_FP16 && c_dtype != ENTWINE_FP32) return ENTWINE_ERR_INVALID;
  if (M < 0 || M > kMaxExtent - 65536 || N < 1 || N > kMaxExtent || K < 1 || K > kMaxK || G < 1 || G > kMaxGroups ||
      G * N > kMaxExtent || ldc < N || lda < K || ldb < K)
    return ENTWINE_ERR_INVALID;
  // a matrix of one row has no row distance, a single expert no distance to the next
  if (M == 1) lda = (K + 15) / 16 * 16;
  if (N == 1) ldb = (K + 15) / 16 * 16;
  if (G == 1) expert_stride = ldb;
  if (lda % 16 || ldb % 16 || expert_stride % 16 || expert_stride < K) return ENTWINE_ERR_INVALID;
  if (G > 1 && expert_stride < (N - 1) * ldb + K) return ENTWINE_ERR_INVALID;
  if (M == 0) return ENTWINE_OK;
  if (bad_pointer(A, 16) || bad_pointer(B, 16) || bad_pointer(scale_a, 4) || bad_pointer(scale_b, 4) ||
      (bias && bad_pointer(bias, 4)) || bad_pointer(C, c_dtype == ENTWINE_FP32 ? 4 : 2))
    return ENTWINE_ERR_INVALID;
  Params P;
  std::memset(&P, 0, sizeof(P));
  P.scale_a = scale_a;
  P.scale_b = scale_b;
  P.bias = bias;
  P.offsets = offsets;
  P.c = C;
  P.ldc = ldc;
  P.M = int(M);
  P.N = int(N);
  P.K = int(K);
  P.G = int(G);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (c_dtype) {
    case ENTWINE_BF16: return run_as<__nv_bfloat16>(A, lda, B, ldb, expert_stride, P, s);
    case ENTWINE_FP16: return run_as<__half>(A, lda, B, ldb, expert_stride, P, s);
    default: return run_as<float>(A, lda, B, ldb, expert_stride, P, s);
  }
}

}  // namespace
}  // namespace entwine

using namespace entwine;

extern "C" {

int entwine_gemm_i8(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb, const float* scale_b,
                    const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M, int64_t N, int64_t K,
                    void* stream) {
  return gemm(A, lda, scale_a, B, ldb, 0, scale_b, bias, nullptr, C, c_dtype, ldc, M, N, K, 1, stream);
}

int entwine_gemm_i8_grouped(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb,
                            int64_t expert_stride, const float* scale_b, const float* bias, const int32_t* offsets,
                            void* C, int c_dtype, int64_t ldc, int64_t M, int64_t N, int64_t K, int64_t G,
                            void* stream) {
  if (M > 0 && bad_pointer(offsets, 4)) return ENTWINE_ERR_INVALID;
  return gemm(A, lda, scale_a, B, ldb, expert_stride, scale_b, bias, offsets, C, c_dtype, ldc, M, N, K, G, stream);
}

int entwine_ops_status(void* stream) {
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &capture) != cudaSuccess) return launched(cudaErrorUnknown);
  if (capture != cudaStreamCaptureStatusNone) return ENTWINE_ERR_INVALID;
  int failed = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&failed, g_wait_failed, sizeof(failed), 0, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && failed) {
    const int none = 0;
    e = cudaMemcpyToSymbolAsync(g_wait_failed, &none, sizeof(none), 0, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  }
  if (e != cudaSuccess) return launched(e);
  return failed ? ENTWINE_ERR_TIMEOUT : ENTWINE_OK;
}

}  // extern "C"
