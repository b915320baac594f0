// Product in 8-bit integers with token and channel scales, for one weight matrix or one per expert
// (entwine_gemm_i8, entwine_gemm_i8_grouped).
//
// The tensor core computes a tile of C transposed: the 128 lanes of an accumulator are output channels (rows of B),
// its columns tokens (rows of A).  With few tokens the instruction is as narrow as their number (16 at least), so
// that a decoding step pays for reading B and nothing else; and a warp's lanes, consecutive channels, store
// consecutive elements of a row of C.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "gemm_tiles.cuh"
#include "ops_common.cuh"
#include "sm100.cuh"

namespace entwine {
namespace {

constexpr int kChannels = 128;       // channels of a tile
constexpr int kKBytes = 128;         // elements of K per pipeline stage (one swizzled row)
constexpr int kThreads = 128;
constexpr int kMaxSplit = 8;
constexpr int64_t kMaxK = 131071;    // 128 * 128 * K < 2^31
constexpr int64_t kMaxExtent = 2147483647;
constexpr int64_t kMaxRows = kMaxExtent - 65536;                  // row and channel numbers of the last tiles, which reach
constexpr int64_t kMaxChannels = kMaxExtent - 255;                // behind the matrix, fit 32 bits

// Bounded waits that ran out on this device.  It only grows: nobody's reading of it takes a failure from anybody else.
__device__ unsigned long long g_waits_failed;

// entwine_ops_set_option
std::atomic<int64_t> g_wait_budget_ns{2000000000}, g_withhold{-1};

struct Maps {
  CUtensorMap a;  // tokens [M][K]
  CUtensorMap b;  // channels [G][N][K]
};

// (a pair tile: 256 channels, up to 256 tokens)
constexpr int kPairThreads = 320;    // TMA warp, MMA warp, eight epilogue warps
constexpr int kPairTokens = 256;
constexpr int kPairStageBytes = 32768;

struct Params {
  const float* scale_a;
  const float* scale_b;
  const float* bias;
  const int32_t* offsets;  // null: one matrix for all rows
  void* c;
  int64_t ldc;
  int c_step;              // bytes, up to 16, on whose multiples all rows of C start
  int M, N, K, G;
  int token_tiles;         // an upper bound with experts
  int split;               // CTAs that share the length K of a tile
  int tile_rows;           // most tokens of a pair tile, a multiple of 32
  int withhold;            // block of K that the first tile's first CTA or pair does not load; -1: none
  unsigned long long wait_ns;  // budget of every wait
};

// Out of line: inlined at every wait, its code cost the loops around them 4 % (8192 x 8192 x 3584: 187 us, 179 without).
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
  static constexpr int kStageBytes = (kChannels + TOKENS) * kKBytes;
  // two CTAs per SM
  static constexpr int kStages = TOKENS >= 128 ? 3 : TOKENS >= 64 ? 4 : TOKENS >= 32 ? 5 : 6;
  static constexpr int kSmem = kStages * kStageBytes + 1024;
  static constexpr int kTmemCols = TOKENS < 32 ? 32 : TOKENS;
};

// One tile of 128 channels x TOKENS tokens per cluster of one to eight CTAs, which share the length K: each sums its
// blocks of K, then the int32 partial sums (exact in any order) meet through distributed shared memory, each CTA
// finishing its share of the tokens.  So a decoding step reads the weights with all SMs.
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
  const int rank = int(cluster_ctarank()), index = int(blockIdx.x) / P.split;
  const int n0 = index / P.token_tiles * kChannels, tile = index % P.token_tiles;
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, done = full + 16 * S;
  const int all = (P.K + kKBytes - 1) / kKBytes;  // blocks of K; this CTA's:
  const int first = int(int64_t(all) * rank / P.split), blocks = int(int64_t(all) * (rank + 1) / P.split) - first;

  int issued = 0;
  bool ok = true;
  int g = 0, m0 = tile * TOKENS, m_end = P.M;
  const int withhold = blockIdx.x == 0 ? P.withhold : -1;
  auto load = [&]() {
    const int s = issued % S;
    const uint32_t at = ring + s * T::kStageBytes;
    if (issued != withhold && elect_one()) {
      mbar_arrive_expect_tx(full + 8 * s, T::kStageBytes);
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
        mbar_init(full + 8 * s, 1);
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
  for (int i = threadIdx.x; i < TOKENS; i += kThreads) token_scale[i] = m0 + i < m_end ? P.scale_a[m0 + i] : 0.0f;
  // this lane's four channels in the last step
  const int n = n0 + 4 * lane;
  float sb[4], add[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sb[i] = n + i < P.N ? P.scale_b[int64_t(g) * P.N + n + i] : 0.0f;
    add[i] = n + i < P.N && P.bias ? P.bias[int64_t(g) * P.N + n + i] : 0.0f;
  }

  if (warp == 0) {
    while (issued < blocks) {
      if (!(ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * (issued % S), (issued / S - 1) & 1)))) break;
      load();
    }
  } else if (warp == 1) {
    // int32 accumulator, signed 8-bit operands, both K-major
    constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (uint32_t(TOKENS >> 3) << 17) |
                               (uint32_t(kChannels >> 4) << 24);
    for (int i = 0; i < blocks; ++i) {
      const int s = i % S;
      if (!(ok = __all_sync(0xffffffffu, wait_bar(P, full + 8 * s, (i / S) & 1)))) break;
      tc_fence_after();
      const uint32_t at = ring + s * T::kStageBytes;
      const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kKBytes / 32; ++k) umma_i8(tmem, da + 2 * k, db + 2 * k, idesc, i > 0 || k > 0);
        tc_commit(empty + 8 * s);
      }
      __syncwarp();
    }
    if (elect_one()) tc_commit(done);
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
  // Every warp finishes tokens, four channels per lane: the sum is exact; its conversion, the two products and the
  // last rounding are the only inexact steps.
  if (ok) {
    const bool vec = P.c_step >= int(4 * sizeof(Out)) && n + 4 <= P.N;
    for (int j = rank + warp * P.split; j < used; j += P.split * (kThreads / 32)) {
      const uint32_t at = ring + (j * kChannels + 4 * lane) * 4;
      int4 part[kMaxSplit];
#pragma unroll
      for (int r = 0; r < kMaxSplit; ++r) part[r] = r < P.split ? ld_cluster_v4(map_to_cta(at, r)) : make_int4(0, 0, 0, 0);
      int4 sum = part[0];
#pragma unroll
      for (int r = 1; r < kMaxSplit; ++r) {
        sum.x += part[r].x;
        sum.y += part[r].y;
        sum.z += part[r].z;
        sum.w += part[r].w;
      }
      const float f = token_scale[j];
      const float o[4] = {fmaf(__int2float_rn(sum.x) * f, sb[0], add[0]), fmaf(__int2float_rn(sum.y) * f, sb[1], add[1]),
                          fmaf(__int2float_rn(sum.z) * f, sb[2], add[2]), fmaf(__int2float_rn(sum.w) * f, sb[3], add[3])};
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

// ------------------------------------------------------------------------------------------
// many tokens: CTA pairs, persistent
// ------------------------------------------------------------------------------------------
// Two CTAs of a cluster compute 256 channels x up to 256 tokens (tcgen05 cta_group::2: 128 channels each, each loading
// half of the tokens), so that an SM takes in 64 bytes per cycle at the full MMA rate instead of 96.  A tile's products
// are as wide as its tokens, in steps of 32 (what is loaded is not: a whole tile's tokens, however few the expert has).
// Two accumulators in TMEM: the epilogue of a tile runs beside the products of the next.
template <typename Out>
struct PairCfg {
  static constexpr int kStages = sizeof(Out) == 4 ? 5 : 6;
  static constexpr int kStagingBytes = 32 * kChannels * sizeof(Out);  // of a group of epilogue warps
  static constexpr int kSmem = kStages * kPairStageBytes + 2 * kStagingBytes + 1024;
};

// Eight rows of 128 staged elements to C by one warp, E elements at a time; `left` channels of the tile lie inside C.
template <typename Out, int E>
__device__ __forceinline__ void store_rows(const Out* in, Out* out, int64_t ldc, int rows, int left, int lane) {
  using V = Piece<Out, E>;
  constexpr int kPerRow = kChannels / E, kTurns = kPerRow / 4, kBatch = kTurns < 8 ? kTurns : 8;
#pragma unroll 1
  for (int t0 = 0; t0 < kTurns; t0 += kBatch) {
    V v[kBatch];
#pragma unroll
    for (int t = 0; t < kBatch; ++t) v[t] = reinterpret_cast<const V*>(in)[(t0 + t) * 32 + lane];
#pragma unroll
    for (int t = 0; t < kBatch; ++t) {
      const int i = (t0 + t) * 32 + lane, r = i / kPerRow, x = i % kPerRow * E;
      if (r >= rows) continue;
      if (x + E <= left) {
        *reinterpret_cast<V*>(out + r * ldc + x) = v[t];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x + e < left) out[r * ldc + x + e] = v[t].e[e];
      }
    }
  }
}

template <typename Out>
__global__ void __launch_bounds__(kPairThreads, 1) gemm_i8_pair_kernel(const __grid_constant__ Maps maps,
                                                                       const __grid_constant__ Params P) {
  using C = PairCfg<Out>;
  constexpr int S = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * S + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ PairGroups groups;
  __shared__ __align__(16) float token_scale[8][32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = int(cluster_ctarank());
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, tfull = full + 16 * S, tempty = tfull + 16,
                 drain = tempty + 16;

  if (threadIdx.x == 0) {
    tma_prefetch_map(&maps.a);
    tma_prefetch_map(&maps.b);
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
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_slot), 512);
  groups.count(P, kPairThreads);
  __syncwarp();
  tc_fence_before();
  cluster_sync_all();  // (of this CTA's threads, too) both CTAs' barriers exist before either signals
  tc_fence_after();
  if (P.G > 1) {
    if (warp == 0) groups.add_up(P, lane);
    __syncthreads();
  }
  const uint32_t tmem = tmem_slot;
  const int channel_tiles = (P.N + kPairChannels - 1) / kPairChannels;
  const int total = groups.first[P.G] * channel_tiles, pair = int(blockIdx.x) / 2, pairs = int(gridDim.x) / 2;
  const int blocks = (P.K + kKBytes - 1) / kKBytes;
  PairWalk walk{groups, channel_tiles};

  if (warp == 0) {
    const uint32_t bytes = kChannels * kKBytes + P.tile_rows / 2 * kKBytes;  // that each CTA brings
    int stage = 0, in_flight = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int t = pair; ok && t < total; t += pairs) {
      const PairTile w = walk.at(t);
      const int n0 = w.n0 + rank * kChannels, m0 = w.m0 + rank * ((w.rows + 31) / 32 * 16);
      for (int b = 0; b < blocks; ++b) {
        if (!(ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * stage, phase ^ 1)))) break;
        const uint32_t at = ring + stage * kPairStageBytes, bar = map_to_cta(full + 8 * stage, 0);
        if (!(t == 0 && b == P.withhold) && elect_one()) {
          if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, 2 * bytes);
          tma_load_3d_pair(at, &maps.b, b * kKBytes, n0, w.g, bar);
          tma_load_2d_pair(at + kChannels * kKBytes, &maps.a, b * kKBytes, m0, bar);
        }
        __syncwarp();
        if (in_flight < S) ++in_flight;
        if (++stage == S) stage = 0, phase ^= 1;
      }
    }
    // All that was loaded is used before the CTA ends, and the arrivals that say so have come (in both CTAs); after a
    // wait that ran out (of the products, too) copies still under way end first.  Those of rank 1 count on rank 0's
    // barriers.
    if (ok && in_flight > 0) {
      const int last = stage > 0 ? stage - 1 : S - 1;
      ok = __all_sync(0xffffffffu, wait_bar(P, empty + 8 * last, stage > 0 ? phase : phase ^ 1));
    }
    for (int i = 0; !ok && rank == 0 && i < in_flight; ++i) {
      if (--stage < 0) stage = S - 1, phase ^= 1;
      wait_bar(P, full + 8 * stage, phase);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      int rows = pair < total ? walk.at(pair).rows : 0, next_rows = 0;
      for (int t = pair; ok && t < total; t += pairs, rows = next_rows) {
        const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (uint32_t((rows + 31) / 32 * 4) << 17) |
                               (uint32_t(kPairChannels >> 4) << 24);
        if (!(ok = __all_sync(0xffffffffu, wait_bar(P, tempty + 8 * acc, acc_phase ^ 1)))) break;
        tc_fence_after();
        const uint32_t d = tmem + acc * kPairTokens;
        for (int b = 0; b < blocks; ++b) {
          if (!(ok = __all_sync(0xffffffffu, wait_bar(P, full + 8 * stage, phase)))) break;
          tc_fence_after();
          const uint32_t at = ring + stage * kPairStageBytes;
          const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kKBytes / 32; ++k) umma_i8_pair(d, da + 2 * k, db + 2 * k, idesc, b > 0 || k > 0);
            tc_commit_pair(empty + 8 * stage);
            if (b == blocks - 1) tc_commit_pair(tfull + 8 * acc);
          }
          __syncwarp();
          if (++stage == S) stage = 0, phase ^= 1;
          if (b == 0 && t + pairs < total) next_rows = walk.at(t + pairs).rows;  // (while these products run)
        }
        if ((acc ^= 1) == 0) acc_phase ^= 1;
      }
      // products under way end before the TMEM is given back (the epilogue may have left after a wait that ran out)
      if (elect_one()) tc_commit_pair(drain, 1);
      __syncwarp();
      wait_bar(P, drain, 0);
    }
  } else {
    // Epilogue: a warp owns 32 channels (its lane quarter of the accumulator), a lane one of them; groups of four
    // warps take turns at the 32-token chunks of a tile.  Values go through the group's staging, [32 tokens][128
    // channels], so that whole lines of C are stored.  The scales of a tile are read before its sums are waited for, a
    // chunk's sums while the chunk before is worked on.  At short K this is what a tile waits for: 4096 x 5120 outputs
    // of K = 512 take 23 us, 14 without it (twice the epilogue warps: 20, but 5 % more at K >= 1024).
    const int q = warp & 3, group = (warp - 2) / 4;
    constexpr int kTurns = kPairTokens / 64;  // chunks of a tile that a group takes
    Out* const staging = reinterpret_cast<Out*>(smem_raw + (ring - smem_u32(smem_raw)) + S * kPairStageBytes +
                                                group * C::kStagingBytes);
    float* const sa = token_scale[warp - 2];
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int t = pair; t < total; t += pairs) {
      const PairTile w = walk.at(t);
      const int n0 = w.n0 + rank * kChannels, n = n0 + q * 32 + lane;
      const float sb = n < P.N ? P.scale_b[int64_t(w.g) * P.N + n] : 0.0f;
      const float add = n < P.N && P.bias ? P.bias[int64_t(w.g) * P.N + n] : 0.0f;
      float scales[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int r = (group + 2 * i) * 32 + lane;
        scales[i] = r < w.rows ? P.scale_a[w.m0 + r] : 0.0f;
      }
      if (!named_bar_and(1 + group, 128, wait_bar(P, tfull + 8 * acc, acc_phase))) break;  // the group leaves together
      __syncwarp();  // (the lanes waited one by one; what follows wants the warp together)
      tc_fence_after();
      const int chunks = (w.rows + 31) / 32;
      const uint32_t sums = tmem + (uint32_t(q) << 21) + acc * kPairTokens;
      // The accumulator has been read: this warp's loads have completed (tcgen05.wait::ld), the lanes have met, and the
      // pair of tcgen05 fences, this one before the arrival and the issuing warp's behind its wait, orders the loads
      // before the products that overwrite it, whatever the arrival's own semantics.  No ordinary memory is handed over
      // (C is not read here), so the arrival is relaxed: a releasing one waits for this warp's stores to C, 1 us a tile.
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(map_to_cta(tempty + 8 * acc, 0));
      };
      auto finish = [&](const uint32_t (&v)[32], float scale, int c) {
        sa[lane] = scale;
        __syncwarp();
        float4 s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = reinterpret_cast<const float4*>(sa)[j];
        Out* const mine = staging + q * 32 + lane;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 s4 = s[j / 4];
          const float f[4] = {fmaf(__int2float_rn(int(v[j + 0])) * s4.x, sb, add),
                              fmaf(__int2float_rn(int(v[j + 1])) * s4.y, sb, add),
                              fmaf(__int2float_rn(int(v[j + 2])) * s4.z, sb, add),
                              fmaf(__int2float_rn(int(v[j + 3])) * s4.w, sb, add)};
          const Piece<Out, 4> o = pack<Out, 4>(f);
#pragma unroll
          for (int u = 0; u < 4; ++u) mine[(j + u) * kChannels] = o.e[u];
        }
        named_bar_sync(1 + group, 128);
        // a quarter of the rows for each warp
        const int row0 = q * 8, rows = min(8, w.rows - c * 32 - row0), left = min(kChannels, P.N - n0);
        Out* const out = static_cast<Out*>(P.c) + int64_t(w.m0 + c * 32 + row0) * P.ldc + n0;
        const Out* const in = staging + row0 * kChannels;
        if (P.c_step >= 16) store_rows<Out, 16 / sizeof(Out)>(in, out, P.ldc, rows, left, lane);
        else if (P.c_step == 8) store_rows<Out, 8 / sizeof(Out)>(in, out, P.ldc, rows, left, lane);
        else if (P.c_step == 4) store_rows<Out, 4 / sizeof(Out)>(in, out, P.ldc, rows, left, lane);
        else store_rows<Out, 1>(in, out, P.ldc, rows, left, lane);
        __syncwarp();
        named_bar_sync(1 + group, 128);
      };
      uint32_t v[2][32];
      if (group < chunks) tmem_ld32(sums + group * 32, v[0]);
      else release();
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int c = group + 2 * i;
        if (c < chunks) {
          tmem_ld_wait(v[i % 2]);
          if (c + 2 < chunks) tmem_ld32(sums + (c + 2) * 32, v[(i + 1) % 2]);
          else release();
          finish(v[i % 2], scales[i], c);
        }
      }
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
  P.token_tiles = int(token_tiles);
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

// The height of the pair tiles.  Four instructions of a tile h tokens high move 32 KB + 128 h bytes through an SM's
// shared memory (operands written by TMA, read by the tensor core, half of the tokens by either CTA), 256 + h cycles;
// the products themselves take 2 h.  So a tile costs 256 + h, and the rows of one matrix are cut so that the waves of
// the pairs cost least together.
int pair_rows(const Params& P) {
  if (P.G > 1) return kPairTokens;
  const int64_t channel_tiles = (P.N + kPairChannels - 1) / kPairChannels, pairs = sm_count() / 2;
  int best = kPairTokens;
  int64_t least = 0;
  for (int rows = kPairTokens; rows >= 96; rows -= 32) {
    const int64_t token_tiles = (P.M + rows - 1) / rows, waves = (token_tiles * channel_tiles + pairs - 1) / pairs;
    const int64_t cost = waves * (rows + 256);
    if (least == 0 || cost < least) least = cost, best = rows;
  }
  return best;
}

template <int TOKENS, typename Out>
int run(const Maps& maps, Params P, cudaStream_t stream) {
  using T = Tile<TOKENS>;
  const int64_t token_tiles = P.offsets ? P.M / TOKENS + P.G : (P.M + TOKENS - 1) / TOKENS;
  const int64_t tiles = token_tiles * ((P.N + kChannels - 1) / kChannels);
  const int blocks = (P.K + kKBytes - 1) / kKBytes;
  // CTAs for all SMs, two each, with two blocks of K or more for every one: 16 tokens through 8192 x 3584 take 11.4,
  // 10.3, 9.6 and 13.8 us with one, two, four and eight CTAs a tile (the rule takes four), through 1024 x 8192 17.7, 11.7,
  // 8.3 and 7.3 (eight); wide tiles exchange more sums: 128 tokens through 4096 x 4096 20.5, 15.0, 11.3 and 12.2 (four).
  P.split = 1;
  while (P.split * TOKENS < 512 && P.split < kMaxSplit && tiles * P.split * 2 <= 2 * int64_t(sm_count()) &&
         blocks >= P.split * 4)
    P.split *= 2;
  if (tiles * P.split > kMaxExtent) return ENTWINE_ERR_INVALID;
  P.token_tiles = int(token_tiles);
  auto kernel = gemm_i8_kernel<TOKENS, Out>;
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
  const int64_t pair_tiles = int64_t(std::min(P.G, P.M)) * ((P.N + kPairChannels - 1) / kPairChannels);
  Maps maps;
  // Pairs where experts alone give every pair two tiles (64 experts of 4096 x 1024 with 4, 6, 16 and 64 rows take 42.2,
  // 43.6, 47.2 and 52.4 us on pairs, 43.5, 48.4, 67.5 and 90.6 on narrow tiles), and for more than 128 tokens where half
  // of the pairs get one (160 tokens through 8192 x 3584: 13.1 and 16.2 us; 300 through 1024 x 4096, where they do not,
  // 13.0 and 10.0).
  if (rows > 128 ? (rows + 127) / 128 * pair_tiles >= sm_count() / 4 : pair_tiles >= sm_count()) {
    Params Q = P;
    Q.tile_rows = pair_rows(P);
    if (!make_maps(&maps, A, lda, B, ldb, expert_stride, Q, Q.tile_rows / 2)) return ENTWINE_ERR_CUDA;
    return run_pairs<Out>(maps, Q, stream);
  }
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

int gemm(const void* A, int64_t lda, const float* scale_a, const void* B, int64_t ldb, int64_t expert_stride,
         const float* scale_b, const float* bias, const int32_t* offsets, void* C, int c_dtype, int64_t ldc, int64_t M,
         int64_t N, int64_t K, int64_t G, void* stream) {
  if (c_dtype != ENTWINE_BF16 && c_dtype != ENTWINE_FP16 && c_dtype != ENTWINE_FP32) return ENTWINE_ERR_INVALID;
  if (M < 0 || M > kMaxRows || N < 1 || N > kMaxChannels || K < 1 || K > kMaxK || G < 1 || G > kMaxGroups ||
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
  const uint64_t starts = reinterpret_cast<uintptr_t>(C) | uint64_t(ldc) * (c_dtype == ENTWINE_FP32 ? 4 : 2);
  P.c_step = int(std::min<uint64_t>(starts & (~starts + 1), 16));
  P.M = int(M);
  P.N = int(N);
  P.K = int(K);
  P.G = int(G);
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

WaitSettings wait_settings() {
  return {static_cast<unsigned long long>(g_wait_budget_ns.load(std::memory_order_relaxed)),
          int(g_withhold.load(std::memory_order_relaxed))};
}

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

int entwine_ops_set_option(int key, int64_t value) {
  switch (key) {
    case ENTWINE_OPS_OPT_WAIT_BUDGET_NS:
      // (a millisecond at least: after a wait that ran out, the same time is given to what is still under way)
      if (value < 1000000) return ENTWINE_ERR_INVALID;
      g_wait_budget_ns.store(value, std::memory_order_relaxed);
      return ENTWINE_OK;
    case ENTWINE_OPS_OPT_WITHHOLD_BLOCK:
      if (value < -1 || value > kMaxK) return ENTWINE_ERR_INVALID;
      g_withhold.store(value, std::memory_order_relaxed);
      return ENTWINE_OK;
    default: return ENTWINE_ERR_INVALID;
  }
}

int entwine_ops_failed_waits(void* stream, uint64_t* count) {
  if (!count) return ENTWINE_ERR_INVALID;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &capture) != cudaSuccess) return launched(cudaErrorUnknown);
  if (capture != cudaStreamCaptureStatusNone) return ENTWINE_ERR_INVALID;
  unsigned long long n = 0, n4 = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&n, g_waits_failed, sizeof(n), 0, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = mxf4_failed_waits(&n4, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return launched(e);
  *count = n + n4;
  return ENTWINE_OK;
}

int entwine_ops_status(void* stream) {
  constexpr int kDevices = 64;
  static thread_local uint64_t told[kDevices];  // failures that this thread has been told of
  uint64_t n = 0;
  const int rc = entwine_ops_failed_waits(stream, &n);
  if (rc != ENTWINE_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return launched(cudaErrorUnknown);
  if (dev < 0 || dev >= kDevices) return n ? ENTWINE_ERR_TIMEOUT : ENTWINE_OK;
  const bool news = n != told[dev];
  told[dev] = n;
  return news ? ENTWINE_ERR_TIMEOUT : ENTWINE_OK;
}

}  // extern "C"
