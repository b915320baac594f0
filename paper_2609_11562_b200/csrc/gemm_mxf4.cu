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

#include "gemm_tiles.cuh"
#include "ops_common.cuh"
#include "sm100.cuh"
#include "tile_rows.h"

namespace entwine {
namespace {

constexpr int kChannels = 128;       // channels of a tile
constexpr int kKBytes = 128;         // bytes of codes per row and pipeline stage (one swizzled row): 256 elements
constexpr int kScaleBytes = 8;       // their scales
constexpr int kThreads = 128;
constexpr int kMaxSplit = 8;
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
  int tile_rows;           // most tokens of a pair tile, a multiple of 32
  int withhold;            // block of K that the first tile's first CTA or pair does not load; -1: none
  unsigned long long wait_ns;  // budget of every wait
};

__device__ __noinline__ void wait_failed() { atomicAdd(&g_waits_failed, 1ull); }

// Bounded wait for a phase of a barrier; CLUSTER: of one that the other CTA arrives at, too.
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_bar(const Params& P, uint32_t bar, uint32_t parity) {
  unsigned long long t0 = 0;
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
      if (CLUSTER ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity)) return true;
    const unsigned long long now = globaltimer_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > P.wait_ns) break;
  }
  wait_failed();
  return false;
}
// The same for a warp that has time: it sleeps between its looks, which leaves the barriers to the warps that have not.
__device__ __forceinline__ bool idle_wait(const Params& P, uint32_t bar, uint32_t parity, int ns) {
  unsigned long long t0 = 0;
  while (!__all_sync(0xffffffffu, mbar_test(bar, parity))) {
    const unsigned long long now = globaltimer_ns();
    if (t0 == 0) t0 = now;
    if (__any_sync(0xffffffffu, now - t0 > P.wait_ns)) {
      wait_failed();
      return false;
    }
    __nanosleep(ns);
  }
  return true;
}
// The same by a whole warp.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(const Params& P, uint32_t bar, uint32_t parity) {
  return __all_sync(0xffffffffu, wait_bar<CLUSTER>(P, bar, parity));
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

// The scales of up to ROWS rows of an operand, fetched stage by stage by THREADS threads: two words of four bytes a row and
// stage.  Word w of row r goes to place w * 512 + r % 32 * 16 + r / 32 * 4 of its 128 rows; a thread's rows are THREADS / 2
// apart, so that its places differ by constants.  Rows and blocks that are not there get zeros, a scale that nothing is
// multiplied with.
template <int ROWS, int THREADS>
struct Scales {
  static constexpr int N = (2 * ROWS + THREADS - 1) / THREADS, kStep = THREADS / 64;  // rows / 32 from one word to the next
  static_assert(THREADS % 64 == 0, "whole groups of 32 rows");
  const uint8_t* from[N];
  uint32_t place, there, word;
  // `rows` rows of the matrix lie at and behind `first`, `most` of them are wanted
  __device__ __forceinline__ Scales(const uint8_t* all, int64_t first, int64_t ld, int rows, int most, int thread) {
    const int r0 = thread / 2;
    word = thread % 2;
    place = word * 512 + r0 % 32 * 16 + r0 / 32 * 4;
    there = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int r = r0 + k * (THREADS / 2);
      const bool ok = r < min(rows, most);
      from[k] = all + (ok ? first + r * ld : 0) + 4 * word;
      there |= uint32_t(ok) << k;
    }
  }
  __device__ __forceinline__ void fetch(uint32_t smem, int at, int row_bytes) const {
    const int left = row_bytes - at - int(4 * word);
    const uint32_t bytes = uint32_t(max(0, min(left, 4)));
    if (left <= 0) at = -int(4 * word);  // (nothing is read there)
#pragma unroll
    for (int k = 0; k < N; ++k)
      cp_async4(smem + place + k * kStep / 4 * 1024 + k * kStep % 4 * 4, from[k] + at, there >> k & 1 ? bytes : 0u);
  }
};

// One tile of 128 channels x TOKENS tokens per cluster of one to eight CTAs, which share the length K: each sums its
// blocks of K, then the partial sums meet through distributed shared memory, added in the order of the CTAs, each CTA
// finishing its share of the tokens.  So a decoding step reads the weights with all SMs.  16 tokens through 8192 x 3584 take
// 8.1 us, the weight's 15.6 MB at 1.9 TB/s: start, the latency of the three or four blocks that a CTA has, and the exchange.
template <int TOKENS, typename Out>
__global__ void __launch_bounds__(kThreads) gemm_mxf4_kernel(const __grid_constant__ Maps maps,
                                                             const __grid_constant__ Params P) {
  using T = Tile<TOKENS>;
  constexpr int S = T::kStages, kScaleThreads = kThreads - 64;
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
        mbar_init(full + 8 * s, 1 + kScaleThreads);  // the codes, every thread's share of the scales
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
      if (!(ok = warp_wait(P, empty + 8 * (issued % S), (issued / S - 1) & 1))) break;
      load();
    }
  } else if (warp == 1) {
    for (int i = 0; i < blocks; ++i) {
      const int s = i % S;
      if (!(ok = warp_wait(P, full + 8 * s, (i / S) & 1))) break;
      // the products that read this buffer of scales are done
      if (i >= 2 && !(ok = warp_wait(P, empty + 8 * ((i - 2) % S), ((i - 2) / S) & 1))) break;
      tc_fence_after();
      fence_async_smem();  // the scales were written by ordinary copies
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
    // Scales, as many stages ahead as the ring holds.  (The copies arrive by themselves: a thread that waited for its oldest
    // ones and fenced them waited for the youngest too.)
    const int thread = threadIdx.x - 64;
    const Scales<kChannels, kScaleThreads> channels(P.scale_b, int64_t(g) * P.scale_stride + int64_t(n0) * P.ldsb, P.ldsb,
                                                    P.N - n0, kChannels, thread);
    const Scales<TOKENS, kScaleThreads> tokens(P.scale_a, int64_t(m0) * P.ldsa, P.ldsa, P.M - m0, TOKENS, thread);
    for (int i = 0; i < blocks; ++i) {
      if (i >= S && !(ok = warp_wait(P, empty + 8 * (i % S), (i / S - 1) & 1))) break;
      const uint32_t at = ring + i % S * T::kStageBytes + T::kCodes;
      channels.fetch(at, (first + i) * kScaleBytes, P.kscales);
      tokens.fetch(at + T::kScales, (first + i) * kScaleBytes, P.kscales);
      cp_async_arrive(full + 8 * (i % S));
    }
    cp_async_wait_all();
  }
  __syncwarp();
  ok = warp_wait(P, done, 0) && ok;
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

// ------------------------------------------------------------------------------------------
// many tokens: CTA pairs, persistent
// ------------------------------------------------------------------------------------------
// Two CTAs of a cluster compute 256 channels x up to 192 tokens (tcgen05 cta_group::2: 128 channels each, each loading
// half of the tokens' codes and all of their scales).  Two accumulators in TMEM, 2 x 192 of its 512 columns, so that the
// epilogue of a tile runs beside the products of the next, and five buffers of scales of 24 columns.  (224 tokens leave
// room for two: the way from products that are done to the next but one's scales is then longer than the products between.)
// 8192 x 8192 x 3584 takes 115 to 118 us, 4.2 PFLOP/s: 670 to 680 cycles a block of K, of which the products are 384 and the
// issuing warp's own instructions 330, at 1.7 GHz; 135 us in a long series, which the power limit holds at 1.44 GHz.
// TMA warp, MMA warp, epilogue warps by groups of four, scale warps, their messenger.  (Eight epilogue warps: 59 us where
// twelve took 53, for 32 experts' 15.6k rows of 4096 x 1024, where the epilogue is what a tile waits for; 16 have too few
// registers.)
constexpr int kEpilogueGroups = 3, kScaleWarps = 4;
constexpr int kFirstScaleWarp = 2 + 4 * kEpilogueGroups, kPairThreads = 32 * (kFirstScaleWarp + kScaleWarps + 1);
constexpr int kPairTokens = 192;
constexpr int kPairCodes = (kChannels + kPairTokens / 2) * kKBytes;  // bytes of a stage
constexpr int kPairStages = 6;
// Scales come by groups of four stages, 32 bytes of a row: eight words of 128 rows each, a little apart from one another so
// that the words of a row, and rows 32 apart, are written to different banks.  (Stage by stage, eight bytes of a row, a
// warp's copies touched four times as many lines: 138 us instead of 112 at 8192 x 8192 x 3584.)
constexpr int kGroupStages = 4, kGroupWords = 2 * kGroupStages, kGroups = 3;
constexpr int kWordBytes = 512 + 16, kSectionBytes = kGroupWords * kWordBytes;  // (a section: 128 rows)
constexpr int kGroupBytes = 3 * kSectionBytes;                                  // channels, tokens, tokens from 128 on
constexpr int kPairSmem = kPairStages * kPairCodes + kGroups * kGroupBytes + 1024;
constexpr int kPairScaleCol = 2 * kPairTokens;
constexpr int kPairBuffers = 5;
static_assert(kPairScaleCol + 24 * kPairBuffers <= 512 && kPairBuffers < kPairStages,
              "TMEM, and barriers that tell a buffer's last use");

// 32 channels (lanes) x 32 tokens (registers) to C, token by token: 64 or 128 bytes side by side with each store.  (Lanes
// that first exchange halves until each has four or eight neighbouring channels store a chunk with 8 or 4 instructions
// instead of 32: no faster, and 20 % slower with 8.)  `rows` tokens and `left` channels lie inside C.
template <typename Out>
__device__ __forceinline__ void store_chunk(const uint32_t (&v)[32], float add, Out* out, int64_t ldc, int rows, int left,
                                            int lane) {
  if (lane >= left) return;
  out += lane;
  if (rows >= 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j) out[j * ldc] = Elem<Out>::down(__uint_as_float(v[j]) + add);
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < rows) out[j * ldc] = Elem<Out>::down(__uint_as_float(v[j]) + add);
  }
}

// What a thread fetches of a section: word lane % 8 of rows lane / 8 * 32 + warp + 4 k, k = 0 to 7, those below `rows`.
struct Section {
  const uint8_t* from;
  int64_t step;
  int count;
  __device__ __forceinline__ Section(const uint8_t* first_row, int64_t ld, int rows, int warp, int lane) {
    const int r = lane / 8 * 32 + warp;
    from = first_row + r * ld + lane % 8 * 4;
    step = 4 * ld;
    count = max(0, min(8, (rows - r + 3) / 4));
  }
  // The group's words, from byte `at` of the rows on; zeros (a scale that nothing is multiplied with) for what is not there.
  __device__ __forceinline__ void fetch(uint32_t smem, int at, int row_bytes, const uint8_t* somewhere, int warp,
                                        int lane) const {
    const int left = row_bytes - at - lane % 8 * 4, n = left > 0 ? count : 0;
    const uint32_t to = smem + lane % 8 * kWordBytes + warp * 16 + lane / 8 * 4;
    const uint8_t* p = from + at;
#pragma unroll
    for (int k = 0; k < 8; ++k, p += step)
      cp_async4(to + k * 64, k < n ? p : somewhere, k < n ? uint32_t(min(left, 4)) : 0u);
  }
};

template <typename Out>
__global__ void __launch_bounds__(kPairThreads, 1) gemm_mxf4_pair_kernel(const __grid_constant__ Maps maps,
                                                                         const __grid_constant__ Params P) {
  constexpr int S = kPairStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * S + 3 * kGroups + 5];
  __shared__ uint32_t tmem_slot;
  __shared__ int tile_columns[8];
  __shared__ PairGroups groups;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = int(cluster_ctarank());
  const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * S, tfull = full + 16 * S, tempty = tfull + 16,
                 drain = tempty + 16, scaled = drain + 8, sempty = scaled + 8 * kGroups, far = sempty + 8 * kGroups;
  const uint32_t scale_ring = ring + S * kPairCodes;

  if (threadIdx.x == 0) {
    tma_prefetch_map(&maps.a);
    tma_prefetch_map(&maps.b);
    for (int s = 0; s < S; ++s) {
      mbar_init(full + 8 * s, 1 + 1);  // both CTAs' codes, rank 0's scales
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < kGroups; ++s) {
      mbar_init(scaled + 8 * s, 32 * kScaleWarps);
      mbar_init(sempty + 8 * s, 1);
      mbar_init(far + 8 * s, 1);  // rank 1's scales
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull + 8 * a, 1);
      mbar_init(tempty + 8 * a, 2 * 4 * kEpilogueGroups);
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
  const int blocks = (P.kbytes + kKBytes - 1) / kKBytes;
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
        if (!(ok = warp_wait(P, empty + 8 * stage, phase ^ 1))) break;
        const uint32_t at = ring + stage * kPairCodes, bar = map_to_cta(full + 8 * stage, 0);
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
      ok = warp_wait(P, empty + 8 * last, stage > 0 ? phase : phase ^ 1);
    }
    for (int i = 0; !ok && rank == 0 && i < in_flight; ++i) {
      if (--stage < 0) stage = S - 1, phase ^= 1;
      wait_bar(P, full + 8 * stage, phase);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // (from uniform registers, where the instructions want their addresses and descriptors)
      const uint32_t base = uniform(tmem);
      const int tiles = int(uniform(uint32_t(total)));
      int stage = 0, acc = 0, turn = 0, group = 0;
      uint32_t phase = 0, acc_phase = 0, group_phase = 0, buffer = 0;
      bool ok = true, there[2] = {false, false};
      for (int t = pair; ok && t < tiles; t += pairs, ++turn) {
        if (!(ok = warp_wait<true>(P, tempty + 8 * acc, acc_phase ^ 1))) break;
        const uint32_t d = base + acc * kPairTokens;
        int columns = 0;
        // two blocks at a time: what a turn costs beside the products is paid half as often (one at a time: 128 us instead of 115)
        for (int b = 0; b < blocks; b += 2) {
          const bool two = b + 1 < blocks, last = b + 2 >= blocks, group_ends = last || b % kGroupStages == kGroupStages - 2;
          const int next = stage + 1 < S ? stage + 1 : 0, after = next + 1 < S ? next + 1 : 0;
          const uint32_t next_phase = stage + 1 < S ? phase : phase ^ 1, after_phase = next + 1 < S ? next_phase : next_phase ^ 1;
          ok = (there[0] || wait_bar<true>(P, full + 8 * stage, phase)) &&
               (!two || there[1] || wait_bar<true>(P, full + 8 * next, next_phase)) &&
               (b % kGroupStages != 0 || wait_bar<true>(P, far + 8 * group, group_phase));
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          if (b == 0) columns = int(uniform(uint32_t(tile_columns[turn % 8])));
          const uint32_t idesc[2] = {instr_desc_mxf4(columns, kPairChannels, 0), instr_desc_mxf4(columns, kPairChannels, 1)};
          // (a look at the next blocks' barriers takes as long as the issue of these products: both at once)
          const int third = after + 1 < S ? after + 1 : 0;
          there[0] = mbar_test_cluster(full + 8 * (two ? after : next), two ? after_phase : next_phase);
          there[1] = mbar_test_cluster(full + 8 * (two ? third : after), two && after + 1 == S ? after_phase ^ 1 : after_phase);
          tc_fence_after();
          auto products = [&](int s, uint32_t buf, int word, bool first) {
            const uint32_t at = ring + s * kPairCodes, scales = base + kPairScaleCol + buf * 24;
            const uint64_t da = smem_desc_sw128(at), db = smem_desc_sw128(at + kChannels * kKBytes);
            const uint64_t ds = smem_desc_scales(scale_ring + group * kGroupBytes + word * kWordBytes);
            // channels: two words of K; tokens: two words of the first 128, of the others
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              tmem_copy_scales_pair(scales + 4 * w, ds + ((w * kWordBytes) >> 4));
              tmem_copy_scales_pair(scales + 8 + 8 * w, ds + ((kSectionBytes + w * kWordBytes) >> 4));
              if (columns > 128) tmem_copy_scales_pair(scales + 12 + 8 * w, ds + ((2 * kSectionBytes + w * kWordBytes) >> 4));
            }
#pragma unroll
            for (int k = 0; k < kKBytes / 32; ++k)
              umma_mxf4_pair(d, da + 2 * k, db + 2 * k, idesc[k % 2], scales + k / 2 * 4, scales + 8 + k / 2 * 8,
                             !first || k > 0);
            tc_commit_pair(empty + 8 * s);
          };
          const uint32_t next_buffer = buffer + 1 < kPairBuffers ? buffer + 1 : 0;
          if (elect_one()) {
            products(stage, buffer, b % kGroupStages * 2, b == 0);
            if (two) products(next, next_buffer, b % kGroupStages * 2 + 2, false);
            if (group_ends) tc_commit_pair(sempty + 8 * group);
            if (last) tc_commit_pair(tfull + 8 * acc);
          }
          __syncwarp();
          buffer = !two ? next_buffer : next_buffer + 1 < kPairBuffers ? next_buffer + 1 : 0;
          stage = two ? after : next;
          phase = two ? after_phase : next_phase;
          if (group_ends && ++group == kGroups) group = 0, group_phase ^= 1;
        }
        if ((acc ^= 1) == 0) acc_phase ^= 1;
      }
      // products under way end before the TMEM is given back (the epilogue may have left after a wait that ran out)
      if (elect_one()) tc_commit_pair(drain, 1);
      __syncwarp();
      wait_bar(P, drain, 0);
    }
  } else if (warp < kFirstScaleWarp) {
    // Epilogue: a warp owns 32 channels (its lane quarter of the accumulator), a lane one of them; groups of four warps
    // take turns at the 32-token chunks of a tile, a chunk's sums read while the chunk before is worked on.
    const int q = warp & 3, group = (warp - 2) / 4;
    // chunks of a tile that a group takes, at most
    constexpr int kTurns = (kPairTokens / 32 + kEpilogueGroups - 1) / kEpilogueGroups;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int t = pair; t < total; t += pairs) {
      const PairTile w = walk.at(t);
      const int n0 = w.n0 + rank * kChannels + q * 32, n = n0 + lane;
      const float add = n < P.N && P.bias ? P.bias[int64_t(w.g) * P.N + n] : 0.0f;
      if (!idle_wait(P, tfull + 8 * acc, acc_phase, 100)) break;
      tc_fence_after();
      const int chunks = (w.rows + 31) / 32;
      const uint32_t sums = tmem + (uint32_t(q) << 21) + acc * kPairTokens;
      // (as in the int8 product: this warp's loads have completed, the lanes have met, the tcgen05 fences order the loads
      // before the products that overwrite the accumulator; no ordinary memory is handed over)
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(map_to_cta(tempty + 8 * acc, 0));
      };
      uint32_t v[2][32];
      if (group < chunks) tmem_ld32(sums + group * 32, v[0]);
      else release();
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int c = group + kEpilogueGroups * i, next = c + kEpilogueGroups;
        if (c < chunks) {
          tmem_ld_wait(v[i % 2]);
          if (next < chunks) tmem_ld32(sums + next * 32, v[(i + 1) % 2]);
          else release();
          store_chunk<Out>(v[i % 2], add, static_cast<Out*>(P.c) + int64_t(w.m0 + c * 32) * P.ldc + n0, P.ldc, w.rows - c * 32,
                           P.N - n0, lane);
          __syncwarp();
        }
      }
      if ((acc ^= 1) == 0) acc_phase ^= 1;
    }
  } else if (warp < kFirstScaleWarp + kScaleWarps) {
    // Scales of both operands, as many groups ahead as there is room for: the copies arrive on their group's barrier by
    // themselves.
    const int w4 = warp - kFirstScaleWarp;
    int group = 0, used = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int t = pair; ok && t < total; t += pairs) {
      const PairTile w = walk.at(t);
      const int n0 = w.n0 + rank * kChannels, tokens = min(P.M - w.m0, (w.rows + 31) / 32 * 32);
      const uint8_t* const row = P.scale_a + int64_t(w.m0) * P.ldsa;
      const Section b0(P.scale_b + int64_t(w.g) * P.scale_stride + int64_t(n0) * P.ldsb, P.ldsb, P.N - n0, w4, lane),
          a0(row, P.ldsa, min(tokens, 128), w4, lane), a1(row + 128 * P.ldsa, P.ldsa, tokens - 128, w4, lane);
      for (int at = 0; at < P.kscales; at += kGroupStages * kScaleBytes) {
        if (!(ok = warp_wait(P, sempty + 8 * group, phase ^ 1))) break;
        const uint32_t to = scale_ring + group * kGroupBytes;
        b0.fetch(to, at, P.kscales, P.scale_b, w4, lane);
        a0.fetch(to + kSectionBytes, at, P.kscales, P.scale_a, w4, lane);
        if (tokens > 128) a1.fetch(to + 2 * kSectionBytes, at, P.kscales, P.scale_a, w4, lane);
        cp_async_arrive(scaled + 8 * group);
        used = 1;
        if (++group == kGroups) group = 0, phase ^= 1;
      }
    }
    cp_async_wait_all();
    // the last arrival that says that a group has been used has come
    if (ok && used) wait_bar(P, sempty + 8 * (group > 0 ? group - 1 : kGroups - 1), group > 0 ? phase : phase ^ 1);
  } else {
    // The messengers tell rank 0's issuing warp, which has both CTAs' scales copied to TMEM, that they are there.  Their fence
    // makes the words, written by ordinary copies, visible to the tensor core, which reads them in this CTA; by a thread that
    // has copies of its own under way it would wait for them (416 us instead of 288 for 8192 x 8192 x 3584).  What rank 1's
    // hands over to the other CTA it releases to the cluster, where it is acquired.  That takes long, so it comes once a group,
    // as soon as the words are there, ahead of the products (from block to block: 244 us instead of 118).
    int group = 0;
    uint32_t group_phase = 0;
    bool ok = true;
    if (rank == 1) {
      for (int t = pair; ok && t < total; t += pairs) {
        for (int b = 0; b < blocks; b += kGroupStages) {
          if (!(ok = warp_wait(P, scaled + 8 * group, group_phase))) break;
          fence_async_smem();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(far + 8 * group, 0));
          __syncwarp();
          if (++group == kGroups) group = 0, group_phase ^= 1;
        }
      }
    } else {
      // Rank 0's says it stage by stage, when the buffer for a stage's scales is free: the products that read it (in both CTAs),
      // five blocks ago, are done.  It also says how wide a tile is, so that the issuing warp need not walk.
      int stage = 0, turn = 0, before = 0;  // before: blocks so far, kPairBuffers at most
      uint32_t phase = 0;
      for (int t = pair; ok && t < total; t += pairs, ++turn) {
        if (lane == 0) tile_columns[turn % 8] = (walk.at(t).rows + 31) / 32 * 32;
        for (int b = 0; b < blocks; ++b) {
          if (b % kGroupStages == 0) {
            if (!(ok = warp_wait(P, scaled + 8 * group, group_phase))) break;
            if (++group == kGroups) group = 0, group_phase ^= 1;
            fence_async_smem();
          }
          if (before == kPairBuffers) {
            const int s = stage >= kPairBuffers ? stage - kPairBuffers : stage + S - kPairBuffers;
            if (!(ok = warp_wait(P, empty + 8 * s, stage >= kPairBuffers ? phase : phase ^ 1))) break;
          } else {
            ++before;
          }
          if (lane == 0) mbar_arrive(full + 8 * stage);
          __syncwarp();
          if (++stage == S) stage = 0, phase ^= 1;
        }
      }
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
  const int64_t token_tiles = P.offsets ? P.M / P.tile_rows + P.G : (P.M + P.tile_rows - 1) / P.tile_rows;
  const int64_t tiles = token_tiles * ((P.N + kPairChannels - 1) / kPairChannels);
  if (tiles > kMaxExtent) return ENTWINE_ERR_INVALID;
  P.token_tiles = int(token_tiles);
  auto kernel = gemm_mxf4_pair_kernel<Out>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
  if (e != cudaSuccess) return launched(e);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(std::min<int64_t>(2 * tiles, sm_count() / 2 * 2)));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = kPairSmem;
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
// the pairs cost least together.  Of experts: expert_tile_rows().
int pair_rows(const Params& P, int rows) {
  if (P.G > 1) return expert_tile_rows(rows, kPairTokens);
  const int64_t channel_tiles = (P.N + kPairChannels - 1) / kPairChannels, pairs = sm_count() / 2;
  int best = kPairTokens;
  int64_t least = 0;
  for (int high = kPairTokens; high >= 32; high -= 32) {
    const int64_t token_tiles = (P.M + high - 1) / high, waves = (token_tiles * channel_tiles + pairs - 1) / pairs;
    const int64_t cost = waves * (high + 256);
    if (least == 0 || cost < least) least = cost, best = high;
  }
  return best;
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
  const int64_t channel_tiles = (P.N + kPairChannels - 1) / kPairChannels;
  const int64_t pair_tiles = int64_t(std::min(P.G, P.M)) * ((rows + kPairTokens - 1) / kPairTokens) * channel_tiles;
  Maps maps;
  if (product_by_pairs(rows, pair_tiles)) {
    Params Q = P;
    Q.tile_rows = pair_rows(P, rows);
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
