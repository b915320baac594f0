// How the products beside the fused call (int8, 4-bit) cut their work: the rows of each expert into token tiles, and the
// walk of a persistent CTA pair over tiles of 256 channels.  A kernel's Params has M, G, offsets, token_tiles, tile_rows.
#pragma once

#include <cuda_runtime.h>

namespace entwine {

constexpr int kMaxGroups = 1024;
constexpr int kPairChannels = 256;
constexpr int kBand = 16;  // token tiles that share a walk over the channels: their rows stay in L2

// Expert and token rows of token tile `tile`, found by one warp: experts have ceil(rows / TOKENS) tiles each.
template <int TOKENS, typename Params>
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

struct PairTile {
  int g, m0, rows, n0;
};

// What the walk over the tiles needs of each expert.
struct PairGroups {
  int first[kMaxGroups + 1];  // token tiles of the experts before
  int start[kMaxGroups];      // first row
  int end[kMaxGroups];
  int height[kMaxGroups];     // rows of a tile: an expert's tiles are as equal as steps of 32 rows allow

  // Token tiles of each expert, by the CTA's `threads`; then (behind a barrier, where there are several) their running sum,
  // by one warp.
  template <typename Params>
  __device__ __forceinline__ void count(const Params& P, int threads) {
    if (threadIdx.x == 0) first[0] = 0;
    for (int g = threadIdx.x; g < P.G; g += threads) {
      int lo = 0, hi = P.M;
      if (P.offsets) {
        lo = min(max(P.offsets[g], 0), P.M);
        hi = min(max(P.offsets[g + 1], lo), P.M);
      }
      const int tiles = (hi - lo + P.tile_rows - 1) / P.tile_rows;
      start[g] = lo;
      end[g] = hi;
      height[g] = tiles > 0 ? ((hi - lo + tiles - 1) / tiles + 31) / 32 * 32 : 0;
      first[g + 1] = tiles;
    }
  }
  template <typename Params>
  __device__ __forceinline__ void add_up(const Params& P, int lane) {
    int before = 0;
    for (int g0 = 0; g0 < P.G; g0 += 32) {
      int sum = g0 + lane < P.G ? first[g0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      // (offsets that decrease can claim rows many times over: no more tiles than the bound, within 32 bits)
      sum = min(sum + before, P.token_tiles);
      if (g0 + lane < P.G) first[g0 + lane + 1] = sum;
      before = __shfl_sync(0xffffffffu, sum, 31);
    }
  }
};

// The tiles of a pair, in order.  An expert's bands of kBand token tiles each walk over the channels together.
struct PairWalk {
  const PairGroups& G;
  int channel_tiles;
  int g = 0;
  __device__ __forceinline__ PairTile at(int t) {
    while (G.first[g + 1] * channel_tiles <= t) ++g;
    const int tiles = G.first[g + 1] - G.first[g];
    int local = t - G.first[g] * channel_tiles, m = 0, in_band = tiles;
    if (tiles > kBand) {
      const int band = local / (kBand * channel_tiles);
      local -= band * kBand * channel_tiles;
      m = band * kBand;
      in_band = min(kBand, tiles - m);
    }
    const int channel = int(unsigned(local) / unsigned(in_band));
    m += local - channel * in_band;
    PairTile r;
    r.g = g;
    r.m0 = G.start[g] + m * G.height[g];
    r.rows = min(G.height[g], G.end[g] - r.m0);
    r.n0 = channel * kPairChannels;
    return r;
  }
};

}  // namespace entwine
