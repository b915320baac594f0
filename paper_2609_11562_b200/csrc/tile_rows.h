// Rules on sizes that need nothing of CUDA.
#pragma once

#include <algorithm>
#include <cstdint>

namespace entwine {

// Which kernel the 4-bit product takes for `rows` tokens, or rows of an average expert, that make `pair_tiles` tiles of 256
// channels: CTA pairs for more than 64 of them where there are 16 tiles, for fewer where nearly every pair gets one; else
// narrow tiles, which share K between CTAs.  In us, pairs and narrow tiles: 32, 64 and 128 tokens through 8192 x 3584 9.8 10.0
// 10.3 and 8.7 9.8 12.5; 64 through 16384 x 8192 18.0 and 20.0; 300 through 1024 x 4096 (8 tiles) 10.1 and 8.8; 600 through 1024
// x 1024 (16) 7.0 and 9.3; 64 experts of 4096 x 1024 with 1, 4 and 16 rows 23.5 28.3 32.7 and 31.2 41.4 68.2; eight experts of
// K = 4096 with 16 rows each and 512, 1024, 2048 and 4096 channels (16, 32, 64, 128 tiles) 12.6 13.4 14.8 22.1 and 8.2 11.2 14.9
// 26.3; four of 100 rows, 1024 x 4096 (16) 13.7 and 12.3, eight of 1024 x 2048 (32) 11.4 and 12.7.
constexpr bool product_by_pairs(int rows, int64_t pair_tiles) { return pair_tiles >= (rows > 64 ? 16 : 64); }

// The height of the pair tiles of the 4-bit product of experts with `rows` rows on average: four times as many, in steps of 32
// rows, at most `most`, a multiple of 32.  (Twice as many: 36.2 us instead of 33.6 for 64 experts of 16 rows, 4096 x 1024, whose
// larger ones are then two tiles, 60.7 instead of 57.5 for 128 of 16 rows, 2048 x 2048, but 35.0 instead of 35.8 for 32 of 16 rows,
// 2048 x 4096; eight times: within 1 % of four.)  The average is cut first: four times it need not fit 32 bits.
constexpr int expert_tile_rows(int rows, int most) { return std::min(most, (4 * std::min(rows, most / 4) + 31) / 32 * 32); }

}  // namespace entwine
