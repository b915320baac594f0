// Rules on sizes that need nothing of CUDA.
#pragma once

#include <algorithm>

namespace entwine {

// The height of the pair tiles of the 4-bit product of experts with `rows` rows on average: four times as many, in steps of 32
// rows, at most `most`, a multiple of 32 (twice as many: 35 us instead of 33 for 64 experts of 16 rows, whose larger ones are
// then two tiles).  The average is cut first: four times it need not fit 32 bits.
constexpr int expert_tile_rows(int rows, int most) { return std::min(most, (4 * std::min(rows, most / 4) + 31) / 32 * 32); }

}  // namespace entwine
