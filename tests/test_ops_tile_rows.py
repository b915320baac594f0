"""CPU tests of the 4-bit product's rules on sizes (csrc/tile_rows.h)."""
import os
import subprocess

import pytest

from paper_2609_11562_b200 import build as B

HEIGHT = """
#include <cstdint>
#include <cstdio>
#include "tile_rows.h"
int main() {
  const int64_t most_rows = 2147418111;
  int64_t step = 1;
  for (int64_t rows = 1; rows <= most_rows; rows += step) {
    int64_t want = (4 * rows + 31) / 32 * 32;
    if (want > 192) want = 192;
    if (entwine::expert_tile_rows(int(rows), 192) != want) return std::printf("%lld\\n", (long long)rows), 1;
    if (rows > 1000) step = 9973;
  }
  return entwine::expert_tile_rows(int(most_rows), 192) != 192 || entwine::expert_tile_rows(1 << 29, 192) != 192;
}
"""


# rows of an average expert, tiles of 256 channels, whether pairs take them: few rows need a tile for nearly every pair
PAIRS = """
#include <cstdio>
#include "tile_rows.h"
int main() {
  const struct { int rows; int64_t tiles; bool pairs; } cases[] = {
      {1, 16, false}, {16, 16, false}, {16, 32, false}, {64, 63, false}, {16, 64, true}, {64, 64, true}, {1, 1024, true}, {65, 15, false},
      {65, 16, true}, {2147418111, 8, false}, {2147418111, int64_t(1) << 40, true}};
  for (const auto& c : cases)
    if (entwine::product_by_pairs(c.rows, c.tiles) != c.pairs) return std::printf("%d %lld\\n", c.rows, (long long)c.tiles), 1;
  return 0;
}
"""


@pytest.mark.parametrize("code", [HEIGHT, PAIRS], ids=["height of experts' tiles", "pairs or narrow tiles"])
def test_rules(tmp_path, code):
    source, program = tmp_path / "rule.cc", tmp_path / "rule"
    source.write_text(code)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-ftrapv", "-I", B.CSRC, str(source), "-o", str(program)], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
