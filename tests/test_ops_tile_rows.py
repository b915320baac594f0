"""CPU test of the height of the experts' tiles (csrc/tile_rows.h) over all numbers of rows that the product takes."""
import os
import subprocess

from paper_2609_11562_b200 import build as B

CODE = """
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


def test_tile_rows_of_experts_stay_within_a_tile(tmp_path):
    source, program = tmp_path / "rows.cc", tmp_path / "rows"
    source.write_text(CODE)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-ftrapv", "-I", B.CSRC, str(source), "-o", str(program)], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
