"""The grids of the layer operators' launches, on the CPU."""
from tests.test_host_code_cpu import run_host


def test_grids_stay_below_the_limits_of_a_launch(tmp_path):
    """fewer than 2^32 threads along x and 2^16 workgroups along y, whatever the sizes
    allow: 2^40 outputs in 64 x 64 tiles, 2^30 rows, 1024 groups"""
    out = run_host(tmp_path, r"""
#include <cstdio>
#include "oz2_layers.h"
int main() {
  int bad = 0, beyond = 0;
  auto take = [&](ll blocks) {
    const Oz2Grid g = oz2_grid(blocks);
    bad += (ll)g.x * 256 >= 1ll << 32 || g.y >= 1u << 16 || (ll)g.x * g.y < blocks || !g.x;
    bad += g.y > 1 ? g.x % 8 != 0 : g.x != blocks;
    beyond += g.y > 1;
  };
  for (ll b : {1ll, 8ll, 255ll, (1ll << 24) - 8, (1ll << 24) - 7, 1ll << 24, (1ll << 28) + 1}) take(b);
  const int off[2] = {0, 0};
  for (int rows : {1, 77, 1 << 20, (1 << 30) - 1, 1 << 30})
    for (int groups : {1, 5, 1024})
      for (int cols = 1; cols <= 1 << 21 && (ll)rows * cols < 1ll << 40; cols = 2 * cols + 7)
        for (int tile : {64, 128, 256}) {
          take(oz2_tile_blocks(Oz2Groups{nullptr, 1, rows}, tile, (cols + tile - 1) / tile));
          take(oz2_tile_blocks(Oz2Groups{off, groups, rows}, tile, (cols + tile - 1) / tile));
        }
  std::printf("%d %s", bad, beyond ? "some beyond" : "none beyond");
}
""")
    assert out == "0 some beyond"
