"""The items of the LoRA factor kernel, compiled for the host: whatever the grid, every slice, token tile and kind occurs exactly once, and a
block's items alternate between the two kinds."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_01703_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include <tuple>
#include "lora_items.h"
int main(int argc, char** argv)
{
    const long tiles = atol(argv[1]), slices = atol(argv[2]), grid = atol(argv[3]), items = 2 * tiles * slices;
    std::set<std::tuple<int, long, bool>> seen;
    long same = 0;
    for (long i = 0; i < items; ++i) {
        const qless::FactorItem f = qless::factor_item(i, tiles, grid);
        if (f.slice < 0 || f.slice >= slices || f.tile < 0 || f.tile >= tiles) { printf("out of range at %ld\n", i); return 1; }
        if (!seen.insert({f.slice, f.tile, f.is_x}).second) { printf("item %ld occurs a second time\n", i); return 1; }
        if (i + grid < items && qless::factor_item(i + grid, tiles, grid).is_x == f.is_x) ++same;
    }
    if ((long)seen.size() != items || same != 0) { printf("%ld of %ld items, %ld steps of one kind\n", (long)seen.size(), items, same); return 1; }
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("items")
    (d / "items.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(d / "items.cpp"), "-o", str(d / "items")], check=True)
    return str(d / "items")


@pytest.mark.parametrize("grid", [1, 2, 3, 74, 131, 132, 147, 148, 149])
@pytest.mark.parametrize("tiles,slices", [(1, 1), (1, 8), (2, 3), (74, 1), (75, 1), (128, 1), (149, 2), (512, 1), (37, 6)])
def test_every_item_once_at_every_grid(program, tiles, slices, grid):
    done = subprocess.run([program, str(tiles), str(slices), str(min(grid, 2 * tiles * slices))], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
