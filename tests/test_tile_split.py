"""How many CTAs share a tile of a product, for devices described by what they hold (host: the
rule is compiled by itself)."""
import os
import subprocess

import pytest

from paper_2608_13966_gb300 import build

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include "linear_plan.h"

// arguments: tiles, k blocks, SMs, then the clusters of 1, 2, ... 8 CTAs that the device holds
// (-1: the question itself fails)
int main(int argc, char** argv)
{
    if (argc != 12) return 2;
    auto held = [&](int size, int* n) {
        const int x = std::atoi(argv[3 + size]);
        if (x < 0) return QUASAR_ERR_CUDA;
        if (x == 0) return QUASAR_ERR_UNSUPPORTED;
        *n = x;
        return QUASAR_OK;
    };
    int split = -1;
    const quasar_status st = quasar::tile_split(std::atoll(argv[1]), std::atoi(argv[2]), std::atoi(argv[3]), held, &split);
    std::printf("%d %d\n", (int)st, split);
    return 0;
}
"""

# clusters of 1 to 8 CTAs: a whole device, and ones that hold none above 4, 2 or 1
WHOLE = (152, 76, 46, 36, 28, 23, 15, 15)
FOUR = (152, 76, 46, 36, 0, 0, 0, 0)
TWO = (20, 8, 0, 0, 0, 0, 0, 0)
ONE = (20, 0, 0, 0, 0, 0, 0, 0)
OK, ERR_CUDA = 0, 3


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    where = tmp_path_factory.mktemp("split")
    (where / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-I" + build.INCLUDE, "-I" + build.CSRC, str(where / "main.cpp"),
                    "-o", str(where / "rule")], check=True)

    def ask(tiles, k_blocks, n_sm, held):
        out = subprocess.run([str(where / "rule"), *map(str, (tiles, k_blocks, n_sm, *held))],
                             check=True, capture_output=True, text=True).stdout
        return tuple(map(int, out.split()))
    return ask


@pytest.mark.parametrize("tiles,k_blocks,held,split", [
    (1, 64, WHOLE, 8), (32, 224, WHOLE, 8), (64, 64, WHOLE, 4), (80, 196, WHOLE, 3), (40, 196, WHOLE, 6),
    (200, 64, WHOLE, 1), (1, 1, WHOLE, 1), (1, 3, WHOLE, 1), (1, 4, WHOLE, 2), (1, 9, WHOLE, 3)])
def test_a_whole_device(rule, tiles, k_blocks, held, split):
    assert rule(tiles, k_blocks, 152, held) == (OK, split)


@pytest.mark.parametrize("tiles,k_blocks,n_sm,held,split", [
    (1, 64, 152, FOUR, 4), (60, 64, 152, FOUR, 4), (1, 64, 20, TWO, 2), (1, 64, 20, ONE, 1), (9, 64, 20, TWO, 2)])
def test_a_device_that_holds_no_large_cluster(rule, tiles, k_blocks, n_sm, held, split):
    """A smaller size that it holds, not a refusal."""
    assert rule(tiles, k_blocks, n_sm, held) == (OK, split)


def test_a_question_that_fails(rule):
    assert rule(1, 64, 152, (152, -1, -1, -1, -1, -1, -1, -1))[0] == ERR_CUDA
