"""Which kernel the loss by W phi takes for up to 64 positions of 16 bits (host arithmetic, no GPU): rules whose other side was measured to be slower."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_09992_amd", "csrc")

MAIN = r"""
#include <stdio.h>
#include <stdlib.h>
#include "default_cross_entropy.hpp"
using namespace pqk::head;
int main(int argc, char** argv) {
    for (int i = 1; i + 1 < argc; i += 2) {
        const int d = atoi(argv[i + 1]);
        const long long tiles = ceil_div(atoll(argv[i]), few_items(d));
        printf("%d", (int)few_tiles_are_many(tiles, tiles < kCUs ? (int)tiles : kCUs, d));
    }
}
"""


@pytest.mark.skipif(not shutil.which("hipcc"), reason="needs hipcc")
def test_few_tiles_a_workgroup_take_the_kernel_with_the_short_start(tmp_path):
    # us by the long pipeline and by two tiles at a time, 64 positions: 300 items of 128 7.4 and 6.7, 10,000 of 256 8.9 and 8.0, 10,000 of 64 7.9 and 7.3, 300,000 of 128 20.8 and 20.4;
    # 20,000 of 512 11.2 and 11.4, 300,000 of 512 55.7 and 61.6, 1.27M of 64 39.0 and 40.4
    short = [(1, 8), (300, 64), (300, 128), (10_000, 64), (10_000, 128), (10_000, 256), (10_000, 512), (16_384, 512), (100_000, 256), (300_000, 64), (300_000, 128), (300_000, 256), (600_000, 64)]
    long = [(17_000, 384), (20_000, 512), (300_000, 512), (1_271_638, 512), (600_000, 256), (1_271_638, 64), (1_271_638, 128), (10_000_000, 64)]
    (tmp_path / "main.hip").write_text(MAIN)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(tmp_path / "main.hip"), "-o",
                    str(tmp_path / "main")], check=True, capture_output=True)
    numbers = [str(x) for case in short + long for x in case]
    out = subprocess.run([str(tmp_path / "main"), *numbers], check=True, capture_output=True, text=True).stdout
    assert out == "0" * len(short) + "1" * len(long)
