"""How products in MXFP4 are computed, by their sizes: the rule as the library is built with it, run on the host.  Every way that it can
name is one that tests/test_gpu_mxfp4_ways.py runs."""
import itertools
import os
import subprocess

import pytest

from paper_2106_10796_amd import build
from test_gpu_mxfp4_ways import WAYS

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    """shapes -> for each of them (ring rows, ring waves, tile, splits, the second launch's tile, it has rows, it has columns); with
    lanes=True the lanes of the largest launch"""
    exe = str(tmp_path_factory.mktemp("choice") / "product_choice")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(build.PKG, "csrc"),
                    os.path.join(HERE, "native", "product_choice.cpp"), "-o", exe], check=True)

    def of(shapes, lanes=False):
        text = "".join("%d %d %d\n" % s for s in shapes)
        out = subprocess.run([exe], input=text, check=True, stdout=subprocess.PIPE, text=True).stdout.split("\n")[:-1]
        assert len(out) == len(shapes)
        rows = [tuple(map(int, line.split())) for line in out]
        return [r[-1] if lanes else r[:-1] for r in rows]
    return of


def test_every_way_is_run(ways):
    sizes = sorted({n + d for n in (16, 32, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384, 65536) for d in (-1, 0, 1)} |
                   {1, 5, 100, 300, 400, 600, 1536, 2304, 2560, 3000, 4352, 5120, 6000, 25088, 36000, 66000, 76800, 1 << 20, 1 << 29})
    sums = (1, 128, 129, 513, 769, 1025, 1793, 2048, 4096, 8191, 8192, 8193, 16383, 16384, 16385, 1 << 24)
    there = set(ways(list(itertools.product(sizes, sizes, sums))))
    run = dict(zip(WAYS, ways(WAYS)))
    assert len(there) >= 14
    assert there == set(run.values()), "not run: %s, run but not there: %s" % (there - set(run.values()), set(run.values()) - there)


def test_every_product_that_fits_the_card_can_be_launched(ways):
    """A launch holds fewer than 2^32 lanes; a result of two bytes an element, 288 GB."""
    sizes = sorted({1, 5, 16, 17, 32, 33, 64, 65, 128, 129, 257, 300, 1000, 4100} | {(1 << k) + d for k in range(12, 30) for d in (-1, 0, 1)} - {(1 << 29) + 1})
    shapes = [(M, N, K) for M in sizes for N in sizes if M * N <= 144e9 for K in (1, 1000, 2000, 20000)]
    many = [(s, n) for s, n in zip(shapes, ways(shapes, lanes=True)) if n >= 1 << 32]
    assert not many, "%d, of them %s" % (len(many), many[:3])
