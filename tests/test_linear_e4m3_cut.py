"""Which kernel and which tiles the 8-bit linear layer takes is plain C++: compiled for the host, it must cut every product within the
kernels' limits, and give the GPU tests of a kernel the kernel that they are written for."""
import os
import shutil
import subprocess

import pytest

import test_gpu_linear_e4m3_pairs as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAIRS = 74                                                   # of a B200: 148 SMs

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host C++ compiler")


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "cut_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2604_17397_b200", "csrc"),
                    os.path.join(ROOT, "tests", "linear_e4m3_cut_check.cpp"), "-o", exe], check=True)

    def ask(products):
        lines = "".join("%d %d %d %d %d\n" % p for p in products)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout
        got = [tuple(map(int, line.split())) for line in out.splitlines()]
        assert len(got) == len(products)
        return got
    return ask


def test_the_pairs_tests_reach_their_tiles(cuts):
    want = [(size, tile // 256, f32) for table in (P.SIZES, P.ODD) for tile, size in table.items() for f32 in (0, 1)]
    want += [(size, tile // 256, f32) for tile, sizes in P.SHORT.items() for size in sizes for f32 in (0, 1)]
    want += [(P.BLOCK, 2, 0)]
    # the layer of the drafter, and what runs between operators of other kinds
    want += [(size, 2, 0) for size in ((4680, 4608, 1536), (4680, 1536, 1536), (4680, 6144, 1536), (4680, 1536, 6144), (777, 9999, 3008))]
    want += [((777, 3008, 1200), 1, 0), ((777, 1200, 3008), 0, 0)]
    got = cuts([(*size, PAIRS, f32) for size, _, f32 in want])
    for (size, subs, f32), (s, *_rest) in zip(want, got):
        assert s == subs, (size, f32)
    for size, (subs, _, _, whole) in zip(P.LONG, cuts([(*s, PAIRS, 1) for s in P.LONG])):
        assert subs == 1 and not whole, size


def test_every_cut_is_within_the_kernels_limits(cuts):
    products = [(r, c, k, pairs, f32) for pairs in (74, 66, 8, 1) for f32 in (0, 1) for r in (1, 2, 15, 16, 17, 33, 64, 65, 128, 333, 777, 4680, 100001)
                for c in (1, 127, 128, 129, 777, 5120, 30720, 2 ** 27) for k in (1, 128, 129, 1111, 5120, 6144, 6145, 20480, 2 ** 20)]
    for (r, c, k, pairs, f32), (subs, tile_t, split, whole) in zip(products, cuts(products)):
        at = (r, c, k, pairs, f32)
        iters = -(-k // 128)
        assert tile_t % 16 == 0 and split in (1, 2, 4, 8) and split <= iters, at
        assert whole or f32, at
        if subs:
            assert r > 64 and 64 <= tile_t <= 240 and split == 1 and (whole or subs == 1), at
        else:
            assert 16 <= tile_t <= 64 and tile_t < r + 16, at
            assert split == 1 or -(-c // 128) * -(-r // tile_t) * split <= 4 * pairs, at
