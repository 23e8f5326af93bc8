"""Grids of paged attention: no more blocks than there can be, and every one of them; no launch beyond what a device takes."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "ccd_attend_grid.h"
extern "C" long long blocks(long long B, long long T, long long G, long long rows, long long few) { return ccd::most_blocks(B, T, G, rows, few); }
extern "C" long long parts(long long workgroups, long long others) { return ccd::most_parts(workgroups, others); }
"""


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    d = tmp_path_factory.mktemp("grid")
    (d / "t.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2410_01518_amd", "csrc"), str(d / "t.cpp"),
                    "-o", str(d / "t.so")], check=True)
    lib = ctypes.CDLL(str(d / "t.so"))
    for f, n in ((lib.blocks, 5), (lib.parts, 2)):
        f.argtypes, f.restype = [ctypes.c_longlong] * n, ctypes.c_longlong
    return lib


@pytest.mark.parametrize("rows", [32, 128])
@pytest.mark.parametrize("few", [0, 16, 32])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16, 32, 40])
def test_every_block_that_there_can_be_is_counted(grid, rows, few, G):
    if few and G > few:
        pytest.skip("heads of one token are more than the other kernels take")
    rng = random.Random(rows * few + G)
    least = few // G + 1                                  # new tokens of a sequence that is listed
    for _ in range(300):
        B = rng.choice((1, 2, 7, 64, 512))
        news = [rng.choice((0, 1, least - 1, least, least, rows // G + 1, rng.randrange(400))) for _ in range(B)]
        T = sum(news)
        filled = sum(-(-m * G // rows) for m in news if m * G > few)
        got = grid.blocks(B, T, G, rows, few)
        assert max(1, filled) <= got <= max(1, T * G // rows + min(B, T // least) + 1)


def test_no_launch_has_more_threads_than_a_device_takes(grid):
    """The descriptors that are accepted have tokens * Hq <= 2^28 and B * Hkv <= 2^21."""
    for rows, few in ((128, 16), (128, 32), (32, 16), (32, 0), (128, 0)):
        for Hkv in (1, 3, 8, 128):
            for G in (1, 4, 16, 32):
                for B in (1, 64, 4096, (1 << 21) // Hkv):
                    for T in (1, 64, 256, (1 << 20) // (Hkv * G), (1 << 28) // (Hkv * G)):
                        listed = grid.blocks(B, T, G, rows, min(few, 32 if G <= 32 else 0))
                        for row_blocks in (1, 8, 4096):
                            workgroups = Hkv * min(listed, B * row_blocks)
                            assert workgroups + 1024 < 1 << 24
                            parts = grid.parts(workgroups, 1024)
                            assert parts >= 1 and (workgroups * parts + 1024) * 256 < 1 << 32


def test_sequences_without_rows_have_no_blocks(grid):
    # 512 slots of 4 heads a group, 64 new tokens: 64 single ones, or one chunk; 575 tokens are one chunk of 64 among 511
    assert grid.blocks(512, 64, 4, 128, 16) <= 14
    assert grid.blocks(512, 575, 4, 128, 16) <= 132
    # a quarter of a million slots and 256 tokens
    assert grid.blocks(1 << 18, 256, 4, 128, 16) <= 64
