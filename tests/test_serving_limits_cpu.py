"""Tiles of products of 8-bit integers by their sizes, and sizes that a launch could not have."""
import ctypes as C

import pytest

from paper_2512_12131_amd import binding as B

THREADS = {(128, 128): 512, (64, 128): 256, (64, 64): 256, (16, 16): 1024}      # of a workgroup per tile; those of 256 x 256 run on 256 workgroups


def test_tiles_by_size():
    assert B.lr_matmul_q8_tile(16, 1024, 4096) == (16, 16)            # a handful of rows
    assert B.lr_matmul_q8_tile(64, 32000, 4096) == (64, 128)          # a vocabulary
    assert B.lr_matmul_q8_tile(2048, 2048, 2048) == (128, 128)
    assert B.lr_matmul_q8_tile(16384, 11008, 4096) == (256, 256)      # the chip full, k long


@pytest.mark.parametrize("N", [1, 8, 100, 129, 512])
def test_a_launch_has_less_than_two_to_the_32_threads(N):
    seen = set()
    for K in (1, 16, 1000, 131071):
        for M in [1 << b for b in range(20, 31)] + [(1 << 30) - 1, (1 << 30) + 1, (1 << 31) - 256]:
            rows, cols = tile = B.lr_matmul_q8_tile(M, N, K)
            seen.add(tile)
            assert -(-M // rows) * -(-N // cols) * THREADS.get(tile, 0) < 1 << 32, (M, K)
    assert (256, 256) in seen and (N > 100 or (64, 128) in seen)


def test_tile_query_refuses():
    for sizes in ((0, 8, 8), (-1, 8, 8), (8, 0, 8), (8, 8, 0), (1 << 31, 8, 8), (8, 8, 131072), (1 << 30, 1 << 20, 8)):
        with pytest.raises(B.LrError):
            B.lr_matmul_q8_tile(*sizes)
    one = C.c_int(0)
    assert B.lib().lr_matmul_q8_tile(8, 8, 8, None, C.byref(one)) == -1
