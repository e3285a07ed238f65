"""Products of 8-bit integers on every kind of tile, against exact sums."""
import pytest
import torch

from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def ints(g, rows, K, room=0):
    """[rows, K] in rows of whole 16 bytes that hold something behind K too."""
    return torch.randint(-127, 128, (rows, -(-K // 16) * 16 + room), generator=g, device=DEV, dtype=torch.int8)[:, :K]


def scales(g, rows):
    return torch.rand((rows,), generator=g, device=DEV) * 0.1 + 1e-3


def test_more_rows_than_a_launch_has_tiles_of_64_for():
    """2^30 rows, 2^24 tiles of 64: 1024 times the same rows, so the result is 1024 times theirs, bit for bit."""
    g = torch.Generator(device=DEV).manual_seed(1)
    rows, times = 1 << 20, 1 << 10
    assert B.lr_matmul_q8_tile(rows * times, 8, 16) == (256, 256) != B.lr_matmul_q8_tile(rows, 8, 16)
    a, sa, b, sb = ints(g, rows, 16), scales(g, rows), ints(g, 8, 16), scales(g, 8)
    few = B.lr_matmul_q8(a, sa, b, sb)
    many = B.lr_matmul_q8(a.repeat(times, 1), sa.repeat(times), b, sb)
    assert many.shape == (rows * times, 8)
    for part in many.view(times, rows, 8).split(64):
        assert torch.equal(part, few[None].expand_as(part))
