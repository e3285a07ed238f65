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


def check(tile, M, N, K, dtype):
    """Rows inside wider ones on either side; the sum is exact, then it is made a float (2^-24) and multiplied twice (2^-24 each) and rounded to dtype."""
    assert B.lr_matmul_q8_tile(M, N, K) == tile
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    a, b, sa, sb = ints(g, M, K, 16), ints(g, N, K, 32), scales(g, M), scales(g, N)
    wide = -(-N // 8) * 8 + 16
    room = torch.full((M + 1, wide), 7.0, dtype=dtype, device=DEV)
    out = room[:M, 8:8 + N]
    B.lr_matmul_q8(a, sa, b, sb, out=out)
    want = (a.double() @ b.double().t().contiguous()) * sa.double()[:, None] * sb.double()[None, :]
    half = torch.finfo(dtype).eps / 2
    tol = want.abs() * (half * (1 + 2.0 ** -7) + (3 * 2.0 ** -24 if dtype == BF else 2 * 2.0 ** -24))
    off = (out.double() - want).abs() - tol
    assert bool((off <= 0).all()), float(off.max())
    out.fill_(7.0)
    assert bool((room == 7.0).all())


# one slice of k and none more, two, three, odd and even numbers of them; what lies behind K in the first, a middle and the last chunk of a slice
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N", [4109, 4112])
@pytest.mark.parametrize("K", [16, 100, 128, 130, 256, 383, 391, 640, 1000, 2047])
def test_stream_of_tiles(K, N, dtype):
    """289 tiles on 256 workgroups: loads run ahead into the next tile, whose rows and columns end inside it."""
    check((256, 256), 4111, N, K, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", [(4096, 4096, 128), (4000, 4090, 77), (4096, 4096, 300), (3900, 4001, 1030), (700, 33001, 270), (16700, 1031, 144), (8200, 8193, 205),
                                   (8200, 8200, 1024)])
def test_stream_of_tiles_of_other_numbers(M, N, K, dtype):
    """A tile for each workgroup at most, and several; a row of tiles longer than another."""
    check((256, 256), M, N, K, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tile,M,N,K", [((128, 128), 2048, 2048, 2048), ((128, 128), 1900, 2041, 1001), ((128, 128), 2047, 2048, 777), ((128, 128), 128, 32003, 4100),
                                        ((128, 128), 127, 32008, 4096), ((128, 128), 100, 32001, 4111), ((64, 128), 777, 2047, 546), ((64, 128), 64, 33003, 515),
                                        ((64, 128), 40, 33000, 528), ((64, 64), 300, 1001, 1003), ((64, 64), 300, 1000, 1024), ((64, 64), 60, 8201, 2050),
                                        ((16, 16), 65, 129, 1000), ((16, 16), 3, 8190, 4097)])
def test_tiles_of_a_ring(tile, M, N, K, dtype):
    """A row of tiles over a weight of 16 MB and more among them, which starts k elsewhere in every tile."""
    check(tile, M, N, K, dtype)


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
