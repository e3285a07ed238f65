"""Page tables of as many columns as a call may have."""
import pytest
import torch

from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_fork_into_the_widest_table():
    """Two new sequences in pages of one token: the second one wants more columns than are left of 2^31 behind the first one's pages.  It gets the pages that are free,
    and every other entry is -1."""
    cols, pages, first = 2 ** 31 - 2048, 6000, 5000
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    refs, table = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.empty((0, cols), dtype=torch.int32, device=DEV)
    refs_out, out, length, copies, missing = B.lr_kv_fork(refs, 1, table, refs[:0], i32([-1, -1]), i32([first, 2 ** 31 - 1]))
    order = torch.arange(pages, dtype=torch.int32, device=DEV)
    assert torch.equal(out[0, :first], order[:first]) and torch.equal(out[1, :pages - first], order[first:])
    for row, held in ((out[0], first), (out[1], pages - first)):
        assert all(bool((part == -1).all()) for part in row[held:].split(2 ** 28))
    assert bool((refs_out == 1).all()) and length.tolist() == [first, 2 ** 31 - 1] and missing.tolist() == [2 ** 31 - 1 - (pages - first)]
    assert all(t.tolist() == v for t, v in zip(copies, ([-1, -1], [-1, -1], [0, 0])))
