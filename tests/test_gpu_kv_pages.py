"""Forked, compacted and copied pages against the oracle: every entry and every element is equal."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def flat(r):
    return [t.cpu().numpy() for t in (*r[:3], *r[3], r[4])] if len(r[3]) == 3 else [t.cpu().numpy() for t in (*r[:2], *r[2], *r[3:])]


def pool(rng, n_in, page, most, cols, pages, shared=0.3, reserve=0):
    """Tables of sequences with lengths below `most`, some of whose full pages are those of the sequence before."""
    length = rng.integers(0, most + 1, n_in)
    table = np.full((n_in, cols), -1, dtype=np.int32)
    order = iter(rng.permutation(pages))
    for b in range(n_in):
        need = min(-(-length[b] // page) + reserve, cols)
        both = min(length[b], length[b - 1]) // page if b and rng.random() < shared else 0
        table[b, :both] = table[b - 1, :both]
        table[b, both:need] = [next(order) for _ in range(need - both)]
    return length, table, np.bincount(table[table >= 0], minlength=pages)


def check_fork(refs, page, table, length, parent, grow, **kw):
    got = B.lr_kv_fork(dev(refs), page, dev(table), dev(length), dev(parent), dev(grow), **kw)
    for name, g, w in zip(("refs", "table", "length", "src", "dst", "rows", "missing"), flat(got), so.kv_fork(refs, page, table, length, parent, grow)):
        assert np.array_equal(g, np.atleast_1d(w)), name
    return got


@pytest.mark.parametrize("n_in,n_out,page,most,grow,pages,reserve", [
    (1, 1, 16, 1, 1, 8, 0), (4, 16, 16, 100, 1, 400, 0), (16, 16, 8, 300, 1, 2000, 1), (5, 0, 16, 90, 1, 300, 0), (0, 7, 24, 0, 77, 100, 0),
    (48, 48, 24, 1500, 3, 4000, 2), (64, 700, 16, 200, 1, 3000, 0), (700, 64, 16, 60, 40, 5000, 0), (2000, 2000, 32, 90, 20, 12000, 1), (3, 9, 1, 40, 5, 300, 0),
    (8, 8, 16, 2000, 3000, 30000, 0), (6, 6, 1000, 9000, 1, 100, 0)])
def test_fork(n_in, n_out, page, most, grow, pages, reserve):
    rng = np.random.default_rng(n_in + n_out)
    cols = -(-(most + grow) // page) + 2
    length, table, refs = pool(rng, n_in, page, most, cols, pages, reserve=reserve)
    refs[rng.integers(0, pages, 5)] += 1                                # pages that somebody else holds too, half filled ones perhaps
    parent = rng.integers(-1, n_in, n_out) if n_in else np.full(n_out, -1)
    check_fork(refs, page, table, length, parent, rng.integers(0, grow + 1, n_out))


def test_fork_of_beams_step_by_step():
    """Beams of a few prompts over 60 steps: the pool never loses a page, and gets them all back."""
    rng = np.random.default_rng(5)
    page, G, W, pages, cols = 8, 3, 4, 300, 20
    state = [dev(np.zeros(pages)), dev(np.full((1, cols), -1)), dev([0])]
    parent, grow = np.full(G * W, -1), np.repeat(rng.integers(5, 30, G), W)
    for step in range(60):
        refs, table, length = (t.cpu().numpy() for t in state)
        state = list(check_fork(refs, page, table, length, parent, grow)[:3])
        held = state[1].cpu().numpy()
        assert np.array_equal(state[0].cpu().numpy(), np.bincount(held[held >= 0], minlength=pages)), step
        parent, grow = np.concatenate([g * W + rng.integers(0, W, W) for g in range(G)]), np.full(G * W, rng.integers(0, 3))
    state = list(check_fork(*(t.cpu().numpy() for t in state[:1]), page, *(t.cpu().numpy() for t in state[1:]), np.zeros(0), np.zeros(0))[:3])
    assert not state[0].any()


def test_fork_with_too_few_pages_and_columns():
    rng = np.random.default_rng(6)
    length, table, refs = pool(rng, 6, 16, 100, 9, 60)
    parent, grow = rng.integers(0, 6, 20), rng.integers(0, 60, 20)
    for left in (0, 1, 7):
        some = refs.copy()
        some[np.flatnonzero(some == 0)[left:]] = 3
        out = check_fork(some, 16, table, length, parent, grow)
        assert int(out[4]) > 0
    assert int(check_fork(refs, 16, table, length, parent, grow * 1000)[4]) > 1000
    check_fork(refs, 16, table, length, parent, np.full(20, 2 ** 31 - 5))


def test_fork_of_lists_that_say_anything():
    """Entries that are no pages, lengths and room below zero or past the table, parents that are not there."""
    rng = np.random.default_rng(7)
    for seed in range(8):
        pages, cols = 50, 6
        refs = rng.integers(-1, 3, pages)
        table = rng.permutation(np.arange(-10, 70))[:24].reshape(4, cols).astype(np.int32)
        refs[table[(table >= 0) & (table < pages)]] = rng.integers(1, 3)
        length = np.array([-5, 95, 96 + seed, 2 ** 31 - 1 if seed % 2 else 40])
        check_fork(refs, 16, table, length, np.array([3, 0, 4, -7, 2, 1, 1, 2 ** 31 - 1]), np.array([1, -3, 20, 33, 0, 5, 5, 17]))


def test_fork_writes_rows_of_wider_tables_and_reuses_results():
    rng = np.random.default_rng(8)
    length, table, refs = pool(rng, 5, 16, 100, 8, 80)
    parent, grow = dev(rng.integers(0, 5, 7)), dev(np.ones(7))
    wide_in, wide_out = torch.full((5, 20), 3, dtype=torch.int32, device=DEV), torch.full((7, 11), 55, dtype=torch.int32, device=DEV)
    wide_in[:, 4:12] = dev(table)
    want = B.lr_kv_fork(dev(refs), 16, dev(table), dev(length), parent, grow)
    out = B.lr_kv_fork(dev(refs), 16, wide_in[:, 4:12], dev(length), parent, grow)
    out = (out[0].fill_(9), wide_out[:, 2:10], out[2].fill_(9), tuple(t.fill_(9) for t in out[3]), out[4].fill_(9))
    nb = B.lr_kv_fork_workspace_bytes(80, 5, 7)
    ws = torch.full((nb + 256,), 99, dtype=torch.uint8, device=DEV)
    got = B.lr_kv_fork(dev(refs), 16, wide_in[:, 4:12], dev(length), parent, grow, out=out, ws=ws[:nb])
    assert got[1].data_ptr() == wide_out[:, 2:10].data_ptr()
    assert all(np.array_equal(a, b) for a, b in zip(flat(got), flat(want)))
    assert bool((wide_out[:, :2] == 55).all()) and bool((wide_out[:, 10:] == 55).all()) and bool((ws[nb:] == 99).all())
    with pytest.raises(B.LrError):
        B.lr_kv_fork(out[0], 16, out[1], out[2], dev(np.zeros(7)), grow, out=out)          # over its own inputs


@pytest.mark.parametrize("pages,live,batch,cols", [(1, 1.0, 1, 1), (1, 0.0, 0, 1), (2, 0.5, 1, 2), (7, 0.5, 2, 3), (1000, 0.5, 8, 70), (2048, 1.0, 3, 10), (4096, 0.5, 4, 2000),
                                                   (4097, 0.02, 2, 50), (5000, 0.98, 2, 5000), (16383, 0.6, 3, 900), (16384, 1.0, 2, 40), (16384, 0.4, 2, 2000), (16385, 0.5, 5, 700),
                                                   (70001, 0.3, 64, 333)])
def test_compact(pages, live, batch, cols):
    rng = np.random.default_rng(pages)
    refs = (rng.random(pages) < live) * rng.integers(1, 4, pages)
    refs[rng.integers(0, pages, 2)] *= -1
    table = rng.integers(-2, pages + 2, (batch, cols))
    want = so.kv_compact(refs, table)
    for name, g, w in zip(("refs", "table", "src", "dst", "page_map", "n_live"), flat(B.lr_kv_compact(dev(refs), dev(table))), want):
        assert np.array_equal(g, np.atleast_1d(w)), name


def test_compact_in_given_memory():
    rng = np.random.default_rng(9)
    refs, table = dev(rng.integers(0, 2, 3000)), dev(rng.integers(-1, 3000, (4, 9)))
    want = B.lr_kv_compact(refs, table)
    out = tuple(t.clone().fill_(5) for t in want[:2]) + (tuple(t.clone().fill_(5) for t in want[2]),) + tuple(t.clone().fill_(5) for t in want[3:])
    nb = B.lr_kv_compact_workspace_bytes(3000)
    ws = torch.full((nb + 256,), 99, dtype=torch.uint8, device=DEV)
    got = B.lr_kv_compact(refs, table, out=out, ws=ws[:nb])
    assert all(np.array_equal(a, b) for a, b in zip(flat(got), flat(want))) and bool((ws[nb:] == 99).all())


@pytest.mark.parametrize("layout", ["token", "head", "wide"])
@pytest.mark.parametrize("page,Hkv,hd", [(8, 1, 8), (16, 8, 128), (24, 3, 64), (128, 2, 128), (16, 5, 192)])
def test_copy(layout, page, Hkv, hd):
    g = torch.Generator(device=DEV).manual_seed(page)
    shape = {"token": (21, page, Hkv, hd), "head": (21, Hkv, page, hd), "wide": (21, 2, page, Hkv, hd + 24)}[layout]
    if layout == "wide":
        both = torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)
        k, v = both[:, 0, ..., :hd], both[:, 1, ..., :hd]
    else:
        k, v = (torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        if layout == "head":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
    order = np.random.default_rng(page).permutation(21)
    src, dst = np.concatenate([order[:6], [-1, order[6], 21, order[0], 99]]), np.concatenate([order[7:13], [order[13], -1, order[14], order[15], order[16]]])
    rows = np.array([page, 1, page // 2, 0, page + 9, -3, page, page, page, page - 1, page])
    for which in (rows, None):
        want = [t.clone() for t in (k, v)]
        for s, d, n in zip(src, dst, rows if which is not None else [page] * len(src)):
            if 0 <= s < 21 and d >= 0:
                for w, t in zip(want, (k, v)):
                    w[d, :max(0, n)] = t[s, :max(0, n)]
        B.lr_kv_copy(k, v, dev(src), dev(dst), None if which is None else dev(which))
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    if layout == "wide":
        assert bool((both[..., hd:] == torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(page), device=DEV).to(torch.bfloat16)[..., hd:]).all())


def test_captured_steps_take_what_the_lists_hold():
    """Fork and copy, compact and copy in two graphs on one workspace, replayed on other lists, each against the eager calls."""
    rng = np.random.default_rng(10)
    page, pages, cols = 16, 400, 12
    cache = torch.randn((2, pages, page, 2, 64), device=DEV).to(torch.bfloat16)
    state = pool(rng, 9, page, 100, cols, pages)
    length, table, refs = (dev(t) for t in state)
    parent, grow = dev(rng.integers(0, 9, 12)), dev(np.ones(12))
    nb = max(B.lr_kv_fork_workspace_bytes(pages, 9, 12), B.lr_kv_compact_workspace_bytes(pages))
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    out_f, out_c = B.lr_kv_fork(refs, page, table, length, parent, grow, ws=ws), B.lr_kv_compact(refs, table, ws=ws)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        B.lr_kv_fork(refs, page, table, length, parent, grow, out=out_f, ws=ws)
        B.lr_kv_copy(cache[0], cache[1], *out_f[3])
    with torch.cuda.graph(g2):
        B.lr_kv_compact(refs, table, out=out_c, ws=ws)
        B.lr_kv_copy(cache[0], cache[1], *out_c[2])
    for turn in range(3):
        for t, w in zip((length, table, refs), pool(rng, 9, page, 100, cols, pages)):
            t.copy_(dev(w))
        parent.copy_(dev(rng.integers(-1, 9, 12)))
        for graph, out, eager in ((g1, out_f, lambda: B.lr_kv_fork(refs, page, table, length, parent, grow)), (g2, out_c, lambda: B.lr_kv_compact(refs, table))):
            before = cache.clone()
            graph.replay()
            want = eager()
            moved = want[3] if len(want[3]) == 3 else (*want[2], None)
            B.lr_kv_copy(before[0], before[1], *moved)
            torch.cuda.synchronize()
            assert all(np.array_equal(a, b) for a, b in zip(flat(out), flat(want))) and torch.equal(cache, before), turn


def test_copies_past_32_bits():
    """A cache of more than 2^31 elements: pages at its two ends."""
    pages = 2 ** 17 + 64
    k, v = (torch.zeros((pages, 16, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[5], v[5], k[-1], v[-1] = 1, 2, 3, 4
    B.lr_kv_copy(k, v, dev([5, pages - 1, pages]), dev([pages - 2, 6, 7]))
    assert bool((k[-2] == 1).all()) and bool((v[-2] == 2).all()) and bool((k[6] == 3).all()) and bool((v[6] == 4).all())
    assert not k[7].any() and not k[-3].any() and not v[-3].any() and not k[4].any()
