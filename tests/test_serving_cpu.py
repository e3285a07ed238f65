"""Beams, pages and 8-bit products on the host: pins of their oracle, and refusals before anything reaches a device."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

EINVAL, EUNSUPPORTED, EWORKSPACE, EALIGN = -1, -2, -3, -4
F32, BF16 = 0, 1


# ---- the oracle -------------------------------------------------------------------------------------
def test_rows_are_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, 33)) * 10.0 ** rng.uniform(-30, 30, (9, 1))
    x[3] = 0
    q, s = so.quant_rows(x)
    assert np.all(np.abs(q) <= 127) and np.all(np.abs(q * s[:, None] - x) <= s[:, None] * (0.5 + 1e-12))
    assert np.all(np.abs(q).max(1)[[0, 1, 2, 4]] == 127) and not q[3].any()
    x[5, 7] = np.inf
    assert np.isnan(so.quant_rows(x)[1][5]) and not so.quant_rows(x)[0][5].any()


def test_select_is_the_sorted_list_of_all_candidates():
    rng = np.random.default_rng(2)
    logits, score = rng.integers(-3, 4, (6, 11)).astype(float), np.array([[-1.0, -1.0, -2.5], [-0.5, -np.inf, -0.25]])
    parent, token, best = so.beam_select(logits, score, 7)
    for b in range(2):
        every = sorted((-(score[b, w] + logits[3 * b + w, v] - np.log(np.exp(logits[3 * b + w]).sum())), w, v) for w in range(3) for v in range(11)
                       if np.isfinite(score[b, w]))
        assert np.allclose(best[b], [-e[0] for e in every[:7]], atol=1e-12)
        assert [(p - 3 * b, t) for p, t in zip(parent[b], token[b])] == [(e[1], e[2]) for e in
                                                                          sorted(((round(e[0], 9), *e[1:]) for e in every))[:7]]
    # one candidate left, then none
    parent, _, best = so.beam_select(np.array([[0.0, -np.inf]]), np.zeros((1, 1)), 2)
    assert parent.tolist() == [[0, -1]] and best.tolist() == [[0.0, -np.inf]]


def test_fork_keeps_the_books():
    """Whatever the parents: counts are those of the new table's entries, keys are where they were or are copied there."""
    rng = np.random.default_rng(3)
    for _ in range(30):
        page, n_in, n_out, cols, pages = 8, rng.integers(1, 6), rng.integers(0, 8), 7, 60
        length = rng.integers(0, 40, n_in)
        order = iter(rng.permutation(pages))
        table = np.full((n_in, cols), -1, dtype=np.int32)
        for b in range(n_in):
            table[b, :-(-length[b] // page)] = [next(order) for _ in range(-(-length[b] // page))]
        refs = np.bincount(table[table >= 0], minlength=pages)
        parent, grow = rng.integers(-1, n_in, n_out), rng.integers(0, 12, n_out)
        new, out, now, src, dst, rows, missing = so.kv_fork(refs, page, table, length, parent, grow)
        assert missing == 0 and np.array_equal(new, np.bincount(out[out >= 0], minlength=pages))
        cell = {s * 1000 + r: s * 1000 + r for s in range(pages) for r in range(page)}      # what is where
        for s, d, r in zip(src, dst, rows):
            for k in range(r):
                cell[d * 1000 + k] = s * 1000 + k
        for i in range(n_out):
            assert np.all(out[i, :-(-int(now[i]) // page)] >= 0)
            for k in range(length[parent[i]] if parent[i] >= 0 else 0):
                assert cell[out[i, k // page] * 1000 + k % page] == table[parent[i], k // page] * 1000 + k % page
            for j in range(i):                                  # new keys have pages of their own
                a, b = (set(out[x, (length[parent[x]] if parent[x] >= 0 else 0) // page:-(-int(now[x]) // page)]) for x in (i, j))
                assert grow[i] == 0 or grow[j] == 0 or not a & b


def test_compact_moves_every_held_page_below():
    rng = np.random.default_rng(4)
    for n in (1, 2, 17, 60):
        refs = rng.integers(0, 3, n) * rng.integers(0, 2, n)
        table = rng.integers(-1, n, (3, 5)).astype(np.int32)
        new, out, src, dst, page_map, live = so.kv_compact(refs, table)
        assert live == np.sum(refs > 0) and np.all(new[:live] > 0) and not new[live:].any() and sorted(new) == sorted(refs)
        assert sorted(page_map[refs > 0]) == list(range(live)) and np.all(page_map[refs <= 0] == -1)
        assert np.all(src[src >= 0] >= live) and np.all(dst[dst >= 0] < live) and np.array_equal(page_map[src[src >= 0]], dst[src >= 0])


# ---- refusals: addresses that are never used --------------------------------------------------------
def _quant(x=0x10000, ldx=64, q=0x20000, ldq=64, scale=0x30000, T=4, n=64, dt=BF16):
    return B.lib().lr_quant_rows(x, ldx, q, ldq, scale, T, n, dt, None)


def test_quant_rows_refuses():
    for args in (dict(n=0), dict(T=-1), dict(ldx=56), dict(ldq=48), dict(dt=3), dict(x=None), dict(q=None), dict(scale=None)):
        assert _quant(**args) == EINVAL, args
    for args in (dict(n=60), dict(ldx=68), dict(ldq=72), dict(x=0x10008), dict(q=0x20008), dict(scale=0x30002), dict(dt=F32, x=0x10002)):
        assert _quant(**args) == EALIGN, args
    assert _quant(T=0, x=None, q=None, scale=None) == 0


def _matmul(a=0x10000, lda=64, sa=0x20000, b=0x30000, ldb=64, sb=0x40000, c=0x50000, ldc=32, M=4, N=30, K=60, dt=BF16):
    return B.lib().lr_matmul_q8(a, lda, sa, b, ldb, sb, c, ldc, M, N, K, dt, None)


def test_matmul_q8_refuses():
    for args in (dict(M=-1), dict(N=0), dict(K=0), dict(K=65), dict(ldc=24), dict(dt=2), dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None)):
        assert _matmul(**args) == EINVAL, args
    for args in (dict(lda=72), dict(ldb=72), dict(a=0x10008), dict(b=0x30004), dict(c=0x50008), dict(ldc=36), dict(sa=0x20001)):
        assert _matmul(**args) == EALIGN, args
    for args in (dict(K=133145, lda=133152, ldb=133152), dict(K=131072, lda=131072, ldb=131072), dict(lda=(1 << 22) + 16), dict(M=1 << 30, N=1 << 20, ldc=1 << 20)):
        assert _matmul(**args) == EUNSUPPORTED, args
    assert _matmul(M=0, a=None, c=None) == 0


def _linear(x=0x10000, ldx=64, wd=0x20000, ldd=64, sd=0x30000, wu=0x40000, ldu=32, su=0x50000, y=0x60000, ldy=48, T=4, d=64, r=32, n=48, act=1,
            dt=BF16, ws=0x70000, nb=1 << 20):
    return B.lib().lr_linear_q8_fwd(x, ldx, wd, ldd, sd, wu, ldu, su, y, ldy, T, d, r, n, act, dt, ws, nb, None)


def test_linear_q8_refuses():
    for args in (dict(act=2), dict(T=-1), dict(r=0), dict(n=0), dict(ldx=56), dict(ldd=48), dict(ldu=16), dict(ldy=40), dict(x=None), dict(wd=None),
                 dict(su=None), dict(y=None)):
        assert _linear(**args) == EINVAL, args
    for args in (dict(r=28), dict(n=44), dict(ldd=72), dict(ldu=40), dict(y=0x60008), dict(ldy=52), dict(dt=F32, ldy=50), dict(ws=0x70010)):
        assert _linear(**args) == EALIGN, args
    need = B.lr_linear_q8_workspace_bytes(4, 64, 32)
    assert need > 0 and _linear(nb=need - 1) == EWORKSPACE and _linear(ws=None) == EWORKSPACE
    assert _linear(T=0, x=None, y=None, ws=None) == 0 and B.lr_linear_q8_workspace_bytes(4, 133145, 32) == 0
    sizes = [B.lr_linear_q8_workspace_bytes(t, 4096, 1024) for t in (1, 16, 777, 16384)]
    assert sizes == sorted(sizes)


def _select(logits=0x10000, ldl=100, score=0x20000, done=None, end=0, parent=0x30000, token=0x40000, best=0x50000, batch=2, beams=4, V=100, n=4,
            dt=BF16, ws=0x60000, nb=1 << 20):
    return B.lib().lr_beam_select(logits, ldl, score, done, end, parent, token, best, batch, beams, V, n, dt, ws, nb, None)


def test_beam_select_refuses():
    for args in (dict(batch=-1), dict(beams=0), dict(V=0), dict(n=0), dict(ldl=99), dict(dt=2), dict(logits=None), dict(score=None), dict(parent=None),
                 dict(token=None), dict(best=None), dict(done=0x1000, end=100), dict(done=0x1000, end=-1), dict(parent=0x10000), dict(parent=0x1063c), dict(best=0x20004),
                 dict(best=0x20000, n=3), dict(token=0x30010), dict(done=0x40004)):
        assert _select(**args) == EINVAL, args
    for args in (dict(logits=0x10001), dict(logits=0x10002, dt=F32), dict(done=0x1002), dict(score=0x20002), dict(ws=0x60010)):
        assert _select(**args) == EALIGN, args
    for args in (dict(beams=65), dict(n=65), dict(V=(1 << 20) + 1, ldl=1 << 21), dict(batch=(1 << 18) + 1)):
        assert _select(**args) == EUNSUPPORTED, args
    need = B.lr_beam_select_workspace_bytes(2, 4, 100, 4)
    assert need > 0 and _select(nb=need - 1) == EWORKSPACE and _select(ws=None) == EWORKSPACE and _select(best=0x20000, ws=None) == EWORKSPACE
    assert _select(batch=0, logits=None, ws=None) == 0 and B.lr_beam_select_workspace_bytes(2, 65, 100, 4) == 0


FORK = dict(refs=0x100000, pages=100, page=16, table=0x200000, ld=10, length=0x300000, n_in=4, parent=0x400000, grow=0x500000, refs_out=0x600000,
            table_out=0x700000, ldo=10, len_out=0x800000, n=6, cols=10, src=0x900000, dst=0xa00000, rows=0xb00000, missing=0xc00000, ws=0xd00000, nb=1 << 20)


def _fork(**over):
    a = {**FORK, **over}
    return B.lib().lr_kv_fork(*a.values(), None)


def test_kv_fork_refuses():
    for args in (dict(pages=0), dict(page=0), dict(n_in=-1), dict(n=-1), dict(cols=0), dict(ld=9), dict(ldo=9), dict(refs=None), dict(table=None),
                 dict(length=None), dict(parent=None), dict(grow=None), dict(refs_out=None), dict(table_out=None), dict(len_out=None), dict(src=None),
                 dict(dst=None), dict(rows=None), dict(missing=None)):
        assert _fork(**args) == EINVAL, args
    # outputs over inputs, or over each other
    for args in (dict(refs_out=FORK["refs"]), dict(table_out=FORK["table"] + 4 * 35), dict(len_out=FORK["length"] + 12), dict(dst=FORK["src"]),
                 dict(missing=FORK["rows"] + 20), dict(src=FORK["parent"])):
        assert _fork(**args) == EINVAL, args
    assert _fork(refs=0x100002) == EALIGN and _fork(ws=0xd00010) == EALIGN
    for args in (dict(pages=(1 << 26) + 1), dict(n_in=(1 << 14) + 1), dict(n=(1 << 14) + 1), dict(cols=1 << 28, ld=1 << 28, ldo=1 << 28)):
        assert _fork(**args) == EUNSUPPORTED, args
    need = B.lr_kv_fork_workspace_bytes(100, 4, 6)
    assert need > 0 and _fork(nb=need - 1) == EWORKSPACE and _fork(ws=None) == EWORKSPACE and B.lr_kv_fork_workspace_bytes(0, 4, 6) == 0


COMPACT = dict(refs=0x100000, pages=100, table=0x200000, ld=10, batch=4, cols=10, refs_out=0x300000, table_out=0x400000, ldo=10, src=0x500000, dst=0x600000,
               where=0x700000, live=0x800000, ws=0x900000, nb=1 << 20)


def _compact(**over):
    return B.lib().lr_kv_compact(*{**COMPACT, **over}.values(), None)


def test_kv_compact_refuses():
    for args in (dict(pages=0), dict(batch=-1), dict(cols=0), dict(ld=9), dict(ldo=9), dict(refs=None), dict(table=None), dict(refs_out=None), dict(table_out=None),
                 dict(src=None), dict(dst=None), dict(where=None), dict(live=None), dict(refs_out=COMPACT["refs"]), dict(table_out=COMPACT["table"]),
                 dict(dst=COMPACT["src"] + 196), dict(where=COMPACT["refs_out"] + 396)):
        assert _compact(**args) == EINVAL, args
    assert _compact(pages=(1 << 26) + 1) == EUNSUPPORTED and _compact(batch=(1 << 16) + 1) == EUNSUPPORTED and _compact(table=0x200001) == EALIGN
    need = B.lr_kv_compact_workspace_bytes(100)
    assert need > 0 and _compact(nb=need - 1) == EWORKSPACE


def _copy(src=0x3000, dst=0x4000, rows=None, n=2, **over):
    c = dict(k=0x1000, v=0x2000, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, page_stride=4096, token_stride=256, head_stride=128, page_table=None, batch=0,
             max_pages=0, table_ld=0, cu_q=None, kv_len=None)
    c.update(over)
    return B.lib().lr_kv_copy(C.byref(B.KvCache(**c)), src, dst, rows, n, None)


def test_kv_copy_refuses():
    for args in (dict(n=-1), dict(src=None), dict(dst=None), dict(k=None), dict(v=None), dict(n_pages=0), dict(page_stride=0)):
        assert _copy(**args) == EINVAL, args
    for args in (dict(src=0x3002), dict(rows=0x5001), dict(k=0x1008), dict(page_size=12), dict(head_dim=100), dict(token_stride=252)):
        assert _copy(**args) == EALIGN, args
    assert _copy(page_size=1 << 20, n_kv_heads=1 << 9, token_stride=1 << 16, page_stride=1 << 36, n_pages=1) == EUNSUPPORTED
    assert B.lib().lr_kv_copy(None, 0x3000, 0x4000, None, 2, None) == EINVAL
    assert _copy(n=0, src=None, dst=None) == 0


# ---- refusals of the binding ------------------------------------------------------------------------
X, Q, S = torch.zeros(4, 32), torch.zeros(6, 32, dtype=torch.int8), torch.zeros(6)
I = lambda *s: torch.zeros(s, dtype=torch.int32)
CACHE = torch.zeros((6, 16, 2, 128), dtype=torch.bfloat16)


@pytest.mark.parametrize("error,call", [
    (B.LrError, lambda: B.lr_quant_rows(X.half())), (ValueError, lambda: B.lr_quant_rows(X[0])), (B.LrError, lambda: B.lr_quant_rows(X, q=X)),
    (ValueError, lambda: B.lr_quant_rows(X, scale=S)), (AssertionError, lambda: B.lr_quant_rows(torch.zeros(32, 4).t())),
    (B.LrError, lambda: B.lr_matmul_q8(X, S[:4], Q, S)), (ValueError, lambda: B.lr_matmul_q8(Q, S, Q[:, :16], S)), (ValueError, lambda: B.lr_matmul_q8(Q, S[:5], Q, S)),
    (B.LrError, lambda: B.lr_matmul_q8(Q, S, Q, S, dtype=torch.float16)), (ValueError, lambda: B.lr_matmul_q8(Q, S, Q, S, out=torch.zeros(6, 7))),
    (B.LrError, lambda: B.lr_matmul_q8(Q[:, :24][:, 16:], S, Q.reshape(-1)[:184].as_strided((6, 24), (32, 1))[:, 16:], S)),   # rows that end with the memory
    (ValueError, lambda: B.lr_linear_q8_fwd(X, Q, S, Q, S)), (B.LrError, lambda: B.lr_linear_q8_fwd(X, Q, S, Q[:, :6], S, y=torch.zeros((4, 6), dtype=torch.bfloat16))),
    (ValueError, lambda: B.lr_beam_select(X, torch.zeros(1, 3))), (B.LrError, lambda: B.lr_beam_select(X, torch.zeros(1, 4).double())),
    (B.LrError, lambda: B.lr_beam_select(X, torch.zeros(1, 4), done=torch.zeros(1, 4))), (ValueError, lambda: B.lr_beam_select(X, torch.zeros(1, 4), done=I(4))),
    (ValueError, lambda: B.lr_beam_select(X, torch.zeros(1, 4), out=(I(1, 3), I(1, 4), torch.zeros(1, 4)))),
    (ValueError, lambda: B.lr_kv_fork(I(9), 16, I(2, 3), I(3), I(4), I(4))), (ValueError, lambda: B.lr_kv_fork(I(9), 16, I(2, 3), I(2), I(4), I(5))),
    (B.LrError, lambda: B.lr_kv_fork(I(9).long(), 16, I(2, 3), I(2), I(4), I(4))), (B.LrError, lambda: B.lr_kv_fork(I(9), 16, I(2, 3), I(2), I(4), I(4), out=(I(9),))),
    (AssertionError, lambda: B.lr_kv_fork(I(9), 16, I(3, 2).t(), I(2), I(4), I(4))), (AssertionError, lambda: B.lr_kv_fork(I(18)[::2], 16, I(2, 3), I(2), I(4), I(4))),
    (B.LrError, lambda: B.lr_kv_compact(I(9), I(2, 3).long())), (ValueError, lambda: B.lr_kv_compact(I(9, 1), I(2, 3))),
    (ValueError, lambda: B.lr_kv_copy(CACHE, CACHE[:5], I(2), I(2))), (ValueError, lambda: B.lr_kv_copy(CACHE, CACHE, I(2), I(3))),
    (B.LrError, lambda: B.lr_kv_copy(CACHE.float(), CACHE.float(), I(2), I(2))), (B.LrError, lambda: B.lr_kv_copy(CACHE, CACHE, I(2).long(), I(2))),
])
def test_binding_refuses(error, call):
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("call", [
    lambda: B.lr_quant_rows(X), lambda: B.lr_matmul_q8(Q, S, Q, S), lambda: B.lr_linear_q8_fwd(X, Q, S, torch.zeros((9, 16), dtype=torch.int8)[:, :6], torch.zeros(9)),
    lambda: B.lr_beam_select(X, torch.zeros(1, 4)), lambda: B.lr_kv_fork(I(9), 16, I(2, 3), I(2), I(4), I(4)), lambda: B.lr_kv_compact(I(9), I(2, 3)),
    lambda: B.lr_kv_copy(CACHE, CACHE, I(2), I(2)),
])
def test_tensors_on_the_host_are_refused(call):
    with pytest.raises(B.LrError, match="current GPU"):
        call()
