"""Keys and values into the pages of a cache, against the fp64 oracle: every element of the cache is compared, those that no token
writes bit for bit."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def make(seqs, Hkv, hd, page, layout="token", lead=0, tail=0, seed=0, extra_pages=2, extra_cols=1):
    """Lists, page table and a cache of random values for seqs = [(new tokens, keys with them)], pages in random order; `lead` and `tail`
    tokens belong to nobody."""
    rng = np.random.default_rng(seed)
    need = [-(-max(kv, 0) // page) for _, kv in seqs]
    cols = max(need + [1]) + extra_cols
    n_pages = sum(need) + extra_pages
    order = iter(rng.permutation(n_pages))
    table = np.full((len(seqs), cols), -1, dtype=np.int32)
    for b, n in enumerate(need):
        table[b, :n] = [next(order) for _ in range(n)]
    cu = np.cumsum([lead] + [n for n, _ in seqs]).astype(np.int32)
    g = torch.Generator(device=DEV).manual_seed(seed)
    if layout == "token":
        shape = (n_pages, page, Hkv, hd)
        k, v = (torch.randn(shape, generator=g, device=DEV).to(BF) for _ in range(2))
    elif layout == "head":                              # heads outside, tokens inside a page
        k, v = (torch.randn((n_pages, Hkv, page, hd), generator=g, device=DEV).to(BF).transpose(1, 2) for _ in range(2))
    else:                                               # keys and values of a page side by side, rows wider than the heads
        both = torch.randn((n_pages, 2, page, Hkv, hd + 24), generator=g, device=DEV).to(BF)
        k, v = both[:, 0, ..., :hd], both[:, 1, ..., :hd]
    return {"k_cache": k, "v_cache": v, "page_table": torch.from_numpy(table).to(DEV), "cu_q": torch.from_numpy(cu).to(DEV),
            "kv_len": torch.tensor([kv for _, kv in seqs], dtype=torch.int32, device=DEV)}, int(cu[-1]) + tail


def np64(t):
    return t.double().cpu().numpy()


def lists(c):
    return tuple(c[n].cpu().numpy() for n in ("cu_q", "kv_len", "page_table"))


CASES = [
    # one token of one sequence, the first of a cache
    ([(1, 1)], 1, 128, 128, 16, 0, "token"),
    # decoding: single tokens, a sequence without any, one whose keys end with a page
    ([(1, 5), (1, 16), (0, 9), (1, 17), (1, 333)], 2, 128, 128, 16, 4, "token"),
    # prompts of odd lengths, some behind earlier keys, half of the head turned
    ([(37, 37), (5, 60), (1, 1), (130, 131)], 3, 128, 64, 24, 5, "head"),
    ([(70, 75), (3, 3)], 2, 64, 16, 8, 6, "wide"),
    # no rotation; more sequences than a wavefront compares at once
    ([(1 + b % 3, 10 + b) for b in range(150)], 1, 192, 0, 32, 2, "token"),
    # more new tokens than keys: those at negative positions have no place
    ([(6, 4), (3, 0), (2, -7)], 2, 128, 128, 16, 2, "token"),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("seqs,Hkv,hd,rot,page,H,layout", CASES)
def test_append(seqs, Hkv, hd, rot, page, H, layout, interleaved):
    print(f"append {len(seqs)} sequences, Hkv={Hkv} hd={hd} rot={rot} page={page} H={H} {layout} interleaved={interleaved}", flush=True)
    c, T = make(seqs, Hkv, hd, page, layout, lead=2, tail=3, seed=len(seqs))
    g = torch.Generator(device=DEV).manual_seed(9)
    qkv = torch.randn((T, (H + 2 * Hkv) * hd + 8), generator=g, device=DEV).to(BF)
    q, k, v = (qkv[:, :H * hd] if H else None), qkv[:, H * hd:(H + Hkv) * hd], qkv[:, (H + Hkv) * hd:(H + 2 * Hkv) * hd]
    cos = sin = None
    if rot:
        cos, sin = B.lr_rope_table(400, rot, device=DEV)
    cu, kv_len, table = lists(c)
    n_pages = c["k_cache"].shape[0]
    placed = po.places(cu, kv_len, table, page, n_pages, T)
    K, V = np64(c["k_cache"]), np64(c["v_cache"])
    magK = np.zeros_like(K)
    out = torch.full((T, H * hd + 16), 7.0, dtype=BF, device=DEV) if H else None
    Q = np.full((T, H, hd), 7.0)
    magQ = np.zeros_like(Q)
    for t, b, p, pg, row in placed:
        kk = np64(k[t]).reshape(Hkv, hd)
        K[pg, row], magK[pg, row] = po.rotate(kk, np64(cos[p]), np64(sin[p]), interleaved) if rot else (kk, np.abs(kk))
        V[pg, row] = np64(v[t]).reshape(Hkv, hd)
        if H:
            qq = np64(q[t]).reshape(H, hd)
            Q[t], magQ[t] = po.rotate(qq, np64(cos[p]), np64(sin[p]), interleaved) if rot else (qq, np.abs(qq))
    got_q = B.lr_kv_append(k, v, rope=(cos, sin) if rot else None, interleaved=interleaved, q=q, H=H, q_out=out, **c)
    torch.cuda.synchronize()
    half, arith = torch.finfo(BF).eps / 2, 3 * 2.0 ** -24
    untouched = magK == 0
    assert np.array_equal(np64(c["k_cache"])[untouched], K[untouched]) and np.array_equal(np64(c["v_cache"]), V)
    assert (np.abs(np64(c["k_cache"]) - K) <= half * np.abs(K) + 2 * arith * magK).all()
    if H:
        got = np64(out)
        assert (got[:, H * hd:] == 7).all()
        assert (np.abs(got[:, :H * hd].reshape(T, H, hd) - Q) <= half * np.abs(Q) + 2 * arith * magQ).all()
        assert got_q.data_ptr() == out.data_ptr()
    else:
        assert got_q is None
    # the queries in place: the same bits, rows without a place as they were
    if H:
        inplace = qkv.clone()
        B.lr_kv_append(k, v, rope=(cos, sin) if rot else None, interleaved=interleaved, q=inplace[:, :H * hd], H=H, q_out=inplace[:, :H * hd], **c)
        torch.cuda.synchronize()
        mine = torch.zeros(T, dtype=torch.bool)
        mine[[t for t, *_ in placed]] = True
        assert torch.equal(inplace[mine.to(DEV)][:, :H * hd], out[mine.to(DEV)][:, :H * hd])
        assert torch.equal(inplace[~mine.to(DEV)], qkv[~mine.to(DEV)]) and torch.equal(inplace[:, H * hd:], qkv[:, H * hd:])


def test_lists_that_lead_nowhere_write_nothing():
    """Page numbers that are none, keys past the table's columns, positions past the rotary tables, lists that point past the tokens."""
    Hkv, hd, page, T = 1, 128, 16, 12
    cos, sin = B.lr_rope_table(40, 128, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v, q = (torch.randn((T, hd), generator=g, device=DEV).to(BF) for _ in range(3))
    big = (1 << 31) - 1
    for cu, kv, table in (([0, 4, 8, 12], [5, 6, 7], [[-1, 0], [4, 0], [big, 0]]), ([0, 4, 8, 12], [900, big, 60], [[0, 1], [2, 3], [0, 1]]),
                          ([0, 12, 12, 12], [-big - 1, 5, 5], [[0, 1], [2, 3], [0, 1]]), ([12, 0, -5, 12], [1, 1, 1], [[-1, -1]] * 3),
                          ([0, 4, 8, 12], [45, 45, 45], [[-1, -1, 0]] * 3)):
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
        kc, vc = (torch.randn((4, page, Hkv, hd), generator=g, device=DEV).to(BF) for _ in range(2))
        before = kc.clone(), vc.clone()
        out = torch.full((T, hd), 7.0, dtype=BF, device=DEV)
        B.lr_kv_append(k, v, kc, vc, i32(table), i32(cu), i32(kv), rope=(cos, sin), q=q, H=1, q_out=out)
        torch.cuda.synchronize()
        assert torch.equal(kc, before[0]) and torch.equal(vc, before[1]) and bool((out == 7).all()), (cu, kv, table)


def test_far_pages():
    """Offsets past 2^32 bytes and 2^31 elements: the last pages of a cache of 5.4 GB."""
    page, Hkv, hd = 256, 8, 128
    n_pages = 10400
    cache = torch.zeros((n_pages, page, Hkv, hd), dtype=BF, device=DEV)
    assert cache.numel() > 1 << 31
    table = torch.tensor([[n_pages - 1, 3], [n_pages - 2, 8200]], dtype=torch.int32, device=DEV)
    cu, kv = (torch.tensor(a, dtype=torch.int32, device=DEV) for a in ([0, 3, 5], [258, 400]))
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((5, Hkv * hd), generator=g, device=DEV).to(BF) for _ in range(2))
    vc = torch.zeros_like(cache)
    B.lr_kv_append(k, v, cache, vc, table, cu, kv)
    torch.cuda.synchronize()
    for t, (pg, row) in enumerate([(n_pages - 1, 255), (3, 0), (3, 1), (8200, 142), (8200, 143)]):
        assert torch.equal(cache[pg, row].flatten(), k[t]) and torch.equal(vc[pg, row].flatten(), v[t])
    assert int((cache.flatten(1).abs().amax(1) > 0).sum()) == 3


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 64, 128])
def test_many_tokens(rot, interleaved):
    """More tokens than find a workgroup each: the bits of lr_rope_at, in their places."""
    H, Hkv, hd, page = 6, 3, 128, 24
    c, T = make([(1500, 1501), (1, 800), (0, 5), (2333, 2333), (31, 40)], Hkv, hd, page, "head", seed=3, lead=1, tail=2)
    g = torch.Generator(device=DEV).manual_seed(9)
    q, k, v = (torch.randn((T, w * hd), generator=g, device=DEV).to(BF) for w in (H, Hkv, Hkv))
    cu, kv_len, table = lists(c)
    placed = np.array(po.places(cu, kv_len, table, page, c["k_cache"].shape[0], T))
    t, pos, pg, row = (torch.from_numpy(placed[:, i].copy()).to(DEV) for i in (0, 2, 3, 4))
    tables = B.lr_rope_table(2400, rot, device=DEV) if rot else None
    want_k, want_v = c["k_cache"].clone(), c["v_cache"].clone()
    all_pos = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    all_pos[t] = pos.to(torch.int32)
    turn = lambda x, w: B.lr_rope_at(x, *tables, w, hd, pos=all_pos, interleaved=interleaved) if rot else x
    want_k[pg, row], want_v[pg, row] = turn(k, Hkv).view(T, Hkv, hd)[t], v.view(T, Hkv, hd)[t]
    got = B.lr_kv_append(k, v, rope=tables, interleaved=interleaved, q=q, H=H, **c)
    torch.cuda.synchronize()
    assert torch.equal(c["k_cache"], want_k) and torch.equal(c["v_cache"], want_v)
    assert torch.equal(got[t], turn(q, H)[t])
