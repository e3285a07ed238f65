"""Rotary tables, rotation at positions, paged cache: what is refused before anything reaches a device, and the oracle against other
formulas."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import gqa_oracle, lowrank_oracle, paged_oracle as po
from paper_2512_12131_amd import binding as B

FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)     # never dereferenced on these paths
EINVAL, EUNSUPPORTED, EWORKSPACE, EALIGN = -1, -2, -3, -4


def test_rope_table_arguments():
    f = lambda *, n=4, rot=8, first=0, base=1e4, factor=1.0, context=0.0, low=0.0, high=1.0, mscale=1.0, cos=FAKE: \
        B.lib().lr_rope_table(cos, FAKE, n, rot, first, base, factor, context, low, high, mscale, None)
    nan, inf = float("nan"), float("inf")
    for bad in ({"n": -1}, {"rot": 0}, {"rot": 7}, {"first": -1}, {"first": (1 << 31) - 3}, {"n": 1 << 40}, {"base": 0.0}, {"base": nan},
                {"base": inf}, {"factor": 0.0}, {"factor": -1.0}, {"context": -1.0}, {"context": 4096.0, "low": 2.0, "high": 2.0},
                {"context": 4096.0, "high": nan}, {"context": inf}, {"mscale": inf}, {"cos": None}):
        assert f(**bad) == EINVAL, bad
    assert f(rot=8194) == EUNSUPPORTED
    assert f(n=0, cos=None) == 0


def _rope(*, x=FAKE, ldx=256, out=FAKE, ldo=256, pos=FAKE, cos=FAKE, rows=8, T=4, H=2, hd=128, rot=128, dt=1):
    return B.lib().lr_rope_at(x, ldx, out, ldo, pos, cos, FAKE, rows, T, H, hd, rot, 0, 0, dt, None)


def test_rope_at_arguments():
    for bad in ({"x": None}, {"ldx": 248}, {"ldo": 248}, {"cos": None}, {"rows": 0}, {"T": -1}, {"H": 0}, {"hd": 0}, {"rot": 0}, {"rot": 144},
                {"rot": 33}, {"dt": 7}, {"pos": None, "T": 9}, {"ldo": 264}, {"T": 1 << 31}):
        assert _rope(**bad) == EINVAL, bad
    for bad in ({"x": ODD, "out": FAKE}, {"ldx": 260, "out": C.c_void_p(0x2000)}, {"cos": ODD}, {"rot": 8}, {"hd": 124, "rot": 16},
                {"pos": C.c_void_p(0x1002)}, {"dt": 0, "x": C.c_void_p(0x1002)}):
        assert _rope(**bad) == EALIGN, bad
    assert _rope(rows=1 << 31) == EUNSUPPORTED
    assert _rope(T=0, x=None, out=None) == 0


def _cache(**over):
    c = dict(k=0x1000, v=0x1000, n_pages=6, page_size=16, n_kv_heads=2, head_dim=128, page_stride=16 * 256, token_stride=256, head_stride=128,
             page_table=0x1000, batch=3, max_pages=4, table_ld=4, cu_q=0x1000, kv_len=0x1000)
    return C.byref(B.KvCache(**{**c, **over}))


BAD_CACHES = [(EINVAL, dict(k=None)), (EINVAL, dict(page_table=None)), (EINVAL, dict(cu_q=None)), (EINVAL, dict(kv_len=None)),
              (EINVAL, dict(n_pages=0)), (EINVAL, dict(page_size=0)), (EINVAL, dict(n_kv_heads=0)), (EINVAL, dict(batch=-1)),
              (EINVAL, dict(max_pages=0)), (EINVAL, dict(table_ld=3)), (EINVAL, dict(token_stride=-256)), (EINVAL, dict(page_stride=0)),
              (EALIGN, dict(page_size=12)), (EALIGN, dict(page_size=1)), (EALIGN, dict(token_stride=260)), (EALIGN, dict(head_stride=132)),
              (EALIGN, dict(page_stride=4100)), (EALIGN, dict(v=0x1008)), (EALIGN, dict(page_table=0x1002)),
              (EUNSUPPORTED, dict(max_pages=1 << 28, table_ld=1 << 28)), (EUNSUPPORTED, dict(page_stride=1 << 33, n_pages=8)),
              (EUNSUPPORTED, dict(page_stride=1 << 62, n_pages=1 << 30)), (EUNSUPPORTED, dict(token_stride=1 << 26)),
              (EUNSUPPORTED, dict(page_size=1 << 40)), (EUNSUPPORTED, dict(batch=1 << 40))]


def _append(cache=None, *, k=FAKE, ldk=256, v=FAKE, ldv=256, q=FAKE, ldq=512, qo=FAKE, ldqo=512, T=4, H=4, cos=FAKE, sin=FAKE, rows=64, rot=128,
            dt=1):
    return B.lib().lr_kv_append(cache or _cache(), k, ldk, v, ldv, q, ldq, qo, ldqo, T, H, cos, sin, rows, rot, 0, dt, None)


def _paged(cache=None, *, q=FAKE, ldq=512, o=FAKE, ldo=512, lse=FAKE, T=4, H=4, scale=0.1, causal=1, dt=1, ws=FAKE, nb=1 << 40):
    return B.lib().lr_attention_paged_fwd(cache or _cache(), q, ldq, o, ldo, lse, T, H, scale, causal, dt, ws, nb, None)


@pytest.mark.parametrize("status,over", BAD_CACHES)
def test_caches_that_are_refused(status, over):
    assert _append(_cache(**over)) == status
    assert _paged(_cache(**over)) == status
    if not {"k", "v", "page_table", "cu_q", "kv_len"} & set(over):
        assert B.lib().lr_attention_paged_workspace_bytes(_cache(**over), 4, 4) == 0


def test_kv_append_arguments():
    for bad in ({"k": None}, {"ldk": 248}, {"ldv": 248}, {"T": -1}, {"H": -1}, {"H": 0}, {"q": None, "qo": None}, {"qo": None}, {"ldq": 504},
                {"ldqo": 504}, {"ldqo": 520}, {"cos": None}, {"sin": None}, {"rows": 0}, {"rot": 0}, {"rot": 144}, {"rot": -16}, {"dt": 9}):
        assert _append(**bad) == EINVAL, bad
    for bad in ({"k": ODD}, {"ldk": 260}, {"rot": 8}, {"q": ODD}, {"cos": ODD}):
        assert _append(**bad) == EALIGN, bad
    assert _append(dt=0) == EUNSUPPORTED and _append(T=(1 << 26) + 1) == EUNSUPPORTED
    assert _append(T=0) == 0 and _append(_cache(batch=0)) == 0


def test_attention_paged_arguments():
    for bad in ({"q": None}, {"o": None}, {"ldq": 504}, {"ldo": 504}, {"T": -1}, {"H": 0}, {"H": 3}, {"scale": 0.0}, {"scale": -1.0},
                {"scale": float("nan")}, {"scale": float("inf")}, {"dt": 5}):
        assert _paged(**bad) == EINVAL, bad
    for bad in ({"q": ODD}, {"o": ODD}, {"ldq": 516}, {"lse": C.c_void_p(0x1002)}):
        assert _paged(**bad) == EALIGN, bad
    for bad in ({"causal": 0}, {"dt": 0}, {"T": (1 << 26) + 1}):
        assert _paged(**bad) == EUNSUPPORTED, bad
    assert _paged(_cache(head_dim=64)) == EUNSUPPORTED
    assert _paged(T=0) == 0 and _paged(_cache(batch=0)) == 0


def test_calls_past_a_launch_are_refused():
    """Sequences and tokens that a launch's lanes (2^32) cannot hold, and lists that every workgroup would read for too long."""
    assert _append(_cache(batch=(1 << 16) + 1)) == EUNSUPPORTED and _paged(_cache(batch=(1 << 16) + 1)) == EUNSUPPORTED
    assert _append(T=(1 << 25) + 1) == EUNSUPPORTED and _paged(T=(1 << 25) + 1) == EUNSUPPORTED
    big = dict(n_kv_heads=256, page_stride=16 * 256 * 128, token_stride=256 * 128, batch=1 << 16)
    for T, kv, batch in ((1 << 16, 256, 1 << 16), (1 << 20, 1024, 1 << 14), ((1 << 25) - 1, 64, 1)):
        cache = lambda: _cache(**{**big, "n_kv_heads": kv, "batch": batch})
        args = dict(T=T, H=kv, ldq=kv * 128, ldo=kv * 128)
        assert B.lib().lr_attention_paged_workspace_bytes(cache(), T, kv) == 0, (T, kv)
        assert _paged(cache(), **args) == EUNSUPPORTED, (T, kv)
    assert B.lib().lr_attention_paged_workspace_bytes(_cache(**{**big, "batch": 1 << 15, "max_pages": 64, "table_ld": 64}), 1 << 15, 256) > 0


@pytest.mark.parametrize("H,kv", [(32, 8), (16, 16), (5, 1)])
def test_a_workspace_for_more_tokens_or_keys_serves_for_fewer(H, kv):
    size = lambda T, batch, cols: B.lib().lr_attention_paged_workspace_bytes(_cache(n_kv_heads=kv, batch=batch, max_pages=cols, table_ld=cols), T, H)
    for batch in (1, 7, 64, 300):
        sizes = [size(T, batch, 100) for T in [*range(1, 200), *range(200, 20000, 333)]]
        assert sizes == sorted(sizes)
        sizes = [size(64, batch, cols) for cols in range(1, 3000, 7)]
        assert sizes == sorted(sizes)
    assert size(1, 1, 8) == 0 and size(1, 1, 9) > 0              # 128 keys are one split
    assert max(size(T, 64, 1 << 20) for T in (1, 64, 4096, 1 << 20)) < 128 << 20


T4 = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
I4 = lambda *s: torch.zeros(s, dtype=torch.int32)
KC, TAB, CU, LEN, COS = T4(6, 16, 2, 128), I4(3, 4), I4(4), I4(3), torch.zeros(64, 64)


@pytest.mark.parametrize("error,call", [
    (ValueError, lambda: B.lr_rope_at(T4(4), COS, COS, 1, 128)), (ValueError, lambda: B.lr_rope_at(T4(4, 128), COS, COS, 2, 128)),
    (ValueError, lambda: B.lr_rope_at(T4(4, 128), COS, COS[:, :8].contiguous(), 1, 128)),
    (ValueError, lambda: B.lr_rope_at(T4(4, 128), COS, COS, 1, 128, pos=I4(3))),
    (B.LrError, lambda: B.lr_rope_at(T4(4, 128), COS, COS, 1, 128, pos=torch.zeros(4, dtype=torch.int64))),
    (B.LrError, lambda: B.lr_rope_at(T4(4, 128), COS.double(), COS, 1, 128)), (B.LrError, lambda: B.lr_rope_at(T4(4, 128).half(), COS, COS, 1, 128)),
    (B.LrError, lambda: B.lr_rope_at(T4(4, 128), COS, COS, 1, 128, out=torch.zeros(4, 128))),
    (AssertionError, lambda: B.lr_rope_at(T4(128, 4).t(), COS, COS, 1, 128)),
    (B.LrError, lambda: B.lr_rope_at(T4(4, 128), COS, COS, 1, 128)),                                   # not on the GPU
    (B.LrError, lambda: B.lr_rope_table(4, 8, device="cpu")), (B.LrError, lambda: B.lr_rope_table(4, 8, ramp=(0.0, 1.0, 2.0))),
    (ValueError, lambda: B.lr_kv_append(T4(4, 256), T4(5, 256), KC, KC, TAB, CU, LEN)),
    (ValueError, lambda: B.lr_kv_append(T4(4, 248), T4(4, 256), KC, KC, TAB, CU, LEN)),
    (ValueError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, TAB, CU, I4(4))),
    (ValueError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, TAB, I4(3), LEN)),
    (ValueError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC[1:], TAB, CU, LEN)),
    (AssertionError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, T4(6, 2, 16, 128).transpose(1, 2), TAB, CU, LEN)),
    (AssertionError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, I4(4, 3).t(), CU, LEN)),
    (AssertionError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, TAB, I4(8)[::2], LEN)),
    (B.LrError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, TAB.long(), CU, LEN)),
    (B.LrError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC.float(), KC.float(), TAB, CU, LEN)),
    (B.LrError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256).float(), KC, KC, TAB, CU, LEN)),
    (B.LrError, lambda: B.lr_kv_append(T4(4, 256), T4(4, 256), KC, KC, TAB, CU, LEN)),                 # not on the GPU
    (ValueError, lambda: B.lr_attention_paged_fwd(T4(4, 256), KC, KC, TAB, CU, LEN, 4)),
    (ValueError, lambda: B.lr_attention_paged_fwd(T4(4, 512), KC[0], KC[0], TAB, CU, LEN, 4)),
    (ValueError, lambda: B.lr_attention_paged_fwd(T4(4, 512), KC, KC, TAB, CU, LEN, 4, lse=torch.zeros(4, 5))),
    (B.LrError, lambda: B.lr_attention_paged_fwd(T4(4, 512), KC, KC, TAB, CU, LEN, 4, o=torch.zeros(4, 512))),
    (B.LrError, lambda: B.lr_attention_paged_fwd(T4(4, 512), KC, KC, TAB, CU, LEN, 4)),                # not on the GPU
])
def test_tensors_that_are_refused(error, call):
    with pytest.raises(error):
        call()


# ---- the oracle ------------------------------------------------------------------------------------------
def test_oracle_tables_are_the_blocks():
    cos, sin = lowrank_oracle.rope_tables(40, 128, 10000.0)
    got = po.rope_table(40, 128)
    assert np.abs(got[0] - cos).max() < 1e-13 and np.abs(got[1] - sin).max() < 1e-13
    # a ramp between "kept" and "divided": its ends are those
    kept, scaled = po.rope_table(40, 64), po.rope_table(40, 64, factor=8.0)
    ramp = po.rope_table(40, 64, factor=8.0, ramp=(2048.0, 1.0, 32.0))
    assert np.allclose(ramp[0][:, 0], kept[0][:, 0], atol=1e-13) and np.allclose(ramp[0][:, -1], scaled[0][:, -1], atol=1e-13)


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotation_is_orthogonal_and_relative(interleaved):
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 80))
    cos, sin = po.rope_table(30, 32)
    turn = lambda v, p, inverse=False: po.rotate(v, cos[p], sin[p], interleaved, inverse)[0]
    assert np.allclose(turn(turn(x, 7), 7, True), x) and np.isclose(turn(x, 7) @ y, x @ turn(y, 7, True))
    assert np.isclose(turn(x, 12) @ turn(y, 9), turn(x, 22) @ turn(y, 19)) and np.array_equal(turn(x, 12)[32:], x[32:])
    if not interleaved:
        full = lowrank_oracle.rope_tables(5, 128, 10000.0)
        z = rng.standard_normal((5, 128))
        ref = lowrank_oracle.rope_apply(z, *full, 1, 5, 1, 128)
        assert np.allclose([po.rotate(z[p], full[0][p], full[1][p])[0] for p in range(5)], ref)


def test_oracle_paged_attention_is_the_dense_one():
    """A whole prompt in pages of any order: causal grouped-query attention."""
    rng = np.random.default_rng(1)
    S, H, Hkv, hd, ps = 21, 4, 2, 16, 8
    q, k, v = rng.standard_normal((S, H * hd)), rng.standard_normal((S, Hkv * hd)), rng.standard_normal((S, Hkv * hd))
    table = np.array([[2, 0, 3]])
    kc, vc = rng.standard_normal((2, 4, ps, Hkv, hd))
    for t, b, p, page, row in po.places([0, S], [S], table, ps, 4, S):
        kc[page, row], vc[page, row] = k[t].reshape(Hkv, hd), v[t].reshape(Hkv, hd)
    o, lse, _, _ = po.attention_paged(q.reshape(S, H, hd), kc, vc, table, [0, S], [S], H, hd ** -0.5)
    o_ref, lse_ref = gqa_oracle.attention_gqa_fwd(q, k, v, 1, S, H, Hkv, hd)
    assert np.allclose(o.reshape(S, -1), o_ref) and np.allclose(lse.T, lse_ref[0])
