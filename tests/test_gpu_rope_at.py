"""Rotary tables and rotation at given positions against the fp64 oracle.  Bounds count roundings: half a step of the storage type
(finfo.eps / 2, relative), and 2^-24 of the magnitudes for each of the three operations in 32 bits."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import lowrank_oracle as orc
from oracle import paged_oracle as po
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# one row and one pair; rows that no workgroup's share divides; the widest; far positions; scaled frequencies
@pytest.mark.parametrize("n,rot,kw", [(1, 2, {}), (7, 128, {}), (300, 6, dict(base=1e6)), (1031, 128, dict(mscale=1.3, factor=4.0)),
                                      (3, 8192, {}), (70, 8190, {}), (5000, 64, dict(first=(1 << 20) - 2500)), (4, 130, dict(first=(1 << 31) - 4)),
                                      (515, 128, dict(factor=32.0, ramp=(4096.0, 1.0, 32.0), base=5e5)),
                                      (33, 48, dict(factor=8.0, ramp=(1e5, 0.0, 2.0), mscale=-0.5))])
def test_tables(n, rot, kw):
    print(f"tables n={n} rot={rot} {kw}", flush=True)
    got = B.lr_rope_table(n, rot, device=DEV, **kw)
    torch.cuda.synchronize()
    m = abs(kw.get("mscale", 1.0))
    far = kw.get("first", 0) + n
    # an angle: its frequency to a few dozen steps of 64 bits on either side; the entry: rounded once
    bound = m * (far * 64 * 2.0 ** -53 + 1e-12)
    for g, ref in zip(got, po.rope_table(n, rot, **kw)):
        assert g.shape == (n, rot // 2) and g.dtype == torch.float32
        assert (np.abs(g.double().cpu().numpy() - ref) <= bound + 2.0 ** -24 * np.abs(ref)).all()


def _expected(x, H, hd, cos, sin, pos, interleaved, inverse):
    """x [T, >= H hd] fp64; rows whose position is in the tables.  Returns result, magnitudes."""
    y, mag = x.copy(), np.abs(x)
    for t, p in enumerate(pos):
        if 0 <= p < len(cos):
            y[t, :H * hd], mag[t, :H * hd] = (a.reshape(-1) for a in po.rotate(x[t, :H * hd].reshape(H, hd), cos[p], sin[p], interleaved, inverse))
    return y, mag


def _close(got, ref, mag, dtype):
    half = torch.finfo(dtype).eps / 2
    err = np.abs(got.double().cpu().numpy() - ref)
    arith = 4 * 2.0 ** -24 * mag                       # two products, their sum, the sign or scale of the table entry
    assert (err <= half * (np.abs(ref) + arith) + arith).all(), float((err - half * np.abs(ref)).max())


# T, H, hd, rot, columns behind the heads
SHAPES = [(1, 1, 128, 128, 0), (2, 1, 8192, 64, 0), (16, 32, 128, 128, 0), (37, 3, 80, 32, 8), (130, 5, 64, 16, 0), (5, 40, 256, 240, 24), (257, 2, 192, 192, 136),
          (3, 7, 16, 16, 0), (1, 300, 96, 48, 0)]


@pytest.mark.parametrize("T,H,hd,rot,extra", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotation(T, H, hd, rot, extra, dtype):
    print(f"rotation T={T} H={H} hd={hd} rot={rot} +{extra} {dtype}", flush=True)
    if dtype == torch.float32:                         # rows may start anywhere, any even part of a head may turn
        extra, rot = extra + 1, max(2, rot - 6)
    rng = np.random.default_rng(T)
    x = si.gaussian(3, "x", (T, H * hd + extra), dtype=dtype).to(DEV)
    rows = 50
    cos, sin = (torch.from_numpy(a).float().to(DEV) for a in po.rope_table(rows, rot, mscale=1.2))
    pos = rng.integers(0, rows, T)
    pos[rng.random(T) < 0.2] = rng.choice([-1, rows, -(1 << 31), (1 << 31) - 1])      # outside the tables
    pd = torch.from_numpy(pos.astype(np.int32)).to(DEV)
    C, S = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    X = x.double().cpu().numpy()
    inside = torch.from_numpy((pos >= 0) & (pos < rows)).to(DEV)
    for interleaved in (False, True):
        for inverse in (False, True):
            ref, mag = _expected(X, H, hd, C, S, pos, interleaved, inverse)
            out = torch.full((T, H * hd + 2 * extra), 7.0, dtype=dtype, device=DEV)
            got = B.lr_rope_at(x, cos, sin, H, hd, pos=pd, interleaved=interleaved, inverse=inverse, out=out)
            torch.cuda.synchronize()
            assert got is out or got.data_ptr() == out.data_ptr()
            _close(out[inside][:, :H * hd], ref[inside.cpu().numpy()][:, :H * hd], mag[inside.cpu().numpy()][:, :H * hd], dtype)
            assert bool((out[~inside] == 7).all()) and bool((out[:, H * hd:] == 7).all())
            place = x.clone()                          # in place: the same bits, what is outside as it was
            B.lr_rope_at(place, cos, sin, H, hd, pos=pd, interleaved=interleaved, inverse=inverse, out=place)
            torch.cuda.synchronize()
            assert torch.equal(place[inside][:, :H * hd], out[inside][:, :H * hd])
            assert torch.equal(place[~inside], x[~inside]) and torch.equal(place[:, H * hd:], x[:, H * hd:])


@pytest.mark.parametrize("hd,rot", [(80, 32), (96, 96), (128, 8)])
def test_fp32_rows_that_start_on_16_bytes(hd, rot):
    """In vectors of four: the bits of the form that takes rows from anywhere."""
    T, H = 123, 3
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((T, H * hd), generator=g, device=DEV)
    pos = torch.randint(0, 300, (T,), generator=g, device=DEV, dtype=torch.int32)
    cos, sin = B.lr_rope_table(300, rot, device=DEV)
    odd = torch.zeros((T, H * hd + 1), device=DEV)
    odd[:, 1:] = x
    for interleaved in (False, True):
        a = B.lr_rope_at(x, cos, sin, H, hd, pos=pos, interleaved=interleaved)
        b = B.lr_rope_at(odd[:, 1:], cos, sin, H, hd, pos=pos, interleaved=interleaved)
        torch.cuda.synchronize()
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H", [(1500, 32), (9000, 5)])
def test_many_rows(T, H, dtype):
    """The positions of rows in order (no list), and a new tensor for the result."""
    print(f"many rows T={T} H={H} {dtype}", flush=True)
    hd = 128
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn((T, H * hd), generator=g, device=DEV).to(dtype)
    cos, sin = B.lr_rope_table(T + 3, 128, device=DEV)
    for interleaved in (False, True):
        got = B.lr_rope_at(x, cos, sin, H, hd, interleaved=interleaved)
        X = x.double().view(T, H, hd)
        a, b = (X[..., 0::2], X[..., 1::2]) if interleaved else (X[..., :64], X[..., 64:])
        c, s = cos[:T].double()[:, None], sin[:T].double()[:, None]
        join = (lambda u, v: torch.stack((u, v), -1).flatten(-2)) if interleaved else (lambda u, v: torch.cat((u, v), -1))
        ref, mag = join(a * c - b * s, b * c + a * s), join((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs())
        torch.cuda.synchronize()
        _close(got, ref.reshape(T, -1).cpu().numpy(), mag.reshape(T, -1).cpu().numpy(), dtype)


def test_half_layout_is_the_blocks_rotation():
    Bn, S, H = 2, 77, 3
    x = si.gaussian(5, "rope_x", (Bn * S, H * 128), dtype=torch.bfloat16).to(DEV)
    cos, sin = B.lr_rope_table(S, 128, device=DEV)
    pos = torch.arange(S, dtype=torch.int32, device=DEV).repeat(Bn)
    for inverse in (False, True):
        ref = B.lr_rope(x.clone(), cos, sin, Bn, S, H, 128, inverse=inverse)
        got = B.lr_rope_at(x, cos, sin, H, 128, pos=pos, inverse=inverse)
        torch.cuda.synchronize()
        err = (got.double() - ref.double()).abs()
        assert bool((err <= 2.0 ** -7 * ref.double().abs()).all())       # a step apart where the two sums round differently


def test_gradient_is_the_transpose_and_agrees_with_differences():
    T, H, hd, rot = 9, 2, 80, 32
    g = torch.Generator(device=DEV).manual_seed(4)
    x, dy = (torch.randn((T, H * hd), generator=g, device=DEV) for _ in range(2))
    pos = torch.randint(0, 1000, (T,), generator=g, device=DEV, dtype=torch.int32)
    cos, sin = B.lr_rope_table(1000, rot, mscale=1.1, device=DEV)
    for interleaved in (False, True):
        f = lambda v: B.lr_rope_at(v, cos, sin, H, hd, pos=pos, interleaved=interleaved)
        dx = B.lr_rope_at(dy, cos, sin, H, hd, pos=pos, interleaved=interleaved, inverse=True)
        # a linear map: differences of any step are its matrix; steps of a power of two round nothing
        for _ in range(6):
            v = torch.randn((T, H * hd), generator=g, device=DEV)
            lhs, rhs = (f(v).double() * dy.double()).sum(), (v.double() * dx.double()).sum()
            scale = (v.abs().double() * dx.abs().double()).sum()
            assert abs(float(lhs - rhs)) <= 2.0 ** -20 * float(scale)
        e = torch.zeros_like(x)
        e[3, 5] = 2.0 ** -6
        diff = ((f(x + e).double() - f(x - e).double()) * dy.double()).sum() / 2.0 ** -5
        assert abs(float(diff - dx[3, 5].double())) <= 2.0 ** -6 * float(dy.abs().max())


def test_tables_feed_the_block():
    """lr_rope_table's tables as a block's rope_cos / rope_sin: the oracle's block with its own tables."""
    Bn, S, H, f, r = 1, 200, 1, 200, 32
    case = si.block_case(Bn, S, 128 * H, H, 128, f, r, seed=41)
    tab = B.lr_rope_table(S, 128, device=DEV)
    desc = B.make_block_desc(Bn, S, 128 * H, H, 128, f, f, r, rope=tab)
    packed = {k: v.to(DEV) for k, v in si.pack_block_params(case["params"], f, f).items()}
    y, _ = B.lr_block_fwd(desc, packed, case["x"].to(DEV))
    torch.cuda.synchronize()
    P = {k: si.f64(v) for k, v in case["params"].items()}
    y_ref, _ = orc.block_fwd(si.f64(case["x"]), P, Bn, S, H, 128, 1e-5, rope=orc.rope_tables(S, 128, 10000.0))
    from parity import check
    check("y", y, y_ref, torch.bfloat16)
