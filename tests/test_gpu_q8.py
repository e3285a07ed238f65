"""Rows as 8-bit integers, their products and the bottleneck layer on them, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def np64(t):
    return t.double().cpu().numpy()


def check_rows(x, q, scale):
    """Whole numbers are the oracle's; a scale is one division, rounded once."""
    want, s = so.quant_rows(np64(x))
    assert np.array_equal(q.cpu().numpy().astype(np.int64), want)
    got = np64(scale)
    assert np.array_equal(np.isnan(got), np.isnan(s))
    assert np.array_equal(got[~np.isnan(s)], s[~np.isnan(s)].astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,n", [(1, 8), (3, 24), (16, 4096), (5, 1024), (7, 1032), (130, 512), (2, 8200), (1, 40000), (3, 16400)])
def test_quant_rows(T, n, dtype):
    g = gen(T * n)
    x = (randn(g, T, n) * 10.0 ** (torch.rand((T, 1), generator=g, device=DEV) * 20 - 10)).to(dtype)
    x[0, n // 2] = x[0].abs().max() / 2                   # 63.5 steps: a tie
    check_rows(x, *B.lr_quant_rows(x))


@pytest.mark.parametrize("n", [1, 3, 17, 1023, 5461])
def test_quant_rows_of_any_width_and_place(n):
    wide = randn(gen(n), 9, n + 5)
    for x in (wide[:, :n], wide[:, 3:n + 3], wide[::2, 1:n + 1]):
        q, scale = B.lr_quant_rows(x)
        check_rows(x, q, scale)
        assert q.stride(0) % 16 == 0 or n <= 16
        behind = torch.as_strided(q, (q.shape[0], -(-n // 16) * 16), (q.stride(0), 1))
        assert not behind[:, n:].any()


def test_quant_rows_ties_and_magnitudes():
    """Every bf16 number below the largest one beside it, as a tie wherever 254 x is an odd multiple of the largest; tiny and huge rows; zeros; no
    numbers."""
    mags = torch.arange(1, 1 << 15, device=DEV, dtype=torch.int16).view(BF)
    mags = mags[torch.isfinite(mags.float()) & (mags.float() > 2.0 ** -12) & (mags.float() <= 1.9921875)].to(F32)
    rows = []
    for most in (1.0, 1.9921875, 1.5, 1.0078125, 1.25):
        row = torch.where(mags <= most, mags, 0.0)
        row[-1] = most
        rows.append(torch.nn.functional.pad(row, (0, -row.numel() % 8)))
    x = torch.stack(rows)
    for dtype in (BF, F32):
        check_rows(x.to(dtype), *B.lr_quant_rows(x.to(dtype)))
    x = randn(gen(3), 12, 64)
    x[0], x[1, 5], x[2, 6], x[3, 63] = 0, float("inf"), float("nan"), -float("inf")
    x[4] *= 1e38 / x[4].abs().max()
    x[5] *= 1e-36
    x[6] *= 1e-38
    x[7] *= 1e-40
    x[8] = torch.arange(64, device=DEV) * 2.0 ** -126 / 2 - 2.0 ** -121
    x[9, :] = 3.4e38
    x[10] = -x[10].abs()
    for dtype in (BF, F32):
        check_rows(x.to(dtype), *B.lr_quant_rows(x.to(dtype)))


def ints(g, rows, K, room=0):
    """[rows, K] in rows of whole 16 bytes that hold something behind K too."""
    wide = torch.randint(-127, 128, (rows, -(-K // 16) * 16 + room), generator=g, device=DEV, dtype=torch.int8)
    return wide[:, :K]


def scales(g, rows):
    return torch.rand((rows,), generator=g, device=DEV) * 0.1 + 1e-3


def product(a, sa, b, sb, dtype):
    """The sum is exact; then it is made a float, and multiplied twice."""
    acc = (a.double() @ b.double().t().contiguous())
    want = acc * sa.double()[:, None] * sb.double()[None, :]
    half = torch.finfo(dtype).eps / 2
    return want, want.abs() * (half * (1 + 2.0 ** -7) + (3 * 2.0 ** -24 if dtype == BF else 2 * 2.0 ** -24))


SHAPES = [(1, 1, 1), (1, 33, 15), (3, 7, 16), (33, 31, 17), (32, 64, 32), (5, 100, 129), (16, 1024, 4096), (16, 4096, 1024), (64, 2048, 512), (65, 129, 1000),
          (100, 777, 333), (128, 128, 128), (129, 257, 640), (256, 512, 255), (777, 2047, 546), (300, 4096, 64), (1031, 768, 256), (2048, 2048, 2048),
          (16, 1024, 11000), (50, 700, 9001), (64, 8200, 2050), (40, 33000, 515), (128, 33000, 523), (100, 4100, 4109), (17, 16500, 1024), (9000, 1, 40), (1, 9000, 40), (40000, 3, 7)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_matmul_q8(M, N, K, dtype):
    g = gen(M + N + K)
    a, b, sa, sb = ints(g, M, K), ints(g, N, K, 32), scales(g, M), scales(g, N)
    got = B.lr_matmul_q8(a, sa, b, sb, dtype=dtype)
    want, tol = product(a, sa, b, sb, dtype)
    assert got.shape == (M, N) and got.dtype == dtype
    assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())


@pytest.mark.parametrize("M,N", [(20, 50), (300, 333)])
def test_matmul_q8_writes_its_columns_alone(M, N):
    g = gen(5)
    a, b, sa, sb = ints(g, M, 100), ints(g, N, 100), scales(g, M), scales(g, N)
    for dtype in (BF, F32):
        room = torch.full((M + 2, 400), 7.0, dtype=dtype, device=DEV)
        out = room[1:-1, 8:8 + N]
        assert B.lr_matmul_q8(a, sa, b, sb, out=out).data_ptr() == out.data_ptr()
        want, tol = product(a, sa, b, sb, dtype)
        assert bool(((out.double() - want).abs() <= tol).all())
        out.fill_(7.0)
        assert bool((room == 7.0).all())


def test_matmul_q8_largest_sums_and_scales_that_are_no_numbers():
    a = torch.full((40, 131072), -128, dtype=torch.int8, device=DEV)[:, :131071]
    b = torch.full((33, 131072), -128, dtype=torch.int8, device=DEV)[:, :131071]
    b[1] = 127
    one = torch.ones(40, device=DEV)
    got = B.lr_matmul_q8(a, one, b, one[:33], dtype=F32)
    want = torch.full((33,), 131071.0 * 128 * 128, dtype=torch.float64, device=DEV)
    want[1] *= -127 / 128
    assert bool(((got.double() - want).abs() <= 2.0 ** -24 * want.abs()).all())
    x = randn(gen(1), 4, 64)
    x[2, 3] = float("nan")
    q, s = B.lr_quant_rows(x)
    w, sw = B.lr_quant_rows(randn(gen(2), 24, 64))
    got = B.lr_matmul_q8(q, s, w, sw, dtype=F32)
    assert bool(torch.isnan(got[2]).all()) and bool(torch.isfinite(got[[0, 1, 3]]).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,d,r,n,silu", [(1, 64, 16, 64, True), (16, 512, 128, 512, True), (7, 136, 40, 72, False), (133, 264, 72, 328, True), (300, 1024, 256, 768, True),
                                          (777, 512, 64, 1368, False), (5, 4096, 1024, 4096, True), (16, 1024, 1024, 4200, True),
                                          (9, 4000, 520, 8504, False)])
def test_linear_q8(T, d, r, n, silu, dtype):
    """Bound, element by element.  z and a are within e = 2^-18 of their size (three roundings; the logistic's exponent is rounded by 2^-23 |z| and |z| is
    below 16 here), so the largest of a row and an element are off by 2 e together, and 127 a / max by 254 e: an element may fall to the other side of a half
    only if it lies within that of one, and then costs one step times its weight.  Everything else is relative: scale e, product 3 * 2^-24, storage half a
    step."""
    g = gen(T + d)
    x = randn(g, T, d).to(dtype)
    wd, sd = B.lr_quant_rows(randn(g, r, d) / d ** 0.5)
    wu, su = B.lr_quant_rows(randn(g, n, r) / r ** 0.5)
    got = np64(B.lr_linear_q8_fwd(x, wd, sd, wu, su, act=B.LR_ACT_SILU if silu else B.LR_ACT_IDENTITY))
    z, a, q, s, want = so.linear_q8(np64(x), wd.cpu().numpy(), np64(sd), wu.cpu().numpy(), np64(su), silu)
    assert np.abs(z).max() < 16
    e = 2.0 ** -18
    most = np.abs(a).max(1, keepdims=True)
    t = 127 * np.abs(a) / most
    open_ = np.abs(t - np.floor(t) - 0.5) <= 254 * e
    w = np.abs(wu.cpu().numpy().astype(np.float64)) * np64(su)[:, None]
    tol = (open_ * s[:, None]) @ w.T + np.abs(want) * (2 * e + torch.finfo(dtype).eps / 2 * (1 + 2.0 ** -7))
    assert got.shape == want.shape and np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) - tol)


def test_linear_q8_rows_apart_and_workspace():
    """Rows inside wider ones, in exactly the workspace that is asked for, with a guard behind its end; a row's result does not depend on the others."""
    g = gen(9)
    T, d, r, n = 70, 264, 72, 136
    x = randn(g, T, d + 24)[:, :d].to(BF)
    x = torch.nn.functional.pad(x, (0, 24))[:, :d]
    wd, sd = B.lr_quant_rows(randn(g, r, d))
    wu, su = B.lr_quant_rows(randn(g, n, r))
    want = B.lr_linear_q8_fwd(x, wd, sd, wu, su)
    nb = B.lr_linear_q8_workspace_bytes(T, d, r)
    ws = torch.full((nb + 256,), 77, dtype=torch.uint8, device=DEV)
    room = torch.full((T, n + 16), 7.0, dtype=BF, device=DEV)
    B.lr_linear_q8_fwd(x, wd, sd, wu, su, y=room[:, 8:8 + n], ws=ws[:nb])
    assert torch.equal(room[:, 8:8 + n], want) and bool((room[:, :8] == 7).all()) and bool((room[:, 8 + n:] == 7).all()) and bool((ws[nb:] == 77).all())
    assert torch.equal(B.lr_linear_q8_fwd(x[31:33].contiguous(), wd, sd, wu, su), want[31:33])
    with pytest.raises(B.LrError):
        B.lr_linear_q8_fwd(x, wd, sd, wu, su, ws=ws[:nb - 1])
    for some in (x[31:32], x[3:19], x[:40]):              # (as many forms as there are for few tokens and many)
        y = B.lr_linear_q8_fwd(some, wd, sd, wu, su)
        assert torch.equal(y, B.lr_linear_q8_fwd(x, wd, sd, wu, su)[some.storage_offset() // x.stride(0):][:len(some)])
    assert B.lr_linear_q8_fwd(x[:0], wd, sd, wu, su).shape == (0, n) and B.lr_quant_rows(x[:0])[0].shape == (0, d)


@pytest.mark.parametrize("T", [1, 16, 130])
def test_captured_layers_share_a_workspace(T):
    """Two captured layers on one workspace, replayed in turn on other tokens with eager calls between; then one on another stream."""
    g = gen(30 + T)
    layers = []
    for d, r, n, dtype in ((512, 128, 264, BF), (1000, 72, 512, F32)):
        layers.append(((randn(g, T, d) * 2).to(dtype), *B.lr_quant_rows(randn(g, r, d)), *B.lr_quant_rows(randn(g, n, r))))
    nb = max(B.lr_linear_q8_workspace_bytes(T, w[0].shape[1], w[1].shape[0]) for w in layers)
    ws = torch.full((nb + 256,), 77, dtype=torch.uint8, device=DEV)
    outs = [B.lr_linear_q8_fwd(*w, ws=ws[:nb]) for w in layers]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in layers]
    for graph, w, y in zip(graphs, layers, outs):
        with torch.cuda.graph(graph):
            B.lr_linear_q8_fwd(*w, y=y, ws=ws[:nb])
    for turn in range(3):
        for graph, w, y in zip(graphs, layers, outs):
            w[0].copy_(randn(g, *w[0].shape) * (turn + 1))
            graph.replay()
            want = B.lr_linear_q8_fwd(*w)
            torch.cuda.synchronize()
            assert torch.equal(y, want), turn
    assert bool((ws[nb:] == 77).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q, s = B.lr_quant_rows(layers[0][0])
        got = B.lr_linear_q8_fwd(*layers[0]), B.lr_matmul_q8(q, s, layers[0][1], layers[0][2])
    side.synchronize()
    q, s = B.lr_quant_rows(layers[0][0])
    assert torch.equal(got[0], B.lr_linear_q8_fwd(*layers[0])) and torch.equal(got[1], B.lr_matmul_q8(q, s, layers[0][1], layers[0][2]))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [3, 90])
def test_tokens_that_are_no_numbers_stay_alone(T, dtype):
    """A token with an infinity or a NaN gives NaN, in every column of its own row; a token of zeros gives zeros."""
    g = gen(T)
    x = randn(g, T, 264).to(dtype)
    w = (*B.lr_quant_rows(randn(g, 72, 264)), *B.lr_quant_rows(randn(g, 136, 72)))
    want = B.lr_linear_q8_fwd(x, *w)
    x[0, 100], x[1, 7], x[2] = float("inf"), float("nan"), 0
    got = B.lr_linear_q8_fwd(x, *w)
    assert got[:2].isnan().all() and not got[2].any() and torch.equal(got[3:], want[3:])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,r,n", [(1024, 256, 1024), (2048, 512, 264), (4096, 64, 136), (1000, 1000, 8), (104, 2048, 3000), (103, 72, 40)])
def test_a_token_alone_and_among_others(d, r, n, dtype):
    """Rows of a layer are the same bits, quantised by a launch of their own (17 tokens) or by the first product (a few), rows at any place in wider ones;
    ties and numbers that are none among them."""
    d += -d % 8 if dtype == BF else 0
    g = gen(d + r)
    wide = (randn(g, 17, d + 8) * 3).to(dtype)
    x = wide[:, 8:] if dtype == BF else wide[:, 3:d + 3]
    x[4, 9], x[5, 0], x[6] = float("nan"), -float("inf"), 0
    x[2, d // 2] = x[2].abs().max() / 2
    w = (*B.lr_quant_rows(randn(g, r, d)), *B.lr_quant_rows(randn(g, n, r)))
    want = B.lr_linear_q8_fwd(x, *w)
    bits = lambda t: t.contiguous().view(torch.int16 if dtype == BF else torch.int32)
    for first, count in ((0, 1), (4, 1), (3, 2), (0, 8), (8, 5), (1, 16)):
        assert torch.equal(bits(B.lr_linear_q8_fwd(x[first:first + count], *w)), bits(want[first:first + count])), (first, count)


def test_offsets_past_32_bits():
    """Rows of 8-bit integers and results with more than 2^31 elements: the last ones are those of the rows alone."""
    g = gen(40)
    M, N = 66000, 33000
    a, b, sa, sb = ints(g, M, 16), ints(g, N, 16), scales(g, M), scales(g, N)
    big = B.lr_matmul_q8(a, sa, b, sb)
    assert big.numel() > 2 ** 31
    for rows in (slice(0, 300), slice(M // 2, M // 2 + 300), slice(M - 300, M)):
        assert torch.equal(big[rows], B.lr_matmul_q8(a[rows].contiguous(), sa[rows].contiguous(), b, sb))
    q, s = B.lr_quant_rows(big)
    for rows in (slice(0, 40), slice(M - 40, M)):
        alone = B.lr_quant_rows(big[rows].clone())
        assert torch.equal(q[rows], alone[0]) and torch.equal(s[rows], alone[1])
