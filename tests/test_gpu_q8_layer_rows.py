"""The rows between a layer's two products are those of lr_quant_rows, whatever the activation and however many tokens there are."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2512_12131_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def apart(x, wd, sd, wu, su, act):
    """The layer in single steps: rows, product, activation, rows, product.  And what the second rows were made of."""
    z = B.lr_matmul_q8(*B.lr_quant_rows(x), wd, sd, dtype=F32)
    a = z if act == B.LR_ACT_IDENTITY else B.lr_act_fwd(z.contiguous(), act)
    return B.lr_matmul_q8(*B.lr_quant_rows(a), wu, su, dtype=x.dtype), a


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)


def before_silu(a):
    """z of which a = z / (1 + exp(-z)), for a >= 0 in 64 bits."""
    z = a.clone() + 0.3
    for _ in range(60):
        s = torch.sigmoid(z)
        z = z - (z * s - a) / (s * (1 + z * (1 - s)))
    return z


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", [B.LR_ACT_IDENTITY, B.LR_ACT_SILU])
def test_elements_next_to_a_half(act, dtype):
    """A row of z is 127 sx sd[j] for tokens that hold one number, so sd puts 127 |a| / max next to k + 1/2 for every k, within a few last places: the
    product with a rounded 127 / max falls to either side there, the quotient does not."""
    g = torch.Generator(device=DEV).manual_seed(act + 5)
    d, r, n, T = 64, 1024, 264, 40
    k = torch.arange(r, device=DEV, dtype=torch.float64) % 127 + 0.5
    target = k / 127 * 5.3
    if act == B.LR_ACT_SILU:
        target = before_silu(target)
    ulps = torch.randint(-3, 4, (r,), generator=g, device=DEV, dtype=torch.int32)
    sd = (target.float().view(torch.int32) + ulps).view(F32)
    sd[-1] = (before_silu(torch.tensor([5.3], dtype=torch.float64, device=DEV)) if act == B.LR_ACT_SILU else torch.tensor([5.3], device=DEV)).float()
    wd = torch.zeros((r, d), dtype=torch.int8, device=DEV)
    wd[:, 3] = 1
    wu, su = B.lr_quant_rows(torch.randn((n, r), generator=g, device=DEV))
    x = torch.zeros((T, d), dtype=dtype, device=DEV)
    x[:, 3] = torch.where(torch.arange(T, device=DEV) % 3 == 0, 1.0, 0.5 + torch.rand(T, generator=g, device=DEV) * 0.7).to(dtype)
    want, a = apart(x, wd, sd, wu, su, act)
    q = 127 * a.double() / a.double().abs().amax(1, keepdim=True)
    near = ((q - torch.floor(q) - 0.5).abs() < 2.0 ** -15).sum()
    assert int(near) > 1000
    for first, count in ((0, T), (0, 1), (3, 1), (1, 8), (4, 16), (2, 17)):
        got = B.lr_linear_q8_fwd(x[first:first + count].contiguous(), wd, sd, wu, su, act=act)
        assert torch.equal(bits(got), bits(want[first:first + count])), (first, count)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", [B.LR_ACT_IDENTITY, B.LR_ACT_SILU])
@pytest.mark.parametrize("d,r,n", [(1024, 256, 1024), (2048, 512, 264), (4096, 1024, 136), (104, 2048, 3000), (96, 72, 40)])
def test_a_layer_is_its_single_steps(d, r, n, act, dtype):
    """For any number of tokens, with ties, zeros and numbers that are none among them: a row's bits depend on the row alone."""
    g = torch.Generator(device=DEV).manual_seed(d + r + act)
    x = (torch.randn((130, d), generator=g, device=DEV) * 3).to(dtype)
    x[4, 9], x[5, 0], x[6] = float("nan"), -float("inf"), 0
    x[2, d // 2] = x[2].abs().max() / 2
    wd, sd = B.lr_quant_rows(torch.randn((r, d), generator=g, device=DEV) / d ** 0.5)
    wu, su = B.lr_quant_rows(torch.randn((n, r), generator=g, device=DEV) / r ** 0.5)
    want, _ = apart(x, wd, sd, wu, su, act)
    for first, count in ((0, 130), (0, 1), (4, 1), (3, 2), (0, 8), (8, 5), (1, 16), (0, 17), (40, 64)):
        got = B.lr_linear_q8_fwd(x[first:first + count].contiguous(), wd, sd, wu, su, act=act)
        assert torch.equal(bits(got), bits(want[first:first + count])), (first, count)


@pytest.mark.parametrize("n", [1016, 8 * 1016, 16 * 1016])
def test_fp32_rows_next_to_a_half(n):
    """Elements at (2 k + 1) max / 254 for every k and up to three last places beside it, and exact halves (max a multiple of 254), for the smallest and largest
    rows there are: whole numbers are those of the quotient, which 64 bits hold exactly where it is a half and else decide (2^-33 off one at least)."""
    rng = np.random.default_rng(n)
    most = np.concatenate([2.0 ** np.array([-126.0, -119, -40, -1, 0, 1, 60, 127]) * (1 + rng.random(8)), 254.0 * 2.0 ** np.array([-120.0, -30, 0, 100]) * rng.integers(1, 2 ** 16, 4),
                           127 * 2.0 ** -126 * np.array([1 - 2.0 ** -20, 1, 1 + 2.0 ** -20])]).astype(np.float32)
    k = np.arange(n) % 127
    x = ((2 * k + 1) * most.astype(np.float64)[:, None] / 254).astype(np.float32)
    x = np.where(most[:, None] % 254 == 0, x, (x.view(np.int32) + rng.integers(-3, 4, x.shape).astype(np.int32)).view(np.float32))
    x *= np.where(rng.random(x.shape) < 0.5, -1, 1).astype(np.float32)
    x[:, n // 2] = most
    want, scale = so.quant_rows(x.astype(np.float64))
    q, s = B.lr_quant_rows(torch.from_numpy(x).to(DEV))
    assert np.array_equal(q.cpu().numpy().astype(np.int64), want)
    assert np.array_equal(s.cpu().numpy(), scale.astype(np.float32))
